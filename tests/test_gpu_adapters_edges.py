"""Low-rank updates of many adapters at the ends of the range, with 32-bit outputs, and rows without an adapter bit for bit: on the GPU against 64 bits."""
import pytest
import torch

from paper_2609_05419_b200 import binding as b

pytestmark = pytest.mark.gpu

from test_gpu_adapters import operands, plain, room, workspace  # noqa: E402


@pytest.mark.parametrize("tokens", [5, 300])
@pytest.mark.parametrize("rank", [4, 40])
@pytest.mark.parametrize("x_size,a_size,w_size", [(1e-10, 1e-10, 1e38), (1e-15, 1e-15, 1e38), (1e-3, 1e-7, 1e37), (1e10, 1e10, 1e-36), (1e15, 1e15, 1e-33), (1e18, 1e17, 1e-34)])
def test_small_numbers_times_large_ones(tokens, rank, x_size, a_size, w_size):
    """X A^T far below 1 beside a B near the end of bf16's range, and the other way round: results well inside 32 bits."""
    x, a, w, index, _, _, _ = operands(tokens, 64, 40, 2, rank, torch.bfloat16, 5, ranks=False, bare=False)
    x, a, w = (torch.tanh(t.float()).mul(size).bfloat16() for t, size in ((x, x_size), (a, a_size), (w, w_size)))
    d = torch.empty(tokens, 40, device="cuda")
    with workspace(tokens, rank, 2):
        b.adapter_add(x, a, w, index, d)
    want, size, beside = plain(x, a, w, index, None, None, None)
    off, most = (d.double() - want).abs(), room(64, rank, want, size, beside, torch.bfloat16, torch.float32)
    assert bool((off <= most).all()), float((off / most).max())


def exact_room(k, rank, want, size):
    """Without any allowance for parts of L: products of 16-bit numbers are exact; sums of k and of 3 rank terms with up to 40 pieces, of which random roundings leave
    the root; the scale, the power of two, C, and D's own rounding."""
    return size * (k + 3 * rank + 48) ** 0.5 * 2.0 ** -23 + 2.0 ** -23 * want.abs()


@pytest.mark.parametrize("tokens,k,n,many,rank", [(1, 64, 40, 1, 1), (40, 256, 320, 3, 16), (40, 100, 33, 3, 30), (200, 64, 256, 2, 64), (256, 96, 90, 5, 128),
                                                  (600, 256, 320, 3, 16), (300, 100, 333, 3, 30), (700, 64, 256, 2, 64), (513, 96, 130, 5, 128), (300, 64, 129, 2, 65)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_outputs_of_32_bits_are_those_of_32_bit_sums(tokens, k, n, many, rank, dtype):
    x, a, w, index, c, scales, _ = operands(tokens, k, n, many, rank, dtype, 21, torch.float32, ranks=False, bare=False)
    d = torch.empty(tokens, n, device="cuda")
    with workspace(tokens, rank, many) as ws:
        ws.buf[4096:].fill_(0xff)
        for add in (None, c):
            b.adapter_add(x, a, w, index, d, C=add, scales=scales)
            b.device_status()
            want, size, _ = plain(x, a, w, index, add, scales, None)
            off, most = (d.double() - want).abs(), exact_room(k, rank, want, size)
            # In the mean the error is that of sums in 32 bits, relative to their partial sums, whose size is the root of the sum of the terms' squares.  (Not of the result: with one
            # token and rank 1 all entries share the error of one sum L, and |L| may be an eighth of the root of 64 terms' squares.)  The tensor cores add 16 products at once and cut the
            # sum, by up to 2^-23 of it and half of that in the mean, always towards zero, so that cuts add up: k / 16 for L, rank / 16 for the update, 2^-24 each; the parts beside the
            # first are below 2^-8 of it and their cuts of no account; four roundings behind.
            squares = torch.zeros_like(want) if add is None else add.double().square()
            for i in range(many):
                rows = (index == i).nonzero()[:, 0]
                squares[rows] += float(scales[i]) ** 2 * (x[rows].double().square() @ a[i].double().square().t()) @ w[i].double().square().t()
            terms = torch.maximum(want.abs(), squares.sqrt())
            assert float(torch.linalg.vector_norm(off) / torch.linalg.vector_norm(terms)) <= (4 + (k + rank) / 16) * 2.0 ** -24
            assert bool((off <= most).all()), float((off / most).max())


@pytest.mark.parametrize("tokens", [30, 300])
def test_outputs_of_32_bits_cancel_what_was_there(tokens):
    """C holds the update with the opposite sign: what is left is the rounding of 32 bits, not of the parts that the product took."""
    x, a, w, index, _, scales, _ = operands(tokens, 128, 70, 2, 8, torch.bfloat16, 31, ranks=False, bare=False)
    update, size, _ = plain(x, a, w, index, None, scales, None)
    d = torch.empty(tokens, 70, device="cuda")
    with workspace(tokens, 8, 2):
        b.adapter_add(x, a, w, index, d, C=-update.float(), scales=scales)
    assert bool((d.abs().double() <= exact_room(128, 8, update, size)).all())


@pytest.mark.parametrize("tokens,k,n,many,rank", [(1, 500, 40, 1, 2), (40, 256, 320, 3, 16), (37, 1000, 33, 3, 30), (200, 256, 256, 2, 64), (256, 600, 90, 5, 128),
                                                  (600, 256, 320, 3, 16), (300, 1000, 333, 3, 30), (700, 256, 256, 2, 64), (513, 400, 130, 5, 128)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_whole_numbers_are_exact(tokens, k, n, many, rank, dtype):
    """Every sum is a whole number below 2^24 and needs more bits than two 16-bit numbers hold (16 and 22): nothing may be rounded anywhere.  Two entries of B per column are not
    zero.  |L| is below 6 x 127^2 / 3 sqrt(1000) < 2^20 (bf16) or 6 x 2047 x 511 / 3 sqrt(k) with k <= 16 entries < 2^23."""
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    whole = lambda most, *shape: torch.randint(-most, most + 1, shape, generator=g, device="cuda").float()
    x, a = (whole(127, tokens, k), whole(127, many, rank, k)) if dtype == torch.bfloat16 else (whole(2047, tokens, k), whole(511, many, rank, k))
    if dtype == torch.float16:
        a[:, :, 16:] = 0
    w = torch.zeros(many, n, rank, device="cuda")
    for _ in range(2):
        w.scatter_(2, torch.randint(0, rank, (many, n, 1), generator=g, device="cuda"), whole(1, many, n, 1))
    x, a, w = x.to(dtype), a.to(dtype), w.to(dtype)
    index = torch.randint(0, many, (tokens,), generator=g, device="cuda").to(torch.int32)
    c, d = whole(1000, tokens, n), torch.empty(tokens, n, device="cuda")
    with workspace(tokens, rank, many):
        b.adapter_add(x, a, w, index, d, C=c)
    want = plain(x, a, w, index, c, None, None)[0]
    assert float(want.abs().max()) < 2 ** 24 and bool((d.double() == want).all())


@pytest.mark.parametrize("tokens", [1, 9, 256, 257])
@pytest.mark.parametrize("n,skip", [(40, 0), (41, 0), (300, 0), (64, 1)])
@pytest.mark.parametrize("d_type", [torch.float32, torch.float16, torch.bfloat16])
def test_rows_without_an_adapter_are_those_of_c_bit_for_bit(tokens, n, skip, d_type):
    """Negative zeros, NaN with payloads and subnormals among them; no adapter, or one of rank 0."""
    x, a, w, index, c, _, _ = operands(tokens, 64, n, 3, 20, torch.bfloat16, 41, d_type, ranks=False)
    index[::2] = -1
    used = torch.tensor([20, 0, 7], dtype=torch.int32, device="cuda")
    whole = torch.int32 if d_type == torch.float32 else torch.int16
    odd = {torch.float32: [-2 ** 31, 0x7f812345, -0x3fedcb, 1, -2 ** 31 + 1], torch.float16: [-2 ** 15, 0x7d23, -0x2ed, 1, -2 ** 15 + 1],
           torch.bfloat16: [-2 ** 15, 0x7fa3, -0x5d, 1, -2 ** 15 + 1]}[d_type]
    c.view(whole)[:, :len(odd) * 7:7] = torch.tensor(odd, dtype=whole, device="cuda")[:c[:, :len(odd) * 7:7].shape[1]]
    store = torch.full((tokens, n + 9), 3.0, device="cuda").to(d_type)
    d = store[:, skip:skip + n]
    with workspace(tokens, 20, 3):
        b.adapter_add(x, a, w, index, d, C=c, ranks=used)
        bare = (index < 0) | (index == 1)
        assert torch.equal(d[bare].view(whole), c[bare].view(whole))
        b.adapter_add(x, a, w, index, d, ranks=used)
        assert bool((d[bare].view(whole) == 0).all())
    assert bool((store[:, :skip] == 3).all()) and bool((store[:, skip + n:] == 3).all())


@pytest.mark.parametrize("tokens,k,rank", [(300, 32768, 16), (300, 32768, 60), (300, 32768, 128), (4096, 8192, 16), (2000, 16384, 32), (257, 32001, 9)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_sums_over_long_rows_of_positive_products(tokens, k, rank, dtype):
    """Sums in which every cut goes the same way.  B is the unit matrix, so D is X A^T.  Up to eight blocks share k, and of a block's steps of 64 entries an accumulator has eight or, where there is not
    room for so many of the padded rank in 256 columns, an even share; a step is four additions, each cut by up to 2^-23 of the partial sum (fp16, whose products are longer than
    bf16's, by up to four times that), which is half of the accumulator's in the mean; then roundings to the nearest."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rank)
    draw = lambda *shape: torch.randn(shape, generator=g, device="cuda").abs()
    x, a = draw(tokens, k).to(dtype), (draw(1, rank, k) / 16).to(dtype)
    w = torch.eye(rank, device="cuda").to(dtype)[None].contiguous()
    d = torch.empty(tokens, rank, device="cuda")
    with workspace(tokens, rank, 1):
        b.adapter_add(x, a, w, torch.zeros(tokens, dtype=torch.int32, device="cuda"), d)
        b.device_status()
    want = x.double() @ a[0].double().t()
    padded = 16 if rank <= 16 else 32 if rank <= 32 else 64 if rank <= 64 else 128
    tiles = tokens // 128 + 2
    blocks = max(1, min(8, 296 // tiles))
    steps = -(-(-(-k // 64)) // blocks)
    cuts = 4 * max(8, -(-steps // (256 // padded)))
    assert bool(((d.double() - want).abs() <= (cuts / 2 * (1 if dtype == torch.bfloat16 else 4) + 8) * 2.0 ** -23 * want).all())

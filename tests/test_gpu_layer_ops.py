"""Layer operators on the GPU against plain implementations in 64 bits: quantisation to 8-bit floating point with block scales, the
product of two such matrices, Newton-Schulz orthogonalisation, and the training example that runs them together."""
import math

import pytest
import torch

from paper_2609_05419_b200 import binding as b

pytestmark = pytest.mark.gpu

from gpu_util import Workspace  # noqa: E402

MAX = {b.E4M3: 448.0, b.E5M2: 57344.0}
DTYPE = {b.E4M3: torch.float8_e4m3fn, b.E5M2: torch.float8_e5m2}


def blocks(v, size=128):
    return -(-v // size)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ------------------------------------------------------------------------------------------------------ quantisation
def plain_quantise(x, block, fmt):
    """(values as 64-bit numbers, scales): the definition, entry by entry of the block grid; scale and inverse scale are single
    divisions in 32 bits, as documented, so the comparison is for equality."""
    x = x.float().cpu()
    rows, cols = x.shape
    s = torch.empty(blocks(rows, block), blocks(cols))
    q = torch.empty(rows, cols, dtype=torch.float64)
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            cut = (slice(i * block, (i + 1) * block), slice(128 * j, 128 * (j + 1)))
            part = x[cut]
            u = torch.clamp(part.abs().max(), min=2.0 ** -100).reshape(1)
            s[i, j] = (u / torch.tensor([MAX[fmt]]))[0] if bool(torch.isfinite(part).all()) else float("nan")
            inv = torch.tensor([MAX[fmt]]) / u
            q[cut] = (part * inv).clamp(-MAX[fmt], MAX[fmt]).to(DTYPE[fmt]).double()
    return q, s


QUANT = [(1, 1), (1, 128), (3, 4096), (16, 1000), (127, 129), (128, 128), (129, 257), (300, 7), (513, 640)]


@pytest.mark.parametrize("rows,cols", QUANT)
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("dtype,fmt", [(torch.bfloat16, b.E4M3), (torch.float32, b.E4M3), (torch.float16, b.E5M2)])
def test_quantise_equals_its_definition(rows, cols, block, dtype, fmt):
    x = (torch.randn(rows, cols, generator=gen(1), device="cuda") * torch.exp(2 * torch.randn(rows, 1, generator=gen(2), device="cuda"))).to(dtype)
    q, s = b.fp8_empty(rows, cols, fmt, block)
    qt, st = b.fp8_empty(cols, rows, fmt, block)
    b.fp8_quantise(x, q, s, qt, st, block_rows=block)
    for got, scale, ref in ((q, s, x), (qt, st, x.t())):
        rq, rs = plain_quantise(ref, block, fmt)
        assert torch.equal(scale.cpu(), rs)
        assert torch.equal(got.double().cpu(), rq)
    # half a unit in the last place of the 8-bit value, in units of x: 2^-4 (2^-3) relative, or half the smallest spacing
    values = q.double() * s.double().repeat_interleave(128, 1)[:, :cols].repeat_interleave(block, 0)[:rows]
    rel, least = (2.0 ** -4, 2.0 ** -10) if fmt == b.E4M3 else (2.0 ** -3, 2.0 ** -17)
    room = torch.maximum(rel * x.double().abs(), least * s.double().repeat_interleave(128, 1)[:, :cols].repeat_interleave(block, 0)[:rows])
    assert bool(((values - x.double()).abs() <= room * (1 + 1e-6)).all())


@pytest.mark.parametrize("form", ["rows", "transposed"])
@pytest.mark.parametrize("block", [1, 128])
def test_quantise_one_form_of_a_strided_unaligned_matrix_and_nothing_beside_it(form, block):
    rows, cols = 200, 333
    store = torch.randn(rows * 400 + 1, generator=gen(3), device="cuda")
    x = store[1:].view(rows, 400)[:, 2:2 + cols]                  # rows start 12 bytes past a 16-byte boundary
    assert x.data_ptr() % 16 != 0
    r, c = (rows, cols) if form == "rows" else (cols, rows)
    buf = torch.full((r + 1, 400), 77, dtype=torch.uint8, device="cuda")
    sbuf = torch.full((blocks(c) + 1, 400), 7.0, device="cuda")
    q, s = buf.view(torch.float8_e4m3fn)[:r, :c], sbuf[:blocks(c), :blocks(r, block)].t()
    b.fp8_quantise(x, *((q, s) if form == "rows" else (None, None, q, s)), block_rows=block)
    rq, rs = plain_quantise(x if form == "rows" else x.t(), block, b.E4M3)
    assert torch.equal(q.double().cpu(), rq) and torch.equal(s.cpu(), rs)
    assert bool((buf[r:] == 77).all()) and bool((buf[:, c:] == 77).all())
    assert bool((sbuf[blocks(c):] == 7).all()) and bool((sbuf[:, blocks(r, block):] == 7).all())


@pytest.mark.parametrize("block", [1, 128])
def test_quantise_zeros_extremes_and_non_finite_blocks(block):
    x = torch.zeros(256, 512, device="cuda")
    x[0, 0], x[1, 130], x[2, 5] = 3e38, 1e-42, -1.0               # the largest, a denormal, an ordinary value
    x[200, 300], x[201, 450] = float("inf"), float("nan")
    q, s = b.fp8_empty(256, 512, b.E4M3, block)
    qt, st = b.fp8_empty(512, 256, b.E4M3, block)
    b.fp8_quantise(x, q, s, qt, st, block_rows=block)
    for got, scale, ref in ((q, s, x), (qt, st, x.t())):
        rq, rs = plain_quantise(ref, block, b.E4M3)
        assert torch.equal(torch.isnan(scale.cpu()), torch.isnan(rs)) and int(torch.isnan(rs).sum()) == 2
        assert torch.equal(torch.nan_to_num(scale.cpu()), torch.nan_to_num(rs))
        fine = ~torch.isnan(rs).repeat_interleave(128, 1)[:, :ref.shape[1]].repeat_interleave(block, 0)[:ref.shape[0]]
        assert torch.equal(got.double().cpu()[fine], rq[fine])


# ----------------------------------------------------------------------------------------------------------- products
def operand(rows, k, block, fmt, seed, ld_extra=0):
    """Random 8-bit values with random scales, laid out with `ld_extra` x 16 bytes of NaN codes behind every row."""
    g = gen(seed)
    width = blocks(k, 16) * 16 + 16 * ld_extra
    buf = torch.full((rows, width), 0x7f, dtype=torch.uint8, device="cuda").view(DTYPE[fmt])
    q = buf[:, :k]
    q.copy_((torch.randn(rows, k, generator=g, device="cuda") * (40 if fmt == b.E4M3 else 400)).clamp(-MAX[fmt], MAX[fmt]))
    s = torch.exp(torch.randn(blocks(k), blocks(rows, block), generator=g, device="cuda")) * 1e-3
    return q, s.t()


def spread(s, block, rows, k):
    return s.double().repeat_interleave(128, 1)[:, :k].repeat_interleave(block, 0)[:rows]


def check_product(m, n, k, ab=1, bb=128, fa=b.E4M3, fb=b.E4M3, dtype=torch.bfloat16, add=False, seed=5, ld_extra=0, d=None):
    qa, sa = operand(m, k, ab, fa, seed, ld_extra)
    qb, sb = operand(n, k, bb, fb, seed + 1, ld_extra)
    a, w = qa.double() * spread(sa, ab, m, k), qb.double() * spread(sb, bb, n, k)
    c = torch.randn(m, n, generator=gen(seed + 2), device="cuda").to(dtype) if add else None
    exact = a @ w.t() + (c.double() if add else 0.0)
    size = a.abs() @ w.abs().t() + (c.double().abs() if add else 0.0)
    d = torch.empty(m, n, dtype=dtype, device="cuda") if d is None else d
    d.fill_(float("nan"))
    b.fp8_gemm(qa, sa, qb, sb, d, C=c, a_block=ab, b_block=bb)
    b.device_status()
    # products of 8-bit values are exact; a block's 128 additions in 32 bits are off by at most 128 x 2^-23 of the sum of
    # magnitudes (aligned and cut, not rounded, is allowed for), scaling by 2 x 2^-24, adding the blocks and C by 2^-24 each; one rounding
    room = size * (128 * 2.0 ** -23 + (blocks(k) + 4) * 2.0 ** -24)
    room += exact.abs() * {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype] * 1.001 + 2.0 ** -24
    off = (d.double() - exact).abs()
    assert bool((off <= room).all()), float((off / room).max())
    return d


SHAPES = [(1, 1, 1), (1, 128, 128), (1, 4096, 512), (2, 130, 1000), (7, 1000, 129), (16, 256, 1024), (33, 515, 640), (64, 64, 64),
          (65, 129, 257), (128, 128, 128), (129, 1, 300), (200, 700, 15), (256, 256, 256), (257, 511, 1111), (300, 520, 4100),
          (1000, 40, 520), (513, 1025, 385)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("ab,bb", [(1, 128), (1, 1), (128, 1), (128, 128)])
def test_product(m, n, k, ab, bb):
    with Workspace(b.workspace_bytes(b.OP_FP8_GEMM, m, n, k, 1)):
        check_product(m, n, k, ab, bb)


# more tiles than fit the GPU at once, in tiles of either width, with ragged edges
@pytest.mark.parametrize("m,n,k", [(2100, 1300, 700), (4100, 4300, 257), (2500, 2600, 1000), (9000, 200, 384), (130, 20000, 130)])
@pytest.mark.parametrize("bb,dtype", [(128, torch.bfloat16), (1, torch.float32)])
def test_product_of_many_tiles(m, n, k, bb, dtype):
    with Workspace(b.workspace_bytes(b.OP_FP8_GEMM, m, n, k, 1)):
        check_product(m, n, k, 1, bb, dtype=dtype, add=bb == 1)


def test_offsets_beyond_32_bits():
    m, n, k = 66000, 33100, 48                                    # m n > 2^31
    qa, sa = operand(m, k, 1, b.E4M3, 91)
    qb, sb = operand(n, k, 128, b.E4M3, 92)
    d = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    with Workspace(b.workspace_bytes(b.OP_FP8_GEMM, m, n, k, 1)):
        b.fp8_gemm(qa, sa, qb, sb, d)
    rows = torch.tensor([0, 1, 32767, 64999, m - 1], device="cuda")
    want = (qa[rows].double() * sa[rows].double()) @ (qb.double() * spread(sb, 128, n, k)).t()
    assert float((d[rows].double() - want).abs().max()) <= 2.0 ** -7 * float(want.abs().max())
    q, s = b.fp8_empty(m, n)
    qt, st = b.fp8_empty(n, m)
    b.fp8_quantise(d, q, s, qt, st)                               # the last rows and columns against a call of their own
    q1, s1 = b.fp8_empty(100, n)
    b.fp8_quantise(d[-100:], q1, s1)
    assert torch.equal(q[-100:].view(torch.uint8), q1.view(torch.uint8)) and torch.equal(s[-100:], s1)
    q2, s2 = b.fp8_empty(100, m)
    b.fp8_quantise(d[:, -100:], None, None, q2, s2)
    assert torch.equal(qt[-100:].view(torch.uint8), q2.view(torch.uint8)) and torch.equal(st[-100:], s2)


@pytest.mark.parametrize("m,n,k", [(3, 300, 700), (200, 300, 700), (600, 1030, 900)])
@pytest.mark.parametrize("fa,fb", [(b.E5M2, b.E4M3), (b.E4M3, b.E5M2), (b.E5M2, b.E5M2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_product_types(m, n, k, fa, fb, dtype):
    with Workspace(b.workspace_bytes(b.OP_FP8_GEMM, m, n, k, 1)):
        check_product(m, n, k, 1, 128, fa, fb, dtype, add=dtype == torch.float32, ld_extra=1)


@pytest.mark.parametrize("m,n,k", [(1, 1000, 1000), (5, 999, 256), (130, 131, 300), (700, 1030, 500)])
@pytest.mark.parametrize("ld,offset", [(1040, 0), (1037, 0), (1040, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_product_into_a_strided_unaligned_matrix_and_nothing_beside_it(m, n, k, ld, offset, dtype):
    store = torch.empty(m * ld + offset + ld, dtype=dtype, device="cuda").fill_(5.0)
    d = store[offset:offset + m * ld].view(m, ld)[:, :n]
    with Workspace(b.workspace_bytes(b.OP_FP8_GEMM, m, n, k, 1)):
        check_product(m, n, k, dtype=dtype, add=True, d=d)
    assert bool((store[offset:offset + m * ld].view(m, ld)[:, n:] == 5).all()) and bool((store[offset + m * ld:] == 5).all())


@pytest.mark.parametrize("m,n,k,bb", [(4, 600, 512, 128), (300, 300, 640, 1), (600, 600, 300, 1)])
def test_product_added_in_place_twice_and_on_another_stream(m, n, k, bb):
    qa, sa = operand(m, k, 1, b.E4M3, 11)
    qb, sb = operand(n, k, bb, b.E4M3, 12)
    with Workspace(b.workspace_bytes(b.OP_FP8_GEMM, m, n, k, 1)):
        once = torch.empty(m, n, device="cuda")
        b.fp8_gemm(qa, sa, qb, sb, once, b_block=bb)
        d = once.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            b.fp8_gemm(qa, sa, qb, sb, d, C=d, b_block=bb)
            b.device_status(side)
        torch.cuda.synchronize()
        assert torch.equal(d, once + once)                     # x + x is exact, and the product is the same every time
        d.fill_(3.0)
        b.fp8_gemm(qa[:, :0], sa[:, :0], qb[:, :0], sb[:, :0], d, C=d, b_block=bb)
        assert bool((d == 3).all())
        b.fp8_gemm(qa[:, :0], sa[:, :0], qb[:, :0], sb[:, :0], d, b_block=bb)
        assert bool((d == 0).all())


@pytest.mark.parametrize("m,n", [(4, 600), (300, 520)])
def test_product_of_nan_scales_and_unread_neighbours(m, n):
    k = 300
    qa, sa = operand(m, k, 1, b.E4M3, 21, ld_extra=2)             # NaN codes behind every row are not data
    qb, sb = operand(n, k, 128, b.E4M3, 22, ld_extra=2)
    sa[1, 1] = float("nan")
    sb[2, 0] = float("nan")
    d = torch.zeros(m, n, device="cuda")
    with Workspace(b.workspace_bytes(b.OP_FP8_GEMM, m, n, k, 1)):
        b.fp8_gemm(qa, sa, qb, sb, d)
    bad = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    bad[1] = True
    bad[:, 256:384] = True
    assert torch.equal(torch.isnan(d), bad)


def test_product_needs_a_workspace_and_replays_from_a_graph():
    m, n, k = 20, 300, 256
    qa, sa = operand(m, k, 1, b.E4M3, 31)
    qb, sb = operand(n, k, 128, b.E4M3, 32)
    d = torch.empty(m, n, device="cuda")
    b.set_workspace(None)
    with pytest.raises(b.Gemm2mError) as err:
        b.fp8_gemm(qa, sa, qb, sb, d)
    assert err.value.status == b.ERR_WORKSPACE
    with Workspace(b.workspace_bytes(b.OP_FP8_GEMM, m, n, k, 1)):
        b.fp8_gemm(qa, sa, qb, sb, d)
        want = d.clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            d.zero_()
            b.fp8_gemm(qa, sa, qb, sb, d, C=d)
            b.fp8_gemm(qa, sa, qb, sb, d, C=d)
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(d, want + want)


# -------------------------------------------------------------------------------------------------------- Newton-Schulz
MUON = (3.4445, -4.7750, 2.0315)


def plain_newton_schulz(g, steps=5, coeffs=None, eps=1e-7):
    x = g.double()
    x = x / (torch.linalg.vector_norm(x) + eps)
    for i in range(steps):
        a, p, q = MUON if coeffs is None else coeffs if not hasattr(coeffs[0], "__len__") else coeffs[i]
        gram = x @ x.t()
        x = a * x + (p * gram + q * gram @ gram) @ x
    return x


def update(m, n, kind, seed):
    g = gen(seed)
    if kind == "flat":
        return torch.randn(m, n, generator=g, device="cuda")
    r = max(1, min(m, n) // 3)
    fall = torch.arange(1, r + 1, device="cuda", dtype=torch.float32) ** -1.0
    return 1e-3 * (torch.randn(m, r, generator=g, device="cuda") * fall) @ torch.randn(r, n, generator=g, device="cuda")


# 2e-3 of the norm before rounding, as documented, and the rounding to bf16: at most 2^-8 of an entry, and over many entries,
# with errors spread evenly over half a unit in the last place, below 2^-9 of the norm
def ns_room(entries):
    return 2e-3 + (2.0 ** -8 if entries < 64 else 2.0 ** -9)


def check_newton_schulz(g, o, **how):
    want = plain_newton_schulz(g, **how)
    rel = float(torch.linalg.vector_norm(o.double() - want) / torch.linalg.vector_norm(want))
    assert rel <= ns_room(g.numel()), rel


# several tiles per pair, every tile width, both orientations, many matrices
@pytest.mark.parametrize("batch,m,n", [(1, 1500, 2300), (1, 2304, 1100), (40, 200, 260), (12, 700, 600), (1, 2500, 2500), (1, 200, 6100), (6, 3900, 130)])
def test_newton_schulz_of_many_tiles(batch, m, n):
    g = torch.stack([update(m, n, "flat" if i % 2 else "falling", 100 + i) for i in range(batch)])
    o = torch.full((batch, m, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    with Workspace(b.workspace_bytes(b.OP_NEWTON_SCHULZ, m, n, batch, 1)):
        b.newton_schulz(g, o)
        b.device_status()
    for i in range(0, batch, 5):
        check_newton_schulz(g[i], o[i])


NS_SHAPES = [(1, 1), (1, 200), (130, 1), (2, 3), (17, 17), (64, 64), (100, 300), (300, 100), (128, 256), (257, 129), (256, 256), (511, 700), (1030, 520)]


@pytest.mark.parametrize("m,n", NS_SHAPES)
@pytest.mark.parametrize("kind,dtype", [("flat", torch.float32), ("falling", torch.float32), ("falling", torch.bfloat16), ("flat", torch.float16)])
def test_newton_schulz(m, n, kind, dtype):
    scale = 100.0 if dtype == torch.float16 else 1.0                 # (keeps the falling spectrum's entries out of the subnormals)
    g = (update(m, n, kind, 41) * scale).to(dtype)
    o = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    with Workspace(b.workspace_bytes(b.OP_NEWTON_SCHULZ, m, n, 1, 1)):
        b.newton_schulz(g, o)
        b.device_status()
    check_newton_schulz(g, o)


@pytest.mark.parametrize("steps,coeffs", [(1, None), (2, (1.5, -0.5, 0.0)), (12, (1.875, -1.25, 0.375)), (3, [(8.2, -22.4, 16.0), (4.0, -2.8, 0.5), (3.8, -2.6, 0.5)])])
def test_newton_schulz_steps_and_coefficients(steps, coeffs):
    g = update(200, 330, "flat", 43)
    o = torch.empty(200, 330, dtype=torch.bfloat16, device="cuda")
    with Workspace(b.workspace_bytes(b.OP_NEWTON_SCHULZ, 200, 330, 1, 1)):
        b.newton_schulz(g, o, steps=steps, coeffs=coeffs)
    check_newton_schulz(g, o, steps=steps, coeffs=coeffs)


@pytest.mark.parametrize("m,n", [(96, 200), (300, 140), (520, 520), (150, 4000)])
def test_newton_schulz_batch_strides_and_independence(m, n):
    batch, ld = 5, n + 13
    store = torch.zeros(batch, m + 2, ld, device="cuda")
    g = store[:, 1:m + 1, 5:5 + n]
    for i in range(batch):
        g[i] = update(m, n, "flat" if i % 2 else "falling", 50 + i) * 10.0 ** (i - 2)
    g[3] = 0.0
    out = torch.full((batch, m + 1, ld), 9.0, dtype=torch.bfloat16, device="cuda")
    o = out[:, :m, 1:1 + n]
    with Workspace(b.workspace_bytes(b.OP_NEWTON_SCHULZ, m, n, batch, 1)):
        b.newton_schulz(g, o)
        one = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
        for i in range(batch):
            if i == 3:
                assert bool((o[i] == 0).all())
                continue
            check_newton_schulz(g[i], o[i])
            b.newton_schulz(g[i], one)
            assert torch.equal(one, o[i])                            # bit for bit what it is alone
    assert bool((out[:, m:] == 9).all()) and bool((out[:, :, :1] == 9).all()) and bool((out[:, :, 1 + n:] == 9).all())


@pytest.mark.parametrize("m,n", [(100, 260), (260, 100)])
def test_newton_schulz_in_place_tiny_huge_and_non_finite(m, n):
    with Workspace(b.workspace_bytes(b.OP_NEWTON_SCHULZ, m, n, 1, 1)):
        g = update(m, n, "flat", 61)
        x = g.bfloat16()
        want = x.clone()
        b.newton_schulz(x, x)
        check_newton_schulz(want, x)
        o = torch.empty_like(x)
        for size in (1e36, 1e-36):                                   # squares leave the 32-bit range on either side
            b.newton_schulz(g * size, o, eps=0.0)
            check_newton_schulz(g * size, o, eps=0.0)
        b.newton_schulz(torch.zeros_like(g), o, eps=0.0)
        assert bool((o == 0).all())
        for bad in (float("inf"), float("nan")):
            h = g.clone()
            h[3, 5] = bad
            b.newton_schulz(h, o)
            assert bool(torch.isnan(o).all())


def test_one_graph_of_copies_quantisation_product_and_newton_schulz():
    m, n, k = 200, 300, 256
    x, w = torch.randn(m, k, device="cuda"), torch.randn(n, k, device="cuda")
    staged, qa, sa = torch.empty_like(x), *b.fp8_empty(m, k)
    qb, sb = b.fp8_empty(n, k, block_rows=128)
    d, o = torch.empty(m, n, device="cuda"), torch.empty(m, n, dtype=torch.bfloat16, device="cuda")

    def step():
        staged.copy_(x)                                             # a copy in front of a kernel that is launched as a dependent
        b.fp8_quantise(staged, qa, sa)
        b.fp8_quantise(w, qb, sb, block_rows=128)
        b.fp8_gemm(qa, sa, qb, sb, d)
        b.newton_schulz(d, o)

    with Workspace(max(b.workspace_bytes(b.OP_FP8_GEMM, m, n, k, 1), b.workspace_bytes(b.OP_NEWTON_SCHULZ, m, n, 1, 1))):
        step()
        want = o.clone()
        x2 = torch.randn(m, k, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)                                 # bit for bit, and again with other inputs
        x.copy_(x2)
        graph.replay()
        got = o.clone()
        step()
        b.device_status()
        assert torch.equal(o, got) and not torch.equal(got, want)


def test_newton_schulz_singular_values_and_small_workspace():
    m, n = 256, 640
    g = update(m, n, "flat", 71)
    o = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    need = b.workspace_bytes(b.OP_NEWTON_SCHULZ, m, n, 1, 1)
    with Workspace(need - 256):
        with pytest.raises(b.Gemm2mError) as err:
            b.newton_schulz(g, o)
        assert err.value.status == b.ERR_WORKSPACE
    with Workspace(need):
        b.newton_schulz(g, o, steps=12, coeffs=(1.875, -1.25, 0.375))
    s = torch.linalg.svdvals(o.double())
    assert float((s - 1).abs().max()) < 0.02                          # the cubic-order iteration converges to the polar factor


# ------------------------------------------------------------------------------------------------------ together
def test_layer_gradients_against_the_formula_and_differences():
    from examples.fp8_layer_training import Fp8Linear, workspace_for
    tokens, n_in, n_out = 200, 264, 136
    g = gen(81)
    layer = Fp8Linear(n_in, n_out, g)
    x = torch.randn(tokens, n_in, generator=g, device="cuda").bfloat16()
    dy = torch.randn(tokens, n_out, generator=g, device="cuda") * 1e-2
    ws = workspace_for([layer])
    b.set_workspace(ws)
    try:
        y = layer.forward(x)
        dx = layer.backward(dy)
        b.device_status()
    finally:
        torch.cuda.synchronize()
        b.set_workspace(None)
    w = layer.qw.double() * spread(layer.sw, 128, n_out, n_in)
    assert torch.equal(w.t(), layer.qwt.double() * spread(layer.swt, 128, n_in, n_out))
    xt = layer.qxt.double() * spread(layer.sxt, 1, n_in, tokens)
    q, s = b.fp8_empty(tokens, n_out)
    qt, st = b.fp8_empty(n_out, tokens)
    b.fp8_quantise(dy, q, s, qt, st)
    dyt = qt.double() * spread(st, 1, n_out, tokens)
    dyr = q.double() * spread(s, 1, tokens, n_out)
    # the formula on the quantised operands: 32-bit sums, one rounding
    close = lambda got, want, unit: float(torch.linalg.vector_norm(got.double() - want) / torch.linalg.vector_norm(want)) <= unit
    assert close(layer.dw, dyt @ xt.t(), 2.0 ** -16) and close(dx, dyr @ w, 2.0 ** -8)
    # differences of the loss sum(dy * (x w^T)) in 64 bits along random directions (it is linear in w and in x)
    for seed in range(3):
        v = torch.randn(n_out, n_in, generator=gen(90 + seed), device="cuda").double()
        loss = lambda step: float((dyt.t() * (xt.t() @ (w + step * v).t())).sum())
        slope = (loss(0.5) - loss(-0.5)) / 1.0
        scale = float(torch.linalg.vector_norm(layer.dw.double()) * torch.linalg.vector_norm(v))
        assert abs(slope - float((layer.dw.double() * v).sum())) <= 2.0 ** -16 * scale
    # quantisation itself: 2^-4 relative per entry of each operand at most
    assert close(y, x.double() @ layer.w.double().t(), 2 * 2.0 ** -4) and close(layer.dw, dy.double().t() @ x.double(), 2 * 2.0 ** -4)


def test_training_example_learns():
    from examples.fp8_layer_training import train
    losses = train(steps=30)
    assert all(math.isfinite(v) for v in losses) and losses[-1] < 0.5 * losses[0], losses

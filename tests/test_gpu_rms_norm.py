"""Root-mean-square norm with 8-bit outputs, and its gradients, on the GPU against plain implementations in 64 bits."""
import pytest
import torch

from paper_2609_05419_b200 import binding as b

pytestmark = pytest.mark.gpu

from gpu_util import Workspace  # noqa: E402

STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}      # half a step, relative
MAX = {b.E4M3: 448.0, b.E5M2: 57344.0}
# A row's sum of squares has positive terms, and no term goes through more than 8 x 4 additions in its thread, 5 in its warp and 32 over the
# warps; square and mean add one rounding each.  The square root halves the relative error and rounds once; H rstd W adds two.
RSTD = (71 / 2 + 2) * 2.0 ** -24
NORM = RSTD + 2 * 2.0 ** -24
LEAST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}  # half the smallest spacing of Y


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(seed, *shape):
    return torch.randn(*shape, generator=gen(seed), device="cuda")


def stream(rows, cols, dtype, seed):
    return (randn(seed, rows, cols) * torch.exp(randn(seed + 1, 1, cols)) * torch.exp(2 * randn(seed + 2, rows, 1))).to(dtype)


def plain(x, r, w, eps):
    """(H as it is stored, rstd, N) in 64 bits."""
    h = x if r is None else (x.float() + r.float()).to(x.dtype)
    rstd = 1 / torch.sqrt(h.double().square().mean(1) + eps)
    n = h.double() * rstd[:, None]
    return h, rstd, n if w is None else n * w.double()


def blocks(v):
    return -(-v // 128)


def check_form(q, s, n, fmt):
    """8-bit values and scales of blocks along the rows of n."""
    rows, cols = n.shape
    top = torch.nn.functional.pad(n.abs(), (0, -cols % 128)).view(rows, -1, 128).amax(2).clamp_min(2.0 ** -100)
    assert bool(((s.double() - top / MAX[fmt]).abs() <= (NORM + 2 * 2.0 ** -24) * top / MAX[fmt]).all())
    spread = s.double().repeat_interleave(128, 1)[:, :cols]
    rel, least = (2.0 ** -4, 2.0 ** -10) if fmt == b.E4M3 else (2.0 ** -3, 2.0 ** -17)
    other = NORM + 4 * 2.0 ** -24                                # of N, of MAX / u, of its product with N, and of s
    room = torch.maximum(rel * n.abs(), least * spread) * (1 + other) + other * n.abs()
    off = (q.double() * spread - n).abs()
    assert bool((off <= room).all()), float((off / room).max())


def outputs(rows, cols, dtype, fmt):
    q, s = b.fp8_empty(rows, cols, fmt)
    qt, st = b.fp8_empty(cols, rows, fmt)
    h, y = (torch.full((rows, cols), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    return dict(H=h, Y=y, Q=q, S=s, Qt=qt, St=st, rstd=torch.full((rows,), float("nan"), device="cuda"))


SIZES = [(1, 1), (1, 8), (1, 4096), (2, 7), (3, 129), (16, 1000), (5, 2048), (127, 128), (128, 512), (129, 513), (300, 1999), (140, 4104), (9, 8200),
         (17, 16384), (3, 20001), (2, 32768)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype,fmt", [(torch.bfloat16, b.E4M3), (torch.float32, b.E4M3), (torch.float16, b.E5M2)])
@pytest.mark.parametrize("residual", [False, True])
def test_norm_against_64_bits(rows, cols, dtype, fmt, residual):
    x = stream(rows, cols, dtype, 1)
    r = stream(rows, cols, dtype, 5) if residual else None
    w = 1 + 0.3 * randn(9, cols)
    out = outputs(rows, cols, dtype, fmt)
    b.rms_norm(x, w, R=r, eps=1e-5, **out)
    h, rstd, n = plain(x, r, w, 1e-5)
    assert torch.equal(out["H"], h)
    assert bool(((out["rstd"].double() - rstd).abs() <= RSTD * rstd).all())
    assert bool(((out["Y"].double() - n).abs() <= (STEP[dtype] * (1 + NORM) + NORM) * n.abs() + LEAST[dtype]).all())
    check_form(out["Q"], out["S"], n, fmt)
    check_form(out["Qt"], out["St"], n.t(), fmt)


@pytest.mark.parametrize("rows,cols", [(1, 1), (130, 700), (257, 4096)])
@pytest.mark.parametrize("fmt", [b.E4M3, b.E5M2])
def test_eight_bit_forms_are_those_of_the_quantiser(rows, cols, fmt):
    x, w = stream(rows, cols, torch.bfloat16, 11), 1 + 0.3 * randn(13, cols)
    out = outputs(rows, cols, torch.float32, fmt)
    b.rms_norm(x.float(), w, **out)
    q, s = b.fp8_empty(rows, cols, fmt)
    qt, st = b.fp8_empty(cols, rows, fmt)
    b.fp8_quantise(out["Y"], q, s, qt, st)                        # Y in 32 bits is N itself
    same = outputs(rows, cols, torch.bfloat16, fmt)
    b.rms_norm(x, w, **same)                                      # and the type of the stream changes nothing
    for got in (out, same):
        assert torch.equal(got["Q"].view(torch.uint8), q.view(torch.uint8)) and torch.equal(got["S"], s)
        assert torch.equal(got["Qt"].view(torch.uint8), qt.view(torch.uint8)) and torch.equal(got["St"], st)
    assert torch.equal(out["Y"].bfloat16(), same["Y"])


def test_every_output_alone_and_none_of_the_others():
    rows, cols = 200, 333
    x, r, w = stream(rows, cols, torch.float32, 21), stream(rows, cols, torch.float32, 25), randn(29, cols)
    want = outputs(rows, cols, torch.float32, b.E4M3)
    b.rms_norm(x, w, R=r, **want)
    for names in (("H",), ("Y",), ("Q", "S"), ("Qt", "St"), ("rstd",), ("H", "Qt", "St"), ("Q", "S", "rstd")):
        got = outputs(rows, cols, torch.float32, b.E4M3)
        with Workspace(b.workspace_bytes(b.OP_RMS_NORM, rows, cols, 1, 1)) as ws:
            ws.buf[4096:].fill_(0xff)
            b.rms_norm(x, w, R=r, **{name: got[name] for name in names})
        for name in names:
            assert torch.equal(got[name].view(torch.uint8) if name[0] == "Q" else got[name], want[name].view(torch.uint8) if name[0] == "Q" else want[name]), (names, name)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strided_unaligned_matrices_and_nothing_beside_them(dtype):
    rows, cols, ld = 130, 333, 352
    mat = lambda seed, skip: torch.cat([randn(seed, skip), stream(rows, ld, torch.float32, seed).flatten()]).to(dtype)[skip:].view(rows, ld)[:, 2:2 + cols]
    x, r = mat(31, 1), mat(35, 3)
    w = torch.cat([randn(39, 1), 1 + 0.3 * randn(40, cols)])[1:]
    assert x.data_ptr() % 16 and w.data_ptr() % 16
    big = {name: torch.full((rows + 2, ld), 7.0, device="cuda").to(dtype) for name in ("H", "Y")}
    bytes8 = {name: torch.full((shape[0] + 1, 400), 77, dtype=torch.uint8, device="cuda") for name, shape in (("Q", (rows, cols)), ("Qt", (cols, rows)))}
    floats = {name: torch.full((shape[0] + 1, 400), 7.0, device="cuda") for name, shape in (("S", (blocks(cols), rows)), ("St", (blocks(rows), cols)))}
    out = {name: t[1:1 + rows, 5:5 + cols] for name, t in big.items()}
    out.update(Q=bytes8["Q"].view(torch.float8_e4m3fn)[:rows, :cols], Qt=bytes8["Qt"].view(torch.float8_e4m3fn)[:cols, :rows],
               S=floats["S"][:blocks(cols), :rows].t(), St=floats["St"][:blocks(rows), :cols].t(), rstd=torch.zeros(rows, device="cuda"))
    b.rms_norm(x, w, R=r, **out)
    want = outputs(rows, cols, dtype, b.E4M3)
    b.rms_norm(x.contiguous(), w.clone(), R=r.contiguous(), **want)
    for name, t in out.items():
        assert torch.equal(t.view(torch.uint8) if name[0] == "Q" else t, want[name].view(torch.uint8) if name[0] == "Q" else want[name]), name
    for t in big.values():
        assert bool((t[0] == 7).all()) and bool((t[-1] == 7).all()) and bool((t[:, :5] == 7).all()) and bool((t[:, 5 + cols:] == 7).all())
    for t, (rr, cc) in ((bytes8["Q"], (rows, cols)), (bytes8["Qt"], (cols, rows))):
        assert bool((t[rr:] == 77).all()) and bool((t[:, cc:] == 77).all())
    for t, (rr, cc) in ((floats["S"], (blocks(cols), rows)), (floats["St"], (blocks(rows), cols))):
        assert bool((t[rr:] == 7).all()) and bool((t[:, cc:] == 7).all())


@pytest.mark.parametrize("cols", [40, 4096])
def test_stream_in_place_of_either_summand(cols):
    x, r = stream(20, cols, torch.bfloat16, 41), stream(20, cols, torch.bfloat16, 45)
    want = outputs(20, cols, torch.bfloat16, b.E4M3)
    b.rms_norm(x, R=r, **want)
    for which in ("x", "r"):
        a, c = x.clone(), r.clone()
        out = outputs(20, cols, torch.bfloat16, b.E4M3)
        out["H"] = a if which == "x" else c
        b.rms_norm(a, R=c, **out)
        for name in ("H", "Y", "S", "St", "rstd"):
            assert torch.equal(out[name], want[name]), name
        assert torch.equal(out["Qt"].view(torch.uint8), want["Qt"].view(torch.uint8))


def test_zero_rows_extremes_and_non_finite_entries():
    rows, cols = 140, 300
    x = stream(rows, cols, torch.float32, 51)
    x[0] = 0
    x[1, 7] = float("nan")
    x[2, 200] = float("inf")
    x[3] = 1e-30                                                  # squares underflow: eps alone is left
    x[4] = 1e18                                                   # squares near the end of the range
    out = outputs(rows, cols, torch.float32, b.E4M3)
    b.rms_norm(x, eps=1e-6, **out)
    assert bool((out["Y"][0] == 0).all()) and bool((out["Q"][0].float() == 0).all()) and bool((out["S"][0] == torch.tensor(2.0 ** -100) / 448).all())
    assert bool(torch.isnan(out["Y"][1]).all()) and bool(torch.isnan(out["S"][1]).all())
    assert bool((out["rstd"][2] == 0)) and torch.isnan(out["Y"][2, 200]) and int(torch.isnan(out["Y"][2]).sum()) == 1
    assert torch.isnan(out["S"][2]).tolist() == [False, True, False]
    assert bool(torch.isnan(out["St"][:, 0]).all())              # the NaN row is in the first block of every column
    assert not bool(torch.isnan(out["St"][:, 1]).any())
    n = plain(x, None, None, 1e-6)[2]
    fine = [3, 4] + list(range(5, rows))
    assert bool(((out["Y"][fine].double() - n[fine]).abs() <= (NORM + 2.0 ** -24) * n[fine].abs()).all())
    y = torch.zeros_like(x)
    b.rms_norm(x[:1], eps=0.0, Y=y[:1])                           # 0 / 0
    assert bool(torch.isnan(y[0]).all())


def test_no_rows_and_no_columns():
    for rows, cols in ((0, 40), (40, 0), (0, 0)):
        out = outputs(rows, cols, torch.bfloat16, b.E4M3)
        x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
        b.rms_norm(x, torch.ones(cols, device="cuda"), R=x, **out)
        dw = torch.full((cols,), 3.0, device="cuda")
        b.rms_norm_backward(x, x, None, out["rstd"], torch.empty_like(x), dW=dw, add=True)
        assert bool((dw == 3).all())
        b.rms_norm_backward(x, x, None, out["rstd"], torch.empty_like(x), dW=dw)
        assert bool((dw == 0).all())


# -------------------------------------------------------------------------------------------------------------- gradients
def plain_backward(dy, h, w, rstd, dr):
    dy, h, rstd = dy.double(), h.double(), rstd.double()[:, None]
    n = h * rstd
    dn = dy if w is None else dy * w.double()
    cols = h.shape[1]
    dx = rstd * (dn - n * (dn * n).sum(1, keepdim=True) / cols)
    # magnitudes, for the error bound
    size = rstd.abs() * (dn.abs() + n.abs() * (dn * n).abs().sum(1, keepdim=True) / cols)
    if dr is not None:
        dx, size = dx + dr.double(), size + dr.double().abs()
    return dx, size, (dy * n).sum(0), (dy * n).abs().sum(0)


def check_backward(rows, cols, dtype, residual, weights, w_type=torch.float32, add=False, seed=61):
    h, dy = stream(rows, cols, dtype, seed), (1e-3 * stream(rows, cols, torch.float32, seed + 3)).to(dtype)
    dr = (1e-3 * stream(rows, cols, torch.float32, seed + 6)).to(dtype) if residual else None
    w = (1 + 0.3 * randn(seed + 9, cols)).to(w_type) if weights else None
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-6)
    dx = torch.full((rows, cols), float("nan"), dtype=dtype, device="cuda")
    start = randn(seed + 10, cols)
    dw = start.clone() if add else torch.full((cols,), float("nan"), device="cuda")
    with Workspace(b.workspace_bytes(b.OP_RMS_NORM_BACKWARD, rows, cols, 1, 1)) as ws:
        ws.buf[4096:].fill_(0xff)                                 # (NaN)
        b.rms_norm_backward(dy, h, w, rstd, dx, dR=dr, dW=dw, add=add)
    want, size, want_w, size_w = plain_backward(dy, h, w, rstd, dr)
    # a mean: 8 x 4 + 5 + 32 additions, four roundings of a term; six roundings around it; one to the type
    off, room = (dx.double() - want).abs(), 80 * 2.0 ** -24 * size + STEP[dtype] * want.abs() * 1.001 + LEAST[dtype]
    assert bool((off <= room).all()), float((off / room).max())
    # a column: fewer than rows / 148 + 1 + 148 x 32 / 32 + 7 additions whatever the width, two roundings of a term
    off, room = (dw.double() - want_w - (start.double() if add else 0)).abs(), (rows + 160) * 2.0 ** -24 * size_w + 2.0 ** -23 * (start.double().abs() + size_w if add else 0)
    assert bool((off <= room).all()), float((off / room).max())
    return dx, dw


@pytest.mark.parametrize("rows,cols", SIZES + [(2000, 96), (700, 2048)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.float16])
@pytest.mark.parametrize("residual", [False, True])
def test_gradients_against_64_bits(rows, cols, dtype, residual):
    check_backward(rows, cols, dtype, residual, True)


@pytest.mark.parametrize("rows,cols", [(300, 8200), (333, 12289), (150, 24584), (111, 24833), (80, 32767)])      # rows shared by two to four blocks, several to a block
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients_of_many_long_rows(rows, cols, dtype):
    check_backward(rows, cols, dtype, True, True, add=True)


@pytest.mark.parametrize("w_type", [torch.float32, torch.float16, torch.bfloat16, None])
def test_gradients_with_weights_of_any_type_added_and_the_same_every_time(w_type):
    first = check_backward(300, 1000, torch.bfloat16, True, w_type is not None, w_type, add=True)
    again = check_backward(300, 1000, torch.bfloat16, True, w_type is not None, w_type, add=True)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("w_type", [torch.float16, torch.bfloat16])
def test_norm_with_weights_of_other_types(w_type):
    x, w = stream(30, 1000, torch.float32, 81), (1 + 0.3 * randn(83, 1000)).to(w_type)
    y, z = torch.empty_like(x), torch.empty_like(x)
    b.rms_norm(x, w, Y=y)
    b.rms_norm(x, w.float(), Y=z)
    assert torch.equal(y, z)


def test_gradients_against_differences():
    rows, cols = 6, 200
    x, w, dy = randn(91, rows, cols), 1 + 0.3 * randn(92, cols), randn(93, rows, cols)
    rstd, dx, dw, y = torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty_like(w), torch.empty_like(x)
    with Workspace(b.workspace_bytes(b.OP_RMS_NORM_BACKWARD, rows, cols, 1, 1)):
        b.rms_norm(x, w, rstd=rstd)
        b.rms_norm_backward(dy, x, w, rstd, dx, dW=dw)
    value = lambda x, w: float((plain(x, None, w, 1e-6)[2] * dy.double()).sum())
    step = 1e-4
    for v, (at, grad, of) in enumerate(((randn(94, rows, cols), dx, "x"), (randn(95, cols), dw, "w"))):
        move = lambda sign: value(x.double() + sign * step * at if of == "x" else x, w.double() + sign * step * at if of == "w" else w)
        slope = (move(1) - move(-1)) / (2 * step)
        # second differences cancel: step^2 times a third derivative of order 1 per entry, and the 32-bit gradients
        room = (step ** 2 * 10 + 100 * 2.0 ** -24) * float((grad.double() * at).abs().sum() + 1)
        assert abs(slope - float((grad.double() * at).sum())) <= room, v


def test_gradient_in_place_of_each_input():
    rows, cols = 50, 600
    h, dy, dr, w = stream(rows, cols, torch.bfloat16, 101), stream(rows, cols, torch.bfloat16, 104), stream(rows, cols, torch.bfloat16, 107), randn(110, cols)
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-6)
    want = torch.empty_like(h)
    b.rms_norm_backward(dy, h, w, rstd, want, dR=dr)
    for which in range(3):
        t = [dy.clone(), h.clone(), dr.clone()]
        b.rms_norm_backward(t[0], t[1], w, rstd, t[which], dR=t[2])
        assert torch.equal(t[which], want)


def test_gradients_of_strided_unaligned_matrices_and_nothing_beside_them():
    rows, cols, ld = 70, 333, 352
    mat = lambda seed, skip: torch.cat([randn(seed, skip), stream(rows, ld, torch.float32, seed).flatten()]).bfloat16()[skip:].view(rows, ld)[:, 2:2 + cols]
    dy, h, dr, w = mat(121, 1), mat(124, 2), mat(127, 3), randn(130, cols + 1)[1:]
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-6)
    big = torch.full((rows + 2, ld), 7.0, dtype=torch.bfloat16, device="cuda")
    want = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    b.rms_norm_backward(dy, h, w, rstd, big[1:-1, 5:5 + cols], dR=dr)
    b.rms_norm_backward(dy.contiguous(), h.contiguous(), w.clone(), rstd, want, dR=dr.contiguous())
    assert torch.equal(big[1:-1, 5:5 + cols], want)
    assert bool((big[0] == 7).all()) and bool((big[-1] == 7).all()) and bool((big[:, :5] == 7).all()) and bool((big[:, 5 + cols:] == 7).all())


def test_row_offsets_beyond_32_bits():
    ld = 2 ** 30 + 8                                              # elements from one row to the next: 6 GB for three rows of 16 bits
    store = torch.empty(2 * ld + 64, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(store, (3, 64), (ld, 1))
    x.copy_(randn(141, 3, 64))
    want, got = torch.empty(3, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(3, 64, dtype=torch.bfloat16, device="cuda")
    b.rms_norm(x, Y=got)
    b.rms_norm(x.contiguous(), Y=want)
    assert torch.equal(got, want)
    rstd = torch.ones(3, device="cuda")
    b.rms_norm_backward(got, x, None, rstd, got)
    b.rms_norm_backward(want, x.contiguous(), None, rstd, want)
    assert torch.equal(got, want)


def test_another_stream_and_a_captured_graph():
    rows, cols = 300, 1024
    x, r, w = stream(rows, cols, torch.bfloat16, 151), stream(rows, cols, torch.bfloat16, 154), randn(157, cols)
    dy, dw, dx = stream(rows, cols, torch.bfloat16, 158), torch.empty(cols, device="cuda"), torch.empty_like(x)
    out = outputs(rows, cols, torch.bfloat16, b.E4M3)

    def step():
        b.rms_norm(x, w, R=r, **out)
        b.rms_norm_backward(dy, out["H"], w, out["rstd"], dx, dR=r, dW=dw)

    with Workspace(b.workspace_bytes(b.OP_RMS_NORM_BACKWARD, rows, cols, 1, 1)):
        step()
        want = {name: t.clone() for name, t in out.items()}, dx.clone(), dw.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for t in (*out.values(), dx, dw):
            t.view(torch.uint8).zero_() if t.dtype == torch.float8_e4m3fn else t.zero_()
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        for name, t in out.items():
            same = torch.equal(t.view(torch.uint8), want[0][name].view(torch.uint8)) if name[0] == "Q" else torch.equal(t, want[0][name])
            assert same, name
        assert torch.equal(dx, want[1]) and torch.equal(dw, want[2])
        del graph

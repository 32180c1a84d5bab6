"""Common norm of many tensors and their clipping on the GPU against a plain implementation in 64 bits."""
import math

import pytest
import torch

from paper_2609_05419_b200 import binding as b

pytestmark = pytest.mark.gpu

from gpu_util import Workspace  # noqa: E402

STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}      # half a step, relative
LEAST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}  # half the smallest spacing, or more
# A sum of 8 squares in 32 bits: 8 roundings, and what underflows 2^-23; the root halves it; rounded once
NORM = (10 / 2 + 1) * 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(seed, *shape, dtype=torch.float32, size=1.0):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * size).to(dtype)


def workspace(count):
    return Workspace(b.workspace_bytes(b.OP_CLIP_GRADIENTS, count, 1, 1, 1))


def plain(grads, limit, eps=1e-6):
    norm = math.sqrt(math.fsum(float(t.double().square().sum()) for t in grads))
    factor = 1.0 if limit >= norm + eps else limit / (norm + eps)
    return norm, factor


def check(grads, limit, out=None, eps=1e-6):
    """Runs the call on a workspace of NaN, in place if out is None, and compares with 64 bits."""
    norm, factor = plain(grads, limit, eps)
    before = [t.clone() for t in grads]
    got = torch.full((), float("nan"), device="cuda")
    with workspace(len(grads)) as ws:
        ws.buf[4096:].fill_(0xff)
        b.clip_gradients(grads, limit, out=out, norm=got, eps=eps)
    assert abs(float(got) - norm) <= NORM * norm, (float(got), norm)
    for was, now in zip(before, grads if out is None else out):
        want = was.double() * factor
        room = ((NORM + 3 * 2.0 ** -24 + STEP[was.dtype] * 1.001) * want.abs() + LEAST[was.dtype]) * (factor != 1.0)
        assert bool(((now.double() - want).abs() <= room).all())
    if out is not None:
        assert all(torch.equal(was, t) for was, t in zip(before, grads))
    return got


SHAPES = [[(1,)], [(7,), (1, 1), (3, 5, 2)], [(200, 200), (300, 200), (200,)], [(8192,), (8193,), (8191,), (16384,)], [(1000, 1000), (), (17,), (3, 40000)],
          [(40,)] * 63, [(40,)] * 64, [(3, 333)] * 65, [(5,)] * 512, [(100,)] * 513, [(33,)] * 1500, [(4000, 4099)]]


@pytest.mark.parametrize("shapes", SHAPES, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("limit", [1.0, 1e30])
@pytest.mark.parametrize("in_place", [True, False])
def test_clip_against_64_bits(shapes, limit, in_place):
    grads = [randn(i, *s, dtype=TYPES[i % 3], size=0.1 + i % 5) for i, s in enumerate(shapes)]
    check(grads, limit, None if in_place else [torch.full_like(t, float("nan")) for t in grads])


@pytest.mark.parametrize("size", [1e-44, 1e-38, 1e-30, 1e-22, 1e-16, 1e-14, 1e14, 1e18, 1e20, 1e30, 1e36])       # (1e36 sqrt(20030) = 1.4e38 is still a 32-bit number)
def test_entries_whose_squares_leave_the_32_bit_range(size):
    for dtype in (torch.float32, torch.bfloat16):
        grads = [randn(1, 500, 40, dtype=dtype, size=size), randn(2, 30, dtype=dtype, size=size)]
        # (the norm itself is a 32-bit number: where it is subnormal its spacing is 2^-149)
        norm, factor = plain(grads, 1.0, 0.0)
        got = torch.empty(1, device="cuda")
        with workspace(2):
            b.clip_gradients(grads, math.inf, norm=got)
        assert abs(float(got) - norm) <= NORM * norm + 2.0 ** -149
    grads = [randn(1, 500, size=size), randn(2, 300), torch.zeros(5000, device="cuda")]     # beside ordinary ones
    check(grads, 1.0)


def test_rows_of_zeros_and_all_zeros():
    g = randn(5, 3000, 100)
    g[torch.rand(3000, device="cuda") < 0.8] = 0
    check([g], 1.0)
    z = [torch.zeros(100, 100, device="cuda")]
    assert float(check(z, 1.0)) == 0 and float(check(z, 0.0)) == 0
    g = [randn(6, 100)]
    check(g, 0.0)
    assert bool((g[0] == 0).all())


@pytest.mark.parametrize("value,everywhere", [(float("nan"), True), (float("inf"), False), (float("-inf"), False)])
@pytest.mark.parametrize("dtype", TYPES)
def test_non_finite_gradients(value, everywhere, dtype):
    grads = [randn(7, 3000, dtype=dtype), randn(8, 20)]
    grads[0][1234] = value
    norm = torch.empty((), device="cuda")
    with workspace(2):
        b.clip_gradients(grads, 1.0, norm=norm)
    if everywhere:                                                # a NaN norm: every entry
        assert bool(torch.isnan(norm)) and all(bool(torch.isnan(t).all()) for t in grads)
    else:                                                         # an infinite one: factor 0
        assert float(norm) == float("inf") and bool(torch.isnan(grads[0][1234])) and int(torch.isnan(grads[0]).sum()) == 1
        assert bool((grads[0].nan_to_num() == 0).all()) and bool((grads[1] == 0).all())


def test_norm_alone_leaves_the_gradients():
    grads = [randn(9, 1000, 30, size=100), randn(10, 77, dtype=torch.bfloat16)]
    before = [t.clone() for t in grads]
    norm = torch.empty(1, device="cuda")
    with workspace(2):
        b.clip_gradients(grads, math.inf, norm=norm)
        assert all(torch.equal(x, y) for x, y in zip(before, grads))
        assert abs(float(norm) - plain(grads, 1)[0]) <= NORM * float(norm)
        out = [torch.empty_like(t) for t in grads]
        b.clip_gradients(grads, math.inf, out=out)
        assert all(torch.equal(x, y) for x, y in zip(before, out))
        b.clip_gradients(grads, 1.0)                              # and the clipping without the norm
        assert abs(plain(grads, 1)[0] - 1) < 1e-2


@pytest.mark.parametrize("rows,cols,ld,skip", [(300, 200, 256, 0), (300, 200, 256, 1), (300, 199, 256, 8), (7, 5000, 5001, 0), (130, 64, 72, 8), (2, 1, 9, 3)])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_apart_unaligned_bases_and_nothing_beside_them(rows, cols, ld, skip, dtype):
    store = randn(11, rows * ld + skip, dtype=dtype)
    g = torch.as_strided(store, (rows, cols), (ld, 1), skip)
    before = store.clone()
    for to_dense in (True, False):
        big = torch.full((rows, ld + 8), 7.0, device="cuda").to(dtype)
        out = torch.full((rows, cols), 7.0, device="cuda").to(dtype) if to_dense else big[:, 3:3 + cols]
        check([g], 1.0, [out])
        assert torch.equal(store, before) and (to_dense or (bool((big[:, :3] == 7).all()) and bool((big[:, 3 + cols:] == 7).all())))
    check([g, randn(12, 10)], 1.0)                                # in place: the gaps stay
    inside = torch.zeros_like(store, dtype=torch.bool)
    torch.as_strided(inside, (rows, cols), (ld, 1), skip).fill_(True)
    assert torch.equal(store[~inside], before[~inside])


def test_transposed_gradients_and_views_side_by_side():
    whole = randn(13, 300, 640)
    grads = [randn(14, 200, 100).t(), whole[:, :200], whole[:, 200:328], whole[:, 328:], randn(15, 4, 5, 6).permute(2, 0, 1)]
    check(grads, 1.0)
    check(grads, 0.5, [torch.empty_like(t) for t in grads])


def test_the_same_every_time_whatever_the_workspace_held():
    grads = [randn(i, 999, 77, dtype=TYPES[i % 3]) for i in range(100)]
    out = [[torch.empty_like(t) for t in grads] for _ in range(2)]
    first = check(grads, 1.0, out[0])
    with workspace(600):
        norm = torch.empty((), device="cuda")
        b.clip_gradients(grads, 1.0, out=out[1], norm=norm)
    assert torch.equal(first, norm) and all(torch.equal(x, y) for x, y in zip(*out))


def test_no_tensors_and_empty_tensors():
    norm = torch.full((), float("nan"), device="cuda")
    with workspace(3):
        b.clip_gradients([], 1.0, norm=norm)
        assert float(norm) == 0
        norm.fill_(float("nan"))
        b.clip_gradients([torch.zeros(0, device="cuda"), torch.zeros(5, 0, device="cuda")], 1.0, norm=norm)
        assert float(norm) == 0
        g = [torch.zeros(0, 4, device="cuda"), torch.full((4,), 2.0, device="cuda"), torch.zeros(0, device="cuda")]
        b.clip_gradients(g, 1.0, norm=norm, eps=0.0)
        assert float(norm) == 4 and bool((g[1] == 0.5).all())


def test_one_tensor_of_more_than_two_to_the_31_entries():
    n = 2 ** 31 + 12345
    g = torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    g[-1] = 64.0
    norm = torch.empty((), device="cuda")
    with workspace(1):
        b.clip_gradients([g], 1.0, norm=norm, eps=0.0)
    want = math.sqrt((n - 1) * 2.0 ** -20 + 4096)
    assert abs(float(norm) - want) <= NORM * want
    step = torch.tensor([64.0, 2.0 ** -10]).double() / want
    assert abs(float(g[-1]) - step[0]) <= 2.0 ** -8 * 1.01 * step[0] and abs(float(g[2 ** 31]) - step[1]) <= 2.0 ** -8 * 1.01 * step[1]
    assert bool((g[:-1] == g[0]).all())


def test_another_stream_and_a_captured_graph():
    grads = [randn(i, 400, 50, dtype=TYPES[i % 3]) for i in range(70)]
    out, norm = [torch.empty_like(t) for t in grads], torch.empty((), device="cuda")
    with workspace(70):
        b.clip_gradients(grads, 1.0, out=out, norm=norm)
        want = [t.clone() for t in out], norm.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.clip_gradients(grads, 1.0, out=out, norm=norm)
        for t in (*out, norm):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, want[1]) and all(torch.equal(x, y) for x, y in zip(out, want[0]))
        grads[3].mul_(2)                                          # a replay reads what is there then
        graph.replay()
        assert abs(float(norm) - plain(grads, 1)[0]) <= NORM * float(norm)
        del graph

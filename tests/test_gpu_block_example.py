"""The residual blocks of the example: norm, products, their gradients, clipping and adapters one after the other, against the formulas in 64 bits on the 8-bit
operands that were formed on the way, and in one captured graph."""
import math

import pytest
import torch

from paper_2609_05419_b200 import binding as b

pytestmark = pytest.mark.gpu

from test_gpu_layer_ops import gen, spread  # noqa: E402


def far(got, want):
    """Distance relative to the norm."""
    return float(torch.linalg.vector_norm(got.double() - want) / torch.linalg.vector_norm(want))


def values(form, block, rows, cols):
    q, s = form
    return q.double() * spread(s, block, rows, cols)


@pytest.fixture
def stack():
    from examples.fp8_block_training import Stack, make_adapters
    g = gen(1)
    tokens, width, inner = 200, 264, 392
    s = Stack(1, width, inner, g)
    s.blocks[0].norm.w.add_(0.2 * torch.randn(width, generator=g, device="cuda"))
    s.adapters = make_adapters(1, 3, 8, width, inner, g)
    s.x, s.r, s.dh = ((torch.randn(tokens, width, generator=g, device="cuda") * size).bfloat16() for size in (2.0, 1.0, 0.01))
    s.index = torch.randint(-1, 3, (tokens,), generator=g, device="cuda").to(torch.int32)
    s.ws = s.workspace(tokens, 8, 3)
    b.set_workspace(s.ws)
    yield s
    torch.cuda.synchronize()
    b.set_workspace(None)


def test_block_and_its_gradients(stack):
    block, x, r, dh = stack.blocks[0], stack.x, stack.r, stack.dh
    (tokens, width), inner = x.shape, block.up.w.shape[0]
    h, summand = block.forward(x, r)
    dx = block.backward(dh)
    b.device_status()
    assert torch.equal(h, (x.float() + r.float()).bfloat16())
    # the 8-bit operands, as they were formed
    rstd = 1 / torch.sqrt(h.double().square().mean(1, keepdim=True) + 1e-6)
    n = h.double() * rstd
    q, s = b.fp8_empty(tokens, width)
    b.rms_norm(x, block.norm.w, R=r, Q=q, S=s)
    wu, wd = values((block.up.qw, block.up.sw), 128, inner, width), values((block.down.qw, block.down.sw), 128, width, inner)
    ntrans, ftrans = values((block.up.qxt, block.up.sxt), 1, width, tokens), values((block.down.qxt, block.down.sxt), 1, inner, tokens)
    # an 8-bit value is off by 2^-4 of itself at most (its subnormals by less of the block's largest entry); the norm itself by 40 x 2^-24
    norm = n * block.norm.w.double()
    assert far(q.double() * spread(s, 1, tokens, width), norm) <= 2.0 ** -4 and far(ntrans.t(), norm) <= 2.0 ** -4
    f = values((q, s), 1, tokens, width) @ wu.t()
    # F is rounded to bf16, then quantised along its columns: 2^-8 and 2^-4
    assert far(ftrans.t(), f.clamp_min(0)) <= 2.0 ** -4 + 2.0 ** -7
    def quantised(t):
        rows, cols = t.shape
        forms = b.fp8_empty(rows, cols), b.fp8_empty(cols, rows)
        b.fp8_quantise(t, *forms[0], *forms[1])
        return values(forms[0], 1, rows, cols), values(forms[1], 1, cols, rows)
    dhr, dht = quantised(dh)
    assert far(block.down.dw, dht @ ftrans.t()) <= 2.0 ** -16                       # 32-bit sums
    df = torch.where(block.active, (dhr @ wd).bfloat16(), torch.zeros(1, dtype=torch.bfloat16, device="cuda"))
    dfr, dft = quantised(df)
    # df was rounded once from a 32-bit sum, here from a 64-bit one: neighbours where it was near a border, each 2^-8 at most; so for what follows from it
    assert far(block.up.dw, dft @ ntrans.t()) <= 2.0 ** -7
    dn = (dfr @ wu).bfloat16().double()
    dnw = dn * block.norm.w.double()
    want = rstd * (dnw - n * (dnw * n).mean(1, keepdim=True)) + dh.double()
    assert far(dx, want) <= 2.0 ** -7 and far(block.norm.dw, (dn * n).sum(0)) <= 2.0 ** -7


def test_norm_and_residual_gradients_against_differences(stack):
    """The block's norm with its residual path, by itself (no quantised product between): loss = sum(dn * N) + sum(dh * H)."""
    block, x, r, dh = stack.blocks[0], stack.x, stack.r, stack.dh
    g = gen(5)
    dn = (torch.randn(x.shape, generator=g, device="cuda") * 0.01).bfloat16()
    h, _, _ = block.norm.forward(x, r)
    dx = block.norm.backward(dn, dh).double()
    for seed in range(3):
        v = torch.randn(x.shape, generator=gen(10 + seed), device="cuda").double()

        def loss(step):
            t = h.double() + step * v
            return float((dn.double() * t / torch.sqrt(t.square().mean(1, keepdim=True) + 1e-6) * block.norm.w.double()).sum() + (dh.double() * t).sum())

        slope = (loss(1e-4) - loss(-1e-4)) / 2e-4
        # dx is rounded to bf16: 2^-8 of it; differences: 1e-8 of third derivatives of order 1
        assert abs(slope - float((dx * v).sum())) <= (2.0 ** -8 + 1e-6) * float(torch.linalg.vector_norm(dx) * torch.linalg.vector_norm(v))


def test_clipping_behind_a_backward_pass(stack):
    block = stack.blocks[0]
    block.forward(stack.x, stack.r)
    block.backward(stack.dh)
    before = [t.clone() for t in stack.gradients()]
    size = math.sqrt(sum(float(t.double().square().sum()) for t in before))
    norm = torch.empty((), device="cuda")
    b.clip_gradients(stack.gradients(), 0.5 * size, norm=norm)
    assert abs(float(norm) - size) <= 6 * 2.0 ** -24 * size
    for was, now in zip(before, stack.gradients()):
        assert bool(((now.double() - 0.5 * was.double() * size / (size + 1e-6)).abs() <= 9 * 2.0 ** -24 * was.double().abs() + 2.0 ** -149).all())


def test_serving_adds_each_tokens_adapter(stack):
    block, x, r, index = stack.blocks[0], stack.x, stack.r, stack.index
    (tokens, width), inner = x.shape, block.up.w.shape[0]
    a, w, scales = stack.adapters[0]
    h, _ = block.serve(x, r, stack.adapters[0], index)
    b.device_status()
    n = torch.empty_like(x)
    q, s = b.fp8_empty(tokens, width)
    b.rms_norm(x, block.norm.w, R=r, Y=n, Q=q, S=s)
    f = torch.empty(tokens, inner, dtype=torch.bfloat16, device="cuda")
    b.fp8_gemm(q, s, block.up.qw, block.up.sw, f)
    want = f.double()
    for i in range(3):
        rows = (index == i).nonzero()[:, 0]
        want[rows] += float(scales[i]) * (n[rows].double() @ a[i].double().t()) @ w[i].double().t()
    # what the second product got: F, rounded to bf16 once more, its positive part in 8 bits along the columns
    got = values((block.down.qxt, block.down.sxt), 1, inner, tokens).t()
    assert far(got, want.clamp_min(0)) <= 2.0 ** -4 + 2.0 ** -7


def test_a_step_captured_into_a_graph_gives_what_it_gives_outside(stack):
    block = stack.blocks[0]
    norm = torch.empty((), device="cuda")
    outputs = {}

    def step():
        for t in stack.gradients():
            t.zero_()
        outputs["h"], outputs["summand"] = block.forward(stack.x, stack.r)
        outputs["dx"] = block.backward(stack.dh)
        b.clip_gradients(stack.gradients(), 0.1, norm=norm)
        outputs["served"] = block.serve(stack.x, stack.r, stack.adapters[0], stack.index)[1]

    step()
    want = {name: t.clone() for name, t in outputs.items()}, [t.clone() for t in stack.gradients()], norm.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(2):
        for t in outputs.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(outputs[name], t) for name, t in want[0].items())
        assert all(torch.equal(x, y) for x, y in zip(stack.gradients(), want[1])) and torch.equal(norm, want[2])
    del graph


def test_example_runs():
    from examples.fp8_block_training import train
    losses, norms, served = train(steps=6)
    assert all(math.isfinite(v) for v in losses + norms) and all(v > 0 for v in norms) and bool(torch.isfinite(served).all())

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

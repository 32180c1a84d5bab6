"""Layer operators on the GPU where they can go wrong: sizes of zero, scales of every size, coefficients and numbers of steps, workspaces
that hold anything."""
import pytest
import torch

from paper_2609_05419_b200 import binding as b

pytestmark = pytest.mark.gpu

from gpu_util import Workspace  # noqa: E402
from test_gpu_layer_ops import gen, operand, plain_newton_schulz, spread  # noqa: E402


# ------------------------------------------------------------------------------------------------------------ sizes of zero
def test_a_batch_without_tokens():
    n_in, n_out = 40, 24
    x, dy = torch.zeros(0, n_in, device="cuda"), torch.zeros(0, n_out, device="cuda")
    forms = {}
    for name, t, cols in (("x", x, n_in), ("dy", dy, n_out)):
        q, s = b.fp8_empty(0, cols)
        qt, st = b.fp8_empty(cols, 0)
        b.fp8_quantise(t, q, s, qt, st)
        forms[name] = q, s, qt, st
    w, sw = b.fp8_empty(n_out, n_in, block_rows=128)
    b.fp8_quantise(torch.ones(n_out, n_in, device="cuda"), w, sw, block_rows=128)
    with Workspace(b.workspace_bytes(b.OP_FP8_GEMM, n_out, n_in, 0, 1)):
        b.fp8_gemm(*forms["x"][:2], w, sw, torch.empty(0, n_out, device="cuda"))
        dw = torch.full((n_out, n_in), 3.0, device="cuda")
        b.fp8_gemm(*forms["dy"][2:], *forms["x"][2:], dw, C=dw, b_block=1)          # the sum over other batches stays
        assert bool((dw == 3).all())
        b.fp8_gemm(*forms["dy"][2:], *forms["x"][2:], dw, b_block=1)                # nothing added: zero
        assert bool((dw == 0).all())
        b.device_status()

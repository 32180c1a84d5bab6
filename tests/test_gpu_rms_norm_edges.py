"""Accuracy of the norm's row sums and the widths between the tested ones, on the GPU against plain implementations in 64 bits."""
import pytest
import torch

from paper_2609_05419_b200 import binding as b

pytestmark = pytest.mark.gpu

from test_gpu_rms_norm import plain, stream  # noqa: E402


@pytest.mark.parametrize("rows,cols", [(4000, 4096), (4000, 1999), (200, 4000), (3000, 8000)])
def test_error_of_rstd_is_hardly_more_than_its_own_rounding(rows, cols):
    """A number rounded once is off by 2^-23 / sqrt(12) of its power of two, 2.5e-8 of itself where numbers are spread over the powers of two (root mean square).  Half the
    error of a sum of squares comes on top: per segment of 256 columns an addition's 3.4e-8 times sqrt(1 + 1/2 + 1/4 + ...) < sqrt(2.5), over the root of 8 segments and
    more at most 1.0e-8: sqrt(2.5^2 + 1.0^2) = 2.7, and a few per cent for the draw."""
    x = stream(rows, cols, torch.float32, 3)
    rstd = torch.empty(rows, device="cuda")
    b.rms_norm(x, rstd=rstd, eps=1e-6)
    want = plain(x, None, None, 1e-6)[1]
    assert float(((rstd.double() - want) / want).square().mean().sqrt()) <= (3.0e-8 if rows > 1000 else 3.3e-8)


@pytest.mark.parametrize("cols", [41, 47, 55, 61, 1999, 8201])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient_of_a_constant_row_along_itself_is_zero(cols, dtype):
    one = torch.ones(3, cols, device="cuda").to(dtype)
    dx = torch.full_like(one, float("nan"))
    b.rms_norm_backward(one, one, None, torch.ones(3, device="cuda"), dx)      # 1 - 1 x mean of ones
    assert bool((dx == 0).all())

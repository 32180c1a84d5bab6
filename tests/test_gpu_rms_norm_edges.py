"""Accuracy of the norm's row sums and the widths between the tested ones, on the GPU against plain implementations in 64 bits."""
import pytest
import torch

from paper_2609_05419_b200 import binding as b

pytestmark = pytest.mark.gpu

from test_gpu_rms_norm import LEAST, NORM, RSTD, STEP, check_backward, check_form, gen, outputs, plain, randn, stream  # noqa: E402


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


@pytest.mark.parametrize("rows,cols", [(5, 3), (5, 300), (4, 4096), (300, 700), (600, 1000), (9, 8200), (3, 20001)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("residual,keep", [(False, False), (True, False), (True, True)])
def test_squares_beyond_the_32_bit_range(rows, cols, dtype, residual, keep):
    """Rows of sizes from 1e-37 to 1e37 beside one another, without an epsilon: their norm is of size 1."""
    size = 10.0 ** torch.linspace(-37, 37, rows, device="cuda", dtype=torch.float64)[torch.randperm(rows, generator=gen(5), device="cuda")]
    draw = lambda seed: (torch.randn(rows, cols, generator=gen(seed), device="cuda").clamp(-5, 5).double() * size[:, None]).to(dtype)
    x, r = draw(7), draw(8) if residual else None
    w = 1 + 0.3 * torch.randn(cols, generator=gen(9), device="cuda")
    h, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda")
    qt, st = b.fp8_empty(cols, rows)
    b.rms_norm(x, w, R=r, H=h if keep else None, Y=y, rstd=rstd, Qt=qt, St=st, eps=0.0)
    stored, want, n = plain(x, r, w, 0.0)
    assert not keep or torch.equal(h, stored)
    # 1.5 roundings of rstd, two of N, one of Y; H itself is of 24 bits or 8 down to 2^-126, N of size 1 and its entries not below 2^-100
    assert bool(((rstd.double() - want) / want).abs().max() <= 3 * 2.0 ** -24)
    step = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}[dtype]
    assert bool(((y.double() - n).abs() <= (5 * 2.0 ** -24 + step * 1.001) * n.abs() + 2.0 ** -126).all())
    assert bool(torch.isfinite(st).all())


def test_squares_beyond_the_range_in_place_and_the_same_for_any_alignment():
    rows, cols = 20, 1000
    x = torch.randn(rows, cols, generator=gen(11), device="cuda") * 10.0 ** torch.linspace(-36, 36, rows, device="cuda", dtype=torch.float64)[:, None].float()
    r = 0.5 * x.flip(1)
    want, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
    b.rms_norm(x, R=r, Y=want, rstd=rstd, eps=0.0)
    for skip in (0, 1):
        store = torch.zeros(rows * cols + 1, device="cuda")
        h = store[skip:skip + rows * cols].view(rows, cols)
        h.copy_(x)
        y, got = torch.empty_like(x), torch.empty(rows, device="cuda")
        b.rms_norm(h, R=r, H=h, Y=y, rstd=got, eps=0.0)
        assert torch.equal(h, x + r) and torch.equal(got, rstd) and torch.equal(y, want)
    many = torch.empty(400 * rows, device="cuda")
    b.rms_norm(x.repeat(400, 1), R=r.repeat(400, 1), rstd=many, eps=0.0)
    assert torch.equal(many.view(400, rows), rstd.expand(400, rows))


@pytest.mark.parametrize("cols", [512, 4096, 32768])
def test_a_sum_that_overflows_although_no_part_of_it_does(cols):
    """Every segment of 256 columns sums to less than 2^128, the row does not."""
    x = torch.full((3, cols), 2.0 ** 59.7, device="cuda")
    x[1] = 1.0
    rstd = torch.empty(3, device="cuda")
    b.rms_norm(x, rstd=rstd, eps=0.0)
    assert bool(((rstd.double() - 1 / x[:, 0].double()).abs() <= 2.0 ** -23 / x[:, 0].double()).all())
    alone = torch.empty(1, device="cuda")
    for row in range(3):
        b.rms_norm(x[row:row + 1], rstd=alone, eps=0.0)
        assert torch.equal(alone[0], rstd[row])


# Widths at which the kernels change: two blocks on an SM up to 5120 columns, one (of 512 threads) up to 8192, clusters beyond
@pytest.mark.parametrize("rows,cols", [(3, 5121), (400, 5376), (333, 6001), (300, 6144), (149, 7160), (301, 8191), (400, 8192), (150, 8193), (700, 4609), (297, 5120)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.float16])
def test_gradients_at_the_widths_where_kernels_change(rows, cols, dtype):
    check_backward(rows, cols, dtype, True, True, add=True, seed=201)
    check_backward(rows, cols, dtype, False, False, seed=211)


@pytest.mark.parametrize("rows,cols", [(297, 2049), (300, 3080), (513, 4096), (298, 5376), (301, 6001), (400, 7168), (297, 8192), (299, 8200), (600, 1025), (2000, 257)])
@pytest.mark.parametrize("dtype,fmt", [(torch.bfloat16, b.E4M3), (torch.float32, b.E5M2)])
def test_norm_of_many_rows_of_any_width(rows, cols, dtype, fmt):
    x, r, w = stream(rows, cols, dtype, 221), stream(rows, cols, dtype, 225), 1 + 0.3 * randn(229, cols)
    out = outputs(rows, cols, dtype, fmt)
    b.rms_norm(x, w, R=r, eps=1e-5, **out)
    h, rstd, n = plain(x, r, w, 1e-5)
    assert torch.equal(out["H"], h)
    assert bool(((out["rstd"].double() - rstd).abs() <= RSTD * rstd).all())
    assert bool(((out["Y"].double() - n).abs() <= (STEP[dtype] * (1 + NORM) + NORM) * n.abs() + LEAST[dtype]).all())
    check_form(out["Q"], out["S"], n, fmt)
    check_form(out["Qt"], out["St"], n.t(), fmt)
    few = torch.empty(8, device="cuda")
    b.rms_norm(x[:8], w, R=r[:8], rstd=few, eps=1e-5)                          # few rows: other warps to a row, the same numbers
    assert torch.equal(few, out["rstd"][:8])

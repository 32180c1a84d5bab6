"""Clipping far above the limit, and views, on the GPU against plain implementations in 64 bits."""
import math

import pytest
import torch

from paper_2609_05419_b200 import binding as b

pytestmark = pytest.mark.gpu

from test_gpu_clip_gradients import LEAST, NORM, STEP, check, randn, workspace  # noqa: E402


@pytest.mark.parametrize("size", [1e30, 1e36])
@pytest.mark.parametrize("limit", [1.0, 0.01, 1e-5, 1e-20])
@pytest.mark.parametrize("in_place", [True, False])
def test_a_factor_below_the_normal_numbers_keeps_its_bits(size, limit, in_place):
    grads = [randn(1, 500, 40, size=size), randn(2, 333, dtype=torch.bfloat16, size=size), randn(3, 41, 7, size=size)[:, 1:]]
    check(grads, limit, None if in_place else [torch.empty(t.shape, dtype=t.dtype, device="cuda") for t in grads])


@pytest.mark.parametrize("limit", [1.0, 0.01, 1e-30])
def test_a_norm_beyond_32_bits(limit):
    grads = [randn(1, 500, 400, size=1e37).clamp(-3e38, 3e38), randn(2, 333, dtype=torch.bfloat16, size=1e37)]
    grads[0][:100] = 3e38
    before = [t.clone() for t in grads]
    norm = torch.empty((), device="cuda")
    with workspace(2):
        b.clip_gradients(grads, limit, norm=norm)
    size = math.sqrt(math.fsum(float(t.double().square().sum()) for t in before))
    assert size > 3.5e38 and float(norm) == math.inf
    for was, now in zip(before, grads):
        want = was.double() * (limit / size)
        assert bool(((now.double() - want).abs() <= (NORM + 3 * 2.0 ** -24 + STEP[was.dtype] * 1.001) * want.abs() + LEAST[was.dtype]).all())

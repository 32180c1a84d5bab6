"""Workspace sizes of the layer operators: what suffices for a call suffices for every smaller one.  No GPU is touched."""
import random

import pytest

from paper_2609_05419_b200 import binding as b

SIZES = {
    b.OP_RMS_NORM: ([0, 1, 7, 8, 100, 129, 5000, 10 ** 6], [0, 1, 512, 513, 8192, 8193, 32768]),
    b.OP_RMS_NORM_BACKWARD: ([0, 1, 2, 7, 8, 9, 147, 148, 149, 295, 296, 297, 1000, 2368, 4096, 10 ** 6],
                             [0, 1, 255, 256, 511, 512, 513, 1024, 1025, 1537, 2048, 2049, 4096, 5119, 5120, 5121, 5633, 8192, 8193, 12288, 12289, 16384, 20000, 32768]),
    b.OP_CLIP_GRADIENTS: ([0, 1, 64, 65, 511, 512, 513, 10000, 2 ** 20],),
    b.OP_ADAPTER_ADD: ([0, 1, 2, 15, 16, 17, 48, 127, 128, 129, 207, 208, 239, 240, 255, 256, 257, 300, 700, 1024, 4992, 8192, 100000], [0, 1, 16, 17, 32, 33, 64, 65, 128],
                       [0, 1, 2, 8, 24, 64, 255, 300, 16384]),
}


def size(op, sizes):
    return b.workspace_bytes(op, *(tuple(sizes) + (1, 1, 1))[:3], 1)


@pytest.mark.parametrize("op", SIZES)
def test_the_size_never_falls_as_one_of_the_sizes_grows(op):
    grids = SIZES[op]
    for at, grid in enumerate(grids):
        rest = [g for i, g in enumerate(grids) if i != at]
        others = [()]
        for g in rest:
            others = [o + (v,) for o in others for v in g]
        for o in others:
            got = [size(op, o[:at] + (v,) + o[at:]) for v in sorted(grid)]
            assert min(got) > 0 and got == sorted(got), (op, at, o, got)


@pytest.mark.parametrize("op,most", [(b.OP_RMS_NORM_BACKWARD, (3000, 32768)), (b.OP_ADAPTER_ADD, (600, 128, 400))])
def test_the_size_of_the_largest_call_suffices_for_any_smaller_one(op, most):
    rng = random.Random(5)
    for _ in range(3000):
        larger = [rng.randint(1, m) for m in most]
        smaller = [rng.randint(1, v) for v in larger]
        assert size(op, smaller) <= size(op, larger), (smaller, larger)

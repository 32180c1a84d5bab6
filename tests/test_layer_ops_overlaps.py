"""Outputs of the layer operators that lie beside something else are taken, those that overlap it are refused.  No GPU is touched: addresses are never dereferenced."""
import ctypes

import pytest

from paper_2609_05419_b200 import binding as b
from test_layer_ops_more_arguments import _clip, _tensor, refused


def view(at, rows, cols, ld=20):
    """Columns (and rows, in `at`) of one matrix at 4096 with `ld` columns of 32 bits."""
    return _tensor(G=4096 + 4 * at, rows=rows, cols=cols, ldg=ld)


def test_clip_takes_a_part_of_one_row_beside_views_of_all_rows():
    columns = view(0, 5, 8)                                                   # columns 0 .. 7 of five rows
    for at, rows, cols in ((8, 1, 12), (28, 1, 12), (40 + 8, 1, 1), (40 + 19, 1, 1), (88, 1, 12), (88, 1, 500)):
        assert not refused(_clip([columns, view(at, rows, cols)], in_place=True)), (at, rows, cols)
        assert not refused(_clip([view(at, rows, cols), columns], in_place=True)), (at, rows, cols)
    for at, rows, cols in ((7, 1, 1), (8, 1, 13), (40, 1, 3), (60 + 19, 1, 2), (87, 1, 1), (28, 1, 60)):
        assert refused(_clip([columns, view(at, rows, cols)], in_place=True)), (at, rows, cols)
        assert refused(_clip([view(at, rows, cols), columns], in_place=True)), (at, rows, cols)
    # a row of gaps taken up by contiguous tensors, one per gap
    assert not refused(_clip([columns] + [view(8 + 20 * i, 1, 12) for i in range(4)] + [view(8 + 80, 3, 4, 4)], in_place=True))

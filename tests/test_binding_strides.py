"""Leading dimensions that the binding derives from strides, for the column-major entry points (no GPU is touched)."""
import pytest
import torch

from paper_2609_05419_b200 import binding as b
from test_layer_ops_arguments import Standin


# one row whose columns all lie on the same entry: memory holds that entry only, and the library refuses a leading dimension of 0
@pytest.mark.parametrize("helper,wrap", [(b._colmajor, Standin), (b._colmajor_host, lambda t: t)])
def test_one_expanded_row_keeps_its_stride(helper, wrap):
    t = torch.zeros(1, 1, dtype=torch.complex128).expand(1, 7)
    assert helper(wrap(t), "A")[3] == 0
    assert b.lib().zgemm2m(1, 4, 7, 256, 0, 256, 7, 256, 1, 16, None) == b.ERR_ARG
    assert b.lib().zgemm2m_host(1, 4, 7, 256, 0, 256, 7, 256, 1, 16, None) == b.ERR_ARG


@pytest.mark.parametrize("helper,wrap", [(b._colmajor, Standin), (b._colmajor_host, lambda t: t)])
def test_leading_dimensions_of_ordinary_and_empty_matrices(helper, wrap):
    colmajor = lambda rows, cols, ld: wrap(torch.zeros(cols, ld, dtype=torch.complex128)[:, :rows].t())
    for rows, cols, ld, want in ((5, 7, 5, 5), (5, 7, 8, 8), (1, 7, 1, 1), (1, 7, 3, 3), (5, 1, 9, 5), (1, 1, 1, 1)):
        assert helper(colmajor(rows, cols, ld), "A")[1:] == (rows, cols, want)
    for rows, cols in ((0, 7), (7, 0), (0, 0)):
        assert helper(wrap(torch.zeros(rows, cols, dtype=torch.complex128)), "A")[3] >= 1
    assert helper(wrap(torch.zeros(0, 1, dtype=torch.complex128).expand(0, 7)), "A")[3] >= 1

"""Leading dimensions that the binding derives from strides, for the column-major entry points (no GPU is touched)."""
import pytest
import torch

from paper_2609_05419_b200 import binding as b
from test_layer_ops_arguments import Standin


@pytest.fixture(autouse=True)
def device_zero(monkeypatch):
    monkeypatch.setattr(b, "_current_device", lambda: 0)


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


# ---------------------------------------------------------------------------------------------- tensors of another than the current device
def test_column_major_operands_and_workspaces_lie_on_the_current_device(monkeypatch):
    seen = []

    class Recorder:
        def __getattr__(self, name):
            return lambda *args: seen.append(name) or b.OK

    monkeypatch.setattr(b, "lib", Recorder)
    monkeypatch.setattr(b, "_current_stream", lambda *device: 0)
    colmajor = lambda rows, cols, device: Standin(torch.zeros(cols, rows, dtype=torch.complex128).t(), device)
    b.zgemm2m(colmajor(3, 4, 0), colmajor(4, 5, 0), colmajor(3, 5, 0))
    b.set_workspace(Standin(torch.zeros(512, dtype=torch.uint8)))
    b.zscale_exponents_static(colmajor(3, 4, 0), Standin(torch.zeros(3, dtype=torch.int32)))
    assert seen == ["zgemm2m", "gemm2m_set_workspace", "gemm2m_zscale_exponents_static"]
    for odd in range(3):
        with pytest.raises(ValueError):
            b.zgemm2m(*(colmajor(r, c, int(i == odd)) for i, (r, c) in enumerate(((3, 4), (4, 5), (3, 5)))))
    with pytest.raises(ValueError):
        b.set_workspace(Standin(torch.zeros(512, dtype=torch.uint8), 1))
    with pytest.raises(ValueError):
        b.zscale_exponents_static(colmajor(3, 4, 0), Standin(torch.zeros(3, dtype=torch.int32), 1))
    assert len(seen) == 3

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


# Matrices of 6 rows of 8 columns of 32 bits in rows 40 columns apart, all in one store; `at`: entries from its start.  An 8-bit matrix there has rows of 160 bytes.
STORE = 1 << 20
at = lambda entries: STORE + 4 * entries
ROWS, COLS, LD = 6, 8, 40
END = ROWS * LD


def norm(**other):
    t = dict(rows=ROWS, cols=COLS, X=at(0), type=b.F32, ldx=LD, R=at(8), ldr=LD, W=at(END), w_type=b.F32, eps=1e-6, H=at(16), ldh=LD, Y=at(24), ldy=LD, fmt=b.E4M3, Q=at(32), ldq=4 * LD,
             S=at(END + 8), lds=ROWS, Qt=at(END + 16), ldqt=16, St=at(END + 48), ldst=COLS, rstd=at(END + 56))
    assert set(other) <= set(t)
    t.update(other)
    t["eps"] = ctypes.c_float(t["eps"])
    return b.lib().gemm2m_rms_norm(*t.values(), None)


def test_norm_takes_operands_side_by_side():
    assert not refused(norm())
    assert not refused(norm(H=at(0))) and not refused(norm(H=at(8)))          # in place of either summand
    assert not refused(norm(R=at(0), H=at(0)))
    assert not refused(norm(rstd=at(34)))                                     # in the gap behind the 8-bit rows
    assert not refused(norm(W=at(END + 62))) and not refused(norm(X=at(1000)))
    assert not refused(norm(Q=None, S=None)) and not refused(norm(rstd=None, Y=None))


@pytest.mark.parametrize("bad", [dict(H=at(1)), dict(H=at(LD)), dict(H=at(12)), dict(H=at(END - 1)), dict(Y=at(1)), dict(Y=at(15)), dict(Y=at(17)), dict(Y=at(LD + 31)), dict(Y=at(LD - 7)),
                                 dict(Q=at(0)), dict(Q=at(28)), dict(Q=at(END)), dict(S=at(0)), dict(S=at(END)), dict(S=at(END + 11)), dict(Qt=at(32)), dict(Qt=at(END + 8)),
                                 dict(Qt=at(END + 4)), dict(St=at(END + 44)), dict(St=at(16)), dict(rstd=at(0)), dict(rstd=at(5 * LD + 30)), dict(rstd=at(END + 3)), dict(rstd=at(END + 10)),
                                 dict(rstd=at(END + 55)), dict(rstd=at(33)), dict(W=at(END + 9)), dict(W=at(18)), dict(X=at(17)), dict(R=at(LD + 16)), dict(X=at(20), ldx=44)])
def test_norm_refuses_outputs_that_overlap(bad):
    assert refused(norm(**bad))


def backward(**other):
    t = dict(rows=ROWS, cols=COLS, dY=at(0), type=b.F32, lddy=LD, H=at(8), ldh=LD, W=at(END), w_type=b.F32, rstd=at(END + 8), dR=at(16), lddr=LD, dX=at(24), lddx=LD, dW=at(END + 16), add=0)
    assert set(other) <= set(t)
    t.update(other)
    return b.lib().gemm2m_rms_norm_backward(*t.values(), None)


def test_norm_backward_takes_operands_side_by_side():
    for fine in (dict(), dict(dX=at(0)), dict(dX=at(8)), dict(dX=at(16)), dict(dY=at(8)), dict(dR=at(0)), dict(dW=at(32)), dict(dW=None), dict(dR=None), dict(dW=at(32 + LD)), dict(rstd=at(32))):
        assert not refused(backward(**fine)), fine


@pytest.mark.parametrize("bad", [dict(dX=at(1)), dict(dX=at(LD)), dict(dX=at(END - 2)), dict(dX=at(LD + 33)), dict(dX=at(END + 1)), dict(dX=at(END + 10)), dict(dX=at(END + 16)), dict(dW=at(0)),
                                 dict(dW=at(END)), dict(dW=at(END + 7)), dict(dW=at(END + 13)), dict(dW=at(25)), dict(dW=at(33)), dict(rstd=at(24)), dict(W=at(30)), dict(dR=at(20)), dict(H=at(LD + 24))])
def test_norm_backward_refuses_outputs_that_overlap(bad):
    assert refused(backward(**bad))


def adapters(**other):
    # B: two matrices of 8 rows of 4 columns of 16 bits, 16 entries of 32 bits each, 100 such entries apart
    t = dict(tokens=ROWS, n=COLS, k=4, adapters=2, rank=4, X=at(5000), type=b.BF16, ldx=4, A=at(6000), lda=4, stride_a=16, B=at(END), ldb=4, stride_b=200, index=at(END + 20), scales=at(END + 26),
             ranks=at(END + 28), C=at(0), ldc=LD, D=at(8), d_type=b.F32, ldd=LD)
    assert set(other) <= set(t)
    t.update(other)
    return b.lib().gemm2m_adapter_add(*t.values(), None)


def test_adapters_take_operands_side_by_side():
    for fine in (dict(), dict(D=at(0)), dict(C=None), dict(X=at(8)), dict(X=at(9)), dict(D=at(END + 30), ldd=8), dict(D=at(END + 116)), dict(scales=None, ranks=None), dict(index=at(16)),
                 dict(B=at(END + 30), adapters=1), dict(B=at(END - 10), adapters=1), dict(k=0, D=at(END + 20), C=None), dict(B=at(20 * LD), stride_b=0)):
        assert not refused(adapters(**fine)), fine


@pytest.mark.parametrize("bad", [dict(D=at(1)), dict(D=at(LD)), dict(D=at(END)), dict(D=at(END + 15)), dict(D=at(END + 14), ldd=8), dict(D=at(END + 18), ldd=8), dict(D=at(END + 25), ldd=8),
                                 dict(D=at(END + 27), ldd=8), dict(D=at(END + 60), ldd=8), dict(D=at(END + 115)), dict(index=at(10)), dict(index=at(LD + 6)), dict(scales=at(15)), dict(ranks=at(7)),
                                 dict(B=at(8)), dict(C=at(10)), dict(k=0, D=at(1)), dict(B=at(END - 30), adapters=1)])
def test_adapters_refuse_outputs_that_overlap(bad):
    assert refused(adapters(**bad))


def test_clip_refuses_a_norm_inside_a_gradient_or_an_output():
    # one gradient of 5 rows of 8 columns 20 apart at 4096, its output contiguous at 8192
    one = [_tensor(G=4096, O=8192, rows=5, cols=8, ldg=20, ldo=8)]
    for inside in (4096, 4096 + 4 * 27, 4096 + 4 * 87, 8192, 8192 + 4 * 39):
        assert refused(_clip(one, norm=inside)), inside
    for beside in (4096 - 4, 4096 + 4 * 8, 4096 + 4 * 39, 4096 + 4 * 88, 8192 - 4, 8192 + 4 * 40):
        assert not refused(_clip(one, norm=beside)), beside
    assert refused(_clip(one, norm=4096, in_place=True)) and not refused(_clip(one, norm=4096 + 32, in_place=True))

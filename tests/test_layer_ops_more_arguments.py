"""Norm, gradient clipping and low-rank adapters: sizes, and the refusals that come before any launch.  No GPU is touched: addresses are never
dereferenced, CPU tensors stand in for CUDA ones and the library is replaced by a recorder."""
import ctypes

import pytest
import torch

from paper_2609_05419_b200 import binding as b
from test_layer_ops_arguments import calls, dense, matrix, Standin  # noqa: F401

ARG, WS = b.ERR_ARG, b.ERR_WORKSPACE
null = None
one, two = 256, 4096         # aligned addresses: argument checks come first


def vector(size, dtype=torch.float32, **where):
    return Standin(torch.zeros(size, dtype=dtype), **where)


# ----------------------------------------------------------------------------------------------------------------- the norm
def _norm(rows=4, cols=4, X=one, type=b.BF16, ldx=4, R=null, ldr=4, W=null, w_type=b.F32, eps=1e-6, H=null, ldh=4, Y=null, ldy=4, fmt=b.E4M3, Q=two, ldq=16,
          S=one, lds=4, Qt=null, ldqt=16, St=null, ldst=4, rstd=null):
    return b.lib().gemm2m_rms_norm(rows, cols, X, type, ldx, R, ldr, W, w_type, ctypes.c_float(eps), H, ldh, Y, ldy, fmt, Q, ldq, S, lds, Qt, ldqt, St, ldst,
                                   rstd, null)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(cols=-1), dict(cols=32769, ldx=40000, ldq=40000), dict(rows=2 ** 31), dict(ldx=3), dict(type=b.E4M3), dict(type=-1),
                                 dict(W=one, w_type=b.E5M2), dict(R=two, ldr=3), dict(H=two, ldh=3), dict(Y=two, ldy=3), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(fmt=b.BF16), dict(ldq=24), dict(ldq=0), dict(Q=264), dict(lds=3), dict(S=null), dict(Q=null), dict(Q=null, S=null),
                                 dict(Qt=one), dict(St=one), dict(Qt=one, St=one, ldqt=8), dict(Qt=one, St=one, ldst=3), dict(Qt=8, St=one), dict(X=null),
                                 dict(H=one, ldh=8), dict(R=two, H=two, ldr=8), dict(Y=one), dict(R=two, Y=two), dict(H=two, Y=two)])
def test_norm_refuses(bad):
    assert _norm(**bad) == ARG


def test_norm_of_nothing_is_fine():
    assert _norm(rows=0, X=null) == 0 and _norm(cols=0, ldx=1) == 0


def _back(rows=4, cols=4, dY=one, type=b.F32, lddy=4, H=two, ldh=4, W=null, w_type=b.F32, rstd=one, dR=null, lddr=4, dX=512, lddx=4, dW=null, add=0):
    return b.lib().gemm2m_rms_norm_backward(rows, cols, dY, type, lddy, H, ldh, W, w_type, rstd, dR, lddr, dX, lddx, dW, add, null)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(cols=-1), dict(cols=32769, lddy=40000, ldh=40000, lddx=40000), dict(type=b.E5M2), dict(W=one, w_type=7), dict(lddy=3),
                                 dict(ldh=3), dict(lddx=3), dict(dR=one, lddr=3), dict(dY=null), dict(H=null), dict(rstd=null), dict(dX=null),
                                 dict(dX=one, lddx=8), dict(dX=two, lddx=8), dict(dR=768, dX=768, lddx=8)])
def test_norm_backward_refuses(bad):
    assert _back(**bad) == ARG


def test_norm_backward_of_nothing_is_fine():
    assert _back(rows=0) == 0 and _back(rows=0, dW=one, add=1) == 0 and _back(cols=0, dW=one) == 0


def test_norm_workspace_sizes():
    size = lambda op, *s: b.workspace_bytes(op, *s, 1, 1)
    assert size(b.OP_RMS_NORM, -1, 4) == 0 and size(b.OP_RMS_NORM, 4, 32769) == 0 and size(b.OP_RMS_NORM_BACKWARD, 4, -1) == 0
    assert 256 <= size(b.OP_RMS_NORM, 0, 0) <= size(b.OP_RMS_NORM, 1000, 64) - 4000
    for rows, cols in ((0, 64), (64, 0), (0, 0)):
        assert size(b.OP_RMS_NORM_BACKWARD, rows, cols) >= 256
    assert size(b.OP_RMS_NORM_BACKWARD, 1, 4096) < size(b.OP_RMS_NORM_BACKWARD, 10 ** 6, 4096) == size(b.OP_RMS_NORM_BACKWARD, 10 ** 8, 4096) < 2 ** 25


def norm_operands(rows=30, cols=50):
    x = lambda: dense(rows, cols, torch.bfloat16)
    (q, s), (qt, st) = matrix(rows, cols), matrix(cols, rows)
    return dict(X=x(), W=vector(cols), R=x(), H=x(), Y=x(), Q=q, S=s, Qt=qt, St=st, rstd=vector(rows))


def backward_operands(rows=30, cols=50):
    x = lambda: dense(rows, cols, torch.bfloat16)
    return dict(dY=x(), H=x(), W=vector(cols), rstd=vector(rows), dX=x(), dR=x(), dW=vector(cols))


OPERANDS = {"rms_norm": norm_operands, "rms_norm_backward": backward_operands}


@pytest.mark.parametrize("name", OPERANDS)
def test_every_operand_lies_on_the_current_device_and_has_its_shape_and_type(calls, name):  # noqa: F811
    call, make = getattr(b, name), OPERANDS[name]
    call(**make())
    assert len(calls) == 1
    wrong = make(rows=29, cols=49)
    for operand in make():
        for elsewhere in (1, -1):
            t = make()
            t[operand].index = elsewhere
            with pytest.raises(ValueError):
                call(**t)
        with pytest.raises(ValueError):
            call(**{**make(), operand: wrong[operand]})
        with pytest.raises(ValueError):
            call(**{**make(), operand: Standin(torch.zeros(make()[operand].shape, dtype=torch.float64))})
    assert len(calls) == 1


def test_norm_refuses_halves_of_forms_and_mixed_formats(calls):  # noqa: F811
    for missing in ("Q", "S", "Qt", "St"):
        t = norm_operands()
        del t[missing]
        with pytest.raises(ValueError):
            b.rms_norm(**t)
    t = norm_operands()
    t["Qt"] = Standin(t["Qt"].tensor.view(torch.float8_e5m2))
    with pytest.raises(ValueError):
        b.rms_norm(**t)
    for missing in ("H", "rstd", "dX"):
        with pytest.raises(ValueError):
            b.rms_norm_backward(**{**backward_operands(), missing: None})
    assert not calls

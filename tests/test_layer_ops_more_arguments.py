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
                                 dict(X=258, ldx=8, type=b.F32), dict(R=513), dict(W=258), dict(H=515), dict(Y=511), dict(S=258), dict(rstd=254),
                                 dict(Qt=one, St=two + 2), dict(H=one, ldh=8), dict(R=two, H=two, ldr=8), dict(Y=one), dict(R=two, Y=two), dict(H=two, Y=two)])
def test_norm_refuses(bad):
    assert _norm(**bad) == ARG


def test_norm_of_nothing_is_fine():
    assert _norm(rows=0, X=null) == 0 and _norm(cols=0, ldx=1) == 0


def _back(rows=4, cols=4, dY=one, type=b.F32, lddy=4, H=two, ldh=4, W=null, w_type=b.F32, rstd=one, dR=null, lddr=4, dX=512, lddx=4, dW=null, add=0):
    return b.lib().gemm2m_rms_norm_backward(rows, cols, dY, type, lddy, H, ldh, W, w_type, rstd, dR, lddr, dX, lddx, dW, add, null)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(cols=-1), dict(cols=32769, lddy=40000, ldh=40000, lddx=40000), dict(type=b.E5M2), dict(W=one, w_type=7), dict(lddy=3),
                                 dict(ldh=3), dict(lddx=3), dict(dR=one, lddr=3), dict(dY=null), dict(H=null), dict(rstd=null), dict(dX=null),
                                 dict(dY=258), dict(H=257), dict(W=258), dict(rstd=255), dict(dR=514), dict(dX=514), dict(dW=258),
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


# ----------------------------------------------------------------------------------------------------------- gradient clipping
def _clip(tensors, max_norm=1.0, eps=1e-6, norm=null, in_place=False, count=None):
    """tensors: (G, O, type, rows, cols, ldg, ldo) each."""
    n = max(len(tensors), 1)
    column = lambda kind, k: (kind * n)(*[t[k] for t in tensors])
    vp, i64 = ctypes.c_void_p, ctypes.c_int64
    return b.lib().gemm2m_clip_gradients(len(tensors) if count is None else count, column(vp, 0), null if in_place else column(vp, 1), column(ctypes.c_int, 2),
                                         *(column(i64, k) for k in (3, 4, 5)), null if in_place else column(i64, 6), max_norm, eps, norm, null)


def _tensor(G=4096, O=8192, type=b.F32, rows=4, cols=4, ldg=4, ldo=4):
    return G, O, type, rows, cols, ldg, ldo


def refused(status):
    """(a call whose arguments are fine fails on this machine for want of a device, or of a workspace)"""
    return status == ARG


@pytest.mark.parametrize("bad", [dict(G=null), dict(O=null), dict(type=b.E4M3), dict(rows=-1), dict(cols=-1), dict(ldg=3), dict(ldo=3), dict(rows=2 ** 30, cols=2 ** 30, ldg=2 ** 30, ldo=2 ** 30),
                                 dict(G=4098), dict(O=8190), dict(type=b.BF16, G=4097), dict(O=4096, ldo=5), dict(O=4100), dict(O=4096 + 60)])
def test_clip_refuses_a_tensor(bad):
    assert not refused(_clip([_tensor()]))
    assert refused(_clip([_tensor(**bad)]))


def test_clip_refuses_numbers():
    for bad in (dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(eps=-1.0), dict(eps=float("nan")), dict(norm=258), dict(count=-1), dict(count=2 ** 20 + 1)):
        assert refused(_clip([_tensor()], **bad))
    for fine in (dict(max_norm=0.0), dict(max_norm=float("inf")), dict(eps=0.0), dict(in_place=True)):
        assert not refused(_clip([_tensor()], **fine))


def test_clip_refuses_outputs_that_overlap():
    a = _tensor()
    assert not refused(_clip([a, _tensor(G=4096, O=8192 + 64)]))              # the same gradient twice, into places of their own
    assert refused(_clip([a, a]))                                            # the same output twice
    assert refused(_clip([_tensor(O=4096), _tensor(O=4096)]))                # in place, twice
    assert refused(_clip([a, _tensor(G=4096 + 32)], in_place=True))
    assert refused(_clip([a, _tensor(G=8192 + 16, O=4 * 4096)]))             # another's input
    assert refused(_clip([a, _tensor(O=8192 + 60)]))
    assert not refused(_clip([a, _tensor(G=4096 + 64)], in_place=True))
    assert not refused(_clip([_tensor(rows=0, G=null, O=null), a, _tensor(cols=0)]))
    # views of one matrix of 20 columns side by side, and ones that share a column
    view = lambda at, cols: _tensor(G=4096 + 4 * at, rows=5, cols=cols, ldg=20)
    assert not refused(_clip([view(0, 8), view(8, 10), view(18, 2)], in_place=True))
    assert not refused(_clip([view(18, 2), view(8, 10), view(0, 8)], in_place=True))
    assert refused(_clip([view(0, 9), view(8, 10)], in_place=True))
    assert refused(_clip([view(0, 4), view(18, 4)], in_place=True))           # around the end of a row
    assert refused(_clip([view(0, 8), view(24, 8)], in_place=True))          # a row further on, four columns shared
    assert not refused(_clip([view(0, 8), view(28, 8)], in_place=True))      # a row further on, other columns
    assert refused(_clip([view(0, 8), _tensor(G=4096 + 32, rows=1, cols=60)], in_place=True))
    # a long span over many short ones
    assert refused(_clip([_tensor(G=4096, rows=1, cols=1000)] + [_tensor(G=9000 + 16 * i, rows=1, cols=4) for i in range(5)] + [_tensor(G=4096 + 3996, rows=1, cols=1)],
                         in_place=True))


def test_clip_workspace_sizes():
    size = lambda n: b.workspace_bytes(b.OP_CLIP_GRADIENTS, n, 1, 1, 1)
    assert 256 <= size(0) <= size(1) <= size(1000) < 10 ** 6 and size(-1) == 0 and size(2 ** 20 + 1) == 0 and size(2 ** 20) > size(1000)


def test_clip_passes_every_tensor_on(calls, monkeypatch):  # noqa: F811
    seen = []

    def record(count, G, O, types, rows, cols, ldg, ldo, max_norm, eps, norm, stream):
        many = lambda at, kind=ctypes.c_int64: at if at is None else list((kind * count).from_address(at))
        seen.append((many(G), many(O), many(types, ctypes.c_int), many(rows), many(cols), many(ldg), many(ldo), max_norm, eps, norm))
        return b.OK

    monkeypatch.setattr(b, "lib", lambda: type("Recorder", (), {"gemm2m_clip_gradients": staticmethod(record)}))
    whole = torch.zeros(6, 40)
    grads = [dense(5, 7), Standin(torch.zeros(3, 4, dtype=torch.bfloat16)), Standin(whole[:, 8:20]), Standin(torch.zeros(8, 9).t()), Standin(torch.zeros(())),
             Standin(torch.zeros(2, 3, 4).permute(2, 0, 1))]
    addresses = lambda tensors: [t.data_ptr() for t in tensors]
    norm = vector(1)
    b.clip_gradients(grads, 2.0, norm=norm)
    g, o, types, rows, cols, ldg, ldo, *rest = seen[-1]
    assert g == addresses(grads) and o is None and ldo is None and rest == [2.0, 1e-6, norm.data_ptr()]
    assert types == [b.F32, b.BF16] + [b.F32] * 4 and rows == [1, 1, 6, 1, 1, 1] and cols == [35, 12, 12, 72, 1, 24] and ldg[2] == 40
    # into outputs whose rows are further apart, or closer together
    outs = [Standin(torch.zeros(5, 20)[:, :7]), dense(3, 4, torch.bfloat16), dense(6, 12), Standin(torch.zeros(8, 9).t()), Standin(torch.zeros(())),
            Standin(torch.zeros(2, 3, 4).permute(2, 0, 1))]
    b.clip_gradients(grads, 2.0, out=outs)
    g, o, types, rows, cols, ldg, ldo, *rest = seen[-1]
    assert o == addresses(outs) and rest == [2.0, 1e-6, None] and rows == [5, 1, 6, 1, 1, 1] and cols == [7, 12, 12, 72, 1, 24]
    assert ldg[0] == 7 and ldo[0] == 20 and ldg[2] == 40 and ldo[2] == 12
    # all of them contiguous
    flat = [dense(5, 7), Standin(torch.zeros(3, 4, 2, dtype=torch.bfloat16)), Standin(torch.zeros(0, 3))]
    for out in (None, [dense(5, 7), Standin(torch.zeros(3, 4, 2, dtype=torch.bfloat16)), Standin(torch.zeros(0, 3))]):
        b.clip_gradients(iter(flat), 2.0, out=out)
        g, o, types, rows, cols, ldg, ldo, *rest = seen[-1]
        assert g == addresses(flat) and (o is None if out is None else o == addresses(out)) and types == [b.F32, b.BF16, b.F32] and rows == [1, 1, 1] and cols == [35, 24, 0]
    b.clip_gradients([], 2.0)
    assert seen[-1][0] == []


def test_clip_refuses_tensors_that_it_cannot_walk(calls):  # noqa: F811
    fine = dense(6, 8)
    for bad in (Standin(torch.zeros(6, 16)[:, ::2]), Standin(torch.zeros(6, 1).expand(6, 8)), Standin(torch.zeros(4, 6, 8)[:, :5]), Standin(torch.zeros(16)[::2]),
                Standin(torch.zeros(6, 8, dtype=torch.float64)), dense(6, 8, device=1), dense(6, 8, device=-1)):
        with pytest.raises(ValueError):
            b.clip_gradients([fine, bad], 1.0)
        with pytest.raises(ValueError):
            b.clip_gradients([fine], 1.0, out=[bad])
    for out in ([], [dense(6, 9)], [dense(6, 8, torch.bfloat16)], [Standin(torch.zeros(8, 6).t())], [fine, fine]):
        with pytest.raises(ValueError):
            b.clip_gradients([fine], 1.0, out=out)
    for norm in (vector(2), vector(1, torch.float64), vector(1, device=1)):
        with pytest.raises(ValueError):
            b.clip_gradients([fine], 1.0, norm=norm)
    assert not calls


# ------------------------------------------------------------------------------------------------------------------- adapters
def _adapters(tokens=4, n=4, k=4, adapters=2, rank=4, X=one, type=b.BF16, ldx=4, A=one, lda=4, sa=16, B=one, ldb=4, sb=16, index=one, scales=null, ranks=null,
              C=null, ldc=4, D=two, d_type=b.F32, ldd=4):
    return b.lib().gemm2m_adapter_add(tokens, n, k, adapters, rank, X, type, ldx, A, lda, sa, B, ldb, sb, index, scales, ranks, C, ldc, D, d_type, ldd, null)


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(n=-1), dict(k=-1), dict(tokens=2 ** 31), dict(adapters=-1), dict(adapters=16385), dict(rank=-1), dict(rank=129, ldb=129),
                                 dict(type=b.F32), dict(type=b.E4M3), dict(d_type=b.E4M3), dict(ldx=3), dict(lda=3), dict(ldb=3), dict(ldd=3), dict(C=one, ldc=3),
                                 dict(C=two, ldc=8), dict(sa=-1), dict(sb=-1), dict(X=null), dict(A=null), dict(B=null), dict(index=null), dict(D=null),
                                 dict(X=257), dict(A=257), dict(B=257), dict(index=258), dict(scales=258), dict(ranks=258), dict(C=258), dict(D=4098), dict(D=4097, d_type=b.F16)])
def test_adapters_refuse(bad):
    assert not refused(_adapters())
    assert refused(_adapters(**bad))


def test_adapters_of_nothing_are_fine():
    assert _adapters(tokens=0, X=null, index=null, D=null) == 0 and _adapters(n=0, B=null, D=null) == 0


def test_adapter_workspace_sizes():
    size = lambda *s: b.workspace_bytes(b.OP_ADAPTER_ADD, *s, 1)
    for bad in ((-1, 4, 4), (4, -1, 4), (4, 129, 4), (4, 4, -1), (4, 4, 16385)):
        assert size(*bad) == 0
    for fine in ((0, 0, 0), (0, 16, 4), (1, 0, 4), (1, 16, 0), (1, 1, 1)):
        assert 256 <= size(*fine) <= size(300, 64, 16)
    assert size(100000, 64, 16) >= 100000 * (4 + 4 * 64)


def adapter_operands(tokens=30, k=50, n=40, many=3, rank=8):
    half = lambda *shape: Standin(torch.zeros(*shape, dtype=torch.bfloat16))
    return dict(X=half(tokens, k), A=half(many, rank, k), B=half(many, n, rank), index=vector(tokens, torch.int32), D=dense(tokens, n), C=dense(tokens, n),
                scales=vector(many), ranks=vector(many, torch.int32))


def test_adapter_operands_lie_on_the_current_device_and_have_their_shapes_and_types(calls):  # noqa: F811
    b.adapter_add(**adapter_operands())
    assert len(calls) == 1
    wrong = adapter_operands(31, 51, 41, 4, 9)
    for operand in adapter_operands():
        for elsewhere in (1, -1):
            t = adapter_operands()
            t[operand].index = elsewhere
            with pytest.raises(ValueError):
                b.adapter_add(**t)
        with pytest.raises(ValueError):
            b.adapter_add(**{**adapter_operands(), operand: wrong[operand]})
        with pytest.raises(ValueError):
            b.adapter_add(**{**adapter_operands(), operand: Standin(torch.zeros(adapter_operands()[operand].shape, dtype=torch.float64))})
    for operand, bad in (("A", torch.zeros(3, 50, 8, dtype=torch.bfloat16).transpose(1, 2)), ("index", torch.zeros(60, dtype=torch.int32)[::2]),
                         ("A", torch.zeros(3, 8, 50, dtype=torch.float16)), ("scales", torch.zeros(6)[::2])):
        with pytest.raises(ValueError):
            b.adapter_add(**{**adapter_operands(), operand: Standin(bad)})
    assert len(calls) == 1


def test_adapters_pass_their_strides_on(calls):  # noqa: F811
    t = adapter_operands()
    t["A"] = Standin(torch.zeros(3, 10, 64, dtype=torch.bfloat16)[:, :8, :50])
    t["B"] = Standin(torch.zeros(1, 40, 8, dtype=torch.bfloat16).expand(3, 40, 8))
    b.adapter_add(**t)
    _, a = calls[-1]
    assert a[:5] == (30, 40, 50, 3, 8) and a[9:11] == (64, 640) and a[12:14] == (8, 0)
    for rank, many in ((1, 3), (8, 1), (1, 1), (0, 2), (3, 0)):
        b.adapter_add(**adapter_operands(rank=rank, many=many))
        _, a = calls[-1]
        assert a[9] >= 50 and a[12] >= max(rank, 1) and a[10] >= 0 and a[13] >= 0

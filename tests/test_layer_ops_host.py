"""Layer operators (8-bit quantisation and products, Newton-Schulz): sizes, and the refusals that come before any launch."""
import ctypes

import pytest
import torch

from paper_2609_05419_b200 import binding as b

ARG, WS = b.ERR_ARG, b.ERR_WORKSPACE
null = None
one = 256            # an aligned address that is never dereferenced: argument checks come first


def _quantise(rows=4, cols=4, X=one, type=b.BF16, ldx=4, fmt=b.E4M3, block=1, Q=one, ldq=16, S=one, lds=4, Qt=null, ldqt=16, St=null, ldst=4):
    return b.lib().gemm2m_fp8_quantise(rows, cols, X, type, ldx, fmt, block, Q, ldq, S, lds, Qt, ldqt, St, ldst, null)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(cols=-1), dict(ldx=3), dict(type=b.E4M3), dict(type=-1), dict(fmt=b.BF16), dict(block=64), dict(ldq=24),
                                 dict(ldq=0), dict(Q=264), dict(lds=3), dict(S=null), dict(Q=null), dict(Q=null, S=null), dict(X=null),
                                 dict(Qt=one), dict(St=one), dict(Qt=one, St=one, ldqt=8), dict(Qt=one, St=one, ldst=3), dict(Qt=8, St=one),
                                 dict(cols=20, ldx=20, ldq=16)])
def test_quantise_refuses(bad):
    assert _quantise(**bad) == ARG


def test_quantise_of_nothing_is_fine():
    assert _quantise(rows=0, lds=1) == 0 and _quantise(cols=0) == 0


def _gemm(m=4, n=4, k=4, A=one, fa=b.E4M3, lda=16, SA=one, ldsa=4, ba=1, B=one, fb=b.E4M3, ldb=16, SB=one, ldsb=4, bb=1, C=null, ldc=4,
          D=one, type=b.BF16, ldd=4):
    return b.lib().gemm2m_fp8_gemm(m, n, k, A, fa, lda, SA, ldsa, ba, B, fb, ldb, SB, ldsb, bb, C, ldc, D, type, ldd, null)


@pytest.mark.parametrize("bad", [dict(m=-1), dict(n=-1), dict(k=-1), dict(lda=20), dict(lda=0), dict(k=17), dict(ldb=8), dict(A=8), dict(B=300),
                                 dict(A=null), dict(B=null), dict(SA=null), dict(SB=null), dict(D=null), dict(ldsa=3), dict(ldsb=3),
                                 dict(ba=2), dict(bb=0), dict(fa=b.BF16), dict(fb=5), dict(type=b.E4M3), dict(ldd=3), dict(C=one + 256, ldc=3),
                                 dict(C=one, ldc=8, ldd=4), dict(m=2 ** 31)])
def test_product_refuses(bad):
    assert _gemm(**bad) == ARG


def test_product_of_nothing_is_fine():
    assert _gemm(m=0, A=null, SA=null) == 0 and _gemm(n=0, B=null, SB=null, D=null) == 0


def _ns(batch=1, m=4, n=4, G=one, type=b.F32, ldg=4, sg=16, O=one, ldo=4, so=16, steps=5, coeffs=null, eps=1e-7):
    return b.lib().gemm2m_newton_schulz(batch, m, n, G, type, ldg, sg, O, ldo, so, steps, coeffs, ctypes.c_float(eps), null)


@pytest.mark.parametrize("bad", [dict(batch=-1), dict(batch=65536), dict(m=-1), dict(n=-1), dict(m=2 ** 20 + 1), dict(ldg=3), dict(ldo=3), dict(type=b.E5M2),
                                 dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(eps=float("nan")), dict(G=null), dict(O=null),
                                 dict(batch=2, so=15), dict(batch=2, sg=-1)])
def test_newton_schulz_refuses(bad):
    assert _ns(**bad) == ARG


def test_newton_schulz_of_nothing_is_fine():
    assert _ns(batch=0) == 0 and _ns(m=0) == 0 and _ns(n=0, ldg=1) == 0


def test_workspace_sizes():
    L = b.lib()
    assert L.gemm2m_workspace_bytes(b.OP_FP8_GEMM, 0, 0, 0, 0) >= 256
    assert L.gemm2m_workspace_bytes(b.OP_FP8_GEMM, -1, 0, 0, 0) == 0
    assert L.gemm2m_workspace_bytes(b.OP_NEWTON_SCHULZ, 100, 200, 70000, 0) == 0
    assert L.gemm2m_workspace_bytes(b.OP_NEWTON_SCHULZ, -1, 200, 1, 0) == 0
    w1, w3 = (L.gemm2m_workspace_bytes(b.OP_NEWTON_SCHULZ, 300, 200, k, 0) for k in (1, 3))
    planes = 2 * 2 * 2 * 300 * 200 + 2 * 2 * 200 * 200      # the iterate twice in two 16-bit planes, two squares
    assert w1 >= planes and w3 >= 3 * planes and w3 <= 3 * w1
    with pytest.raises(b.Gemm2mError):                       # no stages to look at
        b.workspace_layout(b.OP_FP8_GEMM, 4, 4, 4, 1)


def test_binding_refuses_what_the_library_could_not_see():
    x = torch.zeros(4, 4)
    with pytest.raises(ValueError):
        b.fp8_quantise(x, *b.fp8_empty(4, 4, device="cpu"))
    with pytest.raises(ValueError):
        b.fp8_gemm(x, x, x, x, x)
    with pytest.raises(ValueError):
        b.newton_schulz(x, x)
    q, s = b.fp8_empty(5, 300, device="cpu")
    assert q.shape == (5, 300) and q.stride(0) % 16 == 0 and s.shape == (5, 3) and s.stride(0) == 1
    q, s = b.fp8_empty(300, 5, b.E5M2, 128, device="cpu")
    assert q.dtype == torch.float8_e5m2 and s.shape == (3, 1)

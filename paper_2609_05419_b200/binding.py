"""Thin ctypes binding of the gemm2m C-ABI library (include/gemm2m.h): same entry-point names, argument
marshalling only.  Matrices are torch CUDA tensors viewed column-major (stride 1 along the first dimension);
torch is used for device memory and streams, every step of the computation runs in the library's kernels.

There is no fallback: if libgemm2m.so has not been built (``python -m paper_2609_05419_b200.build``) or cannot
be loaded, every call raises.
"""
from __future__ import annotations

import ctypes
import os
from array import array as _array

OP_GAUSSIAN_INT, OP_ZGEMM, OP_CGEMM, OP_ZHERK, OP_ZHER2K, OP_DSYRK, OP_DSYR2K, OP_DGEMM_OZAKI2 = 0, 1, 2, 3, 4, 5, 6, 7
OP_ZGEMM_EISENSTEIN = 8
OP_ZGEMM_HOST = 9
OP_FP8_GEMM, OP_NEWTON_SCHULZ = 10, 11
OP_RMS_NORM, OP_RMS_NORM_BACKWARD, OP_CLIP_GRADIENTS, OP_ADAPTER_ADD = 12, 13, 14, 15
F32, F16, BF16, E4M3, E5M2 = 0, 1, 2, 3, 4              # gemm2m_type
OK = 0
ERR_ARG, ERR_NMOD, ERR_WORKSPACE, ERR_CUDA, ERR_ARCH, ERR_DEVICE_TIMEOUT = 1, 2, 3, 4, 5, 6     # gemm2m_status

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgemm2m.so")
_lib = None


class Gemm2mError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        name = lib().gemm2m_status_string(status).decode()
        extra = ""
        if name == "GEMM2M_ERR_CUDA":
            extra = " (" + lib().gemm2m_last_cuda_error().decode() + ")"
        super().__init__(f"{where}: {name}{extra}")


class Layout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in
                ("off_exp_a", "off_exp_b", "off_apm", "off_bpm", "off_cpm", "kp", "ldp", "total_bytes")]


def lib():
    """The loaded C-ABI library.  Raises if it is missing: there is no CPU or library fallback."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_05419_b200.build` (needs nvcc)")
    L = ctypes.CDLL(LIB_PATH)
    i64, i32, vp, sz = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    L.gemm2m_status_string.restype = ctypes.c_char_p
    L.gemm2m_status_string.argtypes = [i32]
    L.gemm2m_last_cuda_error.restype = ctypes.c_char_p
    L.gemm2m_max_moduli.restype = i32
    L.gemm2m_max_2m_moduli.restype = i32
    L.gemm2m_modulus.argtypes = [i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.gemm2m_workspace_bytes.restype = sz
    L.gemm2m_workspace_bytes.argtypes = [i32, i64, i64, i64, i32]
    L.gemm2m_set_workspace.argtypes = [vp, sz]
    L.gemm2m_gaussian_int.argtypes = [i64, i64, i64, vp, vp, i64, vp, vp, i64, vp, vp, i64, i32, vp]
    L.zgemm2m.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, i32, vp]
    L.cgemm2m.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, i32, vp]
    L.zgemm2m_host.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, i32, vp]
    ex = [ctypes.c_char, ctypes.c_char, i64, i64, i64, vp, vp, i64, vp, i64, vp, vp, i64, i32, vp]
    L.zgemm2m_ex.argtypes = ex
    L.cgemm2m_ex.argtypes = ex
    L.zgemm2m_eisenstein.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, i32, vp]
    L.zgemm2m_eisenstein_ex.argtypes = ex
    L.gemm2m_max_eisenstein_moduli.restype = i32
    L.gemm2m_eisenstein_modulus.argtypes = [i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.gemm2m_debug_tables_eisenstein.argtypes = [i32, i64] + [vp] * 10
    L.zherk2m.argtypes = [i64, i64, vp, i64, vp, i64, i32, vp]
    L.dsyrk2m.argtypes = [i64, i64, vp, i64, vp, i64, i32, vp]
    L.zher2k2m.argtypes = [i64, i64, vp, i64, vp, i64, vp, i64, i32, vp]
    L.dsyr2k2m.argtypes = [i64, i64, vp, i64, vp, i64, vp, i64, i32, vp]
    L.gemm2m_device_status.argtypes = [vp]
    L.gemm2m_zscale_exponents_static.argtypes = [i64, i64, vp, i64, i32, vp, vp]
    L.gemm2m_set_profiling.argtypes = [i32]
    L.gemm2m_phase_ms.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i32)]
    L.gemm2m_last_launch_count.argtypes = [ctypes.POINTER(i32)]
    L.gemm2m_workspace_layout.argtypes = [i32, i64, i64, i64, i32, ctypes.POINTER(Layout)]
    L.gemm2m_debug_set_gemm_kernel.argtypes = [i32]
    L.gemm2m_debug_wait_selftest.argtypes = [ctypes.c_uint64, vp]
    L.gemm2m_debug_newton_schulz_wait_ns.argtypes, L.gemm2m_debug_newton_schulz_wait_ns.restype = [i64] * 3, ctypes.c_uint64
    L.gemm2m_debug_set_panels.argtypes = [i32]
    L.dgemm_ozaki2.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, i32, vp]
    L.gemm2m_debug_tables_real.argtypes = [i32, i64] + [vp] * 10
    L.gemm2m_set_scaling.argtypes = [i32]
    L.gemm2m_debug_tables.argtypes = [i32, i64, i32, vp, vp, vp, vp, vp, vp]
    L.gemm2m_debug_residue_reduction.argtypes = [i32, vp, vp, vp, vp, vp]
    L.gemm2m_debug_post_operands.argtypes = [i32, i32, vp, vp, vp]
    L.gemm2m_fp8_quantise.argtypes = [i64, i64, vp, i32, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp]
    L.gemm2m_fp8_gemm.argtypes = [i64, i64, i64] + [vp, i32, i64, vp, i64, i32] * 2 + [vp, i64, vp, i32, i64, vp]
    L.gemm2m_newton_schulz.argtypes = [i64, i64, i64, vp, i32, i64, i64, vp, i64, i64, i32, vp, ctypes.c_float, vp]
    L.gemm2m_rms_norm.argtypes = [i64, i64, vp, i32, i64, vp, i64, vp, i32, ctypes.c_float] + [vp, i64] * 2 + [i32] + [vp, i64] * 4 + [vp, vp]
    L.gemm2m_rms_norm_backward.argtypes = [i64, i64, vp, i32, i64, vp, i64, vp, i32, vp, vp, i64, vp, i64, vp, i32, vp]
    L.gemm2m_clip_gradients.argtypes = [i64] + [vp] * 7 + [ctypes.c_float, ctypes.c_float, vp, vp]
    L.gemm2m_adapter_add.argtypes = [i64, i64, i64, i32, i32, vp, i32, i64] + [vp, i64, i64] * 2 + [vp] * 3 + [vp, i64, vp, i32, i64, vp]
    _lib = L
    return L


def _check(status, where):
    if status != OK:
        raise Gemm2mError(status, where)


_raw_device = _raw_stream = None


def _current_device():
    """Index of torch's current device, by torch's own look-up (0.1 us) once it is initialised."""
    global _raw_device
    if _raw_device is None:
        import torch
        device = getattr(torch._C, "_cuda_getDevice", None)
        if not device or not torch.cuda.is_initialized():
            return torch.cuda.current_device()
        _raw_device = device
    return _raw_device()


def _current_stream(device=None):
    """Handle of torch's current stream on the current device.  torch's own look-up by device index takes 0.1 us, a Stream object 3 us."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if not raw or not torch.cuda.is_initialized():
            return torch.cuda.current_stream().cuda_stream
        _raw_stream = raw
    return _raw_stream(_current_device() if device is None else device)


def _stream_ptr(stream):
    if stream is None:
        return ctypes.c_void_p(_current_stream())
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _launch_device(t, name):
    """Index of the device that a call with `t` runs on: the current one, which `t` has to lie on."""
    device = t.get_device()                         # (-1: not a CUDA tensor)
    if device < 0 or device != _current_device():
        raise ValueError(f"{name}: need a CUDA tensor on the current device")
    return device


def _colmajor(t, name):
    """(pointer, rows, cols, leading dimension) of a 2-D CUDA tensor stored column-major."""
    if t.dim() != 2:
        raise ValueError(f"{name}: need a 2-D CUDA tensor")
    _launch_device(t, name)
    rows, cols = t.shape
    if rows > 1 and t.stride(0) != 1:
        raise ValueError(f"{name}: need column-major storage (stride 1 along dim 0), e.g. torch.empty(cols, rows).t()")
    ld = t.stride(1) if cols > 1 else max(rows, 1)
    return ctypes.c_void_p(t.data_ptr()), rows, cols, ld if rows > 0 else max(ld, 1)      # (0: an expanded row, which the library refuses)


def max_moduli():
    return int(lib().gemm2m_max_moduli())


def max_2m_moduli():
    return int(lib().gemm2m_max_2m_moduli())


def modulus(j):
    m, s = ctypes.c_int(), ctypes.c_int()
    _check(lib().gemm2m_modulus(j, ctypes.byref(m), ctypes.byref(s)), "gemm2m_modulus")
    return m.value, s.value


def workspace_bytes(op, m, n, k, nmod):
    return int(lib().gemm2m_workspace_bytes(op, m, n, k, nmod))


def workspace_layout(op, m, n, k, nmod):
    lay = Layout()
    _check(lib().gemm2m_workspace_layout(op, m, n, k, nmod, ctypes.byref(lay)), "gemm2m_workspace_layout")
    return {name: getattr(lay, name) for name, _ in Layout._fields_}


def set_workspace(tensor):
    """Register a torch uint8 CUDA tensor (kept alive by the caller) as the library's workspace on the current device; None unregisters."""
    if tensor is None:
        _check(lib().gemm2m_set_workspace(None, 0), "gemm2m_set_workspace")
    else:
        _launch_device(tensor, "workspace")
        _check(lib().gemm2m_set_workspace(ctypes.c_void_p(tensor.data_ptr()), tensor.numel() * tensor.element_size()),
               "gemm2m_set_workspace")


def gemm2m_gaussian_int(Ar, Ai, Br, Bi, Cr, Ci, nmod, stream=None):
    pa, m, k, lda = _colmajor(Ar, "Ar")
    pai, _, _, ldai = _colmajor(Ai, "Ai")
    pb, k2, n, ldb = _colmajor(Br, "Br")
    pbi, _, _, ldbi = _colmajor(Bi, "Bi")
    pc, _, _, ldc = _colmajor(Cr, "Cr")
    pci, _, _, ldci = _colmajor(Ci, "Ci")
    if k != k2 or Ai.shape != Ar.shape or Bi.shape != Br.shape or Cr.shape != (m, n) or Ci.shape != (m, n):
        raise ValueError("shape mismatch")
    if (lda, ldb, ldc) != (ldai, ldbi, ldci):
        raise ValueError("real and imaginary planes must share their leading dimension")
    _check(lib().gemm2m_gaussian_int(m, n, k, pa, pai, lda, pb, pbi, ldb, pc, pci, ldc, nmod, _stream_ptr(stream)),
           "gemm2m_gaussian_int")


def _xgemm(fn, name, A, B, C, nmod, stream):
    pa, m, k, lda = _colmajor(A, "A")
    pb, k2, n, ldb = _colmajor(B, "B")
    pc, mc, nc, ldc = _colmajor(C, "C")
    if k != k2 or (mc, nc) != (m, n):
        raise ValueError("shape mismatch")
    _check(fn(m, n, k, pa, lda, pb, ldb, pc, ldc, nmod, _stream_ptr(stream)), name)


def zgemm2m(A, B, C, nmod=16, stream=None):
    _xgemm(lib().zgemm2m, "zgemm2m", A, B, C, nmod, stream)


def _colmajor_host(t, name):
    """(pointer, rows, cols, leading dimension) of a 2-D CPU tensor stored column-major."""
    if t.dim() != 2 or t.is_cuda:
        raise ValueError(f"{name}: need a 2-D CPU tensor")
    rows, cols = t.shape
    if rows > 1 and t.stride(0) != 1:
        raise ValueError(f"{name}: need column-major storage (stride 1 along dim 0), e.g. torch.empty(cols, rows).t()")
    ld = t.stride(1) if cols > 1 else max(rows, 1)
    return ctypes.c_void_p(t.data_ptr()), rows, cols, ld if rows > 0 else max(ld, 1)      # (0: an expanded row, which the library refuses)


def zgemm2m_host(A, B, C, nmod=16, stream=None):
    """C = A B with A, B, C complex128 CPU tensors (column-major views; pinned memory lets the copies overlap the kernels).
    Asynchronous on `stream`: C is valid, and A, B may be changed, once the stream has completed."""
    pa, m, k, lda = _colmajor_host(A, "A")
    pb, k2, n, ldb = _colmajor_host(B, "B")
    pc, mc, nc, ldc = _colmajor_host(C, "C")
    if k != k2 or (mc, nc) != (m, n):
        raise ValueError("shape mismatch")
    _check(lib().zgemm2m_host(m, n, k, pa, lda, pb, ldb, pc, ldc, nmod, _stream_ptr(stream)), "zgemm2m_host")


def cgemm2m(A, B, C, nmod=7, stream=None):
    _xgemm(lib().cgemm2m, "cgemm2m", A, B, C, nmod, stream)


def _xgemm_ex(fn, name, ctype, transa, transb, alpha, A, B, beta, C, nmod, stream):
    """C = alpha op(A) op(B) + beta C; A, B as stored (column-major views), trans in 'N', 'T', 'C'."""
    pa, ra, ca, lda = _colmajor(A, "A")
    pb, rb, cb, ldb = _colmajor(B, "B")
    pc, m, n, ldc = _colmajor(C, "C")
    ma, ka = (ra, ca) if transa in "Nn" else (ca, ra)
    kb, nb = (rb, cb) if transb in "Nn" else (cb, rb)
    if ka != kb or (ma, nb) != (m, n):
        raise ValueError("shape mismatch")
    pair = lambda z: None if z is None else (ctype * 2)(complex(z).real, complex(z).imag)
    al, be = pair(alpha), pair(beta)
    ptr = lambda a: None if a is None else ctypes.cast(a, ctypes.c_void_p)
    _check(fn(transa.encode(), transb.encode(), m, n, ka, ptr(al), pa, lda, pb, ldb, ptr(be), pc, ldc, nmod, _stream_ptr(stream)), name)


def zgemm2m_ex(transa, transb, alpha, A, B, beta, C, nmod=16, stream=None):
    _xgemm_ex(lib().zgemm2m_ex, "zgemm2m_ex", ctypes.c_double, transa, transb, alpha, A, B, beta, C, nmod, stream)


def cgemm2m_ex(transa, transb, alpha, A, B, beta, C, nmod=7, stream=None):
    _xgemm_ex(lib().cgemm2m_ex, "cgemm2m_ex", ctypes.c_float, transa, transb, alpha, A, B, beta, C, nmod, stream)


def zgemm2m_eisenstein(A, B, C, nmod=16, stream=None):
    """C = A B through the Eisenstein-integer variant (complex128 CUDA tensors, column-major views)."""
    _xgemm(lib().zgemm2m_eisenstein, "zgemm2m_eisenstein", A, B, C, nmod, stream)


def zgemm2m_eisenstein_ex(transa, transb, alpha, A, B, beta, C, nmod=16, stream=None):
    _xgemm_ex(lib().zgemm2m_eisenstein_ex, "zgemm2m_eisenstein_ex", ctypes.c_double, transa, transb, alpha, A, B, beta, C, nmod, stream)


def max_eisenstein_moduli():
    return int(lib().gemm2m_max_eisenstein_moduli())


def eisenstein_modulus(j):
    m, s = ctypes.c_int(0), ctypes.c_int(0)
    _check(lib().gemm2m_eisenstein_modulus(j, ctypes.byref(m), ctypes.byref(s)), "gemm2m_eisenstein_modulus")
    return m.value, s.value


def debug_tables_eisenstein(nmod, k):
    """Host-side constants of the Eisenstein variant (see gemm2m_debug_tables_eisenstein)."""
    import numpy as np
    scale = np.zeros(4, dtype=np.int32)
    gr = np.zeros((nmod, 5), dtype=np.float64)
    gi = np.zeros((nmod, 5), dtype=np.float64)
    mc = np.zeros(5, dtype=np.float64)
    nch = np.zeros(1, dtype=np.int32)
    y0 = np.zeros(nmod, dtype=np.int32)
    cq = np.zeros(nmod, dtype=np.float32)
    inv = np.zeros(nmod, dtype=np.float32)
    xmax = np.zeros(nmod, dtype=np.int32)
    margin = np.zeros(nmod, dtype=np.float64)
    ptr = lambda a: ctypes.c_void_p(a.ctypes.data)
    _check(lib().gemm2m_debug_tables_eisenstein(nmod, k, ptr(scale), ptr(gr), ptr(gi), ptr(mc), ptr(nch), ptr(y0), ptr(cq), ptr(inv),
                                                ptr(xmax), ptr(margin)), "gemm2m_debug_tables_eisenstein")
    return dict(Pt=int(scale[0]), PA=int(scale[1]), PB=int(scale[2]), ck=int(scale[3]), gr=gr, gi=gi, Mc=mc, nchunks=int(nch[0]),
                y0_bits=y0, cq=cq, inv_m=inv, xmax=xmax, margin=margin)


def dgemm_ozaki2(A, B, C, nmod=15, stream=None):
    """Real C = A B by the real Ozaki-II scheme (float64 CUDA tensors, column-major views)."""
    _xgemm(lib().dgemm_ozaki2, "dgemm_ozaki2", A, B, C, nmod, stream)


def zherk2m(A, C, nmod=16, stream=None):
    pa, n, k, lda = _colmajor(A, "A")
    pc, n1, n2, ldc = _colmajor(C, "C")
    if (n1, n2) != (n, n):
        raise ValueError("shape mismatch")
    _check(lib().zherk2m(n, k, pa, lda, pc, ldc, nmod, _stream_ptr(stream)), "zherk2m")


STATIC_MAX_ROWS = 65536


def zscale_exponents_static(A, e, nmod=16, stream=None):
    """Scale exponents of the rows of A (the ones zgemm2m uses for `nmod` moduli) into the int32 CUDA tensor `e`, for
    callers that may not allocate device memory: the library's built-in scratch replaces the workspace.  At most
    STATIC_MAX_ROWS rows; calls on one GPU must not overlap."""
    pa, m, k, lda = _colmajor(A, "A")
    if m > STATIC_MAX_ROWS:
        raise ValueError(f"zscale_exponents_static: {m} rows exceed the built-in scratch ({STATIC_MAX_ROWS} rows)")
    _launch_device(e, "e")
    if e.numel() != m or e.element_size() != 4 or not e.is_contiguous():
        raise ValueError("e: need a contiguous int32 CUDA tensor with one entry per row of A")
    _check(lib().gemm2m_zscale_exponents_static(m, k, pa, lda, nmod, ctypes.c_void_p(e.data_ptr()), _stream_ptr(stream)),
           "gemm2m_zscale_exponents_static")


def _rank(fn, name, A, B, C, nmod, stream):
    pa, n, k, lda = _colmajor(A, "A")
    pc, n1, n2, ldc = _colmajor(C, "C")
    if (n1, n2) != (n, n):
        raise ValueError("shape mismatch")
    if B is None:
        _check(fn(n, k, pa, lda, pc, ldc, nmod, _stream_ptr(stream)), name)
    else:
        pb, nb, kb, ldb = _colmajor(B, "B")
        if (nb, kb) != (n, k):
            raise ValueError("shape mismatch")
        _check(fn(n, k, pa, lda, pb, ldb, pc, ldc, nmod, _stream_ptr(stream)), name)


def zher2k2m(A, B, C, nmod=16, stream=None):
    _rank(lib().zher2k2m, "zher2k2m", A, B, C, nmod, stream)


def dsyrk2m(A, C, nmod=16, stream=None):
    _rank(lib().dsyrk2m, "dsyrk2m", A, None, C, nmod, stream)


def dsyr2k2m(A, B, C, nmod=16, stream=None):
    _rank(lib().dsyr2k2m, "dsyr2k2m", A, B, C, nmod, stream)


# ---- layer operators: row-major matrices (torch's default order), column-major scales ----

_type_codes = {}


def _type_of(t, name, allowed):
    if not _type_codes:
        import torch
        _type_codes.update({torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3, torch.float8_e5m2: E5M2})
    code = _type_codes.get(t.dtype, -1)
    if code not in allowed:
        raise ValueError(f"{name}: unsupported type {t.dtype}")
    return code


def _rowmajor(t, name, allowed, device):
    """(pointer, type code, rows, cols, leading dimension) of a 2-D CUDA tensor with contiguous rows."""
    shape = t.shape
    if len(shape) != 2 or t.get_device() != device:
        raise ValueError(f"{name}: need a 2-D CUDA tensor on the current device")
    rows, cols = shape
    ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError(f"{name}: need row-major storage (stride 1 along dim 1)")
    if rows <= 1 or cols == 0:                      # the stride of a single row, or of rows without entries, says nothing
        ld = (max(cols, 1) + 15) // 16 * 16
    return t.data_ptr(), _type_of(t, name, allowed), rows, cols, ld


def _scales(t, name, rows, cols, device):
    """(pointer, leading dimension) of a column-major float32 scale matrix of the given shape."""
    if t.shape != (rows, cols) or t.get_device() != device:
        raise ValueError(f"{name}: need a CUDA tensor of shape {(rows, cols)} on the current device")
    _type_of(t, name, (F32,))
    step, ld = t.stride()
    if rows > 1 and step != 1:
        raise ValueError(f"{name}: need column-major storage (stride 1 along dim 0), e.g. torch.empty(cols, rows).t()")
    if cols <= 1 or rows == 0:                      # the stride of a single column says nothing
        return t.data_ptr(), max(rows, 1)
    if ld < rows:                                   # an expanded column of scales: the kernels read (or write) one column per block
        raise ValueError(f"{name}: columns of scales overlap (stride {ld} along dim 1, {rows} rows); store one scale per block")
    return t.data_ptr(), ld


def _stream_of(stream, device):
    return _current_stream(device) if stream is None else stream if isinstance(stream, int) else stream.cuda_stream


_FP8 = (E4M3, E5M2)
_FLOATS = (F32, F16, BF16)
_HALVES = (F16, BF16)
_int32 = None
_NO_FORM = (None, 0, None, 0)


def fp8_empty(rows, cols, fmt=E4M3, block_rows=1, device="cuda"):
    """Uninitialised (values, scales) for a rows x cols matrix, laid out as fp8_quantise and fp8_gemm take them."""
    import torch
    dtype = {E4M3: torch.float8_e4m3fn, E5M2: torch.float8_e5m2}[fmt]
    q = torch.empty((rows, -(-cols // 16) * 16), dtype=dtype, device=device)[:, :cols]
    return q, torch.empty((-(-cols // 128), -(-rows // block_rows)), dtype=torch.float32, device=device).t()


def fp8_quantise(X, Q=None, S=None, Qt=None, St=None, block_rows=1, stream=None):
    """X (row-major, float32 / float16 / bfloat16) to 8-bit values Q with scales S, and / or its transpose Qt with scales St."""
    device = _launch_device(X, "X")
    px, tx, rows, cols, ldx = _rowmajor(X, "X", _FLOATS, device)
    if block_rows not in (1, 128):
        raise ValueError("block_rows: need 1 or 128")
    fmt, form, form_t = None, _NO_FORM, _NO_FORM
    if Q is not None:
        pq, fmt, r, c, ldq = _rowmajor(Q, "Q", _FP8, device)
        if r != rows or c != cols or S is None:
            raise ValueError("Q, S: shape mismatch")
        form = (pq, ldq, *_scales(S, "S", rows if block_rows == 1 else -(-rows // 128), -(-cols // 128), device))
    if Qt is not None:
        pq, fmt_t, r, c, ldq = _rowmajor(Qt, "Qt", _FP8, device)
        if r != cols or c != rows or St is None or fmt not in (None, fmt_t):
            raise ValueError("Qt, St: shape or type mismatch")
        fmt = fmt_t
        form_t = (pq, ldq, *_scales(St, "St", cols if block_rows == 1 else -(-cols // 128), -(-rows // 128), device))
    if fmt is None or (Q is None and S is not None) or (Qt is None and St is not None):
        raise ValueError("need Q and S, or Qt and St, or all four")
    _check(lib().gemm2m_fp8_quantise(rows, cols, px, tx, ldx, fmt, block_rows, *form, *form_t, _stream_of(stream, device)), "gemm2m_fp8_quantise")


def fp8_gemm(A, SA, B, SB, D, C=None, a_block=1, b_block=128, stream=None):
    """D = C + A B^T with A (m x k), B (n x k) in 8 bits and their scales; D, C float32 / float16 / bfloat16 (C may be D)."""
    device = _launch_device(A, "A")
    pa, fa, m, k, lda = _rowmajor(A, "A", _FP8, device)
    pb, fb, n, k2, ldb = _rowmajor(B, "B", _FP8, device)
    pd, td, md, nd, ldd = _rowmajor(D, "D", _FLOATS, device)
    if k != k2 or (md, nd) != (m, n):
        raise ValueError("shape mismatch")
    if a_block not in (1, 128) or b_block not in (1, 128):
        raise ValueError("a_block, b_block: need 1 or 128")
    kb = -(-k // 128)
    sa, ldsa = _scales(SA, "SA", -(-m // a_block), kb, device)
    sb, ldsb = _scales(SB, "SB", -(-n // b_block), kb, device)
    pc, ldc = None, ldd
    if C is not None:
        pc, tc, mc, nc, ldc = _rowmajor(C, "C", _FLOATS, device)
        if (mc, nc) != (m, n) or tc != td:
            raise ValueError("C: need the shape and type of D")
    _check(lib().gemm2m_fp8_gemm(m, n, k, pa, fa, lda, sa, ldsa, a_block, pb, fb, ldb, sb, ldsb, b_block, pc, ldc, pd, td, ldd,
                                 _stream_of(stream, device)), "gemm2m_fp8_gemm")


def newton_schulz(G, O, steps=5, coeffs=None, eps=1e-7, stream=None):
    """O (bfloat16) = G orthogonalised by Newton-Schulz steps; 2-D, or 3-D for a batch.  coeffs: (a, b, c), or one such per step."""
    device = _launch_device(G, "G")
    if G.dim() not in (2, 3) or O.get_device() != device or O.shape != G.shape:
        raise ValueError("G, O: need CUDA tensors of the same 2-D or 3-D shape on the current device")
    tg = _type_of(G, "G", _FLOATS)
    _type_of(O, "O", (BF16,))
    batch = G.shape[0] if G.dim() == 3 else 1
    m, n = G.shape[-2:]
    if n > 1 and (G.stride(-1) != 1 or O.stride(-1) != 1):
        raise ValueError("G, O: need row-major storage (stride 1 along the last dim)")
    ld = lambda t: t.stride(-2) if m > 1 else max(n, 1)
    stride = lambda t: t.stride(0) if batch > 1 and t.dim() == 3 else m * max(n, 1)
    co = None
    if coeffs is not None:
        first = coeffs[0]
        rows = [coeffs] * steps if not hasattr(first, "__len__") or getattr(first, "ndim", 1) == 0 else list(coeffs)      # (an entry of a tensor has both)
        if len(rows) != steps or any(len(r) != 3 for r in rows):
            raise ValueError("coeffs: need (a, b, c), or one such per step")
        co = ctypes.cast((ctypes.c_float * (3 * steps))(*[float(v) for r in rows for v in r]), ctypes.c_void_p)
    _check(lib().gemm2m_newton_schulz(batch, m, n, G.data_ptr(), tg, ld(G), stride(G), O.data_ptr(), ld(O), stride(O), steps, co, eps,
                                      _stream_of(stream, device)), "gemm2m_newton_schulz")


def _like(t, name, like, shape, device):
    """(pointer, leading dimension) of a matrix that has to have this shape and the type of `like`, (None, 0) for None."""
    if t is None:
        return None, 0
    if t.shape != shape or t.dtype is not like.dtype or t.get_device() != device:
        raise ValueError(f"{name}: need a CUDA tensor of shape {tuple(shape)} and type {like.dtype} on the current device")
    ld, step = t.stride()
    rows, cols = shape
    if step != 1 and cols > 1:
        raise ValueError(f"{name}: need row-major storage (stride 1 along dim 1)")
    if rows <= 1 or cols == 0:
        ld = (max(cols, 1) + 15) // 16 * 16
    return t.data_ptr(), ld


def _vector(t, name, size, allowed, device):
    """(pointer, type code) of a contiguous vector, (None, F32) for None."""
    if t is None:
        return None, F32
    if t.shape != (size,) or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name}: need a contiguous CUDA tensor of {size} entries on the current device")
    return t.data_ptr(), _type_of(t, name, allowed)


def _fp8_form(Q, S, names, rows, cols, device):
    """(format or None, (pointer, ld, scales, ld)) of an 8-bit form with 1 x 128 blocks that may be absent."""
    if Q is None and S is None:
        return None, _NO_FORM
    if Q is None or S is None:
        raise ValueError(f"{names}: need both or neither")
    p, fmt, r, c, ld = _rowmajor(Q, names, _FP8, device)
    if (r, c) != (rows, cols):
        raise ValueError(f"{names}: shape mismatch")
    return fmt, (p, ld, *_scales(S, names, rows, -(-cols // 128), device))


def rms_norm(X, W=None, R=None, H=None, Y=None, Q=None, S=None, Qt=None, St=None, rstd=None, eps=1e-6, stream=None):
    """Root-mean-square norm of the rows of H = X + R with weights W, into any of H, Y (type of X), 8-bit Q with scales S, the
    transposed Qt with St (both as fp8_empty lays them out), rstd (float32, one per row)."""
    device = _launch_device(X, "X")
    px, tx, rows, cols, ldx = _rowmajor(X, "X", _FLOATS, device)
    shape = X.shape
    pr, ldr = _like(R, "R", X, shape, device)
    ph, ldh = _like(H, "H", X, shape, device)
    py, ldy = _like(Y, "Y", X, shape, device)
    pw, tw = _vector(W, "W", cols, _FLOATS, device)
    fmt, form = _fp8_form(Q, S, "Q, S", rows, cols, device)
    fmt_t, form_t = _fp8_form(Qt, St, "Qt, St", cols, rows, device)
    if fmt is not None and fmt_t is not None and fmt != fmt_t:
        raise ValueError("Q, Qt: types differ")
    fmt = fmt if fmt is not None else fmt_t if fmt_t is not None else E4M3
    _check(lib().gemm2m_rms_norm(rows, cols, px, tx, ldx, pr, ldr, pw, tw, eps, ph, ldh, py, ldy, fmt, *form, *form_t,
                                 _vector(rstd, "rstd", rows, (F32,), device)[0], _stream_of(stream, device)), "gemm2m_rms_norm")


def rms_norm_backward(dY, H, W, rstd, dX, dR=None, dW=None, add=False, stream=None):
    """dX = the gradient of rms_norm's X (and R) from dY, joined with dR; dW (float32) = the gradient of W, added to dW for add=True.
    H and rstd as rms_norm left them; W None: ones."""
    device = _launch_device(dY, "dY")
    pg, tg, rows, cols, ldg = _rowmajor(dY, "dY", _FLOATS, device)
    shape = dY.shape
    if H is None or dX is None or rstd is None:
        raise ValueError("need H, rstd and dX")
    ph, ldh = _like(H, "H", dY, shape, device)
    px, ldx = _like(dX, "dX", dY, shape, device)
    pr, ldr = _like(dR, "dR", dY, shape, device)
    pw, tw = _vector(W, "W", cols, _FLOATS, device)
    _check(lib().gemm2m_rms_norm_backward(rows, cols, pg, tg, ldg, ph, ldh, pw, tw, _vector(rstd, "rstd", rows, (F32,), device)[0], pr, ldr, px, ldx,
                                          _vector(dW, "dW", cols, (F32,), device)[0], 1 if add else 0, _stream_of(stream, device)), "gemm2m_rms_norm_backward")


def _rows_of(t, name):
    """(rows, columns, leading dimension) of a tensor of any shape: dense in any order of its axes, or 2-D with rows apart."""
    if t.is_contiguous():
        size = t.numel()
        return 1, size, size
    shape, strides = t.shape, t.stride()
    if len(shape) == 2 and strides[1] == 1 and strides[0] >= shape[1]:
        return shape[0], shape[1], strides[0]
    dense = 1
    for stride, size in sorted(zip(strides, shape)):
        if size > 1:
            if stride != dense:
                raise ValueError(f"{name}: need tensors that are dense, or 2-D with contiguous rows")
            dense *= size
    return 1, dense, dense


def _dtypes_of(tensors, name, device):
    if any([t.get_device() != device for t in tensors]):
        raise ValueError(f"{name}: need CUDA tensors on the current device")
    return [t.dtype for t in tensors]


def clip_gradients(grads, max_norm, out=None, norm=None, eps=1e-6, stream=None):
    """Common 2-norm of a list of tensors (float32 / float16 / bfloat16) into `norm` (float32, one entry), and the tensors times
    min(1, max_norm / (norm + eps)), in place or into the list `out` (of the same types, shapes and orders of axes, or contiguous both and as many entries).
    max_norm = inf: the norm alone, unless there is an `out`."""
    grads = list(grads)
    count = len(grads)
    device = _current_device()
    if norm is not None:
        if norm.numel() != 1 or norm.get_device() != device:
            raise ValueError("norm: need a CUDA tensor of one entry on the current device")
        _type_of(norm, "norm", (F32,))
    dtypes = _dtypes_of(grads, "grads", device)
    if count:
        _type_of(grads[0], "grads", _FLOATS)        # (fills the table of codes)
    types = [_type_codes.get(d, -1) for d in dtypes]
    if count and (min(types) < F32 or max(types) > BF16):
        raise ValueError("grads: unsupported type")
    contiguous = all([t.is_contiguous() for t in grads])
    if out is not None:
        out = list(out)
        if _dtypes_of(out, "out", device) != dtypes:
            raise ValueError("out: need as many tensors as grads, of their types")
        contiguous = contiguous and all([t.is_contiguous() for t in out])
    # host arrays for the library: 64-bit numbers, one array for each argument
    array = lambda values: _array("q", values)
    address = lambda a: a.buffer_info()[0]
    if contiguous:
        rows, cols = array([1]) * count, array([t.numel() for t in grads])
        if out is not None and array([t.numel() for t in out]) != cols:
            raise ValueError("out: need the shapes of grads")
        lds = ld_out = cols
    else:
        walks, walks_out = [], []
        for g, o in zip(grads, grads if out is None else out):
            if g.shape != o.shape:
                raise ValueError("out: need the shapes of grads")
            walk, walk_out = _rows_of(g, "grads"), _rows_of(o, "out")
            if walk != walk_out or any(size > 1 and a != c for size, a, c in zip(g.shape, g.stride(), o.stride())):
                # the same order of entries, with rows of their own distance
                if g.dim() != 2 or any(t.shape[1] > 1 and t.stride(1) != 1 for t in (g, o)):
                    raise ValueError("out: need the order of the gradient's axes in memory")
                m, n = g.shape
                walk, walk_out = ((m, n, t.stride(0) if m > 1 else n) for t in (g, o))
            walks.append(walk)
            walks_out.append(walk_out)
        rows, cols, lds = (array([w[k] for w in walks]) for k in range(3))
        ld_out = array([w[2] for w in walks_out])
    types = _array("i", types)
    pointers = array([t.data_ptr() for t in grads])
    p_out = None if out is None else array([t.data_ptr() for t in out])
    _check(lib().gemm2m_clip_gradients(count, address(pointers), p_out and address(p_out), address(types), address(rows), address(cols), address(lds),
                                       None if out is None else address(ld_out), max_norm, eps, None if norm is None else norm.data_ptr(), _stream_of(stream, device)),
           "gemm2m_clip_gradients")


def _stack(t, name, like, device):
    """(pointer, matrices, rows, cols, leading dimension, stride) of a 3-D CUDA tensor of row-major matrices of the type of `like`."""
    shape = t.shape
    if len(shape) != 3 or t.get_device() != device or t.dtype is not like.dtype:
        raise ValueError(f"{name}: need a 3-D CUDA tensor of type {like.dtype} on the current device")
    many, rows, cols = shape
    stride, ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError(f"{name}: need row-major storage (stride 1 along the last dim)")
    if rows <= 1 or cols == 0:
        ld = max(cols, 1)
    return t.data_ptr(), many, rows, cols, ld, stride if many > 1 else rows * max(cols, 1)


def _indexes(t, name, size, device):
    """Pointer of a contiguous vector of 32-bit whole numbers."""
    global _int32
    if _int32 is None:
        import torch
        _int32 = torch.int32
    if t.shape != (size,) or t.dtype is not _int32 or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name}: need a contiguous int32 CUDA tensor of {size} entries on the current device")
    return t.data_ptr()


def adapter_add(X, A, B, index, D, C=None, scales=None, ranks=None, stream=None):
    """D[t] = C[t] + scales[a] (X[t] A[a]^T) B[a]^T with a = index[t] (int32; no adapter where it is not an index of A): X tokens x k,
    A adapters x rank x k, B adapters x n x rank in float16 / bfloat16; D, C float32 / float16 / bfloat16 (C may be D, or None for zero).
    ranks (int32): how many rows of A[a] and columns of B[a] are in use."""
    device = _launch_device(X, "X")
    px, tx, tokens, k, ldx = _rowmajor(X, "X", _HALVES, device)
    pa, many, rank, k2, lda, stride_a = _stack(A, "A", X, device)
    pb, many2, n, rank2, ldb, stride_b = _stack(B, "B", X, device)
    pd, td, md, nd, ldd = _rowmajor(D, "D", _FLOATS, device)
    if k2 != k or many2 != many or rank2 != rank or md != tokens or nd != n:
        raise ValueError("shape mismatch")
    pc, ldc = _like(C, "C", D, D.shape, device)
    pi = _indexes(index, "index", tokens, device)
    pr = None if ranks is None else _indexes(ranks, "ranks", many, device)
    _check(lib().gemm2m_adapter_add(tokens, n, k, many, rank, px, tx, ldx, pa, lda, stride_a, pb, ldb, stride_b, pi,
                                    _vector(scales, "scales", many, (F32,), device)[0], pr, pc, ldc, pd, td, ldd, _stream_of(stream, device)),
           "gemm2m_adapter_add")


def device_status(stream=None):
    _check(lib().gemm2m_device_status(_stream_ptr(stream)), "gemm2m_device_status")


def set_profiling(enabled):
    _check(lib().gemm2m_set_profiling(1 if enabled else 0), "gemm2m_set_profiling")


def phase_ms():
    """Average per-call milliseconds of (scan, residues, GEMMs, post) over the profiled calls, and their number."""
    ms = (ctypes.c_float * 4)()
    calls = ctypes.c_int()
    _check(lib().gemm2m_phase_ms(ms, ctypes.byref(calls)), "gemm2m_phase_ms")
    return [float(x) for x in ms], calls.value


def last_launch_count():
    per = (ctypes.c_int * 4)()
    total = int(lib().gemm2m_last_launch_count(per))
    return total, [int(x) for x in per]


def debug_newton_schulz_wait_ns(batch, m, n):
    return int(lib().gemm2m_debug_newton_schulz_wait_ns(batch, m, n))


def debug_wait_selftest(budget_ns, stream=None):
    """Enqueue the bounded-wait self-test (see gemm2m_debug_wait_selftest)."""
    _check(lib().gemm2m_debug_wait_selftest(int(budget_ns), _stream_ptr(stream)), "gemm2m_debug_wait_selftest")


def debug_set_gemm_kernel(which):
    _check(lib().gemm2m_debug_set_gemm_kernel(which), "gemm2m_debug_set_gemm_kernel")


def set_scaling(mode):
    """0 = scale factors from the largest part of each row / column (default), 1 = from a bound of its 2-norm."""
    _check(lib().gemm2m_set_scaling(int(mode)), "gemm2m_set_scaling")


def debug_set_overlap(enabled):
    _check(lib().gemm2m_debug_set_overlap(1 if enabled else 0), "gemm2m_debug_set_overlap")


def debug_set_chained_launch(enabled):
    _check(lib().gemm2m_debug_set_chained_launch(1 if enabled else 0), "gemm2m_debug_set_chained_launch")


def debug_set_panels(max_panels):
    _check(lib().gemm2m_debug_set_panels(max_panels), "gemm2m_debug_set_panels")


def debug_tables(nmod, k, herk=False):
    """Host-side constants of the library for `nmod` moduli (see gemm2m_debug_tables)."""
    import numpy as np
    scale = np.zeros(4, dtype=np.int32)
    gr = np.zeros((nmod, 5), dtype=np.float64)
    gi = np.zeros((nmod, 5), dtype=np.float64)
    mc = np.zeros(5, dtype=np.float64)
    nch = np.zeros(1, dtype=np.int32)
    w = np.zeros((nmod, 16), dtype=np.int8)
    ptr = lambda a: ctypes.c_void_p(a.ctypes.data)
    _check(lib().gemm2m_debug_tables(nmod, k, 1 if herk else 0, ptr(scale), ptr(gr), ptr(gi), ptr(mc), ptr(nch), ptr(w)),
           "gemm2m_debug_tables")
    return dict(Pt=int(scale[0]), PA=int(scale[1]), PB=int(scale[2]), ck=int(scale[3]), gr=gr, gi=gi, Mc=mc,
                nchunks=int(nch[0]), res_w=w)


def debug_post_operands(nmod, eisenstein=False, herk=False):
    """Operand of the post-processing contraction (see gemm2m_debug_post_operands)."""
    import numpy as np
    dims = np.zeros(3, dtype=np.int32)
    consts = np.zeros(19, dtype=np.float64)
    ptr = lambda a: ctypes.c_void_p(a.ctypes.data)
    variant = 2 if herk else 1 if eisenstein else 0
    _check(lib().gemm2m_debug_post_operands(variant, nmod, None, ptr(dims), None), "gemm2m_debug_post_operands")
    digits = np.zeros((2, int(dims[0]), 24), dtype=np.uint8)
    _check(lib().gemm2m_debug_post_operands(variant, nmod, ptr(digits), ptr(dims), ptr(consts)), "gemm2m_debug_post_operands")
    return dict(planes=int(dims[0]), ks=int(dims[1]), nb=int(dims[2]), digits=digits, Mc=consts[0:6], off=consts[6:18].reshape(2, 6),
                inv_M=float(consts[18]))


def debug_residue_reduction(nmod):
    """Constants of the residue kernels' reduction modulo m_j (see gemm2m_debug_residue_reduction)."""
    import numpy as np
    y0 = np.zeros(nmod, dtype=np.int32)
    cq = np.zeros(nmod, dtype=np.float32)
    inv = np.zeros(nmod, dtype=np.float32)
    xmax = np.zeros(nmod, dtype=np.int32)
    margin = np.zeros(nmod, dtype=np.float64)
    ptr = lambda a: ctypes.c_void_p(a.ctypes.data)
    _check(lib().gemm2m_debug_residue_reduction(nmod, ptr(y0), ptr(cq), ptr(inv), ptr(xmax), ptr(margin)),
           "gemm2m_debug_residue_reduction")
    return dict(y0_bits=y0, cq=cq, inv_m=inv, xmax=xmax, margin=margin)


def debug_tables_real(nmod, k):
    """Host-side constants of the real scheme (see gemm2m_debug_tables_real)."""
    import numpy as np
    mods = np.zeros(nmod, dtype=np.int32)
    scale = np.zeros(4, dtype=np.int32)
    g = np.zeros((nmod, 5), dtype=np.float64)
    mc = np.zeros(5, dtype=np.float64)
    nch = np.zeros(1, dtype=np.int32)
    y0 = np.zeros(nmod, dtype=np.int32)
    cq = np.zeros(nmod, dtype=np.float32)
    inv = np.zeros(nmod, dtype=np.float32)
    xmax = np.zeros(nmod, dtype=np.int32)
    margin = np.zeros(nmod, dtype=np.float64)
    ptr = lambda a: ctypes.c_void_p(a.ctypes.data)
    _check(lib().gemm2m_debug_tables_real(nmod, k, ptr(mods), ptr(scale), ptr(g), ptr(mc), ptr(nch), ptr(y0), ptr(cq), ptr(inv),
                                          ptr(xmax), ptr(margin)), "gemm2m_debug_tables_real")
    return dict(moduli=mods, Pt=int(scale[0]), PA=int(scale[1]), PB=int(scale[2]), ck=int(scale[3]), g=g, Mc=mc, nchunks=int(nch[0]),
                y0_bits=y0, cq=cq, inv_m=inv, xmax=xmax, margin=margin)

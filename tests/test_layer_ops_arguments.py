"""What the binding of the layer operators passes on to the library, and what it refuses: no GPU is touched, CPU tensors stand in for
CUDA ones and the library is replaced by a recorder."""
import ast
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2609_05419_b200 import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Standin:
    """A CPU tensor that says it is a CUDA one."""
    is_cuda = True

    def __init__(self, tensor, device=0):
        self.tensor, self.index = tensor, device

    def __getattr__(self, name):
        return getattr(self.tensor, name)

    def get_device(self):
        return self.index


@pytest.fixture
def calls(monkeypatch):
    """Calls that would have reached the library: (name, arguments) each."""
    seen = []

    class Recorder:
        def __getattr__(self, name):
            return lambda *args: seen.append((name, args)) or b.OK

    monkeypatch.setattr(b, "lib", Recorder)
    monkeypatch.setattr(b, "_current_stream", lambda *device: 0)
    monkeypatch.setattr(b, "_current_device", lambda: 0, raising=False)
    return seen


def matrix(rows, cols, block=1, **where):
    q, s = b.fp8_empty(rows, cols, b.E4M3, block, device="cpu")
    return Standin(q, **where), Standin(s, **where)


def dense(rows, cols, dtype=torch.float32, **where):
    return Standin(torch.zeros(rows, cols, dtype=dtype), **where)


# ------------------------------------------------------------------------------------- scales with a stride below their rows
# one scale per row for all of k, spelled as an expanded column: memory holds one column of scales, not one per block
@pytest.mark.parametrize("m", [1, 2, 300])
@pytest.mark.parametrize("side", ["A", "B"])
def test_product_refuses_expanded_scales(calls, m, side):
    k = 500
    qa, sa = matrix(m, k)
    qb, sb = matrix(m, k)
    one = Standin(torch.ones(m, 1).expand(m, 4))
    sa, sb = (one, sb) if side == "A" else (sa, one)
    with pytest.raises(ValueError):
        b.fp8_gemm(qa, sa, qb, sb, dense(m, m), b_block=1)
    assert not calls


@pytest.mark.parametrize("rows", [1, 300])
def test_quantise_refuses_to_write_expanded_scales(calls, rows):
    q, _ = matrix(rows, 500)
    with pytest.raises(ValueError):
        b.fp8_quantise(dense(rows, 500), q, Standin(torch.ones(rows, 1).expand(rows, 4)))
    if rows > 128:                                             # transposed form with a scale per 128 x 128: 4 x 3 of them
        qt, _ = matrix(500, rows, 128)
        with pytest.raises(ValueError):
            b.fp8_quantise(dense(rows, 500), None, None, qt, Standin(torch.ones(4, 1).expand(4, 3)), block_rows=128)
    assert not calls


def test_scales_pass_their_own_leading_dimension(calls):
    for rows, cols, want in ((300, 500, 300), (1, 500, 1), (300, 100, 300), (1, 1, 1)):
        q, s = matrix(rows, cols)
        b.fp8_quantise(dense(rows, cols), q, s)
        assert calls[-1][1][10] == want                        # lds
    wide = Standin(torch.zeros(4, 400).t()[:300])               # columns further apart than their rows
    b.fp8_quantise(dense(300, 500), matrix(300, 500)[0], wide)
    assert calls[-1][1][10] == 400


# ------------------------------------------------------------------------------------------------------------ sizes of nothing
# (in a process of its own: an arithmetic signal would end the test run)
@pytest.mark.parametrize("op", ["OP_NEWTON_SCHULZ", "OP_FP8_GEMM"])
def test_workspace_sizes_of_empty_matrices(op):
    code = ("from paper_2609_05419_b200 import binding as b\n"
            f"op = b.{op}\n"
            "print([b.workspace_bytes(op, *size, 1) for size in ((0, 8, 1), (8, 0, 1), (0, 0, 1), (0, 0, 0), (8, 8, 0), (8, 8, 1))])")
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert done.returncode == 0, (done.returncode, done.stderr)
    sizes = ast.literal_eval(done.stdout)
    assert all(256 <= v <= sizes[-1] for v in sizes)


# a batch without tokens: both forms of X, the forward product, and the weight gradient whose inner dimension is empty
@pytest.mark.parametrize("rows,cols", [(0, 40), (40, 0), (0, 0), (1, 0), (0, 1)])
def test_empty_matrices_have_leading_dimensions_that_the_library_takes(calls, rows, cols):
    q, s = matrix(rows, cols)
    qt, st = matrix(cols, rows)
    b.fp8_quantise(dense(rows, cols), q, s, qt, st)
    _, args = calls[-1]
    ldx, ldq, ldqt = args[4], args[8], args[12]
    assert ldx >= max(cols, 1) and ldq >= max(cols, 1) and ldq % 16 == 0 and ldqt >= max(rows, 1) and ldqt % 16 == 0
    for (a, sa), n in ((matrix(rows, cols), 24), (matrix(24, rows), 8)):
        m, k = a.shape
        bq, sb = matrix(n, k)
        b.fp8_gemm(a, sa, bq, sb, dense(m, n), C=dense(m, n), b_block=1)
        _, args = calls[-1]
        for ld, scales, count in ((args[5], args[7], m), (args[11], args[13], n)):
            assert ld >= max(k, 1) and ld % 16 == 0 and scales >= max(count, 1)
        assert args[16] >= n and args[19] >= n                  # ldc, ldd


# ------------------------------------------------------------------------------------------------ tensors on more than one device
def quantise_operands():
    return dense(300, 500), *matrix(300, 500), *matrix(500, 300)


def product_operands():
    return *matrix(300, 500), *matrix(200, 500), dense(300, 200), dense(300, 200)


def newton_schulz_operands():
    return dense(30, 50), dense(30, 50, torch.bfloat16)


def run(name, t):
    if name == "product":
        b.fp8_gemm(*t[:5], C=t[5], b_block=1)
    else:
        {"quantise": b.fp8_quantise, "newton_schulz": b.newton_schulz}[name](*t)


@pytest.mark.parametrize("name,make", [("quantise", quantise_operands), ("product", product_operands), ("newton_schulz", newton_schulz_operands)])
def test_every_operand_lies_on_the_current_device(calls, monkeypatch, name, make):
    run(name, make())
    assert len(calls) == 1
    for i in range(len(make())):
        for elsewhere in (1, -1):
            operands = make()
            operands[i].index = elsewhere
            with pytest.raises(ValueError):
                run(name, operands)
    operands = make()
    for t in operands:
        t.index = 1
    with pytest.raises(ValueError):
        run(name, operands)
    assert len(calls) == 1
    monkeypatch.setattr(b, "_current_device", lambda: 1)
    run(name, operands)
    assert len(calls) == 2


# ------------------------------------------------------------------------------------------------------- halves of an output form
def test_quantise_refuses_scales_without_their_values(calls):
    q, s = matrix(300, 500)
    qt, st = matrix(500, 300)
    x = dense(300, 500)
    for args in ((None, s, qt, st), (q, s, None, st), (q, None, qt, st), (q, s, qt, None), (None, s, None, None), ()):
        with pytest.raises(ValueError):
            b.fp8_quantise(x, *args)
    assert not calls


# ------------------------------------------------------------------------------------------------------- limits of device-side waits
# a CTA without tiles waits for a whole product, 2 s^2 l operations, at no less than 5e14 per second (a third of the 16-bit rate)
@pytest.mark.parametrize("batch,m,n", [(1, 1, 1), (1, 300, 200), (16, 1024, 1024), (1, 16384, 4096), (1, 40000, 130000), (1, 110000, 100000), (3, 65536, 20000)])
def test_newton_schulz_waits_outlast_a_step(batch, m, n):
    limit, product = b.debug_newton_schulz_wait_ns(batch, m, n) * 1e-9, 2.0 * min(m, n) ** 2 * max(m, n) * batch
    assert limit >= 1.0 + product / 5e14
    assert limit <= 2.5 + product / 5e13                           # and end all the same
    assert b.debug_newton_schulz_wait_ns(1, -1, 4) == 0


# ----------------------------------------------------------------------------------------------------------- coefficients as arrays
@pytest.mark.parametrize("steps", [3, 5])
@pytest.mark.parametrize("kind", [tuple, list, np.array, torch.tensor])
def test_newton_schulz_coefficients_in_any_container(calls, kind, steps):
    one, each = (1.5, -0.5, 0.25), [(i + 1.5, i - 0.5, i + 0.25) for i in range(steps)]
    for coeffs, rows in ((one, [one] * steps), (each, each)):
        b.newton_schulz(*newton_schulz_operands(), steps=steps, coeffs=kind(coeffs))
        passed = ctypes.cast(calls[-1][1][11], ctypes.POINTER(ctypes.c_float))
        assert [passed[i] for i in range(3 * steps)] == [v for row in rows for v in row]
    for bad in (one[:2], each[1:], [row[:2] for row in each]):
        with pytest.raises(ValueError):
            b.newton_schulz(*newton_schulz_operands(), steps=steps, coeffs=kind(bad))

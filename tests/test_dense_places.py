"""Dense layers of 8- and 16-bit operands: scales, addends and workspaces that begin where a result or an operand does are refused at the C ABI (no GPU:
a refused call launches nothing)."""
import ctypes

import pytest

from paper_2008_08272_b200 import binding
from paper_2008_08272_b200.binding import Matrix

F32, I8, BF16 = 1, 3, 16
UNSUPPORTED = 4


def mat(index, rows, cols, kind, ld=None):
    return Matrix((index + 1) << 24, rows, cols, ld or cols, kind, 0)


def at(m):
    return ctypes.c_void_p(m.data)


SCALE, WS = ctypes.c_void_p(1 << 40), ctypes.c_void_p(1 << 41)


def test_scale_of_quantised_rows():
    lib = binding.load()
    X, Q = mat(0, 4, 40, F32), mat(1, 4, 40, I8)
    for scale in (X, Q):
        assert lib.onnx_quantize_rows_run(X, Q, at(scale), None) == UNSUPPORTED


@pytest.mark.parametrize("which", range(3))
def test_result_in_the_place_of_a_vector(which):
    lib = binding.load()
    A, B, Y = mat(0, 4, 48, I8), mat(1, 30, 48, I8), mat(2, 4, 30, F32)
    vectors = [at(Y) if i == which else SCALE for i in range(3)]
    assert lib.onnx_gemm_int8_run(A, vectors[0], B, vectors[1], vectors[2], 0, Y, None, 0, None) == UNSUPPORTED
    assert lib.onnx_gated_int8_run(A, vectors[0], B, vectors[1], mat(3, 30, 48, I8), vectors[2], 0, Y, None, 0, None) == UNSUPPORTED


def test_workspace_in_the_place_of_a_tensor():
    """(rows of 41 elements do not begin at multiples of 16 bytes: a workspace is asked for)"""
    lib = binding.load()
    A, B, Y = mat(0, 4, 41, I8), mat(1, 30, 41, I8), mat(2, 4, 30, F32)
    for m in (A, B, Y):
        assert lib.onnx_gemm_int8_run(A, SCALE, B, SCALE, None, 0, Y, at(m), 1 << 30, None) == UNSUPPORTED
    W, H = mat(3, 30, 41, I8), mat(4, 4, 30, BF16)
    for m in (A, B, W, H):
        assert lib.onnx_gated_int8_run(A, SCALE, B, SCALE, W, SCALE, 0, H, at(m), 1 << 30, None) == UNSUPPORTED
    X, Wg, Wu, dH, G, U, dX, dWg, dWu = (mat(5 + i, *size, BF16) for i, size in enumerate([(4, 41)] + [(30, 41)] * 2 + [(4, 30)] * 3 + [(4, 41)] + [(30, 41)] * 2))
    for m in (X, Wg, Wu, dH, G, U):
        assert lib.onnx_gated_run(X, Wg, Wu, 0, dH, G, U, at(m), 1 << 30, None) == UNSUPPORTED
    for m in (X, Wg, Wu, dH, G, U, dX, dWg, dWu):
        assert lib.onnx_gated_backward_run(dH, X, Wg, Wu, G, U, 0, dX, dWg, dWu, at(m), 1 << 30, None) == UNSUPPORTED

"""What the dense layers of 8- and 16-bit operands refuse, at the C ABI (no GPU: a refused call launches nothing), and that the definitions the
GPU tests compare with have the gradients that differences give."""
import ctypes
import math

import pytest
import torch

import dense_reference as ref
from paper_2008_08272_b200 import binding
from paper_2008_08272_b200.binding import Matrix

F32, I8, F16, BF16 = 1, 3, 10, 16
NULL, ATTR, SHAPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5
_next = [1 << 20]


def mat(rows, cols, kind, ld=None, data=None, reserved=0):
    """A view at an address of its own (never read: the call is refused before anything is launched)."""
    if data is None:
        _next[0] += 1 << 24
        data = _next[0]
    return Matrix(data or None, rows, cols, cols if ld is None else ld, kind, reserved)


def change(m, **kw):
    n = Matrix(m.data, m.rows, m.cols, m.ld, m.type, m.reserved)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


SCALE = ctypes.c_void_p(1 << 40)
WS = ctypes.c_void_p(1 << 41)
BAD_VIEWS = [(dict(type=2), ATTR), (dict(reserved=1), ATTR), (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(ld=7), SHAPE),
             (dict(rows=(1 << 30) + 1), UNSUPPORTED), (dict(ld=1 << 31), UNSUPPORTED), (dict(data=None), NULL)]


def each_view(call, views, good):
    """Every view of a call spoilt in every way; a type that is none is refused in whatever order the checks come."""
    for name in views:
        for bad, status in BAD_VIEWS:
            got = call({**good, name: change(good[name], **bad)})
            # (a spoilt size disagrees with the other views' as well)
            assert got == status or (status == UNSUPPORTED and got == SHAPE), (name, bad, got)
        assert call({**good, name: None}) == NULL, name


def test_quantize_rows():
    lib = binding.load()
    good = dict(X=mat(4, 40, BF16), Q=mat(4, 40, I8))

    def call(a, scale=SCALE):
        return lib.onnx_quantize_rows_run(a["X"], a["Q"], scale, None)

    each_view(call, ("X", "Q"), good)
    assert call({**good, "X": mat(4, 40, I8)}) == ATTR and call({**good, "Q": mat(4, 40, F16)}) == ATTR
    assert call({**good, "Q": mat(4, 41, I8)}) == SHAPE and call({**good, "Q": mat(3, 40, I8)}) == SHAPE
    assert call(good, None) == NULL and call(good, ctypes.c_void_p(6)) == UNSUPPORTED
    assert call({**good, "X": change(good["X"], data=good["X"].data + 1)}) == UNSUPPORTED
    assert call({**good, "Q": change(good["Q"], data=good["X"].data)}) == UNSUPPORTED
    assert call(dict(X=mat(0, 40, BF16, data=0), Q=mat(0, 40, I8, data=0)), None) == 0


def test_gemm_int8():
    lib = binding.load()
    good = dict(A=mat(4, 40, I8), B=mat(30, 40, I8), Y=mat(4, 30, F32))

    def call(a, sa=SCALE, sb=SCALE, C=None, ws=WS, n=1 << 30):
        return lib.onnx_gemm_int8_run(a["A"], sa, a["B"], sb, C, 0, a["Y"], ws, n, None)

    each_view(call, ("A", "B", "Y"), good)
    for name, kind in (("A", BF16), ("B", F32), ("Y", I8)):
        assert call({**good, name: change(good[name], type=kind)}) == ATTR
    for name, size in (("A", (5, 40)), ("B", (30, 41)), ("Y", (4, 31)), ("B", (0, 40))):
        assert call({**good, name: mat(*size, good[name].type)}) == SHAPE
    assert call(good, sa=None) == NULL and call(good, sb=None) == NULL
    for k in ("sa", "sb", "C"):
        assert call(good, **{k: ctypes.c_void_p(258)}) == UNSUPPORTED
    assert call(dict(A=mat(4, 131072, I8), B=mat(30, 131072, I8), Y=mat(4, 30, F32))) == UNSUPPORTED
    assert call({**good, "Y": change(good["Y"], data=good["B"].data)}) == UNSUPPORTED
    assert call(dict(A=mat(0, 40, I8, data=0), B=good["B"], Y=mat(0, 30, F32, data=0)), sa=None) == 0


def test_gated():
    lib = binding.load()
    good = dict(X=mat(4, 40, BF16), Wg=mat(30, 40, BF16), Wu=mat(30, 40, BF16), H=mat(4, 30, BF16), G=mat(4, 30, BF16), U=mat(4, 30, BF16))

    def call(a, activation=0, ws=WS, n=1 << 30):
        return lib.onnx_gated_run(a["X"], a["Wg"], a["Wu"], activation, a["H"], a["G"], a["U"], ws, n, None)

    each_view(call, ("X", "Wg", "Wu", "H", "G", "U"), good)
    for name in good:
        for kind in (F32, F16, I8):
            assert call({**good, name: change(good[name], type=kind)}) == ATTR
    assert call({k: change(v, type=I8) for k, v in good.items()}) == ATTR
    assert call(good, activation=4) == ATTR and call(good, activation=-1) == ATTR
    for name, size in (("X", (5, 40)), ("Wg", (30, 41)), ("Wu", (31, 40)), ("H", (4, 31)), ("G", (3, 30)), ("U", (4, 29))):
        assert call({**good, name: mat(*size, BF16)}) == SHAPE
    for a, b in (("G", "U"), ("G", "H"), ("U", "H"), ("H", "X"), ("G", "X"), ("H", "Wg"), ("G", "Wg"), ("U", "Wu")):
        assert call({**good, a: change(good[a], data=good[b].data)}) == UNSUPPORTED
    assert call({**good, "H": change(good["H"], data=good["H"].data + 1)}) == UNSUPPORTED


def test_gated_int8():
    lib = binding.load()
    good = dict(A=mat(4, 40, I8), Wg=mat(30, 40, I8), Wu=mat(30, 40, I8), H=mat(4, 30, F16))

    def call(a, activation=0, scales=(SCALE,) * 3):
        return lib.onnx_gated_int8_run(a["A"], scales[0], a["Wg"], scales[1], a["Wu"], scales[2], activation, a["H"], WS, 1 << 30, None)

    each_view(call, ("A", "Wg", "Wu", "H"), good)
    assert call({**good, "H": change(good["H"], type=I8)}) == ATTR and call({**good, "Wu": change(good["Wu"], type=F16)}) == ATTR
    assert call({k: change(v, type=F16) for k, v in good.items()}) == ATTR and call(good, activation=7) == ATTR
    for i in range(3):
        assert call(good, scales=[None if j == i else SCALE for j in range(3)]) == NULL
        assert call(good, scales=[ctypes.c_void_p(2) if j == i else SCALE for j in range(3)]) == UNSUPPORTED
    assert call(dict(A=mat(4, 131072, I8), Wg=mat(30, 131072, I8), Wu=mat(30, 131072, I8), H=mat(4, 30, F16))) == UNSUPPORTED


def test_gated_backward():
    lib = binding.load()
    good = dict(dH=mat(4, 30, F16), X=mat(4, 40, F16), Wg=mat(30, 40, F16), Wu=mat(30, 40, F16), G=mat(4, 30, F16), U=mat(4, 30, F16),
                dX=mat(4, 40, F16), dWg=mat(30, 40, F16), dWu=mat(30, 40, F16))

    def call(a, activation=0, ws=WS, n=1 << 30):
        return lib.onnx_gated_backward_run(a["dH"], a["X"], a["Wg"], a["Wu"], a["G"], a["U"], activation, a["dX"], a["dWg"], a["dWu"], ws, n, None)

    each_view(call, ("dH", "G", "U", "X", "Wg", "Wu"), good)
    for name in ("dX", "dWg", "dWu"):
        for bad, status in BAD_VIEWS:
            got = call({**good, name: change(good[name], **bad)})
            assert got == status or got == SHAPE, (name, bad, got)
    for name in good:
        for kind in (F32, BF16, I8):
            assert call({**good, name: change(good[name], type=kind)}) == ATTR
    for name in good:
        assert call({**good, name: change(good[name], rows=good[name].rows + 1)}) == SHAPE
        assert call({**good, name: change(good[name], cols=good[name].cols - 1)}) == SHAPE
    assert call(good, activation=9) == ATTR
    assert call({**good, "dX": None, "dWg": None, "dWu": None}) == NULL
    assert call(good, ws=None, n=0) == WORKSPACE
    need = lib.onnx_gated_backward_workspace_bytes(*(good[k] for k in ("dH", "X", "Wg", "Wu", "dX", "dWg", "dWu")))
    assert need >= 2 * 4 * 30 * 2 and call(good, n=need - 1) == WORKSPACE
    assert call(good, ws=ctypes.c_void_p((1 << 41) + 8)) == UNSUPPORTED
    for a, b in (("dWg", "dWu"), ("dX", "dH"), ("dWg", "X"), ("dX", "G"), ("dWu", "Wu")):
        assert call({**good, a: change(good[a], data=good[b].data)}) == UNSUPPORTED


def test_binding_refuses_what_is_no_cuda_matrix():
    x = torch.zeros(4, 40, dtype=torch.bfloat16)
    q, s = torch.zeros(4, 40, dtype=torch.int8), torch.zeros(4)
    for call in (lambda: binding.onnx_quantize_rows(x), lambda: binding.onnx_gemm_int8(q, s, q, s), lambda: binding.onnx_gated(x, x, x),
                 lambda: binding.onnx_gated_int8(q, s, q, s, q, s), lambda: binding.onnx_gated_backward(x, x, x, x, x, x)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("kind", ref.KINDS)
def test_reference_gradients_are_those_of_differences(kind):
    g = torch.Generator().manual_seed(20)

    def normal(*s):
        return torch.randn(*s, generator=g, dtype=torch.float64)

    M, K, F, e = 5, 7, 6, 1e-5
    X, Wg, Wu, dH = normal(M, K), normal(F, K), normal(F, K), normal(M, F)

    def loss(X, Wg, Wu):
        return float((ref.act(kind, X @ Wg.T)[0] * (X @ Wu.T) * dH).sum())

    value, slope = ref.act(kind, X @ Wg.T)
    dG, dU = dH * (X @ Wu.T) * slope, dH * value
    formula = (dG @ Wg + dU @ Wu, dG.T @ X, dU.T @ X)
    for i, w in enumerate((X, Wg, Wu)):
        for _ in range(3):
            step = normal(*w.shape)
            at = [X, Wg, Wu]
            up, down = [list(at), list(at)]
            up[i], down[i] = w + e * step, w - e * step
            by_difference = (loss(*up) - loss(*down)) / (2 * e)
            assert math.isclose(by_difference, float((formula[i] * step).sum()), rel_tol=1e-6, abs_tol=1e-7)

"""What layer normalisation and the products by group refuse, at the C ABI (no GPU: a refused call launches nothing)."""
import ctypes

import pytest

from paper_2008_08272_b200 import binding
from paper_2008_08272_b200.binding import Matrices, Matrix

F32, I8, F16, BF16 = 1, 3, 10, 16
NULL, ATTR, SHAPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5
_next = [1 << 20]
OFFSETS, SCALE, WS = ctypes.c_void_p(1 << 40), ctypes.c_void_p(1 << 42), ctypes.c_void_p(1 << 41)


def address():
    _next[0] += 1 << 24
    return _next[0]


def mat(rows, cols, kind=F16, ld=None, data=None):
    return Matrix(data or address(), rows, cols, cols if ld is None else ld, kind, 0)


def mats(count, rows, cols, kind=F16, ld=None, stride=None, data=None):
    ld = cols if ld is None else ld
    return Matrices(data or address(), count, rows, cols, ld, rows * ld if stride is None else stride, kind, 0)


def change(m, **kw):
    n = type(m)(*[getattr(m, f) for f, _ in m._fields_])
    for k, v in kw.items():
        setattr(n, k, v)
    return n


BAD_VIEWS = [(dict(type=2), ATTR), (dict(type=F32), ATTR), (dict(type=I8), ATTR), (dict(reserved=1), ATTR), (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE),
             (dict(ld=7), SHAPE), (dict(rows=(1 << 30) + 1), UNSUPPORTED), (dict(ld=1 << 31), UNSUPPORTED), (dict(data=None), NULL)]
BAD_GROUPS = BAD_VIEWS[:4] + [(dict(count=0), SHAPE), (dict(rows=0), SHAPE), (dict(cols=0), SHAPE), (dict(ld=7), SHAPE), (dict(count=1025), UNSUPPORTED),
                              (dict(stride=0), SHAPE), (dict(stride=39), SHAPE), (dict(stride=-4000), SHAPE), (dict(stride=(1 << 36) + 1), UNSUPPORTED),
                              (dict(ld=1 << 31, stride=1 << 36), UNSUPPORTED), (dict(rows=1 << 29, stride=1 << 36), UNSUPPORTED), (dict(data=None), NULL)]




# Each call is spoilt in one way more than the one that is tried (no workspace where one is needed), so that none is ever launched here.
@pytest.fixture
def lib():
    return binding.load()


def test_grouped_gemm(lib):
    good = dict(X=mat(90, 41), W=mats(4, 50, 41), Y=mat(90, 50))

    def call(a, offsets=OFFSETS, ws=None, size=0):
        return lib.onnx_grouped_gemm_run(a["X"], a["W"], offsets, a["Y"], ws, size, None)

    for name, m in good.items():
        for bad, status in BAD_GROUPS if isinstance(m, Matrices) else BAD_VIEWS:
            got = call({**good, name: change(m, **bad)})
            assert got == status or (status == UNSUPPORTED and got == SHAPE), (name, bad, got)
        assert call({**good, name: None}) == NULL
    need = lib.onnx_grouped_gemm_workspace_bytes(good["X"], good["W"])
    assert need == 128 * (90 + 4 * 50) and call(good) == WORKSPACE and call(good, ws=WS, size=need - 1) == WORKSPACE
    assert call(good, None, WS, need) == NULL and call(good, ctypes.c_void_p(6), WS, need) == UNSUPPORTED
    assert call(good, ws=ctypes.c_void_p(8), size=need) == UNSUPPORTED
    for name in ("X", "W", "Y"):
        assert call(good, ws=ctypes.c_void_p(good[name].data), size=need) == UNSUPPORTED
        if name != "Y":
            assert call({**good, "Y": change(good["Y"], data=good[name].data)}, ws=WS, size=need) == UNSUPPORTED
    assert call({**good, "Y": change(good["Y"], data=1 << 40)}, ws=WS, size=need) == UNSUPPORTED
    for other in (dict(X=mat(90, 40)), dict(Y=mat(90, 51)), dict(Y=mat(89, 50)), dict(W=mats(4, 50, 40))):
        assert call({**good, **other}) == SHAPE
    for name, m in good.items():
        assert call({**good, name: change(m, type=BF16)}) == ATTR
    # groups that lie between one another's rows are fine, groups that overlap are not
    between = mats(4, 50, 40, ld=4 * 40, stride=40)
    assert lib.onnx_grouped_gemm_workspace_bytes(mat(90, 40), between) == 0
    assert call(dict(X=mat(90, 40), W=change(between, ld=159), Y=mat(90, 50))) == SHAPE
    assert call(dict(X=mat(90, 40), W=change(between, stride=39), Y=mat(90, 50))) == SHAPE
    assert lib.onnx_grouped_gemm_workspace_bytes(mat(90, 40), change(between, stride=41, ld=164)) == 128 * 200


def test_grouped_gated(lib):
    good = dict(X=mat(90, 41), Wg=mats(4, 50, 41), Wu=mats(4, 50, 41), H=mat(90, 50), G=mat(90, 50), U=mat(90, 50))

    def call(a, act=0, offsets=OFFSETS, ws=None, size=0):
        ref = lambda m: None if m is None else ctypes.byref(m)
        return lib.onnx_grouped_gated_run(a["X"], a["Wg"], a["Wu"], offsets, act, a["H"], ref(a["G"]), ref(a["U"]), ws, size, None)

    for name, m in good.items():
        for bad, status in BAD_GROUPS if isinstance(m, Matrices) else BAD_VIEWS:
            got = call({**good, name: change(m, **bad)})
            assert got == status or (status == UNSUPPORTED and got == SHAPE), (name, bad, got)
        assert call({**good, name: None}) == NULL
    assert call(good) == WORKSPACE and call({**good, "G": None, "U": None}) == WORKSPACE
    assert call(good, act=4) == ATTR and call(good, act=-1) == ATTR
    need = lib.onnx_grouped_gated_workspace_bytes(good["X"], good["Wg"], good["Wu"])
    assert need == 128 * (90 + 2 * 4 * 50)
    for a, b in (("H", "G"), ("H", "U"), ("G", "U"), ("H", "X"), ("G", "Wg"), ("U", "Wu")):
        assert call({**good, a: change(good[a], data=good[b].data)}, ws=WS, size=need) == UNSUPPORTED
    assert call({**good, "Wu": mats(3, 50, 41)}) == SHAPE and call({**good, "Wu": mats(4, 49, 41)}) == SHAPE


def test_grouped_backward(lib):
    ref = lambda m: None if m is None else ctypes.byref(m)
    good = dict(dY=mat(90, 50), X=mat(90, 41), W=mats(4, 50, 41), dX=mat(90, 41), dW=mats(4, 50, 41))

    def call(a, offsets=OFFSETS, ws=None, size=0):
        return lib.onnx_grouped_gemm_backward_run(ref(a["dY"]), ref(a["X"]), ref(a["W"]), offsets, ref(a["dX"]), ref(a["dW"]), ws, size, None)

    for name, m in good.items():
        for bad, status in BAD_GROUPS if isinstance(m, Matrices) else BAD_VIEWS:
            got = call({**good, name: change(m, **bad)})
            assert got == status or (status == UNSUPPORTED and got == SHAPE), (name, bad, got)
    for name in ("dY", "X", "W"):
        assert call({**good, name: None}) == NULL
    assert call({**good, "dX": None, "dW": None}) == NULL and call(good) == WORKSPACE
    need = lib.onnx_grouped_gemm_backward_workspace_bytes(*[ctypes.byref(good[n]) for n in ("dY", "X", "W", "dX", "dW")])
    assert need == 128 * (90 + 90 + 200)
    for a, b in (("dX", "dY"), ("dX", "X"), ("dW", "W"), ("dX", "dW"), ("dW", "X")):
        assert call({**good, a: change(good[a], data=good[b].data)}, ws=WS, size=need) == UNSUPPORTED

    full = dict(dH=mat(90, 50), X=mat(90, 41), Wg=mats(4, 50, 41), Wu=mats(4, 50, 41), G=mat(90, 50), U=mat(90, 50), dX=mat(90, 41), dWg=mats(4, 50, 41),
                dWu=mats(4, 50, 41))

    def gated(a, act=0, offsets=OFFSETS, ws=None, size=0):
        return lib.onnx_grouped_gated_backward_run(ref(a["dH"]), ref(a["X"]), ref(a["Wg"]), ref(a["Wu"]), ref(a["G"]), ref(a["U"]), offsets, act, ref(a["dX"]),
                                                   ref(a["dWg"]), ref(a["dWu"]), ws, size, None)

    for name, m in full.items():
        for bad, status in BAD_GROUPS if isinstance(m, Matrices) else BAD_VIEWS:
            got = gated({**full, name: change(m, **bad)})
            assert got == status or (status == UNSUPPORTED and got == SHAPE), (name, bad, got)
    for name in ("dH", "X", "Wg", "Wu", "G", "U"):
        assert gated({**full, name: None}) == NULL
    assert gated(full) == WORKSPACE and gated(full, act=9) == ATTR and gated(full, offsets=None) == NULL
    assert gated({**full, "dX": None, "dWg": None, "dWu": None}) == NULL
    assert gated({**full, "dWg": change(full["dWg"], data=full["dWu"].data)}, ws=WS, size=1 << 30) == UNSUPPORTED


def test_sums_of_too_many_terms(lib):
    """(Without the limit each of these would ask for a workspace.)"""
    ref = ctypes.byref
    long, most = (1 << 27) + 1, 1 << 27
    for K, status in ((long, UNSUPPORTED), (most, WORKSPACE)):
        X = mat(90, K, ld=K + 3)
        assert lib.onnx_grouped_gemm_run(X, mats(2, 8, K), OFFSETS, mat(90, 8), None, 0, None) == status
        assert lib.onnx_grouped_gated_run(X, mats(2, 8, K), mats(2, 8, K), OFFSETS, 0, mat(90, 8), None, None, None, 0, None) == status
    for R, N, wanted, status in ((long, 9, (0, 1), UNSUPPORTED), (most, 9, (0, 1), WORKSPACE), (long, 9, (1, 0), WORKSPACE), (90, long, (1, 0), UNSUPPORTED),
                                 (90, most, (1, 0), WORKSPACE), (90, long, (0, 1), WORKSPACE)):
        dY, X, W = mat(R, N, ld=N + 4 - N % 2), mat(R, 9), mats(2, N, 9)
        dX, dW = mat(R, 9) if wanted[0] else None, mats(2, N, 9) if wanted[1] else None
        assert lib.onnx_grouped_gemm_backward_run(ref(dY), ref(X), ref(W), OFFSETS, dX and ref(dX), dW and ref(dW), None, 0, None) == status
        assert lib.onnx_grouped_gated_backward_run(ref(dY), ref(X), ref(W), ref(W), ref(dY), ref(dY), OFFSETS, 0, dX and ref(dX), dW and ref(dW), None, None, 0,
                                                   None) == status


def test_layer_normalization(lib):
    ref = lambda m: None if m is None else ctypes.byref(m)
    X, s, b, Y = mat(4, 40, BF16), mat(1, 40, BF16), mat(1, 40, BF16), mat(4, 40, BF16)
    mean, inv = ctypes.c_void_p(1 << 43), ctypes.c_void_p(1 << 44)

    def norm(X=X, s=s, b=b, eps=1e-5, Y=Y, mean=mean, inv=inv):
        return lib.onnx_layer_normalization_run(ref(X), ref(s), ref(b), eps, ref(Y), mean, inv, None)

    for kw in (dict(X=None), dict(s=None), dict(Y=None), dict(mean=None), dict(inv=None)):
        assert norm(**kw) == NULL
    for kw in (dict(X=change(X, type=I8)), dict(Y=change(Y, type=F16)), dict(s=change(s, type=F16)), dict(b=change(b, type=F32)), dict(eps=-1.0),
               dict(eps=float("inf")), dict(eps=float("nan"))):
        assert norm(**kw) == ATTR
    for kw in (dict(s=mat(1, 41, BF16)), dict(s=mat(2, 40, BF16)), dict(b=mat(1, 39, BF16)), dict(Y=mat(4, 41, BF16)), dict(X=change(X, ld=39))):
        assert norm(**kw) == SHAPE
    for kw in (dict(mean=inv), dict(mean=ctypes.c_void_p(6)), dict(Y=change(Y, data=X.data)), dict(Y=change(Y, data=s.data)), dict(mean=ctypes.c_void_p(Y.data)),
               dict(inv=ctypes.c_void_p(X.data)), dict(X=change(X, data=X.data + 1))):
        assert norm(**kw) == UNSUPPORTED
    dY, dX, dS, dB = mat(4, 40, BF16), mat(4, 40, BF16), mat(1, 40, BF16), mat(1, 40, BF16)

    def back(dY=dY, X=X, s=s, mean=mean, inv=inv, dX=dX, dS=dS, dB=dB, ws=WS, size=1 << 20):
        return lib.onnx_layer_normalization_backward_run(ref(dY), ref(X), ref(s), mean, inv, ref(dX), ref(dS), ref(dB), ws, size, None)

    for kw in (dict(dY=None), dict(X=None), dict(s=None), dict(mean=None), dict(inv=None), dict(dX=None, dS=None, dB=None)):
        assert back(**kw) == NULL
    for kw in (dict(dY=change(dY, type=F16)), dict(dX=change(dX, type=F32)), dict(dS=change(dS, type=F32)), dict(dB=change(dB, type=F16)), dict(s=change(s, type=F32))):
        assert back(**kw) == ATTR
    for kw in (dict(dY=mat(5, 40, BF16)), dict(dX=mat(4, 41, BF16)), dict(dS=mat(1, 41, BF16)), dict(dB=mat(2, 40, BF16))):
        assert back(**kw) == SHAPE
    for kw in (dict(dX=change(dX, data=X.data)), dict(dX=change(dX, data=dY.data)), dict(dS=change(dS, data=s.data)), dict(dS=change(dS, data=dB.data)),
               dict(dB=change(dB, data=dX.data)), dict(mean=ctypes.c_void_p(dX.data)), dict(ws=ctypes.c_void_p(X.data)), dict(ws=mean), dict(ws=ctypes.c_void_p(8))):
        assert back(**kw) == UNSUPPORTED
    assert back(ws=None, size=0) == WORKSPACE and back(size=16) == WORKSPACE
    assert lib.onnx_layer_normalization_backward_workspace_bytes(X, None, None) == 0


def test_how_many_rows_take_weights_as_they_lie(lib):
    """Weights that begin anywhere are read as they lie (no workspace) by up to 128 rows of 4 a group on average, however many groups there are: those that one
    group may have are few passes over its weights.  Else they are copied."""
    for E, R, K, as_they_lie in ((1024, 16, 41, True), (1024, 128, 513, True), (32, 128, 513, True), (31, 128, 513, False), (1024, 129, 513, False), (1024, 4096, 513, False),
                                 (1024, 128, 511, False), (1, 17, 513, False), (1, 16, 513, True)):
        X, W = mat(R, K), mats(E, 24, K)
        assert (lib.onnx_grouped_gemm_workspace_bytes(X, W) == 0) == as_they_lie, (E, R, K)
        assert (lib.onnx_grouped_gated_workspace_bytes(X, W, W) == 0) == as_they_lie, (E, R, K)
        aligned = mats(E, 24, K + 7 & ~7)
        assert (lib.onnx_grouped_gemm_workspace_bytes(mat(R, aligned.cols), aligned) == 0)

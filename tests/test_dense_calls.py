"""Dense layers of 8- and 16-bit operands, call by call: through the checked path of the binding, captured before anything else has run,
with non-finite values, with what the binding refuses."""
import os
import subprocess
import sys

import pytest
import torch

import dense_reference as ref
from paper_2008_08272_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def normal(g, *size):
    return torch.randn(*size, generator=g, device="cuda")


def operands(M, K=136, F=200, t=torch.bfloat16, seed=31):
    g = torch.Generator(device="cuda").manual_seed(seed)
    X, Wg, Wu, dH = normal(g, M, K).to(t), (normal(g, F, K) / 12).to(t), (normal(g, F, K) / 12).to(t), normal(g, M, F).to(t)
    return X, Wg, Wu, dH


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 30, 200])
def test_checked_path_gives_the_same(M, monkeypatch):
    """The calls over ctypes, which take over where the native path declines: the same results bit by bit, and on another stream."""
    X, Wg, Wu, dH = operands(M)

    def calls():
        Q, s = binding.onnx_quantize_rows(X)
        (QW, sw), (QU, su) = binding.onnx_quantize_rows(Wg), binding.onnx_quantize_rows(Wu)
        H, G, U = binding.onnx_gated(X, Wg, Wu, save=True)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        on_side = binding.onnx_gated(X, Wg, Wu, activation="relu", stream=side)
        torch.cuda.current_stream().wait_stream(side)
        return [Q, s, binding.onnx_gemm_int8(Q, s, QW, sw, sw, fuse_relu=True, dtype=torch.float16), binding.onnx_gemm_int8(Q, s, QW, sw),
                binding.onnx_gated_int8(Q, s, QW, sw, QU, su, activation="gelu", dtype="bfloat16"), H, G, U, on_side,
                *binding.onnx_gated_backward(dH, X, Wg, Wu, G, U)]

    native = calls()
    monkeypatch.setattr(binding, "_fast_mod", binding._Declined())
    checked = calls()
    torch.cuda.synchronize()
    assert all(a.dtype == b.dtype and torch.equal(a, b) for a, b in zip(native, checked)) and len(native) == len(checked)


@pytest.mark.gpu
def test_captured_before_anything_has_run():
    """In a process of its own: the first call of every kind inside a capture, replayed on inputs that have changed."""
    program = """
import sys; sys.path[:0] = [%r, %r]
import torch
from paper_2008_08272_b200 import binding
import test_dense_calls as t
for M in (3, 150):
    X, Wg, Wu, dH = t.operands(M)
    W8 = torch.randint(-9, 9, (200, 136), dtype=torch.int8, device="cuda"); s = torch.rand(200, device="cuda")
    def calls():
        Q, sq = binding.onnx_quantize_rows(X)
        H, G, U = binding.onnx_gated(X, Wg, Wu, save=True)
        return [Q, sq, binding.onnx_gemm_int8(Q, sq, W8, s), binding.onnx_gated_int8(Q, sq, W8, s, W8, s), H, G, U,
                *binding.onnx_gated_backward(dH, X, Wg, Wu, G, U)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        kept = calls()
    X.mul_(-0.5)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, calls())), M
assert binding.last_device_status() == 0
print("captured")
""" % (ROOT, os.path.join(ROOT, "tests"))
    done = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "captured" in done.stdout, done.stderr[-2000:]


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("M", [4, 14, 60, 300])
def test_non_finite_values_stay_where_they_belong(M, value):
    """A token's makes its own results NaN or infinite and no other's; a channel's its own column."""
    X, Wg, Wu, dH = operands(M)
    want = binding.onnx_gated(X, Wg, Wu, save=True)
    bad = X.clone()
    bad[2, 5] = value
    for y, w in zip(binding.onnx_gated(bad, Wg, Wu, save=True), want):
        assert not bool(y[2].isfinite().any()) and torch.equal(torch.cat([y[:2], y[3:]]), torch.cat([w[:2], w[3:]]))
    worse = Wg.clone()
    worse[7, 135] = value
    H, G, U = binding.onnx_gated(X, worse, Wu, save=True)
    others = [i for i in range(200) if i != 7]
    assert not bool(G[:, 7].isfinite().any()) and torch.equal(H[:, others], want[0][:, others]) and torch.equal(U, want[2])
    clean = binding.onnx_gated_backward(dH, X, Wg, Wu, want[1], want[2])
    spoilt = dH.clone()
    spoilt[3, 9] = value
    dX, dWg, dWu = binding.onnx_gated_backward(spoilt, X, Wg, Wu, want[1], want[2])
    assert not bool(dX[3].isfinite().any()) and torch.equal(torch.cat([dX[:3], dX[4:]]), torch.cat([clean[0][:3], clean[0][4:]]))
    channels = [i for i in range(200) if i != 9]
    assert not bool(dWg[9].isfinite().any()) and torch.equal(dWg[channels], clean[1][channels]) and torch.equal(dWu[channels], clean[2][channels])


@pytest.mark.gpu
@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("size", [(1, 64, 69), (1, 368, 192), (2, 33, 1100), (5, 200, 64), (17, 96, 256), (31, 520, 77), (32, 64, 64)], ids=str)
def test_gradients_of_few_tokens_round_once(size, t):
    """Up to 32 tokens dG and dU keep what rounding leaves of them: the gradients are as near as rounding the results lets them be."""
    M, K, F = size
    X, Wg, Wu, dH = operands(M, K, F, t, 51)
    H, G, U = binding.onnx_gated(X, Wg, Wu, activation="gelu_tanh", save=True)
    dense = binding.onnx_gated_backward(dH, X, Wg, Wu, G, U, activation="gelu_tanh")
    odd = torch.full((M, K + 3), 7.0, dtype=t, device="cuda")
    odd[:, 1:K + 1] = X
    strided = binding.onnx_gated_backward(dH, odd[:, 1:K + 1], Wg, Wu, G, U, activation="gelu_tanh")
    want = ref.gated_backward(dH, X, Wg, Wu, G, U, "gelu_tanh", twice=True)
    for y, z, pair in zip(dense, strided, want):
        assert ref.worst(y, pair) <= 1 and torch.equal(y, z)
        once = float((pair[0].to(t).double() - pair[0]).norm())
        # (the products' sums in 32 bits and the activation's 2^-15 besides)
        assert float((y.double() - pair[0]).norm()) <= 1.1 * once + 2.0 ** -13 * float(pair[0].norm())


@pytest.mark.gpu
def test_what_the_binding_refuses():
    X, Wg, Wu, dH = operands(6)
    Q, s = binding.onnx_quantize_rows(X)
    W8, sw = binding.onnx_quantize_rows(Wg)
    shape, attr, unsupported = 3, 2, 4

    def status(call):
        with pytest.raises(binding.OnnxB200Error) as e:
            call()
        return e.value.status

    assert status(lambda: binding.onnx_gated(X[:1].expand(6, 136), Wg, Wu)) == shape              # rows that overlap
    assert status(lambda: binding.onnx_gated(X, Wg, Wu, activation="tanh")) == attr
    assert status(lambda: binding.onnx_gated(X, Wg, Wu[:-1])) == shape
    assert status(lambda: binding.onnx_gated(X, Wg, Wu, H=dH, G=dH)) == unsupported               # two results in one place
    assert status(lambda: binding.onnx_gemm_int8(Q, s, W8, sw[:-1])) == shape
    assert status(lambda: binding.onnx_gemm_int8(Q, s, W8[:, :-1], sw)) == shape
    assert status(lambda: binding.onnx_gemm_int8(Q, None, W8, sw)) == 1
    assert status(lambda: binding.onnx_quantize_rows(X, scale=s[:-1])) == shape
    assert status(lambda: binding.onnx_gated_backward(dH, X, Wg, Wu, dH, dH, wanted=(False, False, False))) == 1
    for call in (lambda: binding.onnx_gated(X.float(), Wg, Wu), lambda: binding.onnx_gated(X, Wg, Wu.half()), lambda: binding.onnx_gated(X.T, Wg, Wu),
                 lambda: binding.onnx_gated(X[0], Wg, Wu), lambda: binding.onnx_gated(X.cpu(), Wg, Wu), lambda: binding.onnx_gemm_int8(X, s, W8, sw),
                 lambda: binding.onnx_gemm_int8(Q, s.half(), W8, sw), lambda: binding.onnx_gemm_int8(Q, s, W8, sw, dtype=torch.int8),
                 lambda: binding.onnx_gemm_int8(Q, s, W8, sw, sw[::2].repeat(2)[::1].half()), lambda: binding.onnx_quantize_rows(Q)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        binding.onnx_gated_backward(dH, X, Wg, Wu, dH, dH, wanted=(True, True))
    # a workspace that is too small, and one that is as large as asked for
    odd = X[:, 1:]
    need = (136 * 2 + 127) // 128 * 128 * 6
    assert status(lambda: binding.onnx_gated(odd, Wg[:, 1:], Wu[:, 1:], workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))) == 5
    before = binding.launch_count()
    with pytest.raises(binding.OnnxB200Error):
        binding.onnx_gated(X, Wg, Wu[:-1])
    assert binding.launch_count() == before


@pytest.mark.gpu
def test_two_streams_at_once():
    """The same calls on two streams side by side, again and again: each with workspaces of its own."""
    jobs = []
    for seed in (41, 42):
        X, Wg, Wu, dH = operands(300, 131, 257, seed=seed)
        jobs.append((X, Wg, Wu, dH, torch.cuda.Stream()))

    def run(X, Wg, Wu, dH, stream=None):
        H, G, U = binding.onnx_gated(X, Wg, Wu, save=True, stream=stream)
        Q, s = binding.onnx_quantize_rows(X, stream=stream)
        W8, sw = binding.onnx_quantize_rows(Wg, stream=stream)
        return [H, G, U, binding.onnx_gemm_int8(Q, s, W8, sw, stream=stream), *binding.onnx_gated_backward(dH, X, Wg, Wu, G, U, stream=stream)]

    want = [run(*job[:4]) for job in jobs]
    torch.cuda.synchronize()
    for _ in range(10):
        got = [run(*job) for job in jobs]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


def test_reference_activations_against_torch():
    g = torch.Generator().manual_seed(43)
    x = 4 * torch.randn(1000, generator=g, dtype=torch.float64)
    for kind, f in (("silu", torch.nn.functional.silu), ("relu", torch.relu), ("gelu", torch.nn.functional.gelu),
                    ("gelu_tanh", lambda v: torch.nn.functional.gelu(v, approximate="tanh"))):
        assert torch.allclose(ref.act(kind, x)[0], f(x), rtol=1e-12, atol=1e-14)

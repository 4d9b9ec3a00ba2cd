"""Sums of the dense layers in 32 bits all the way, also where a reduction is shared or goes through planes: errors in the norm (dense_norms.py), which
sums in 16 bits would not keep to (shown on the CPU).  And the activations in 32 bits, by value."""
import math

import pytest
import torch

import dense_norms as norms
import dense_reference as ref
from paper_2008_08272_b200 import binding

HALVES = (torch.bfloat16, torch.float16)
# (tokens, width, channels) of few tiles and a long reduction
LONG = [(20, 5000, 33), (40, 2000, 70), (130, 3001, 200), (300, 4104, 130), (150, 4096, 200)]


def normal(g, *size):
    return torch.randn(*size, generator=g, device=g.device)


def gen(seed, device="cuda"):
    return torch.Generator(device=device).manual_seed(seed)


def block(g, M, K, F, t):
    return normal(g, M, K).to(t), (normal(g, F, K) / math.sqrt(K)).to(t), (normal(g, F, K) / math.sqrt(K)).to(t)


# --------------------------------------------------------------------- what the bound lets pass (no GPU)
def in_parts(x, w, t, parts, between):
    """x w^T in 64 bits, the running sum rounded by `between` after each of `parts` parts but the last, the whole to t."""
    n, total = x.shape[1], torch.zeros(x.shape[0], w.shape[0], dtype=torch.float64)
    for i in range(parts):
        at = slice(i * n // parts, (i + 1) * n // parts)
        total = total + x[:, at] @ w[:, at].T
        if i + 1 < parts:
            total = total.to(between).double()
    return total.to(t)


@pytest.mark.parametrize("t", HALVES, ids=str)
@pytest.mark.parametrize("size", LONG, ids=str)
def test_the_bound_tells_sums_in_16_bits_from_those_in_32(size, t):
    X, Wg, _ = (v.double() for v in block(gen(81, "cpu"), *size, t))
    pair = norms.product(X, Wg)
    for parts in (2, 4, 8):
        assert norms.ratio(in_parts(X, Wg, t, parts, torch.float32), pair) <= 1
        if parts > 2 or t == torch.bfloat16:                   # (one rounding to fp16 half way is 1.22 of the result's own; the bound is up to 1.25)
            assert norms.ratio(in_parts(X, Wg, t, parts, t), pair) > 1, parts
    chain = torch.zeros(X.shape[0], Wg.shape[0])
    for k in range(0, X.shape[1], 16):                         # in 32 bits, 16 products at a time
        chain += (X[:, k:k + 16] @ Wg[:, k:k + 16].T).float()
    assert norms.ratio(chain.to(t), pair) <= 1


# --------------------------------------------------------------------- the kernels
def check(pairs, got):
    torch.cuda.synchronize()
    assert binding.last_device_status() == 0
    for name, pair, y in zip("HGU" if len(got) == 3 else "H", pairs, got):
        assert norms.ratio(y, pair) <= 1, name


@pytest.mark.gpu
@pytest.mark.parametrize("t", HALVES, ids=str)
@pytest.mark.parametrize("size", LONG + [(1, 8192, 512), (7, 6000, 300), (16, 5000, 257), (1000, 4096, 640)], ids=str)
@pytest.mark.parametrize("tile", ["", "1x64", "2x128", "1x64/2", "1x128/4", "1x64/8", "1x256/8"])
def test_gated(tile, size, t, monkeypatch):
    if tile:
        monkeypatch.setenv("ONNXB_DENSE_TILE", tile)
    X, Wg, Wu = block(gen(82), *size, t)
    for kind in ("silu", "gelu"):
        want = norms.gated(X, Wg, Wu, kind)
        check(want, binding.onnx_gated(X, Wg, Wu, activation=kind, save=True))
        check(want[:1], (binding.onnx_gated(X, Wg, Wu, activation=kind),))


@pytest.mark.gpu
@pytest.mark.parametrize("t", HALVES, ids=str)
@pytest.mark.parametrize("size", [(40, 512, 3000), (100, 1030, 2056), (512, 1024, 4096), (1024, 512, 4096), (300, 200, 8000), (4000, 130, 72), (64, 4096, 10240)], ids=str)
@pytest.mark.parametrize("parts", ["", "1", "2", "4", "8"])
def test_gated_backward(parts, size, t, monkeypatch):
    if parts:
        monkeypatch.setenv("ONNXB_DENSE_PARTS", parts)
    g = gen(83)
    M, K, F = size
    X, Wg, Wu = block(g, M, K, F, t)
    dH, G, U = (normal(g, M, F).to(t) for _ in range(3))
    got = binding.onnx_gated_backward(dH, X, Wg, Wu, G, U, activation="gelu_tanh")
    torch.cuda.synchronize()
    for name, pair, y in zip(("dX", "dWg", "dWu"), norms.gated_backward(dH, X, Wg, Wu, G, U, "gelu_tanh"), got):
        assert norms.ratio(y, pair) <= 1, name


# --------------------------------------------------------------------- activations in 32 bits
def argument(kind, g):
    """How large the exponential's argument is, which it is off by steps of."""
    if kind == "silu":
        return g.abs()
    if kind == "gelu":
        return g * g / 2
    return math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3).abs() if kind == "gelu_tanh" else torch.zeros_like(g)


def gate(kind, g, u):
    """(act(g) u, how far 32 bits may be off it): g and u by 4 steps each; act(g) by 16 steps and 3 for every unit of the argument (2 + 1.2 of
    the exponential's, up to 1.5 where the argument itself is rounded; 2 of a quotient; the polynomial of the normal distribution's tail 1.7e-7,
    and 8 for its terms, which are 1.8 times their sum); two roundings."""
    value, slope = ref.act(kind, g)
    h = value * u
    off = (16 + 3 * argument(kind, g)) * ref.STEP * h.abs() + 4 * ref.STEP * (slope * g * u).abs() + (4 + 2) * ref.STEP * h.abs() + 1e-37 * u.abs()
    return h, off


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("M", [1, 6, 30, 200])
def test_activations_in_32_bits(kind, M):
    """Gates of 8-bit operands, whose sums are exact, with 32-bit results: single values, from 0 to some 12."""
    g = gen(84)
    A, Wg, Wu = (torch.randint(-127, 128, (n, 96), generator=g, device="cuda", dtype=torch.int8) for n in (M, 500, 500))
    sa, one = torch.exp(normal(g, M)) / 127, torch.rand(500, generator=g, device="cuda") / 127 / 2
    H = binding.onnx_gated_int8(A, sa, Wg, one, Wu, one, activation=kind)
    torch.cuda.synchronize()
    gu = [ref.gemm_int8(A, sa, W, one, None, False, torch.float32)[0] for W in (Wg, Wu)]
    inside = gu[0].abs() <= 12
    h, off = gate(kind, *gu)
    assert float(inside.float().mean()) > 0.7
    assert ref.worst(H[inside], (h[inside], off[inside])) <= 1


@pytest.mark.parametrize("kind", ref.KINDS[:3])
def test_the_bound_tells_activations_of_fewer_bits(kind):
    """What 32 bits give passes, and what is off by 2^-17 of the value (64 steps, of the 256 that the elementwise bound for sums lets pass) does not."""
    g = torch.linspace(-12, 12, 4001, dtype=torch.float64)
    u = torch.ones_like(g)
    h, off = gate(kind, g.float().double(), u)
    assert ref.worst(ref.act(kind, g.float())[0] if kind != "gelu" else h.float(), (h, off)) <= 1
    assert ref.worst(h * (1 + 2.0 ** -17), (h, off)) > 1

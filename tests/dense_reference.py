"""The dense layers of 8- and 16-bit operands from their definitions, in 64 bits (torch, any device), and how far a result may be off.

Tolerances, all from the formats: a rounding to a type t is off by at most half a step, eps(t)/2 of the value (and half the smallest number
where that is more); a sum of n products that are exact in 32 bits, taken in 32 bits in any order, with every addition off by as much as
a whole step, by n 2^-23 sum|products|; the activation in 32 bits by 2^-15 of its value (an exponential with its argument rounded in
32 bits is off by about |argument| 2^-23, the argument at most 100 where the value counts; a polynomial of the normal distribution's tail by
2^-22 and a quotient besides), its slope, which is a sum, by 2^-15 of 1.2, its largest value.  Two numbers given to 64-bit functions are exact.
"""
import math

import torch

KINDS = ("silu", "gelu", "gelu_tanh", "relu")
ACT, SLOPE, STEP = 2.0 ** -15, 1.2 * 2.0 ** -15, 2.0 ** -23


def half_step(t, value):
    info = torch.finfo(t)
    return (value.abs() * (info.eps / 2)).clamp(min=info.smallest_normal * info.eps / 2)


def act(kind, g):
    """act(g) and act'(g)."""
    if kind == "relu":
        return g.clamp(min=0), (g > 0).to(g.dtype)
    if kind == "silu":
        p = torch.sigmoid(g)
        return g * p, p + g * p * (1 - p)
    if kind == "gelu":
        p = torch.special.erfc(-g / math.sqrt(2)) / 2
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(8 / math.pi)
    p = torch.sigmoid(c * (g + 0.044715 * g ** 3))
    return g * p, p + g * p * (1 - p) * c * (1 + 3 * 0.044715 * g * g)


def quantize_rows(X):
    """(Q, scale) as the definition has them: equal bit by bit."""
    x = X.double()
    bad = ~torch.isfinite(x).all(1)
    scale = (torch.where(bad[:, None], torch.zeros_like(x), x).abs().amax(1) / 127).float()
    s = scale.double()
    q = torch.where((s[:, None] > 0) & ~bad[:, None], torch.round(x / s.clamp(min=1e-300)[:, None]), torch.zeros_like(x))
    return q.nan_to_num().clamp(-127, 127).to(torch.int8), torch.where(bad, torch.full_like(scale, math.nan), scale)


def gemm_int8(A, a_scale, B, b_scale, C, relu, t):
    """(Y, tolerance): the sum's conversion, two products and the addend's sum are off by a step each at most."""
    v = (A.double() @ B.double().T) * a_scale.double()[:, None] * b_scale.double()[None, :]
    y = v if C is None else v + C.double()
    off = 4 * STEP * v.abs() + (0 if C is None else STEP * y.abs())
    y = y.clamp(min=0) if relu else y
    return y, off + half_step(t, y) * (1 + 2.0 ** -10)


def projection(X, W):
    """(sum, how far 32 bits may be off it)."""
    x, w = X.double(), W.double()
    return x @ w.T, X.shape[1] * STEP * (x.abs() @ w.abs().T)


def _gate(kind, g, dg, u, du, t):
    value, _ = act(kind, g)
    h = value * u
    off = (ACT * value.abs() + 1.2 * dg) * (u.abs() + du) + value.abs() * du + 2 * STEP * h.abs()
    return h, off + half_step(t, h.abs() + off)


def gated(X, Wg, Wu, kind):
    """((H, tolerance), (G, tolerance), (U, tolerance))."""
    g, dg = projection(X, Wg)
    u, du = projection(X, Wu)
    return _gate(kind, g, dg, u, du, X.dtype), (g, dg + half_step(X.dtype, g.abs() + dg)), (u, du + half_step(X.dtype, u.abs() + du))


def gated_int8(A, a_scale, Wg, g_scale, Wu, u_scale, kind, t):
    g, u = (gemm_int8(A, a_scale, W, s, None, False, torch.float32)[0] for W, s in ((Wg, g_scale), (Wu, u_scale)))
    return _gate(kind, g, 4 * STEP * g.abs(), u, 4 * STEP * u.abs(), t)


def gated_backward(dH, X, Wg, Wu, G, U, kind, twice=False):
    """((dX, tolerance), (dWg, tolerance), (dWu, tolerance)); dG and dU are rounded to the type on the way, or (`twice`) what that leaves
    of them is, which is half a step at most."""
    t = dH.dtype
    dh, g, u, x, wg, wu = (v.double() for v in (dH, G, U, X, Wg, Wu))
    value, slope = act(kind, g)
    dg, du = dh * u * slope, dh * value
    off_g = SLOPE * (dh * u).abs() + 3 * STEP * dg.abs()
    off_u = ACT * du.abs() + STEP * du.abs()
    rest_g, rest_u = half_step(t, dg.abs() + off_g), half_step(t, du.abs() + off_u)
    if twice:
        rest_g, rest_u = half_step(t, rest_g), half_step(t, rest_u)
    off_g, off_u = off_g + rest_g, off_u + rest_u
    F, M = dH.shape[1], dH.shape[0]

    def product(terms, n):
        y = sum(a @ b for a, _, b in terms)
        size = sum((a.abs() + o) @ b.abs() for a, o, b in terms)
        off = sum(o @ b.abs() for _, o, b in terms) + n * STEP * size
        return y, off + half_step(t, y.abs() + off)

    n = 2 if twice else 1
    return (product([(dg, off_g, wg), (du, off_u, wu)], 2 * n * F),
            product([(dg.T, off_g.T, x)], n * M), product([(du.T, off_u.T, x)], n * M))


def worst(got, pair):
    """The largest |got - want| / tolerance; where the definition has an infinity or NaN the result has to have it too."""
    want, off = pair
    assert got.shape == want.shape, (got.shape, want.shape)
    if want.numel() == 0:
        return 0.0
    d = (got.double() - want).abs()
    return float((d / off).nan_to_num(nan=math.inf).max())

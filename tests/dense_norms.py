"""How far whole results of the dense layers may be off in the norm, where a bound for each element would let sums in 16 bits pass.

A sum of n products: the tensor cores add 16 of them (16-bit floats) at once to what is there in 32 bits, and are off each time by at most a step
(2^-23) of the largest of these numbers; up to 8 further additions join parts.  The terms have random signs, so that running sums are no larger in
the mean square than S = sqrt(sum (x w)^2), which the whole sum is too: off by (n / 16 + 8) 2^-23 S.  Rounding what is that far off in place
of the exact value changes the norm of the rounding error by less than 5 % (it is 2 % of a step of 16 bits or less, and moves to the neighbour
where it crosses a half: 4 % of the elements, of whose error it changes the sign).  A running sum that were rounded to 16 bits k times on its
way, at equal distances, would be off by sqrt(1 + sum (i / (k + 1), i <= k)) times the result's own rounding: 1.22 times for k = 1, 1.58 for 3.
"""
import torch

import dense_reference as ref

SLACK, STEP = 1.05, ref.STEP
ACT = 16 * STEP          # of the activation's value: an exponential (2 + 1.2 |argument| steps), a quotient (2), products and sums


def steps(n):
    return (n / 16 + 8) * STEP


def product(x, w):
    """x [M,n] and w [N,n] in 64 bits: (x w^T, how far a sum in 32 bits is off it)."""
    return x @ w.T, steps(x.shape[1]) * torch.sqrt((x * x) @ (w * w).T)


def allowed(exact, off, t):
    return SLACK * float((exact.to(t).double() - exact).norm()) + float(off.norm())


def ratio(got, pair):
    """||got - exact|| over what it may be."""
    exact, off = pair
    return float((got.double() - exact).norm()) / allowed(exact, off, got.dtype)


def gated(X, Wg, Wu, kind):
    (g, dg), (u, du) = (product(X.double(), W.double()) for W in (Wg, Wu))
    value, slope = ref.act(kind, g)
    h = value * u
    return (h, slope.abs() * dg * u.abs() + value.abs() * du + ACT * h.abs()), (g, dg), (u, du)


def gated_backward(dH, X, Wg, Wu, G, U, kind):
    """More than 32 tokens: of dG and dU rounded to the type."""
    dh, g, u, x, wg, wu = (v.double() for v in (dH, G, U, X, Wg, Wu))
    value, slope = ref.act(kind, g)
    dg, du = ((dh * v).to(dH.dtype).double() for v in (u * slope, value))
    return product(torch.cat([dg, du], 1), torch.cat([wg.T, wu.T], 1)), product(dg.T, x.T), product(du.T, x.T)

"""Plain 64-bit evaluation of the gated recurrence and its gradients, token by token, with the error bounds that the tests use.

u = 2^-24 is the roundoff of the 32-bit arithmetic.  exp(-|g|) is off by at most 5 u of itself (ex2.approx 2 ulp, the correction), 1 + a by u,
the quotient by 4 u: the smaller one of f and 1 - f by 10 u of itself, the other one by that and its rounding.  With rest = 1 - f
(and one of the two at least 1/2) f is off by at most u (1 + 20 rest) of itself, rest by u (1 + 20 f); sqrt(rest (1 + f)) by half of
that, two roundings and 2 ulp, all inputs' factors within 18 u.
A value h_t is a sum of products of factors f and one b = i x.  Every factor adds its own error, a rounding of the product it
becomes part of and, once in 8 tokens, of the composition of warps, at most u (1 + 20 rest) + 2 u + u; every sum a rounding, in a
lane and where the parts meet.  With A the same recurrence on absolute values,
    E_t = f (E_{t-1} + u (4 + 20 rest) A_{t-1}) + 20 u |b_t| + 2 u A_t
bounds the error of h_t in 32 bits; outputs are rounded once more to their type.  exp(-|g|) below 2^-126 (|g| above 87.3) is zero in 32 bits,
so f, rest and both slopes are off by up to F = 2^-126 besides - with sqrt(rest (1 + f)) its factor by up to sqrt(2 F), and that one's
slope: this times what they multiply is added.
"""
from __future__ import annotations

import numpy as np

from tests.lm_reference import U

u = 2.0 ** -24
F = 2.0 ** -126
LOST = {"complement": F, "one": 0.0, "root": (2.0 * F) ** 0.5}       # of an input's factor


def gates(g, kind):
    """f, 1 - f, i, df, di"""
    with np.errstate(over="ignore"):
        f, rest = 1.0 / (1.0 + np.exp(-g)), 1.0 / (1.0 + np.exp(g))
    if kind == "complement":
        return f, rest, rest, f * rest, -f * rest
    if kind == "one":
        return f, rest, np.ones_like(f), f * rest, np.zeros_like(f)
    i = np.sqrt(rest * (1.0 + f))
    return f, rest, i, f * rest, -f * f * i / (1.0 + f)


def recurrence(f, rest, b, first, lost):
    """(t, d) arrays, lost what an input may be off by beside its relative error: h, the bound of its error in 32 bits, and the states before each token with theirs."""
    t, d = b.shape
    h, e, a = first.copy(), np.zeros(d), np.abs(first)
    hs, es, before, e_before = np.zeros((t, d)), np.zeros((t, d)), np.zeros((t, d)), np.zeros((t, d))
    for k in range(t):
        before[k], e_before[k] = h, e
        e = f[k] * (e + u * (4.0 + 20.0 * rest[k]) * a) + 20.0 * u * np.abs(b[k]) + F * a + lost[k]
        h = f[k] * h + b[k]
        a = f[k] * a + np.abs(b[k])
        e = e + 2.0 * u * a
        hs[k], es[k] = h, e
    return hs, es, before, e_before, h, e


def rounded(value, error, dtype):
    """Bound after one rounding to the type."""
    r = U[dtype]
    return error * (1.0 + r) + r * np.abs(value) + (2.0 ** -25 if r == 2.0 ** -11 else 0.0) + 1e-37


def forward(x, g, kind, first, dtype):
    """(value, bound) of h and of the last state, for one sequence of (t, d)."""
    f, rest, i, _, _ = gates(g, kind)
    h, e, _, _, last, e_last = recurrence(f, rest, i * x, first, LOST[kind] * np.abs(x))
    return (h, rounded(h, e, dtype)), (last, e_last + 1e-37)


def backward(x, g, d_y, kind, first, d_last, dtype):
    """(value, bound) of dx, dgate and the gradient of the first state."""
    f, rest, i, df, di = gates(g, kind)
    _, _, h, e_h, _, _ = recurrence(f, rest, i * x, first, LOST[kind] * np.abs(x))
    t, d = x.shape
    flow, e, a = d_last.copy(), np.zeros(d), np.abs(d_last)
    grad, e_g = np.zeros((t, d)), np.zeros((t, d))
    for k in range(t - 1, -1, -1):
        grad[k] = d_y[k] + flow
        a = a + np.abs(d_y[k])
        e = e + 2.0 * u * a
        e_g[k] = e
        flow = f[k] * grad[k]
        e = f[k] * (e + u * (4.0 + 20.0 * rest[k]) * a) + F * a
        a = f[k] * a
    slopes = np.abs(h) * df + np.abs(x * di)
    dx, dg = i * grad, grad * (h * df + x * di)
    # products of up to four factors, each within 20 u
    return ((dx, rounded(dx, i * e_g + 24.0 * u * np.abs(dx) + LOST[kind] * np.abs(grad), dtype)),
            (dg, rounded(dg, (e_g * slopes + np.abs(grad) * e_h * df) * 1.01 + 64.0 * u * np.abs(grad) * slopes + np.abs(grad) * (F * np.abs(h) + LOST[kind] * np.abs(x)), dtype)), (flow, e + 1e-37))

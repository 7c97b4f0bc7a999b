"""Plain 64-bit layer norm and its gradients, with the error bounds that the tests use.

u = 2^-24.  A sum over a row is one of at most 32 terms in a thread, 5 levels of a warp and 5 of a block: off by at most k = 48 u times
the sum of absolute values, the product in every term included.  The first mean may be off by `off` = k mean|x| + u |mean|, which the second one takes out again: what is left in
a centred value is its two roundings and the second mean's error, dv = 2 u (|v| + off) + k (mean|v| + off).  The variance is a sum of
squares, off by at most 2 k of itself, r = 1/sqrt(variance + eps) by k and 4 u (2 ulp): 1.2 k.  The rest is the sum of what its factors are off by.
Gradients of the parameters are sums over rows: in a block at most rows/100 + 8 in order, then the blocks' (at most 1184) in eight groups.
"""
from __future__ import annotations

import numpy as np

from tests.lm_reference import U

u = 2.0 ** -24
k = 48 * u


def rounded(value, error, dtype):
    r = U[dtype]
    return error * (1.0 + r) + r * np.abs(value) + (2.0 ** -25 if r == 2.0 ** -11 else 0.0) + 1e-37


def parts(x, eps):
    mean = x.mean(1, keepdims=True)
    v = x - mean
    off = k * np.abs(x).mean(1, keepdims=True) + u * np.abs(mean)
    dv = 2 * u * (np.abs(v) + off) + k * (np.abs(v).mean(1, keepdims=True) + off)
    r = 1.0 / np.sqrt((v * v).mean(1, keepdims=True) + eps)
    # variance: from the squares of values off by dv
    loose = 1.2 * k + r * r * (np.abs(v) * dv).mean(1, keepdims=True)
    return v, dv, r, loose


def forward(x, w, b, eps, dtype):
    v, dv, r, loose = parts(x, eps)
    y = w * v * r + b
    error = np.abs(w) * r * (dv + np.abs(v) * loose) + 3 * u * (np.abs(w * v * r) + np.abs(b))
    return y, rounded(y, error, dtype)


def backward(d_y, x, w, eps, dtype, param_type):
    v, dv, r, loose = parts(x, eps)
    n = v * r
    dn = r * dv + loose * np.abs(n) + u * np.abs(n)
    e = w * d_y
    me, men = e.mean(1, keepdims=True), (e * n).mean(1, keepdims=True)
    d_me = (k + 2 * u) * np.abs(e).mean(1, keepdims=True)
    d_men = (k + 4 * u) * np.abs(e * n).mean(1, keepdims=True) + (np.abs(e) * dn).mean(1, keepdims=True) + loose * np.abs(men)
    d_x = r * (e - me - n * men)
    size = np.abs(e) + np.abs(me) + np.abs(n * men)
    error = r * (u * np.abs(e) + d_me + np.abs(n) * d_men + np.abs(men) * dn) + r * size * (loose + 4 * u)
    many = x.shape[0] / 100 + 8 + 1184 / 8 + 8
    d_w, d_b = (d_y * n).sum(0), d_y.sum(0)
    e_w = (np.abs(d_y) * dn).sum(0) + (many + 1) * u * np.abs(d_y * n).sum(0)
    e_b = many * u * np.abs(d_y).sum(0)
    return (d_x, rounded(d_x, error, dtype)), (d_w, rounded(d_w, e_w, param_type)), (d_b, rounded(d_b, e_b, param_type))

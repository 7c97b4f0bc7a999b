"""Plain 64-bit evaluation of the language-model operators, and the error bounds that their tests use.

A mixing is the token-by-token definition: with lead = 1 forward in time, X <- a X + in_scale k v^T, o = out_scale X^T q; with
lead = 0 backward in time, X <- X + in_scale k v^T, o = out_scale X^T q, X <- a X.  Run on absolute values it gives the
sum A of the absolute values of the products behind every output, which the bounds are multiples of:

 - outputs are sums of products in which one factor (a score, or a value of the state) was rounded to the 16-bit type,
   unit roundoff u = 2^-8 (bfloat16) or 2^-11 (float16), then the output was: |error| <= u |o| + u A, plus what 32-bit
   sums of a few hundred terms and the exponentials add (1e-5 A) and what products of rounding errors add (0.02 u A);
 - float16 has a smallest step of 2^-24: a score below 2^-14 is off by up to 2^-25, in each of the 128 tokens of a group:
   128 * 2^-24 * max |v| covers scores and keys;
 - states are 32-bit sums of products with keys held in two 16-bit terms, off by u^2 <= 2^-16: (2^-16 + 1e-5) A.
"""
from __future__ import annotations

import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def f64(x) -> np.ndarray:
    return x.detach().double().cpu().numpy()


def mix(q, k, v, log_decay, lead, init=None, in_scale=1.0, out_scale=1.0):
    """(b, t, h, d) float64 -> outputs (b, t, h, dv) and the last state (b, h, dk, dv)."""
    b, t, h, dk = q.shape
    dv = v.shape[-1]
    a = np.exp(log_decay)[None, :, None, None]
    x = np.zeros((b, h, dk, dv)) if init is None else init.copy()
    o = np.zeros((b, t, h, dv))
    for i in (range(t) if lead else range(t - 1, -1, -1)):
        x = (a * x if lead else x) + in_scale * k[:, i, :, :, None] * v[:, i, :, None, :]
        o[:, i] = out_scale * np.einsum("bhk,bhkv->bhv", q[:, i], x)
        if not lead:
            x = a * x
    return o, x


def bounded_mix(dtype, q, k, v, log_decay, lead, init=None, in_scale=1.0, out_scale=1.0):
    """mix() with the bounds of its outputs and of its last state."""
    o, x = mix(q, k, v, log_decay, lead, init, in_scale, out_scale)
    ab = [np.abs(y) for y in (q, k, v)]
    ao, ax = mix(*ab, log_decay, lead, None if init is None else np.abs(init), abs(in_scale), abs(out_scale))
    u = U[dtype]
    step = 128 * 2.0 ** -24 * (ab[2].max() if ab[2].size else 0.0) if dtype == torch.float16 else 0.0
    return o, u * np.abs(o) + (1.02 * u + 1e-5) * ao + step + 1e-30, x, (2.0 ** -16 + 1e-5) * ax + 1e-30


def transpose(x):
    return None if x is None else np.swapaxes(x, -1, -2)


def gradients(dtype, q, k, v, log_decay, scale, init, d_o, d_last):
    """(value, bound) of dq, dk, dv and of the gradient of the first state."""
    dq, eq, _, _ = bounded_mix(dtype, d_o, v, k, log_decay, 1, transpose(init), 1.0, scale)
    dv, ev, d0, e0 = bounded_mix(dtype, k, q, d_o, log_decay, 0, d_last, scale, 1.0)
    dk, ek, _, _ = bounded_mix(dtype, v, d_o, q, log_decay, 0, transpose(d_last), scale, 1.0)
    return (dq, eq), (dk, ek), (dv, ev), (d0, e0)


def assert_within(got, want, bound, what=""):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, f"{what}: shape {got.shape}, want {want.shape}"
    assert np.isfinite(got).all(), f"{what}: {np.count_nonzero(~np.isfinite(got))} values are not finite"
    err = np.abs(got - want)
    if not (err <= bound).all():
        i = np.unravel_index(np.argmax(err - bound), err.shape)
        raise AssertionError(f"{what}: {np.count_nonzero(err > bound)} of {err.size} out of bounds, worst at {i}: got {got[i]}, want {want[i]}, bound {bound[i]}")

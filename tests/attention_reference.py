"""Linear attention with one decay per head and its gradients from the definition, in 64 bits, and what the tests compare with.

Everything is computed a second time on absolute values: the sums of the terms' sizes, which rounding errors are measured by."""
from __future__ import annotations

import numpy as np

UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
# What the products may round before the output's own rounding: weighted scores to bf16 once (2^-8); to 16 bits in two bf16 parts, the
# product of the two low parts dropped (< 4 * 2^-16); to 24 bits in three parts, products below 2^-24 dropped (< 8 * 2^-24).
INNER = {"bf16": 2.0 ** -8, "f16": 2.0 ** -14, "f32": 2.0 ** -21}


def power(g, n):
    """exp(g n), 1 for n = 0."""
    n = np.asarray(n, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        return np.where(n == 0, 1.0, np.exp(g * n))


def weights(length, g):
    """a^(t - s) for s <= t, else 0."""
    t = np.arange(length)
    apart = t[:, None] - t[None, :]
    return np.where(apart >= 0, power(g, np.maximum(apart, 0)), 0.0)


def forward_row(q, k, v, g, s0, scale):
    n = len(q)
    t = np.arange(n)
    o = ((q @ k.T) * weights(n, g)) @ v + power(g, t + 1)[:, None] * (q @ s0)
    return scale * o, power(g, n) * s0 + (k * power(g, n - 1 - t)[:, None]).T @ v


def backward_row(q, k, v, g, s0, scale, do, ds):
    n = len(q)
    t, w = np.arange(n), weights(n, g)
    p, dp = (q @ k.T) * w * scale, (do @ v.T) * w * scale
    up, down = power(g, t + 1)[:, None], power(g, n - 1 - t)[:, None]
    return (dp @ k + scale * up * (do @ s0.T), dp.T @ q + down * (v @ ds.T), p.T @ do + down * (k @ ds),
            power(g, n) * ds + scale * (q * up).T @ do)


def _head(x, h, heads):
    return x[:, h * x.shape[1] // heads]


def forward(q, k, v, log_decay, offsets, scale, state_in, absolute=False):
    """out [total, heads, dv] (NaN where no row is) and the states [rows, heads, dk, dv]."""
    q, k, v, state_in = (np.abs(np.asarray(x, np.float64)) if absolute else np.asarray(x, np.float64) for x in (q, k, v, state_in))
    heads, scale = len(log_decay), abs(scale) if absolute else scale
    out, states = np.full((len(q), heads, v.shape[2]), np.nan), np.array(state_in)
    for r in range(len(offsets) - 1):
        rows = slice(offsets[r], offsets[r + 1])
        for h in range(heads):
            out[rows, h], states[r, h] = forward_row(_head(q, h, heads)[rows], _head(k, h, heads)[rows], _head(v, h, heads)[rows], log_decay[h],
                                                     state_in[r, h], scale)
    return out, states


def backward(q, k, v, log_decay, offsets, scale, state_in, d_out, d_state, absolute=False):
    """dq, dk, dv (NaN where no row is) and the gradient by state_in."""
    q, k, v, state_in, d_out, d_state = (np.abs(np.asarray(x, np.float64)) if absolute else np.asarray(x, np.float64) for x in (q, k, v, state_in, d_out, d_state))
    heads, scale = len(log_decay), abs(scale) if absolute else scale
    grads, d_in = [np.full(x.shape, np.nan) for x in (q, k, v)], np.empty_like(state_in)
    for r in range(len(offsets) - 1):
        rows = slice(offsets[r], offsets[r + 1])
        for g in grads:
            g[rows] = 0.0
        for h in range(heads):
            *parts, d_in[r, h] = backward_row(_head(q, h, heads)[rows], _head(k, h, heads)[rows], _head(v, h, heads)[rows], log_decay[h], state_in[r, h], scale,
                                              d_out[rows, h], d_state[r, h])
            for g, part in zip(grads, parts):
                g[rows, h * g.shape[1] // heads] += part
    return *grads, d_in


def close(got, want, size, kind, longest, features, state=False):
    """Asserts |got - want| <= (the output's rounding of `want`) + (what is rounded inside, of the sum of the terms' sizes): INNER (states: three parts
    always), and 2^-24 for every addition in a chain of fp32 sums as long as a row is in blocks of 16 tokens and `features` are wide.
    Places of no row (NaN in `want`) are not compared."""
    inside = (2.0 ** -21 if state else INNER[kind]) + (features + 64 + longest / 16) * 2.0 ** -24
    there = ~np.isnan(want)
    bound = UNIT["f32" if state else kind] * np.abs(want) + inside * size + 1e-30
    if kind == "f16" and not state:
        bound = bound + 2.0 ** -25                              # half of the smallest subnormal
    off = np.abs(got.astype(np.float64) - want)[there] / bound[there]
    assert np.isfinite(off).all() and (off <= 1.0).all(), f"{kind}: {off.max() if off.size else 0:.3g} of what rounding explains"

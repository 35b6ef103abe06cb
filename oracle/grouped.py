"""Rotary positions, attention over any length with shared key/value heads, and
the 8-bit key/value cache -- TEST INFRASTRUCTURE ONLY (CPU oracle).

Written out from the definitions in float64 with numpy.  Only the tests may use
it; it shares nothing with the GPU library.

Beside each result `bounds` gives how far a computation may be off that rounds
where the library says it does, element by element, with u the half step of bf16
(2^-8 relative):
  out   u |out| (rounded once) + u sum_j P |v| (P rounded for the product),
  dv    u |dv| + u sum_i P |dout|,
  dq    u |dq| + u scale sum_j |dS| |k|                (dS rounded)
              + scale sum_j P dD |k|,  dD = u sum_d |dout| |out|   (out rounded),
  dk    likewise over the queries of the group,
and for what is held in 32 bits (scores, exponentials, sums) F = 2^-12 of the
same sums of magnitudes: a score is a sum of at most 128 products off by 2^-24
of their magnitudes each, an exponential off by that times the score's size.
"""
from __future__ import annotations

import numpy as np

U, F = 2.0 ** -8, 2.0 ** -12
E4M3_MAX = 448.0
BLOCK = 64


def rotary(x, positions, freqs, half, scale=1.0, inverse=False):
    """x [batch, n, heads, head_dim], positions [batch, n]."""
    x = np.asarray(x, dtype=np.float64)
    rot = 2 * len(freqs)
    t = np.asarray(positions, dtype=np.float64)[..., None] * np.asarray(freqs, dtype=np.float64)
    c, s = np.cos(t)[:, :, None] * scale, np.sin(t)[:, :, None] * scale * (-1 if inverse else 1)
    y = x.copy()
    ia = slice(0, rot // 2) if half else slice(0, rot, 2)
    ib = slice(rot // 2, rot) if half else slice(1, rot, 2)
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y


def _seen(n_q, n_k, causal, length):
    seen = np.broadcast_to(np.arange(n_k) < length, (n_q, n_k)).copy()
    if causal:
        seen &= np.arange(n_k)[None] <= np.arange(n_q)[:, None] + (n_k - n_q)
    return seen


def _probs(q, k, seen, scale):
    s = np.where(seen, scale * (q @ k.T), -np.inf)
    m = s.max(axis=1, initial=-np.inf)
    e = np.where(seen, np.exp(s - np.where(np.isinf(m), 0.0, m)[:, None]), 0.0)
    z = e.sum(axis=1)
    with np.errstate(divide="ignore", invalid="ignore"):
        p = np.where(z[:, None] > 0, e / z[:, None], 0.0)
        return p, np.where(z > 0, m + np.log(z), -np.inf)


def _operands(q, k, v, lengths, scale):
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    scale = q.shape[3] ** -0.5 if scale is None else scale
    lengths = [k.shape[1]] * len(q) if lengths is None else [min(max(int(n), 0), k.shape[1])
                                                            for n in lengths]
    return q, k, v, lengths, scale, q.shape[2] // k.shape[2]


def forward(q, k, v, causal=True, lengths=None, scale=None):
    """(out, lse, bound of out)."""
    q, k, v, lengths, scale, group = _operands(q, k, v, lengths, scale)
    out, bound = np.zeros_like(q), np.zeros_like(q)
    lse = np.full((q.shape[0], q.shape[2], q.shape[1]), -np.inf)
    for b, n in enumerate(lengths):
        seen = _seen(q.shape[1], k.shape[1], causal, n)[:, :n]
        for h in range(q.shape[2] if n else 0):
            vh = v[b, :n, h // group]
            p, lse[b, h] = _probs(q[b, :, h], k[b, :n, h // group], seen, scale)
            out[b, :, h] = p @ vh
            bound[b, :, h] = U * np.abs(out[b, :, h]) + (U + F) * (p @ np.abs(vh))
    return out, lse, bound


def backward(q, k, v, dout, causal=True, lengths=None, scale=None, exact=0):
    """((dq, dk, dv), (their bounds)); out's rounding plays no part in rows that see at
    most `exact` keys."""
    q, k, v, lengths, scale, group = _operands(q, k, v, lengths, scale)
    dout = np.asarray(dout, dtype=np.float64)
    g = [np.zeros_like(t) for t in (q, k, v)]
    e = [np.zeros_like(t) for t in (q, k, v)]
    for b, n in enumerate(lengths):
        seen = _seen(q.shape[1], k.shape[1], causal, n)[:, :n]
        for h in range(q.shape[2] if n else 0):
            c = h // group
            qh, kh, vh, do = q[b, :, h], k[b, :n, c], v[b, :n, c], dout[b, :, h]
            p, _ = _probs(qh, kh, seen, scale)
            o, dp = p @ vh, do @ vh.T
            ds = p * (dp - (do * o).sum(axis=1)[:, None])
            g[0][b, :, h] = scale * ds @ kh
            g[1][b, :n, c] += scale * ds.T @ qh
            g[2][b, :n, c] += p.T @ do
            dd = np.abs(do * o).sum(axis=1)[:, None]
            off = scale * (U * np.abs(ds) + U * p * dd * (seen.sum(axis=1) > exact)[:, None]
                           + F * p * (np.abs(do) @ np.abs(vh).T + dd))
            e[0][b, :, h] = off @ np.abs(kh)
            e[1][b, :n, c] += off.T @ np.abs(qh)
            e[2][b, :n, c] += (U + F) * (p.T @ np.abs(do))
    return tuple(g), tuple(x + U * np.abs(t) for x, t in zip(e, g))


def e4m3(x):
    """The nearest e4m3 number (ties to even), magnitudes held to 448; NaN stays."""
    x = np.asarray(x, dtype=np.float64)
    mag = np.minimum(np.abs(x), E4M3_MAX)
    e = np.maximum(np.frexp(np.where(mag > 0, mag, 1.0))[1] - 1, -6)
    step = np.ldexp(1.0, e - 3)
    return np.where(np.isnan(x), np.nan, np.sign(x) * np.round(mag / step) * step)


def held(x, s):
    """x as e4m3 numbers times s; at the largest scale, 2^120, finite ones are held to 240,
    the last below 2^128."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        q = x / s
    return e4m3(np.where(np.isfinite(q), np.clip(q, -240, 240), q) if s == 2.0 ** 120 else q) * s


def needed_scale(x):
    """The least power of two from 2^-118 to 2^120 by which |x| / 2^e <= 448."""
    mag = np.abs(x[~np.isnan(x)])
    amax = mag.max() if mag.size else 0.0
    e = -118
    while e < 120 and amax > E4M3_MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Cache:
    """One sequence's keys or values: [capacity, heads, head_dim] values held."""

    def __init__(self, capacity, heads, head_dim):
        self.capacity = capacity
        self.held = np.zeros((capacity, heads, head_dim))
        self.scale = np.zeros((-(-capacity // BLOCK), heads))

    def append(self, x, pos):
        if not 0 <= pos < self.capacity:
            return
        x = np.asarray(x, dtype=np.float64)[:self.capacity - pos]
        t = 0
        while t < len(x):
            blk = (pos + t) // BLOCK
            n = min(len(x) - t, (blk + 1) * BLOCK - (pos + t))
            for h in range(x.shape[1]):
                s = needed_scale(x[t:t + n, h])
                old = slice(blk * BLOCK, pos + t)
                if pos + t > blk * BLOCK:
                    s = max(s, self.scale[blk, h])
                    self.held[old, h] = held(self.held[old, h], s)
                self.held[pos + t:pos + t + n, h] = held(x[t:t + n, h], s)
                self.scale[blk, h] = s
            t += n

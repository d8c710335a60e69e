"""CPU oracle of what stands around the sparse path, numpy fp64, from the formulas alone: norm and rotation of queries and keys, attention over a
window and a few first keys, and the backward passes of both.  One head at a time: x [tokens, d], q [n, d], k and v [m, d]."""
from __future__ import annotations

import numpy as np


def turns(pos, dims, theta, interleaved, d):
    """cos, sin [tokens, pairs], and the two channels of every pair."""
    ang, first, second, at = [], [], [], 0
    for axis, n in enumerate(dims):
        i = np.arange(n // 2)
        ang.append(pos[:, axis, None].astype(np.float64) * theta ** (-2.0 * i / n))
        first.append(at + (2 * i if interleaved else i))
        second.append(at + (2 * i + 1 if interleaved else i + n // 2))
        at += n
    a = np.concatenate(ang, axis=1)
    return np.cos(a), np.sin(a), np.concatenate(first), np.concatenate(second)


def qk_norm_rope(x, pos, dims, theta, interleaved, w, eps):
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    c, s, i, j = turns(pos, dims, theta, interleaved, x.shape[-1])
    out = y.copy()
    out[:, i] = y[:, i] * c - y[:, j] * s
    out[:, j] = y[:, i] * s + y[:, j] * c
    return out


def qk_norm_rope_bwd(x, up, pos, dims, theta, interleaved, w, eps):
    """(dx, dw) for the gradient `up` of the result."""
    c, s, i, j = turns(pos, dims, theta, interleaved, x.shape[-1])
    g = up.copy()
    g[:, i] = up[:, i] * c + up[:, j] * s
    g[:, j] = up[:, j] * c - up[:, i] * s
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    gw = g * w
    return r * (gw - n * (gw * n).mean(-1, keepdims=True)), (g * n).sum(0)


def window_mask(n_q, n_k, left, right, sinks):
    """[n_q, n_k]: what a query at position n_k - n_q + i sees."""
    p = (n_k - n_q + np.arange(n_q))[:, None]
    j = np.arange(n_k)[None, :]
    see = np.ones((n_q, n_k), bool) if right < 0 else j <= p + right
    return see if left < 0 else see & ((j >= p - left) | (j < sinks))


def window_attn(q, k, v, see, scale):
    """(o, lse, weights); rows that see nothing have o = 0 and lse = -inf."""
    s = np.where(see, q @ k.T * scale, -np.inf)
    if s.shape[1] == 0:
        return np.zeros(q.shape), np.full(len(q), -np.inf), s
    m = s.max(-1, keepdims=True)
    m = np.where(np.isneginf(m), 0.0, m)
    p = np.exp(s - m)
    total = p.sum(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (m + np.log(total))[:, 0]
    p = p / np.where(total == 0, 1.0, total)
    return p @ v, lse, p


def window_attn_bwd(q, k, v, see, scale, d_o):
    o, _, p = window_attn(q, k, v, see, scale)
    ds = p * (d_o @ v.T - (d_o * o).sum(-1, keepdims=True))
    return scale * ds @ k, scale * ds.T @ q, p.T @ d_o

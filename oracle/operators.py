"""CPU float64 definitions of the transformer operators (linear, rope, qk_norm_rope, attention).

TEST INFRASTRUCTURE ONLY, as oracle/decoder.py: plain loops and numpy float64, sharing no code with
the HIP path. Each function also returns what a rounding bound needs (sums of magnitudes).
"""
from __future__ import annotations

import math

import numpy as np

ERF = np.vectorize(math.erf, otypes=[np.float64])


def activate(v: np.ndarray, act: str) -> np.ndarray:
    if act == "relu":
        return np.where(v < 0, 0.0, v)
    if act == "gelu":
        return 0.5 * v * (1 + ERF(v / math.sqrt(2)))
    if act == "gelu_tanh":
        return 0.5 * v * (1 + np.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    if act == "silu":
        with np.errstate(over="ignore"):
            return v / (1 + np.exp(-v))
    assert act == "none"
    return v


def linear(x, w, bias=None, act="none", residual=None):
    """act(x w^T + bias) + residual, and the magnitudes |x| |w|^T + |bias| its sum runs over."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    v, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        v, mag = v + bias, mag + np.abs(bias)
    y = activate(v, act)
    return (y if residual is None else y + residual), mag


def angles(positions, pairs, theta, shared):
    """[tokens][P] rotation angles; positions [tokens][axes]."""
    out, total, j = [], sum(pairs), 0
    for a, n in enumerate(pairs):
        for i in range(n):
            out.append(np.asarray(positions)[:, a].astype(np.float64) * theta ** -(j / total if shared else i / n))
            j += 1
    return np.stack(out, 1) if out else np.zeros((len(positions), 0))


def rope(x, positions, pairs, theta=10000.0, layout="half", shared=False, inverse=False):
    """Rotates x [tokens][heads][dh]."""
    y = np.array(x, np.float64)
    ang = angles(positions, pairs, theta, shared) * (-1 if inverse else 1)
    P = ang.shape[1]
    for j in range(P):
        a, b = (j, j + P) if layout == "half" else (2 * j, 2 * j + 1)
        c, s = np.cos(ang[:, j])[:, None], np.sin(ang[:, j])[:, None]
        u, v = x[..., a].astype(np.float64), x[..., b].astype(np.float64)
        y[..., a], y[..., b] = u * c - v * s, u * s + v * c
    return y


def rms_norm(x, gain=None, eps=1e-6):
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return y if gain is None else y * gain


def visible(i, n_q, n_k, left, right, sinks):
    """Keys that query i of n_q sees among n_k: a bool [n_k]."""
    j, pos = np.arange(n_k), n_k - n_q + i
    see = np.ones(n_k, bool)
    if right >= 0:
        see &= j <= pos + right
    if left >= 0:
        see &= (j >= pos - left) | (j < sinks)
    return see


def attention(q, k, v, left=-1, right=-1, sinks=0, scale=None, q_lengths=None, k_lengths=None):
    """softmax(scale q k^T) v; q [b][sq][hq][dh], k and v [b][sk][hk][dh]. Rows past a sequence's queries
    are NaN (not defined). Returns (out, sum of weights times |v|, largest |score| bound per row)."""
    b, sq, hq, dh = q.shape
    hk = k.shape[2]
    scale = dh ** -0.5 if scale is None else scale
    out = np.full(q.shape, np.nan)
    mag, top = np.zeros(q.shape), np.zeros((b, sq, hq))
    for s in range(b):
        nq = sq if q_lengths is None else min(max(int(q_lengths[s]), 0), sq)
        nk = k.shape[1] if k_lengths is None else min(max(int(k_lengths[s]), 0), k.shape[1])
        for h in range(hq):
            kk, vv = k[s, :nk, h * hk // hq].astype(np.float64), v[s, :nk, h * hk // hq].astype(np.float64)
            for i in range(nq):
                see = visible(i, nq, nk, left, right, sinks)
                if not see.any():
                    out[s, i, h] = 0.0
                    continue
                qi = q[s, i, h].astype(np.float64)
                z = scale * (kk[see] @ qi)
                p = np.exp(z - z.max())
                p /= p.sum()
                out[s, i, h] = p @ vv[see]
                mag[s, i, h] = p @ np.abs(vv[see])
                top[s, i, h] = scale * (np.abs(kk[see]) @ np.abs(qi)).max()
    return out, mag, top

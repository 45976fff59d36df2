"""Linear attention with decays, the norms of heads with their rotation, and 8-bit
products, from their definitions: numpy, fp64, position by position and with no
regard for speed.  Shares no code with the library."""
from __future__ import annotations

import numpy as np


def attend(q, k, v, decay, scale, state):
    """One sequence: q [T, H, K], k [T, G, K], v [T, G, V], decay [G], state [G, K, V].  Returns (y [T, H, V], state)."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    S, keep = np.array(state, np.float64), np.exp(np.asarray(decay, np.float64))[:, None, None]
    T, H = q.shape[:2]
    G = k.shape[1]
    y = np.zeros((T, H, v.shape[2]))
    with np.errstate(invalid="ignore", over="ignore"):
        for t in range(T):
            S = keep * S + k[t][:, :, None] * v[t][:, None, :]
            # (no library product: those differ in what they make of 0 * inf)
            y[t] = scale * (q[t].reshape(G, H // G, -1)[..., None] * S[:, None]).sum(2).reshape(H, -1)
    return y, S


def heads(x, P, norm, weight, eps, positions, freqs, pairs):
    """Rows x [T, heads P] normed head by head and turned by positions [T] times freqs [rotary / 2]."""
    x = np.asarray(x, np.float64)
    v = x.reshape(len(x), -1, P)
    with np.errstate(invalid="ignore", over="ignore"):
        if norm == "layer":
            v = v - v.mean(-1, keepdims=True)
        if norm != "none":
            v = v / np.sqrt((v * v).mean(-1, keepdims=True) + eps)
            v = v * (1.0 if weight is None else np.asarray(weight, np.float64))
        out, half = np.array(v), len(freqs)
        for j in range(half):
            a, b = (j, j + half) if pairs == "half" else (2 * j, 2 * j + 1)
            # the angle modulo a turn before anything is rounded to it: positions are whole
            angle = np.asarray(positions, np.float64) * freqs[j]
            c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
            out[..., a], out[..., b] = v[..., a] * c - v[..., b] * s, v[..., b] * c + v[..., a] * s
    return out.reshape(x.shape)


def codes(x):
    """(codes, scales) of rows x [R, K] of fp32 values."""
    x = np.asarray(x, np.float64)
    most = np.abs(x).max(-1)
    with np.errstate(invalid="ignore"):
        s = np.where(np.isfinite(most), (most / 127).astype(np.float32), np.nan).astype(np.float64)
        q = np.rint(x / np.where(s > 0, s, 1.0)[:, None])  # ties to even
    q = np.where((s > 0)[:, None], np.clip(q, -127, 127), 0.0)
    return q.astype(np.int64), s


def q8(x, weight_codes, scales, bias):
    """(y, |y| before the bias) of rows x [R, K] against codes [N, K] with scales [N]."""
    c, s = codes(x)
    with np.errstate(invalid="ignore"):
        y = (c @ np.asarray(weight_codes, np.int64).T) * np.asarray(scales, np.float64) * s[:, None]
    return (y if bias is None else y + np.asarray(bias, np.float64)), np.abs(y)

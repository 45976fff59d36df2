"""The selective state space mixer with its short causal convolution, and the
other operators of the gated layer, from their definitions: numpy, fp64,
position by position and with no regard for speed.  Shares no code with the
library."""
from __future__ import annotations

import numpy as np


def silu(v):
    with np.errstate(over="ignore"):
        return v / (1.0 + np.exp(-v))


def scan(xbc, dt, z, conv_w, conv_b, A, skip, dt_bias, G, N, state, window):
    """One sequence: xbc [T, C], dt [T, H], z [T, D] or None, conv_w [C, W], state [H, P, N], window [W-1, C].
    Returns (y [T, D], state, window) after it."""
    xbc, dt, conv_w, conv_b, A, skip, dt_bias = (np.asarray(v, np.float64) for v in
                                                 (xbc, dt, conv_w, conv_b, A, skip, dt_bias))
    S, rows = np.array(state, np.float64), np.concatenate([np.asarray(window, np.float64), xbc])
    H, P, W = S.shape[0], S.shape[1], conv_w.shape[1]
    D, T = H * P, xbc.shape[0]
    y = np.zeros((T, D))
    group = np.arange(H) // (H // G)
    with np.errstate(invalid="ignore", over="ignore"):
        for t in range(T):
            u = conv_b.copy()
            for k in range(W):
                u += conv_w[:, k] * rows[t + k]
            u = silu(u)
            x, Bm, Cm = u[:D].reshape(H, P), u[D:D + G * N].reshape(G, N), u[D + G * N:].reshape(G, N)
            s = np.logaddexp(0.0, dt[t] + dt_bias)
            S = np.exp(s * A)[:, None, None] * S + (s[:, None] * x)[:, :, None] * Bm[group][:, None, :]
            v = (S * Cm[group][:, None, :]).sum(-1) + skip[:, None] * x
            y[t] = v.reshape(D)
        if z is not None:
            y *= silu(np.asarray(z, np.float64))
    return y, S, rows[T:]


def normed(v, kind, w, b, eps):
    """Rows of v [R, D] ("none", "rms" or "layer")."""
    if kind == "none":
        return v
    m = v.mean(-1, keepdims=True) if kind == "layer" else 0.0
    v = (v - m) / np.sqrt(((v - m) ** 2).mean(-1, keepdims=True) + eps)
    return v if w is None and b is None else v * (1.0 if w is None else w) + (0.0 if b is None else b)


def block_norm(o, g, r, post, pre, act, groups, alpha, eps, post_w, post_b, scale, pre_w, pre_b):
    """(r', n) of rows o (or None), g (or None) and r [R, D]."""
    r = alpha * np.asarray(r, np.float64)
    if o is not None:
        v = np.asarray(o, np.float64)
        if act != "none":
            g = np.asarray(g, np.float64)
            v = v * (silu(g) if act == "silu" else 1.0 / (1.0 + np.exp(-g)))
        R, D = v.shape
        v = normed(v.reshape(R * groups, D // groups), post, None, None, eps).reshape(R, D)
        if post != "none":
            v = v * (1.0 if post_w is None else post_w) + (0.0 if post_b is None else post_b)
        r = r + (1.0 if scale is None else scale) * v
    return r, normed(r, pre, pre_w, pre_b, eps)


def q4_weights(codes, scales, zeros, K, group):
    """[N, K] weights that codes [N, ceil(K/2)], scales and zeros (or None) [N, ceil(K/group)] stand for."""
    k = np.arange(K)
    q = (codes[:, k // 2] >> (4 * (k % 2))) & 15
    z = 8 if zeros is None else (zeros[:, k // group] & 15).astype(np.int64)
    return scales[:, k // group].astype(np.float64) * (q.astype(np.int64) - z)

"""The linear attention layer's operators in fp64, straight from their definitions."""

from __future__ import annotations

import numpy as np


def spans(B, T, lengths=None, offsets=None):
    """(row, first token, length) of each sequence."""
    if offsets is not None:
        o = [min(max(int(x), 0), T) for x in offsets]
        return [(0, o[b], max(o[b + 1] - o[b], 0)) for b in range(len(o) - 1)]
    n = [T] * B if lengths is None else [min(max(int(x), 0), T) for x in lengths]
    return [(b, 0, n[b]) for b in range(B)]


def sequence(q, k, v, g, scale, s0):
    """o [n][H][Dv] and the last state of one sequence; q [n][H][Dk], k and v with K heads, s0 [H][Dk][Dv]."""
    share = q.shape[1] // k.shape[1]
    S, o = s0.copy(), np.zeros((q.shape[0], q.shape[1], v.shape[2]))
    a = np.exp(g)[:, None, None]
    for t in range(q.shape[0]):
        S = a * S + np.repeat(k[t][:, :, None] * v[t][:, None, :], share, axis=0)
        o[t] = scale * np.einsum("hd,hde->he", q[t], S)
    return o, S


def sequence_gradients(do, q, k, v, g, scale, s0, ds_last):
    """dq, dk, dv, ds0 of one sequence."""
    n, H, K = q.shape[0], q.shape[1], k.shape[1]
    share = H // K
    S, a = s0.copy(), np.exp(g)[:, None, None]
    dq, dk, dv = np.zeros(q.shape), np.zeros((n, H, k.shape[2])), np.zeros((n, H, v.shape[2]))
    for t in range(n):
        S = a * S + np.repeat(k[t][:, :, None] * v[t][:, None, :], share, axis=0)
        dq[t] = scale * np.einsum("hde,he->hd", S, do[t])
    R = ds_last.copy()
    for t in reversed(range(n)):
        R = R + scale * q[t][:, :, None] * do[t][:, None, :]
        dk[t] = np.einsum("hde,he->hd", R, np.repeat(v[t], share, axis=0))
        dv[t] = np.einsum("hde,hd->he", R, np.repeat(k[t], share, axis=0))
        R = a * R
    return dq, dk.reshape(n, K, share, k.shape[2]).sum(2), dv.reshape(n, K, share, v.shape[2]).sum(2), R


def frequencies(R, base=10000.0, factor=1.0, original=0.0, low=1.0, high=32.0):
    f = base ** (-np.arange(0, R, 2) / R) if R else np.zeros(0)
    stay = np.clip((original * f / (2 * np.pi) - low) / (high - low), 0, 1) if original else 0.0
    return f * (stay + (1 - stay) / factor)


def rotary(x, freq, positions, interleaved, inverse, magnitude):
    """x [B][T][H][D]"""
    R = 2 * len(freq)
    angle = (-1.0 if inverse else 1.0) * positions[..., None].astype(np.longdouble) * freq.astype(np.longdouble)
    angle = angle - np.round(angle / (2 * np.pi)) * (2 * np.longdouble(np.pi)) if np.finfo(np.longdouble).nmant > 60 else angle
    c, s = np.cos(angle).astype(np.float64)[:, :, None], np.sin(angle).astype(np.float64)[:, :, None]
    out = x.copy()
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])
    a, b = magnitude * (a * c - b * s), magnitude * (a * s + b * c)
    if interleaved:
        out[..., 0:R:2], out[..., 1:R:2] = a, b
    else:
        out[..., :R // 2], out[..., R // 2:R] = a, b
    return out


def act(name, u):
    """(act(u), act'(u))"""
    if name == "none":
        return 1.0, 0.0
    with np.errstate(over="ignore"):
        s, rest = 1 / (1 + np.exp(-u)), 1 / (1 + np.exp(u))
    return (u * s, s * (1 + u * rest)) if name == "silu" else (s, s * rest)


def gated_norm(x, weight, gate, residual, next_weight, groups, name, scale, eps):
    rows, cols = x.shape
    xg = x.reshape(rows, groups, -1)
    rstd = 1 / np.sqrt((xg ** 2).mean(-1) + eps)
    y = scale * act(name, gate)[0] * (xg * rstd[..., None]).reshape(rows, cols) * weight
    y = y if residual is None else residual + y
    if next_weight is None:
        return y, rstd, None, None
    next_rstd = 1 / np.sqrt((y ** 2).mean(-1) + eps)
    return y, rstd, y * next_rstd[:, None] * next_weight, next_rstd


def gated_norm_gradients(dy, x, weight, rstd, gate, dz, y, next_weight, next_rstd, groups, name, scale):
    rows, cols = x.shape
    split = lambda t: t.reshape(rows, groups, -1)   # noqa: E731
    t, dnext = 0.0 if dy is None else dy, None
    if dz is not None:
        m, u = y * next_rstd[:, None], dz * next_weight
        t = t + next_rstd[:, None] * (u - m * (u * m).mean(-1, keepdims=True))
        dnext = (dz * m).sum(0)
    n = (split(x) * rstd[..., None]).reshape(rows, cols)
    a, slope = act(name, gate)
    e = scale * t
    p = e * a * weight
    dx = (rstd[..., None] * (split(p) - split(n) * split(p * n).mean(-1, keepdims=True))).reshape(rows, cols)
    return {"dx": dx, "dgate": e * n * weight * slope, "dresidual": t, "dweight": (e * a * n).sum(0), "dnext_weight": dnext}

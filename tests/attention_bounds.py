"""Forward error bounds of the linear attention layer's operators, evaluated in fp64 beside the exact values.

With u = 2^-24 (one fp32 rounding):

* Attention.  o is a sum of terms w q_c k_c v, w = e^(g n), over the contracted c and the tokens.  In any
  order a sum of N terms takes at most N roundings on any term's way; the ways here are at most a head's C
  terms, a block's own tokens, and one addition a block for what has come before: C + T + 40 covers
  them with the products' and the weights' own roundings.  Additions inside a tensor core may cut off instead of rounding to
  nearest, so each counts 2u.  w's exponent is off by |g| n u, and a state that is decayed block by block by one
  rounding for each.  Two-byte types are multiplied by tensor cores whose 16-bit operands hold what is between two
  products (weighted scores, states) as a sum of parts: at least 2^-16 of the larger factor's magnitude
  is kept for a stored output, and 2^-23 for fp32 states.
* Rotary.  Angle: 2^-53 of the frequency times the position (in turns) and 2^-25 half-turns; sine, cosine, and the
  products and the sum: 8u of the pair's magnitude.
* Norms.  As for the norm after dropout (layer_bounds); the gate's exponential is off by (|u| + 4) u and its sigmoid by 4u
  more.

Bounds are doubled once, for terms of second order.  A stored result adds its own rounding (layer_bounds.stored).
"""

from __future__ import annotations

import numpy as np

from tests.layer_bounds import U

SPLIT = {"f32": 0.0, "f16": 2.0 ** -16, "bf16": 2.0 ** -16}


def walk(q, k, v, g, first, dtype, after):
    """Bounds of what one head reads from the state at each position, without its scale, and of the last state, for
    queries [n][C], keys [n][C], values [n][D]; after: tokens between `first` and the first read."""
    n, C = q.shape
    q, k, v, first = np.abs(q), np.abs(k), np.abs(v), np.abs(first)
    count = 2 * (C + n + 40) * U
    i = np.arange(n)
    d = i[:, None] - i[None, :]
    w = np.where(d >= 0, np.exp(g * np.maximum(d, 0)), 0.0)
    e = w * (count + SPLIT[dtype] + np.abs(g) * np.maximum(d, 0) * U)
    far = np.exp(g * (i + after)) * (count + SPLIT[dtype] + np.abs(g) * (i + after) * U)
    out = ((q @ k.T) * e) @ v + far[:, None] * (q @ first)
    end = np.exp(g * (n - 1 - i + 1 - after)) * (count + np.abs(g) * n * U)
    last = (k * end[:, None]).T @ v + np.exp(g * n) * (count + np.abs(g) * n * U) * first
    return 2 * out, 2 * last


def rotary(x, freq, positions, interleaved, magnitude):
    R = 2 * len(freq)
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])
    size = np.sqrt(a * a + b * b) * abs(magnitude)
    angle = np.abs(positions)[..., None] * np.abs(freq) * 2.0 ** -52 + 2.0 ** -24 * np.pi
    e = 2 * size * (angle[:, :, None] + 8 * U)
    out = np.zeros(x.shape)
    if interleaved:
        out[..., 0:R:2] = out[..., 1:R:2] = e
    else:
        out[..., :R // 2] = out[..., R // 2:R] = e
    return out


def _gate(name, u):
    """Size and error of act(u) and of its slope."""
    from oracle import attention

    if name == "none":
        return 1.0, 0.0, 0.0, 0.0
    a, slope = attention.act(name, u)
    rel = (np.abs(u) + 10) * U
    s = attention.act("sigmoid", u)[0]
    big = s * (1 + np.abs(u) * (1 - s)) if name == "silu" else slope
    return np.abs(a), np.abs(a) * rel, np.abs(slope), big * 3 * rel


def gated_norm(x, weight, gate, residual, next_weight, groups, name, scale, eps):
    """Bounds of y, relative ones of rstd, and of z and next_rstd."""
    from oracle import attention

    rows, cols = x.shape
    width = cols // groups
    rel = (width + 10) * U
    size, err, _, _ = _gate(name, gate)
    n = np.abs(attention.gated_norm(x, weight, None, None, None, groups, "none", scale, eps)[0])
    e = n * err + n * size * (rel + 6 * U)
    y = attention.gated_norm(x, weight, gate, residual, None, groups, name, scale, eps)[0]
    e = e + U * np.abs(y)
    if next_weight is None:
        return 2 * e, 2 * rel, None, None
    mean = (y ** 2).mean(-1, keepdims=True) + eps
    rel2 = (cols + 10) * U + (np.abs(y) * 2 * e).mean(-1, keepdims=True) / mean
    r2 = 1 / np.sqrt(mean)
    return 2 * e, 2 * rel, 2 * np.abs(next_weight) * r2 * (np.abs(y) * (rel2 + 3 * U) + 2 * e), 2 * rel2[:, 0]


def gated_norm_gradients(dy, x, weight, rstd, gate, dz, y, next_weight, next_rstd, groups, name, scale):
    rows, cols = x.shape
    width = cols // groups
    split = lambda t: t.reshape(rows, groups, -1)   # noqa: E731
    t, et, dnext = (0.0, 0.0, None) if dy is None else (np.abs(dy), U * np.abs(dy), None)
    if dz is not None:
        m, u = np.abs(y * next_rstd[:, None]), np.abs(dz * next_weight)
        mean = (u * m).mean(-1, keepdims=True)
        part = next_rstd[:, None] * (u + m * mean)
        t, et = t + part, et + U * (t + next_rstd[:, None] * (5 * u + m * mean * (cols + 14)))
        dnext = 2 * U * (rows + 6) * (np.abs(dz) * m).sum(0)
    n = np.abs(split(x) * rstd[..., None]).reshape(rows, cols)
    a, ea, s, es = _gate(name, gate)
    e, ee, w = abs(scale) * t, abs(scale) * (et + U * t), np.abs(weight)
    p, ep = e * a * w, (ee * a + e * ea) * w + 3 * U * e * a * w
    pn, epn = split(p * n), split(ep * n + 3 * U * p * n)
    mean, emean = pn.mean(-1, keepdims=True), epn.mean(-1, keepdims=True) + (width + 4) * U * pn.mean(-1, keepdims=True)
    r = rstd[..., None]
    dx = r * (split(ep) + split(n) * emean + 5 * U * (split(p) + split(n) * mean))
    dw = (e * ea + ee * a) * n + 4 * U * e * a * n
    return {"dx": 2 * dx.reshape(rows, cols), "dgate": 2 * n * w * (ee * s + e * es + 4 * U * e * s), "dresidual": 2 * et,
            "dweight": 2 * (dw.sum(0) + (rows + 6) * U * (e * a * n).sum(0)), "dnext_weight": dnext}

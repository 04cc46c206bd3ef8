"""Forward error bounds of the recurrent layer's operators computed in fp32, evaluated in fp64
beside the exact values.

With u = 2^-24 (one fp32 rounding) and, for the GPU's approximate functions, the documented
2^-22 of the base-two exponential and one ulp (2u) of reciprocal and square root:

* sigmoid(v): the exponent's product is off by |v| u, the exponential by 4u, sum and reciprocal
  by 3u: (|v| + 7) u.
* rate = c softplus(decay): 8u.  log a: eps_l = (|r| + 17) u.  a: eps_a = |log a| eps_l + 4u.
* 1 - a^2: log a's error enters with a factor of at most one (|q| e^q / (1 - e^q) <= 1), the
  evaluation with at most 16u on either branch; the square root halves that and adds 3u.
* the recurrence E_t = a (E_{t-1} + (eps_a + 2u) M_{t-1}) + (eps_b + u) |b_t| with M_t = a M_{t-1} + |b_t|
  bounds the error of h whichever way the maps of runs are composed: every product of decays takes
  one more rounding for each factor, every sum one of a partial result that M bounds.

Bounds are doubled once, for terms of second order.  A stored result adds its own rounding.
"""

from __future__ import annotations

import numpy as np

from oracle import layer

U = 2.0 ** -24
ROUND = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
SMALLEST = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}


def stored(exact, err, dtype: str):
    """Allowed distance of a stored value from `exact` when the value before storing is off by err."""
    return err + ROUND[dtype] * (np.abs(exact) + err) + SMALLEST[dtype]


def gate_errors(x, r, i, decay, c):
    """Magnitudes and relative errors of what a token's gates give."""
    sr, si, la, a, gain = layer.gates(r, i, decay, c)
    e = {"sr": (np.abs(r) + 7) * U, "si": (np.abs(i) + 7) * U, "l": (np.abs(r) + 17) * U}
    e["a"] = np.abs(la) * e["l"] + 4 * U
    e["gain"] = (e["l"] + 16 * U) / 2 + 3 * U
    e["b"] = e["gain"] + e["si"] + 3 * U
    return sr, si, la, a, gain, e


def recurrence(x, r, i, decay, h0, reset, lengths, c, dy=None, dh_last=None):
    """Bounds (before storing) of y and h_last, and with dy of the gradients."""
    x, r, i = (np.asarray(v, dtype=np.float64) for v in (x, r, i))
    B, T, D = x.shape
    n = [T if lengths is None else min(max(int(l), 0), T) for l in (lengths if lengths is not None else [T] * B)]
    sr, si, la, a, gain, e = gate_errors(x, r, i, decay, c)
    if reset is not None:
        cut = np.asarray(reset).astype(bool)
        a, gain = np.where(cut[..., None], 0.0, a), np.where(cut[..., None], 1.0, gain)
    E, M = np.zeros((B, T + 1, D)), np.zeros((B, T + 1, D))
    M[:, 0] = np.abs(h0) if h0 is not None else 0.0
    for b in range(B):
        for t in range(n[b]):
            at, bt = a[b, t], gain[b, t] * si[b, t] * np.abs(x[b, t])
            carry, size = (E[b, t], M[b, t]) if not (reset is not None and cut[b, t]) else (0.0, 0.0)
            E[b, t + 1] = at * (carry + (e["a"][b, t] + 2 * U) * size) + (e["b"][b, t] + U) * bt
            M[b, t + 1] = at * size + bt
        E[b, n[b] + 1:] = 0.0
    out = {"y": 2 * E[:, 1:], "h_last": 2 * np.stack([E[b, n[b]] for b in range(B)])}
    if dy is None:
        return out
    dy = np.abs(np.asarray(dy, dtype=np.float64))
    for k in ("dx", "dr", "di"):
        out[k] = np.zeros((B, T, D))
    out["dh0"], dd, slope = np.zeros((B, D)), np.zeros(D), c * layer.sigmoid(np.asarray(decay, dtype=np.float64))
    total = np.zeros(D)
    for b in range(B):
        ef, mf = np.zeros(D), np.abs(dh_last[b]) if dh_last is not None else np.zeros(D)
        for t in range(n[b] - 1, -1, -1):
            s = (b, t)
            eg, mg = ef + U * (mf + dy[s]), mf + dy[s]
            k, ax = gain[s], np.abs(x[s])
            out["dx"][s] = k * si[s] * (eg + mg * (e["gain"][s] + e["si"][s] + 3 * U))
            out["di"][s] = k * ax * si[s] * ((1 - si[s]) * (eg + mg * (e["gain"][s] + e["si"][s] + 4 * U))
                                             + mg * (si[s] * e["si"][s] + U))
            if reset is not None and cut[s]:
                ef, mf = np.zeros(D), np.zeros(D)
                continue
            inv = np.divide(1.0, k, out=np.zeros_like(k), where=k > 0)
            t1, t2 = a[s] * mg * M[b, t], a[s] ** 2 * mg * si[s] * ax * inv
            edla = (a[s] * (eg * M[b, t] + mg * E[b, t]) + t1 * (e["a"][s] + 4 * U)
                    + a[s] ** 2 * eg * si[s] * ax * inv + t2 * (2 * e["a"][s] + e["gain"][s] + e["si"][s] + 6 * U))
            la_, sr_ = np.abs(la[s]), sr[s]
            out["dr"][s] = la_ * ((1 - sr_) * (edla + (t1 + t2) * (e["l"][s] + 4 * U)) + (t1 + t2) * (sr_ * e["sr"][s] + U))
            dd += sr_ * (edla + (t1 + t2) * (e["sr"][s] + U))
            total += sr_ * (t1 + t2)
            ef, mf = a[s] * (eg + (e["a"][s] + 2 * U) * mg), a[s] * mg
        out["dh0"][b] = ef
    # the sum over all tokens, in any order: one rounding for each addition
    out["ddecay"] = slope * (dd + total * U * (sum(n) + 20))
    for k in ("dx", "dr", "di", "dh0", "ddecay"):
        out[k] = 2 * out[k]
    return out


def dropout(x, scale: float, residual=None):
    """Three roundings: of the scale, the product and the sum."""
    x = np.where(np.isfinite(x), np.abs(x), 0.0)
    return 3 * U * (x * scale + (0 if residual is None else np.abs(residual)))


def add_norm(y, e_y, weight, cols: int):
    """(err of z, relative err of rstd): a sum of squares takes at most one rounding for each of
    its terms, so cols + 8 with the mean, eps, and the square root's own."""
    mean = np.mean(y * y, axis=-1, keepdims=True)
    rel = (cols + 8) * U + np.mean(np.abs(y) * e_y, axis=-1, keepdims=True) / np.maximum(mean, 1e-30)
    rstd = 1 / np.sqrt(np.maximum(mean, 1e-30))
    return 2 * np.abs(weight) * rstd * (np.abs(y) * (rel + 3 * U) + e_y), 2 * rel[..., 0]


def add_norm_backward(dz, dy, y, weight, rstd):
    """(err of dresidual, err of dweight) before storing."""
    rows, cols = y.shape
    n, u = np.abs(y * rstd[:, None]), np.abs(dz * weight)
    mean = np.mean(u * n, axis=1, keepdims=True)
    d = 0.0 if dy is None else np.abs(dy)
    e_t = U * (rstd[:, None] * (4 * u + n * mean * (cols + 12)) + 2 * d)
    return 2 * e_t, 2 * U * (rows + 4) * (np.abs(dz) * n).sum(axis=0)

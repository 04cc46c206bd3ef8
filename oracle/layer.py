"""The recurrent layer's operators in fp64 numpy, token by token and element by element, from
their definitions: the counter-based generator, dropout, dropout + residual + RMS norm, and the
gated linear recurrence, each with its gradient.  Shares nothing with the CUDA code.
"""

from __future__ import annotations

import numpy as np

_LOW = np.uint64(0xFFFFFFFF)


def philox4x32(counter, key, rounds: int = 10):
    """Philox4x32 (Salmon, Moraes, Dror and Shaw, SC 2011) on four arrays of 32-bit counter words
    and two key words; returns four uint64 arrays of 32-bit words."""
    c = [np.asarray(w, dtype=np.uint64) & _LOW for w in counter]
    k0, k1 = int(key[0]) & 0xFFFFFFFF, int(key[1]) & 0xFFFFFFFF
    for _ in range(rounds):
        m0 = c[0] * np.uint64(0xD2511F53)
        m1 = c[2] * np.uint64(0xCD9E8D57)
        c = [(m1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), m1 & _LOW,
             (m0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), m0 & _LOW]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def dropout_threshold(p: float) -> int:
    return int(np.floor(float(np.float32(p)) * 65536.0 + 0.5))


def dropout_kept(n: int, p: float, seed: int, offset: int, first: int = 0) -> np.ndarray:
    """Whether the elements first ... first + n - 1 are kept."""
    e = np.arange(first, first + n, dtype=np.uint64)
    block = e >> np.uint64(3)
    words = philox4x32((block & _LOW, block >> np.uint64(32), offset & 0xFFFFFFFF, offset >> 32),
                       (seed & 0xFFFFFFFF, seed >> 32))
    which = (e & np.uint64(7)).astype(np.int64)
    word = np.choose(which // 2, words)
    u = np.where(which % 2 == 0, word & np.uint64(0xFFFF), word >> np.uint64(16))
    return u >= np.uint64(dropout_threshold(p))


def dropout(x, p: float, seed: int, offset: int, residual=None) -> np.ndarray:
    x = np.asarray(x, dtype=np.float64)
    t = dropout_threshold(p)
    kept = dropout_kept(x.size, p, seed, offset).reshape(x.shape)
    out = np.zeros_like(x)
    if t < 65536:
        out[kept] = x[kept] * (65536.0 / (65536 - t))
    return out if residual is None else out + np.asarray(residual, dtype=np.float64)


def add_norm(x, residual, weight, p: float, seed: int, offset: int, eps: float):
    """(y, z, rstd)."""
    y = dropout(x, p, seed, offset, residual)
    rstd = 1.0 / np.sqrt(np.mean(y * y, axis=-1) + eps)
    return y, y * rstd[..., None] * np.asarray(weight, dtype=np.float64), rstd


def add_norm_backward(dz, dy, y, weight, rstd, p: float, seed: int, offset: int):
    """(dx, dresidual, dweight) for 2-d arrays."""
    dz, y, rstd = (np.asarray(v, dtype=np.float64) for v in (dz, y, rstd))
    n = y * rstd[:, None]
    u = dz * np.asarray(weight, dtype=np.float64)
    dt = rstd[:, None] * (u - n * np.mean(u * n, axis=1, keepdims=True))
    if dy is not None:
        dt = dt + np.asarray(dy, dtype=np.float64)
    return dropout(dt, p, seed, offset), dt, (dz * n).sum(axis=0)


def sigmoid(x):
    return np.where(x >= 0, 1.0, np.exp(np.minimum(x, 0))) / (1.0 + np.exp(-np.abs(x)))


def softplus(x):
    return np.maximum(x, 0) + np.log1p(np.exp(-np.abs(x)))


def gates(r, i, decay, c: float):
    """(sigmoid(r), sigmoid(i), log a, a, sqrt(1 - a^2))."""
    sr, si = sigmoid(np.asarray(r, dtype=np.float64)), sigmoid(np.asarray(i, dtype=np.float64))
    la = -c * softplus(np.asarray(decay, dtype=np.float64)) * sr
    return sr, si, la, np.exp(la), np.sqrt(-np.expm1(2 * la))


def recurrence(x, r, i, decay, h0=None, reset=None, lengths=None, c: float = 8.0):
    """(y, h_last, h): h[:, t] is the state before token t, in [B][T][D] arrays."""
    x = np.asarray(x, dtype=np.float64)
    B, T, D = x.shape
    _, si, _, a, gain = gates(r, i, decay, c)
    state = np.zeros((B, D)) if h0 is None else np.array(h0, dtype=np.float64)
    y, before = np.zeros((B, T, D)), np.zeros((B, T, D))
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        for t in range(n):
            before[b, t] = state[b]
            if reset is not None and reset[b, t]:
                state[b] = si[b, t] * x[b, t]
            else:
                state[b] = a[b, t] * state[b] + gain[b, t] * si[b, t] * x[b, t]
            y[b, t] = state[b]
    return y, state, before


def recurrence_backward(dy, dh_last, x, r, i, decay, h0=None, reset=None, lengths=None, c: float = 8.0):
    """Dict of dx, dr, di, ddecay, dh0."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    B, T, D = x.shape
    sr, si, la, a, gain = gates(r, i, decay, c)
    before = recurrence(x, r, i, decay, h0, reset, lengths, c)[2]
    out = {k: np.zeros((B, T, D)) for k in ("dx", "dr", "di")}
    out["ddecay"] = np.zeros(D)
    flow = np.zeros((B, D)) if dh_last is None else np.array(dh_last, dtype=np.float64)
    slope = -c * sigmoid(np.asarray(decay, dtype=np.float64))
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        for t in range(n - 1, -1, -1):
            at = (b, t)
            g = dy[at] + flow[b]
            cut = reset is not None and reset[at]
            k = np.ones(D) if cut else gain[at]
            out["dx"][at] = g * k * si[at]
            out["di"][at] = g * k * x[at] * si[at] * (1 - si[at])
            if cut:
                flow[b] = 0.0
                continue
            inverse = np.divide(1.0, k, out=np.zeros_like(k), where=k > 0)
            dla = g * (a[at] * before[at] - si[at] * x[at] * a[at] ** 2 * inverse)
            out["dr"][at] = dla * la[at] * (1 - sr[at])
            out["ddecay"] += dla * sr[at] * slope
            flow[b] = a[at] * g
    out["dh0"] = flow
    return out


def recurrence_step(x, r, i, decay, state, slots=None, c: float = 8.0):
    """(y, new state)."""
    x, state = np.asarray(x, dtype=np.float64), np.array(state, dtype=np.float64)
    _, si, _, a, gain = gates(r, i, decay, c)
    y = np.zeros_like(x)
    for b in range(x.shape[0]):
        s = b if slots is None else int(slots[b])
        if 0 <= s < state.shape[0]:
            state[s] = a[b] * state[s] + gain[b] * si[b] * x[b]
            y[b] = state[s]
    return y, state

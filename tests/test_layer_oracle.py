"""Pins of the recurrent layer's fp64 oracle (CPU): the generator's published vectors, closed
forms, and every gradient against central differences."""

import numpy as np
import pytest

from oracle import layer


def test_philox_published_vectors():
    """The known-answer vectors published with the generator (10 rounds)."""
    ones = 0xFFFFFFFF
    cases = [((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
             ((ones,) * 4, (ones,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
             ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
              (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]
    for counter, key, want in cases:
        got = layer.philox4x32([np.array([w]) for w in counter], key)
        assert tuple(int(w[0]) for w in got) == want


def test_dropout_rate_and_slices():
    n, p = 400_000, 0.1
    kept = layer.dropout_kept(n, p, 12345, 6)
    t = layer.dropout_threshold(p)
    mean, sd = 1 - t / 65536, np.sqrt(t / 65536 * (1 - t / 65536) / n)
    assert abs(kept.mean() - mean) < 5 * sd
    assert np.array_equal(layer.dropout_kept(1000, p, 12345, 6, first=777), kept[777:1777])
    assert not np.array_equal(layer.dropout_kept(n, p, 12345, 7), kept)
    assert not np.array_equal(layer.dropout_kept(n, p, 12346, 6), kept)
    assert layer.dropout_kept(n, 0.0, 1, 2).all() and not layer.dropout_kept(n, 1.0, 1, 2).any()


def test_dropout_is_zero_where_dropped_whatever_was_there():
    x = np.full(64, np.inf)
    out = layer.dropout(x, 0.5, 3, 4)
    kept = layer.dropout_kept(64, 0.5, 3, 4)
    assert np.all(out[~kept] == 0) and np.all(np.isinf(out[kept]))


def test_recurrence_closed_forms():
    rng = np.random.default_rng(0)
    B, T, D = 2, 9, 3
    x, i = rng.standard_normal((2, B, T, D))
    decay, h0 = rng.standard_normal(D), rng.standard_normal((B, D))
    # a closed recurrence gate keeps the state and lets nothing in
    y, h, _ = layer.recurrence(x, np.full((B, T, D), -1e3), i, decay, h0)
    assert np.allclose(y, h0[:, None]) and np.allclose(h, h0)
    # a very fast decay forgets everything: y is the gated input
    y, _, _ = layer.recurrence(x, np.full((B, T, D), 1e3), i, np.full(D, 100.0), h0)
    assert np.allclose(y, layer.sigmoid(i) * x)
    # a reset at every token does the same, whatever the state was
    y, _, _ = layer.recurrence(x, i, i, decay, np.full((B, D), np.inf), np.ones((B, T)))
    assert np.allclose(y, layer.sigmoid(i) * x)
    # constant gates: a geometric sum
    r = np.zeros((B, T, D))
    _, si, _, a, gain = layer.gates(r, i, decay, 8.0)
    y, _, _ = layer.recurrence(np.ones((B, T, D)), r, np.full((B, T, D), 1e3), decay, np.zeros((B, D)))
    k = np.arange(1, T + 1)[None, :, None]
    assert np.allclose(y, gain * (1 - a ** k) / (1 - a))


def test_recurrence_lengths():
    rng = np.random.default_rng(1)
    B, T, D = 3, 6, 2
    x, r, i = rng.standard_normal((3, B, T, D))
    decay, h0 = rng.standard_normal(D), rng.standard_normal((B, D))
    y, h, _ = layer.recurrence(x, r, i, decay, h0, lengths=[0, 4, 6])
    assert np.all(y[0] == 0) and np.array_equal(h[0], h0[0]) and np.all(y[1, 4:] == 0)
    y4, h4, _ = layer.recurrence(x[1:2, :4], r[1:2, :4], i[1:2, :4], decay, h0[1:2])
    assert np.array_equal(y[1, :4], y4[0]) and np.array_equal(h[1], h4[0])


def test_recurrence_step_is_one_token():
    rng = np.random.default_rng(2)
    B, D = 4, 5
    x, r, i = rng.standard_normal((3, B, D))
    decay, state = rng.standard_normal(D), rng.standard_normal((6, D))
    y, after = layer.recurrence_step(x, r, i, decay, state, [5, -1, 0, 6])
    want, h, _ = layer.recurrence(x[[0, 2], None], r[[0, 2], None], i[[0, 2], None], decay, state[[5, 0]])
    assert np.array_equal(y[[0, 2]], want[:, 0]) and np.all(y[[1, 3]] == 0)
    assert np.array_equal(after[[5, 0]], h) and np.array_equal(after[1:5], state[1:5])


def _differences(f, v, step=1e-6):
    out = np.empty(v.size)
    flat = v.reshape(-1)
    for k in range(v.size):
        keep = flat[k]
        flat[k] = keep + step
        hi = f()
        flat[k] = keep - step
        lo = f()
        flat[k] = keep
        out[k] = (hi - lo) / (2 * step)
    return out.reshape(v.shape)


@pytest.mark.parametrize("masked", [False, True])
def test_recurrence_gradient_against_differences(masked):
    rng = np.random.default_rng(3)
    B, T, D = 2, 7, 3
    x, r, i, dy = rng.standard_normal((4, B, T, D))
    decay, h0, dh = rng.standard_normal(D) - 2, rng.standard_normal((B, D)), rng.standard_normal((B, D))
    reset = (rng.random((B, T)) < 0.25) if masked else None
    lengths = [5, 7] if masked else None

    def loss():
        y, h, _ = layer.recurrence(x, r, i, decay, h0, reset, lengths)
        return float((y * dy).sum() + (h * dh).sum())

    got = layer.recurrence_backward(dy, dh, x, r, i, decay, h0, reset, lengths)
    for name, v in (("dx", x), ("dr", r), ("di", i), ("ddecay", decay), ("dh0", h0)):
        # central differences of step 1e-6 in fp64: truncation 1e-12, rounding 1e-16 / 1e-6 of a loss of order 10
        np.testing.assert_allclose(got[name], _differences(loss, v), rtol=1e-6, atol=2e-8, err_msg=name)


def test_add_norm_gradient_against_differences():
    rng = np.random.default_rng(4)
    rows, cols, p, seed, offset, eps = 3, 11, 0.3, 9, 2, 1e-3
    x, residual, dz, dy = rng.standard_normal((4, rows, cols))
    weight = rng.standard_normal(cols)

    def loss():
        y, z, _ = layer.add_norm(x, residual, weight, p, seed, offset, eps)
        return float((z * dz).sum() + (y * dy).sum())

    y, _, rstd = layer.add_norm(x, residual, weight, p, seed, offset, eps)
    dx, dres, dw = layer.add_norm_backward(dz, dy, y, weight, rstd, p, seed, offset)
    for got, v in ((dx, x), (dres, residual), (dw, weight)):
        np.testing.assert_allclose(got, _differences(loss, v), rtol=1e-6, atol=2e-8)

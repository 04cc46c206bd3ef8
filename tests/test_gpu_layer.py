"""The recurrent layer's operators on the GPU against their fp64 oracle, within the bounds of
tests/layer_bounds.py, at the sizes, strides and masks where they can go wrong."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layer  # noqa: E402
from tests import layer_bounds as bounds  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
C = 8.0


@pytest.fixture(scope="module")
def gs():
    import paper_2108_06004_gb300 as lib
    lib.load_library()
    torch.cuda.set_device(0)
    return lib


def put(a, dtype="f32", pad=0, shift=0):
    """A device tensor of these values, `pad` unused elements after each row, the first element
    `shift` elements past an aligned address; and the values as stored, in fp64."""
    a = np.asarray(a)
    shape = a.shape[:-1] + (a.shape[-1] + pad,)
    flat = torch.full((int(np.prod(shape)) + shift,), float("nan"), dtype=DT[dtype], device="cuda")
    t = flat[shift:].view(shape)[..., :a.shape[-1]]
    t.copy_(torch.from_numpy(np.ascontiguousarray(a)).to(DT[dtype]))
    return t, host(t)


def host(t):
    return t.detach().double().cpu().numpy()


def empty(shape, dtype="f32", pad=0, shift=0, fill=float("nan")):
    return put(np.full(shape, fill), dtype, pad, shift)[0]


def close(got, exact, tol, what):
    got = host(got) if torch.is_tensor(got) else got
    bad = ~(np.abs(got - exact) <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} outside, first at {np.argwhere(bad)[0]}: "
                           f"{got[bad][0]!r} for {exact[bad][0]!r} +- {tol[bad][0]!r}")


# ---- dropout ----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (1, 7, 0, 0), (1, 8, 0, 0), (3, 5, 0, 0), (5, 1001, 0, 0),
                                                 (4, 64, 8, 0), (4, 64, 5, 0), (7, 61, 3, 0), (2, 4099, 0, 1),
                                                 (33, 256, 0, 3), (1, 100_003, 0, 0)])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(gs, dtype, rows, cols, pad, shift, residual):
    rng = np.random.default_rng(rows * 1000 + cols)
    p, seed, offset = 0.3, 0xFEDCBA9876543210, (1 << 33) + 5
    x, xv = put(rng.standard_normal((rows, cols)), dtype, pad, shift)
    res, rv = put(rng.standard_normal((rows, cols)), dtype, 0, shift) if residual else (None, None)
    out = empty((rows, cols), dtype, pad, shift)
    gs.gs_dropout(x, out, p, seed, offset, residual=res)
    exact = layer.dropout(xv, p, seed, offset, rv)
    scale = 65536 / (65536 - layer.dropout_threshold(p))
    close(out, exact, bounds.stored(exact, bounds.dropout(xv, scale, rv), dtype), "out")
    if not residual:
        kept = layer.dropout_kept(rows * cols, p, seed, offset).reshape(rows, cols)
        assert np.array_equal(host(out) != 0, kept & (xv != 0))
        dx = empty((rows, cols), dtype)
        gs.gs_dropout_backward(x, dx, p, seed, offset)
        assert torch.equal(dx, out)


@pytest.mark.parametrize("p", [0.0, 1.0, 2.0 ** -17, 2.0 ** -16, 1 - 2.0 ** -16, 0.5])
def test_dropout_probabilities(gs, p):
    n = 200_003
    x = torch.randn(n, device="cuda")
    out = torch.empty_like(x)
    gs.gs_dropout(x, out, p, 5, 6)
    exact = layer.dropout(host(x), p, 5, 6)
    t = layer.dropout_threshold(p)
    close(out, exact, bounds.stored(exact, bounds.dropout(host(x), 65536 / max(65536 - t, 1)), "f32"), "out")
    if t == 0:
        assert torch.equal(out, x)
    if t == 65536:
        assert not out.any()


def test_dropout_masks_what_is_not_finite(gs):
    n, p = 4096, 0.4
    kept = layer.dropout_kept(n, p, 8, 9)
    x = torch.ones(n, device="cuda")
    x[torch.from_numpy(~kept).cuda()] = float("nan")
    x[3::7] = float("inf")
    out = torch.empty_like(x)
    gs.gs_dropout(x, out, p, 8, 9)
    got = host(out)
    assert np.all(got[~kept] == 0) and not np.isnan(got).any()
    assert np.all(np.isinf(got[3::7]) == kept[3::7])


def test_dropout_in_place_and_shapes(gs):
    x = torch.randn(3, 4, 5, 24, device="cuda", dtype=torch.bfloat16)
    want = torch.empty_like(x)
    gs.gs_dropout(x, want, 0.2, 1, 2)
    flat = torch.empty(x.numel(), device="cuda", dtype=torch.bfloat16)
    gs.gs_dropout(x.view(-1), flat, 0.2, 1, 2)
    assert torch.equal(flat.view_as(x), want)
    y = x.clone()
    gs.gs_dropout(y, y, 0.2, 1, 2)
    assert torch.equal(y, want)
    # a slice of a wider tensor takes the same mask: it is indexed by the slice's own positions
    wide = torch.zeros(60, 40, device="cuda", dtype=torch.bfloat16)
    wide[:, 8:32] = x.view(60, 24)
    out = torch.empty(60, 24, device="cuda", dtype=torch.bfloat16)
    gs.gs_dropout(wide[:, 8:32], out, 0.2, 1, 2)
    assert torch.equal(out.view_as(x), want)
    # one row for all (stride 0)
    row = torch.randn(1, 24, device="cuda", dtype=torch.bfloat16)
    a, b = torch.empty(60, 24, device="cuda", dtype=torch.bfloat16), torch.empty(60, 24, device="cuda", dtype=torch.bfloat16)
    gs.gs_dropout(row.expand(60, 24), a, 0.2, 1, 2)
    gs.gs_dropout(row.expand(60, 24).contiguous(), b, 0.2, 1, 2)
    assert torch.equal(a, b)


def test_dropout_past_32_bits(gs):
    n = (1 << 32) + 8 * 1000 + 3
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    gs.gs_dropout(x, x, 0.25, 77, 3)
    for first in (0, (1 << 31) - 500, (1 << 32) - 500, n - 1003):
        kept = layer.dropout_kept(1003, 0.25, 77, 3, first=first)
        assert np.array_equal(host(x[first:first + 1003]) != 0, kept), first


# ---- dropout, add, norm -------------------------------------------------------------------------

NORM_SHAPES = [(1, 1, 0, 0), (3, 7, 0, 0), (9, 256, 0, 0), (5, 257, 0, 0), (17, 512, 8, 0), (6, 1001, 0, 0),
               (5, 1024, 0, 1), (4, 2048, 24, 0), (3, 2056, 5, 0), (700, 64, 0, 0), (3, 4096, 0, 0), (2, 8192, 0, 0),
               (2, 8200, 0, 0), (2, 16384, 0, 0), (1, 16383, 0, 0)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,shift", NORM_SHAPES)
def test_add_norm(gs, dtype, rows, cols, pad, shift):
    rng = np.random.default_rng(rows + cols)
    p, seed, offset, eps = 0.1, 99, 7, 1e-5
    x, xv = put(rng.standard_normal((rows, cols)), dtype, pad, shift)
    res, rv = put(rng.standard_normal((rows, cols)), dtype, 0, shift)
    w, wv = put(1 + 0.1 * rng.standard_normal(cols))
    y, z = empty((rows, cols), dtype, pad, shift), empty((rows, cols), dtype)
    rstd = empty((rows,))
    gs.gs_dropout_add_norm(x, res, w, y, z, rstd, p, seed, offset, eps=eps)
    ey, ez, er = layer.add_norm(xv, rv, wv, p, seed, offset, eps)
    e_y = bounds.dropout(xv, 65536 / (65536 - layer.dropout_threshold(p)), rv)
    close(y, ey, bounds.stored(ey, e_y, dtype), "y")
    e_z, rel = bounds.add_norm(ey, e_y, wv, cols)
    close(z, ez, bounds.stored(ez, e_z, dtype), "z")
    close(rstd, er, er * rel, "rstd")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,shift", NORM_SHAPES)
@pytest.mark.parametrize("with_dy", [True, False])
def test_add_norm_backward(gs, dtype, rows, cols, pad, shift, with_dy):
    rng = np.random.default_rng(rows * 3 + cols)
    p, seed, offset = 0.1, 99, 7
    y, yv = put(rng.standard_normal((rows, cols)), dtype, pad, shift)
    dz, dzv = put(rng.standard_normal((rows, cols)), dtype, 0, shift)
    dy, dyv = put(rng.standard_normal((rows, cols)), dtype, pad, shift) if with_dy else (None, None)
    w, wv = put(1 + 0.1 * rng.standard_normal(cols))
    rstd, rv = put(1 / np.sqrt((yv * yv).mean(axis=1) + 1e-6))
    dx, dres, dw = empty((rows, cols), dtype, pad, shift), empty((rows, cols), dtype), empty((cols,))
    ws = torch.empty(gs.gs_dropout_add_norm_workspace_size(rows, cols), dtype=torch.uint8, device="cuda")
    gs.gs_dropout_add_norm_backward(dz, dy, y, w, rstd, dx, dres, dw, p, seed, offset, ws)
    ex, et, ew = layer.add_norm_backward(dzv, dyv, yv, wv, rv, p, seed, offset)
    e_t, e_w = bounds.add_norm_backward(dzv, dyv, yv, wv, rv)
    scale = 65536 / (65536 - layer.dropout_threshold(p))
    close(dres, et, bounds.stored(et, e_t, dtype), "dresidual")
    close(dx, ex, bounds.stored(ex, scale * (e_t + 2 * bounds.U * np.abs(et)), dtype), "dx")
    close(dw, ew, e_w + 1e-30, "dweight")
    # either gradient alone, and again: the same bits
    one, two, dw2 = empty((rows, cols), dtype), empty((rows, cols), dtype), empty((cols,))
    gs.gs_dropout_add_norm_backward(dz, dy, y, w, rstd, one, None, dw2, p, seed, offset, ws)
    gs.gs_dropout_add_norm_backward(dz, dy, y, w, rstd, None, two, dw2, p, seed, offset, ws)
    assert torch.equal(one, dx) and torch.equal(two, dres) and torch.equal(dw2, dw)


def test_add_norm_many_rows(gs):
    """More rows than the backward pass has CTAs, several times over."""
    rows, cols = 20_011, 96
    rng = np.random.default_rng(5)
    y, yv = put(rng.standard_normal((rows, cols)))
    dz, dzv = put(rng.standard_normal((rows, cols)))
    w, wv = put(rng.standard_normal(cols))
    rstd, rv = put(1 / np.sqrt((yv * yv).mean(axis=1)))
    dx, dres, dw = empty((rows, cols)), empty((rows, cols)), empty((cols,))
    ws = torch.empty(gs.gs_dropout_add_norm_workspace_size(rows, cols), dtype=torch.uint8, device="cuda")
    gs.gs_dropout_add_norm_backward(dz, None, y, w, rstd, dx, dres, dw, 0.0, 1, 2, ws)
    _, et, ew = layer.add_norm_backward(dzv, None, yv, wv, rv, 0.0, 1, 2)
    e_t, e_w = bounds.add_norm_backward(dzv, None, yv, wv, rv)
    close(dres, et, bounds.stored(et, e_t, "f32"), "dresidual")
    close(dw, ew, e_w, "dweight")


def test_add_norm_all_zero_row_and_no_rows(gs):
    z = torch.zeros(4, 32, device="cuda")
    w, rstd, out, y = torch.ones(32, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(z), torch.empty_like(z)
    gs.gs_dropout_add_norm(z, z, w, y, out, rstd, 0.5, 1, 2, eps=1e-6)
    assert not out.any() and not y.any()
    np.testing.assert_allclose(host(rstd), 1e3, rtol=1e-5)
    e = torch.empty(0, 32, device="cuda")
    gs.gs_dropout_add_norm(e, e, w, e, e, torch.empty(0, device="cuda"), 0.5, 1, 2)
    dw = torch.full((32,), float("nan"), device="cuda")
    ws = torch.empty(gs.gs_dropout_add_norm_workspace_size(0, 32), dtype=torch.uint8, device="cuda")
    gs.gs_dropout_add_norm_backward(e, None, e, w, torch.empty(0, device="cuda"), e, e, dw, 0.5, 1, 2, ws)
    assert not dw.any()
    gs.gs_dropout(e, e, 0.5, 1, 2)


# ---- the recurrence -----------------------------------------------------------------------------

def rec_inputs(B, T, D, dtype, seed, masks, pad=0, shift=0, spread=1.0):
    rng = np.random.default_rng(seed)
    s = {}
    s["x"], xv = put(rng.standard_normal((B, T, D)), dtype, pad, shift)
    gate, gv = put(spread * rng.standard_normal((B, T, 2 * D)), dtype, 0, shift)
    s["r"], s["i"], rv, iv = gate[..., :D], gate[..., D:], gv[..., :D], gv[..., D:]
    u = rng.uniform(0.9, 0.999, D)
    s["decay"], dv = put(np.log(np.expm1(-np.log(u) / C)))
    s["h0"], hv = put(rng.standard_normal((B, D)))
    s["dy"], yv = put(rng.standard_normal((B, T, D)), dtype, pad, shift)
    s["dh"], dhv = put(rng.standard_normal((B, D)))
    reset = lengths = None
    if "reset" in masks:
        reset = (rng.random((B, T)) < 0.05).astype(np.uint8)
        if T:
            reset[0, 0] = 1
    if "lengths" in masks:
        lengths = rng.integers(0, T + 1, B).astype(np.int32)
        lengths[0], lengths[-1] = T, 0
        for b in range(B):      # what lies past a row's end is never looked at
            for k in ("x", "r", "i", "dy"):
                s[k][b, int(lengths[b]):] = float("nan")
    s["reset"] = None if reset is None else torch.from_numpy(reset).cuda()
    s["lengths"] = None if lengths is None else torch.from_numpy(lengths).cuda()
    return s, dict(x=xv, r=rv, i=iv, decay=dv, h0=hv, dy=yv, dh=dhv, reset=reset, lengths=lengths)


def rec_run(gs, s, dtype, pad=0, shift=0, train=True, h0=True, dh=True):
    B, T, D = s["x"].shape
    out = {"y": empty((B, T, D), dtype, pad, shift), "h_last": empty((B, D))}
    states = torch.empty(gs.gs_recurrence_states_size(B, T, D), dtype=torch.uint8, device="cuda") if train else None
    gs.gs_recurrence_forward(s["x"], s["r"], s["i"], s["decay"], out["y"], h0=s["h0"] if h0 else None, reset=s["reset"],
                             lengths=s["lengths"], h_last=out["h_last"], states=states, c=C)
    if train:
        for k in ("dx", "dr", "di"):
            out[k] = empty((B, T, D), dtype, pad, shift)
        out["ddecay"], out["dh0"] = empty((D,)), empty((B, D))
        ws = torch.empty(gs.gs_recurrence_workspace_size(B, T, D), dtype=torch.uint8, device="cuda")
        gs.gs_recurrence_backward(s["dy"], s["x"], s["r"], s["i"], s["decay"], states, out["dx"], out["dr"], out["di"],
                                  out["ddecay"], ws, dh_last=s["dh"] if dh else None, reset=s["reset"],
                                  lengths=s["lengths"], dh0=out["dh0"], c=C)
    return out


def rec_check(out, v, dtype, h0=True, dh=True):
    a = (v["x"], v["r"], v["i"], v["decay"], v["h0"] if h0 else None, v["reset"], v["lengths"], C)
    y, h, _ = layer.recurrence(*a)
    exact = {"y": y, "h_last": h}
    train = "dx" in out
    if train:
        exact.update(layer.recurrence_backward(v["dy"], v["dh"] if dh else None, *a))
    tol = bounds.recurrence(*a, dy=v["dy"] if train else None, dh_last=v["dh"] if dh and train else None)
    for k, e in exact.items():
        close(out[k], e, bounds.stored(e, tol[k], dtype if k in ("y", "dx", "dr", "di") else "f32"), k)


REC_SHAPES = [(1, 1, 1, 0, 0), (2, 2, 3, 0, 0), (1, 16, 64, 0, 0), (2, 17, 66, 0, 0), (3, 127, 5, 0, 0), (1, 128, 130, 6, 0),
              (2, 129, 64, 0, 0), (1, 300, 63, 0, 1), (2, 515, 34, 2, 0), (1, 1100, 70, 0, 0), (1, 2100, 8, 0, 0),
              (1, 1024, 128, 8, 0), (2, 640, 192, 0, 0)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,T,D,pad,shift", REC_SHAPES)
def test_recurrence(gs, dtype, B, T, D, pad, shift):
    s, v = rec_inputs(B, T, D, dtype, 11 * T + D, (), pad, shift)
    rec_check(rec_run(gs, s, dtype, pad, shift), v, dtype)


@pytest.mark.parametrize("masks", [("reset",), ("lengths",), ("reset", "lengths")])
@pytest.mark.parametrize("B,T,D", [(3, 5, 4), (4, 40, 66), (5, 200, 7), (3, 700, 64), (2, 1500, 31), (3, 1290, 96)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_recurrence_masks(gs, dtype, masks, B, T, D):
    s, v = rec_inputs(B, T, D, dtype, T + D, masks)
    # the values past a row's end are NaN on the device; the oracle never reads them either
    rec_check(rec_run(gs, s, dtype), v, dtype)


@pytest.mark.parametrize("train", [False, True])
def test_recurrence_without_optional_arguments(gs, train):
    s, v = rec_inputs(2, 150, 70, "bf16", 3, ())
    rec_check(rec_run(gs, s, "bf16", train=train, h0=False, dh=False), v, "bf16", h0=False, dh=False)


def test_recurrence_many_columns(gs):
    """More (row, channel group) columns than the device holds CTAs: no cluster."""
    s, v = rec_inputs(70, 150, 321, "bf16", 4, ("reset", "lengths"))
    rec_check(rec_run(gs, s, "bf16"), v, "bf16")


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_recurrence_wide_gates(gs, dtype):
    """Gate values far out on both sides: open, shut, and in between."""
    s, v = rec_inputs(2, 260, 64, dtype, 5, (), spread=30.0)
    rec_check(rec_run(gs, s, dtype), v, dtype)


def test_recurrence_infinite_gates(gs):
    """A gate of minus infinity holds the state and has no gradient; plus infinity opens it."""
    s, v = rec_inputs(1, 40, 64, "f32", 6, ())
    s["r"][0, 10:30] = float("-inf")
    s["i"][0, 35:38] = float("-inf")
    s["r"][0, 38:] = float("inf")
    out = {k: host(t) for k, t in rec_run(gs, s, "f32").items()}
    assert all(np.isfinite(t).all() for t in out.values())
    # held: equal but for the order in which the tokens before are combined, at most one rounding
    # for each of them of partial results that the sum of all inputs' magnitudes bounds
    size = np.abs(v["h0"]) + np.abs(v["x"][:, :10]).sum(axis=1)
    assert np.all(np.abs(out["y"][0, 10:30] - out["y"][0, 9]) <= 40 * bounds.U * size)
    assert not out["dr"][0, 10:30].any() and not out["dx"][0, 10:30].any() and not out["dx"][0, 35:38].any()


@pytest.mark.parametrize("T", [50, 1400])
def test_recurrence_reset_shuts_out_infinities(gs, T):
    """Nothing before a reset is seen after it, and no gradient before it sees one past it."""
    s, v = rec_inputs(1, T, 64, "f32", 7, ())
    at = T - 20
    reset = torch.zeros(1, T, dtype=torch.uint8, device="cuda")
    reset[0, at] = 1
    s["reset"], clean = reset, {k: (t.clone() if torch.is_tensor(t) else t) for k, t in s.items()}
    clean["reset"] = reset
    want = rec_run(gs, clean, "f32")
    s["x"][0, 3, ::2] = float("inf")
    s["x"][0, 4, ::3] = float("nan")
    got = rec_run(gs, s, "f32")
    assert torch.equal(got["y"][0, at:], want["y"][0, at:]) and torch.equal(got["h_last"], want["h_last"])
    for k in ("dx", "dr", "di"):
        assert torch.equal(got[k][0, at:], want[k][0, at:])
    # a gradient that is not finite after the reset stays there
    bad = {k: (t.clone() if torch.is_tensor(t) else t) for k, t in clean.items()}
    bad["dy"][0, at + 3] = float("nan")
    back = rec_run(gs, bad, "f32")
    for k in ("dx", "dr", "di"):
        assert torch.equal(back[k][0, :at], want[k][0, :at])
    assert torch.equal(back["dh0"], want["dh0"])


@pytest.mark.parametrize("lengths", [[0, 0], [0, 1], [300, 0]])
def test_recurrence_empty_rows(gs, lengths):
    s, v = rec_inputs(2, 300, 66, "bf16", 8, ())
    v["lengths"] = np.array(lengths, dtype=np.int32)
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    rec_check(rec_run(gs, s, "bf16"), v, "bf16")


def test_recurrence_lengths_out_of_range_are_clamped(gs):
    s, v = rec_inputs(2, 150, 64, "f32", 9, ())
    v["lengths"] = np.array([-5, 1000], dtype=np.int32)
    s["lengths"] = torch.tensor([-5, 1000], dtype=torch.int32, device="cuda")
    rec_check(rec_run(gs, s, "f32"), v, "f32")


def test_recurrence_of_no_tokens(gs):
    h0, out = torch.randn(3, 70, device="cuda"), torch.empty(3, 70, device="cuda")
    e = torch.empty(3, 0, 70, device="cuda")
    decay, states = torch.zeros(70, device="cuda"), torch.empty(gs.gs_recurrence_states_size(3, 0, 70), dtype=torch.uint8, device="cuda")
    gs.gs_recurrence_forward(e, e, e, decay, e, h0=h0, h_last=out, states=states)
    assert torch.equal(out, h0)
    dd, dh0 = torch.full((70,), float("nan"), device="cuda"), torch.empty(3, 70, device="cuda")
    ws = torch.empty(gs.gs_recurrence_workspace_size(3, 0, 70), dtype=torch.uint8, device="cuda")
    gs.gs_recurrence_backward(e, e, e, e, decay, states, e, e, e, dd, ws, dh_last=h0, dh0=dh0)
    assert not dd.any() and torch.equal(dh0, h0)
    none = torch.empty(0, 4, 70, device="cuda")
    gs.gs_recurrence_forward(none, none, none, decay, none)
    gs.gs_recurrence_backward(none, none, none, none, decay, states, none, none, none, dd.fill_(1), ws)
    assert not dd.any()


def test_recurrence_orders_and_broadcasts(gs):
    """[T][B][D] memory, a gate shared by all tokens, and a state carried over in place."""
    B, T, D = 3, 290, 66
    s, v = rec_inputs(B, T, D, "bf16", 10, ())
    want = rec_run(gs, s, "bf16")
    t = dict(s)
    for k in ("x", "r", "i", "dy"):
        t[k] = s[k].transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.empty(T, B, D, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    h = s["h0"].clone()
    gs.gs_recurrence_forward(t["x"], t["r"], t["i"], t["decay"], out, h0=h, h_last=h, c=C)
    assert torch.equal(out, want["y"]) and torch.equal(h, want["h_last"])
    one = s["r"][:, :1].contiguous()
    a, b = torch.empty_like(out), torch.empty_like(out)
    gs.gs_recurrence_forward(s["x"], one.expand(B, T, D), s["i"], s["decay"], a, c=C)
    gs.gs_recurrence_forward(s["x"], one.expand(B, T, D).contiguous(), s["i"], s["decay"], b, c=C)
    assert torch.equal(a, b)


def test_recurrence_alignment_does_not_matter(gs):
    for dtype in ("f32", "bf16"):
        s, _ = rec_inputs(2, 333, 128, dtype, 12, ("reset", "lengths"))
        want = rec_run(gs, s, dtype)
        moved = dict(s)
        for k in ("x", "r", "i", "dy"):
            moved[k] = empty(s[k].shape, dtype, 3, 1)
            moved[k].copy_(s[k])
        got = rec_run(gs, moved, dtype, 3, 1)
        for k in want:
            assert torch.equal(got[k], want[k]), k


def test_recurrence_strides_past_32_bits(gs):
    """The second row of the batch lies more than 2^32 elements after the first."""
    T, D, far = 200, 66, (1 << 32) + 64
    s, v = rec_inputs(2, T, D, "bf16", 13, ())
    want = rec_run(gs, s, "bf16")
    buf = torch.empty(far + 3 * T * D, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, T, D), (far, D, 1), T * D)
    x.copy_(s["x"])
    y = buf.as_strided((2, T, D), (far, D, 1), 2 * T * D)
    h = torch.empty(2, D, device="cuda")
    gs.gs_recurrence_forward(x, s["r"], s["i"], s["decay"], y, h0=s["h0"], h_last=h, c=C)
    assert torch.equal(y, want["y"]) and torch.equal(h, want["h_last"])


def test_recurrence_pieces_are_the_whole(gs):
    """A sequence in two calls, the state handed over, agrees with one call (another order of the
    same operations, so within the bounds and not bit for bit)."""
    s, v = rec_inputs(2, 500, 64, "f32", 14, ())
    y, h = empty((2, 500, 64)), s["h0"].clone()
    for lo, hi in ((0, 201), (201, 500)):
        gs.gs_recurrence_forward(s["x"][:, lo:hi], s["r"][:, lo:hi], s["i"][:, lo:hi], s["decay"], y[:, lo:hi], h0=h,
                                 h_last=h, c=C)
    rec_check({"y": y, "h_last": h}, v, "f32")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,D,pad,shift", [(1, 1, 0, 0), (3, 64, 0, 0), (5, 1001, 0, 0), (130, 256, 8, 0), (7, 66, 3, 1), (2, 8, 0, 0)])
def test_recurrence_step(gs, dtype, B, D, pad, shift):
    rng = np.random.default_rng(B + D)
    x, xv = put(rng.standard_normal((B, D)), dtype, pad, shift)
    gate, gv = put(rng.standard_normal((B, 2 * D)), dtype, 0, shift)
    decay, dv = put(rng.standard_normal(D) - 4)
    n = B + 3
    state, sv = put(rng.standard_normal((n, D)), "f32", pad, shift)
    slots = rng.permutation(n)[:B].astype(np.int32)
    if B > 2:
        slots[1], slots[2] = -1, n
    y = empty((B, D), dtype, pad, shift)
    gs.gs_recurrence_step(x, gate[:, :D], gate[:, D:], decay, state, y, slots=torch.from_numpy(slots).cuda(), c=C)
    ey, es = layer.recurrence_step(xv, gv[:, :D], gv[:, D:], dv, sv, slots)
    idle = (slots < 0) | (slots >= n)
    at = np.where(idle, 0, slots)
    tol = bounds.recurrence(xv[:, None], gv[:, None, :D], gv[:, None, D:], dv, sv[at], None, None, C)["h_last"]
    tol[idle] = 0
    close(y, ey, np.where(idle[:, None], 0, bounds.stored(ey, tol, dtype)), "y")
    full = np.zeros((n, D))
    full[at[~idle]] = bounds.stored(es[at[~idle]], tol[~idle], "f32")
    close(state, es, full, "state")


def test_recurrence_step_continues_a_prompt(gs):
    B, T, D = 2, 65, 96
    s, v = rec_inputs(B, T, D, "bf16", 15, ())
    state, y = s["h0"].clone(), empty((B, T, D), "bf16")
    gs.gs_recurrence_forward(s["x"][:, :-3], s["r"][:, :-3], s["i"][:, :-3], s["decay"], y[:, :-3], h0=state, h_last=state, c=C)
    for t in range(T - 3, T):
        gs.gs_recurrence_step(s["x"][:, t], s["r"][:, t], s["i"][:, t], s["decay"], state, y[:, t], c=C)
    rec_check({"y": y, "h_last": state}, v, "bf16")


# ---- streams, graphs, repetition ----------------------------------------------------------------

def test_side_stream_graph_and_repeats(gs):
    s, _ = rec_inputs(2, 1300, 130, "bf16", 16, ("reset",))
    want = rec_run(gs, s, "bf16")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            got = rec_run(gs, s, "bf16")
    side.synchronize()
    for k in want:
        assert torch.equal(got[k], want[k]), k
    x = torch.randn(300, 520, device="cuda", dtype=torch.bfloat16)
    out, ref = torch.empty_like(x), torch.empty_like(x)
    gs.gs_dropout(x, ref, 0.1, 3, 4, residual=x)
    w, z, rstd = torch.ones(520, device="cuda"), torch.empty_like(x), torch.empty(300, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    y, h = torch.empty_like(s["x"]), torch.empty(2, 130, device="cuda")
    with torch.cuda.graph(graph):
        gs.gs_dropout(x, out, 0.1, 3, 4, residual=x)
        gs.gs_dropout_add_norm(x, x, w, x, z, rstd, 0.0, 3, 4)
        gs.gs_recurrence_forward(s["x"], s["r"], s["i"], s["decay"], y, h0=s["h0"], reset=s["reset"], h_last=h, c=C)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ref) and torch.equal(y, want["y"]) and torch.equal(h, want["h_last"])

"""The recurrence over the range of its parameters: decay rates from the smallest to the largest, with
gates that bring the decay into play, against the fp64 oracle within the bounds of tests/layer_bounds.py."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layer  # noqa: E402
from tests import layer_bounds as bounds  # noqa: E402
from tests.test_gpu_layer import close, empty, put  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs():
    import paper_2108_06004_gb300 as lib
    lib.load_library()
    torch.cuda.set_device(0)
    return lib


def check(gs, dtype, c, decay, x, r, i, dy, h0, dh, reset=None, lengths=None):
    """Forward, backward and step on these values (fp64 arrays, rounded to the types of the call)."""
    B, T, D = x.shape
    (x, xv), (r, rv), (i, iv), (dy, yv) = (put(a, dtype) for a in (x, r, i, dy))
    (decay, dv), (h0, hv), (dh, dhv) = (put(a) for a in (decay, h0, dh))
    masks = {"reset": None if reset is None else torch.from_numpy(reset).cuda(),
             "lengths": None if lengths is None else torch.from_numpy(lengths).cuda()}
    got = {"y": empty((B, T, D), dtype), "h_last": empty((B, D)), "ddecay": empty((D,)), "dh0": empty((B, D))}
    got.update({k: empty((B, T, D), dtype) for k in ("dx", "dr", "di")})
    states = torch.empty(gs.gs_recurrence_states_size(B, T, D), dtype=torch.uint8, device="cuda")
    ws = torch.empty(gs.gs_recurrence_workspace_size(B, T, D), dtype=torch.uint8, device="cuda")
    gs.gs_recurrence_forward(x, r, i, decay, got["y"], h0=h0, h_last=got["h_last"], states=states, c=c, **masks)
    gs.gs_recurrence_backward(dy, x, r, i, decay, states, got["dx"], got["dr"], got["di"], got["ddecay"], ws, dh_last=dh,
                              dh0=got["dh0"], c=c, **masks)
    a = (xv, rv, iv, dv, hv, reset, lengths, float(np.float32(c)))
    y, h, _ = layer.recurrence(*a)
    exact = {"y": y, "h_last": h, **layer.recurrence_backward(yv, dhv, *a)}
    tol = bounds.recurrence(*a, dy=yv, dh_last=dhv)
    for k, e in exact.items():
        close(got[k], e, bounds.stored(e, tol[k], dtype if k in ("y", "dx", "dr", "di") else "f32"), k)
    if reset is None and lengths is None:
        state, ys = h0.clone(), empty((B, D), dtype)
        gs.gs_recurrence_step(x[:, 0], r[:, 0], i[:, 0], decay, state, ys, c=c)
        t = bounds.recurrence(xv[:, :1], rv[:, :1], iv[:, :1], dv, hv, None, None, a[-1])["h_last"]
        close(state, y[:, 0], bounds.stored(y[:, 0], t, "f32"), "state")
        close(ys, y[:, 0], bounds.stored(y[:, 0], t, dtype), "step y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rate", [1e3, 1e9, 1e16, 1e22, 1e28])
@pytest.mark.parametrize("by_c", [False, True])
@pytest.mark.parametrize("B,T,D", [(2, 60, 70), (1, 700, 8)])
def test_fast_decays_behind_nearly_shut_gates(gs, dtype, rate, by_c, B, T, D):
    """Rates so large that a gate of 1/rate is what lets the state live; input gates far out too."""
    rng = np.random.default_rng(int(np.log10(rate)) + T)
    c, decay = (rate / layer.softplus(-4.0), np.full(D, -4.0)) if by_c else (8.0, np.full(D, rate / 8))
    r = -np.log(rate) + 2 * rng.standard_normal((B, T, D))
    i = 30 * rng.standard_normal((B, T, D))
    check(gs, dtype, float(c), decay, rng.standard_normal((B, T, D)), r, i, rng.standard_normal((B, T, D)),
          rng.standard_normal((B, D)), rng.standard_normal((B, D)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c,decay", [(8.0, 3e38), (3e38, -4.0), (3e38, 3e38)])
def test_rates_past_the_largest_number(gs, dtype, c, decay):
    """c softplus(decay) overflows or is close to it: with gates that are not shut the state lives for one token."""
    B, T, D = 2, 60, 66
    rng = np.random.default_rng(9)
    r, i = rng.uniform(-40, 30, (B, T, D)), 30 * rng.standard_normal((B, T, D))
    x = rng.standard_normal((B, T, D))
    (xg, xv), (rg, _), (ig, iv) = put(x, dtype), put(r, dtype), put(i, dtype)
    dy, yv = put(rng.standard_normal((B, T, D)), dtype)
    y, h = empty((B, T, D), dtype), torch.ones(B, D, device="cuda")
    dg = torch.full((D,), decay, device="cuda")
    states = torch.empty(gs.gs_recurrence_states_size(B, T, D), dtype=torch.uint8, device="cuda")
    ws = torch.empty(gs.gs_recurrence_workspace_size(B, T, D), dtype=torch.uint8, device="cuda")
    dx, dr, di, dd, dh0 = (empty(s, t) for s, t in (((B, T, D), dtype),) * 3 + (((D,), "f32"), ((B, D), "f32")))
    gs.gs_recurrence_forward(xg, rg, ig, dg, y, h0=h, h_last=h, states=states, c=c)
    gs.gs_recurrence_backward(dy, xg, rg, ig, dg, states, dx, dr, di, dd, ws, dh0=dh0, c=c)
    si = layer.sigmoid(iv)
    # the sigmoid, the root of 1 and their products: (|i| + 7) + 16 / 2 + 6 roundings, doubled
    rel = 2 * (np.abs(iv) + 21) * bounds.U
    close(y, si * xv, bounds.stored(si * xv, rel * np.abs(si * xv), dtype), "y")
    close(h, (si * xv)[:, -1], bounds.stored((si * xv)[:, -1], (rel * np.abs(si * xv))[:, -1], "f32"), "h_last")
    close(dx, si * yv, bounds.stored(si * yv, rel * np.abs(si * yv), dtype), "dx")
    for t in (dr, dd, dh0):
        assert not t.any()

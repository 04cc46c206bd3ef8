"""The gradients of gates that are far open keep their digits: 1 - sigmoid is never a difference from 1.

The bounds are those of tests/layer_bounds.py but for 1 - sigmoid(v), which may be off by its own roundings
alone: the exponent's product by |v| u, the exponential by 4u, sum, root or reciprocal and square by 9u."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layer  # noqa: E402
from tests import layer_bounds as bounds  # noqa: E402
from tests.layer_bounds import U  # noqa: E402
from tests.test_gpu_layer import close, empty, put  # noqa: E402

pytestmark = pytest.mark.gpu

C = 8.0


@pytest.fixture(scope="module")
def gs():
    import paper_2108_06004_gb300 as lib
    lib.load_library()
    torch.cuda.set_device(0)
    return lib


def tolerances(x, r, i, decay, h0, dy, dh):
    """Of di and dr, before storing; x ... are fp64 arrays without masks."""
    B, T, D = x.shape
    sr, si, la, a, gain, e = bounds.gate_errors(x, r, i, decay, C)
    off_r, off_i = 1 / (1 + np.exp(r)), 1 / (1 + np.exp(i))
    bt = gain * si * np.abs(x)
    E, M = np.zeros((B, T + 1, D)), np.zeros((B, T + 1, D))
    M[:, 0] = np.abs(h0)
    for t in range(T):
        E[:, t + 1] = a[:, t] * (E[:, t] + (e["a"][:, t] + 2 * U) * M[:, t]) + (e["b"][:, t] + U) * bt[:, t]
        M[:, t + 1] = a[:, t] * M[:, t] + bt[:, t]
    di, dr = np.zeros_like(x), np.zeros_like(x)
    ef, mf = np.zeros((B, D)), np.abs(dh)
    for t in range(T - 1, -1, -1):
        mg = mf + np.abs(dy[:, t])
        eg = ef + U * mg
        k, s, ax, ea = gain[:, t], si[:, t], np.abs(x[:, t]), e["a"][:, t]
        di[:, t] = k * ax * s * off_i[:, t] * (eg + mg * (e["gain"][:, t] + e["si"][:, t] + (np.abs(i[:, t]) + 18) * U))
        t1, t2 = a[:, t] * mg * M[:, t], a[:, t] ** 2 * mg * s * ax / k
        edla = (a[:, t] * (eg * M[:, t] + mg * E[:, t]) + t1 * (ea + 4 * U) + a[:, t] ** 2 * eg * s * ax / k
                + t2 * (2 * ea + e["gain"][:, t] + e["si"][:, t] + 6 * U))
        dr[:, t] = np.abs(la[:, t]) * off_r[:, t] * (edla + (t1 + t2) * (e["l"][:, t] + (np.abs(r[:, t]) + 17) * U))
        ef, mf = a[:, t] * (eg + (ea + 2 * U) * mg), a[:, t] * mg
    return 2 * di, 2 * dr


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,T,D", [(40, 1, 66), (2, 256, 64), (1, 1500, 24), (57, 64, 512)])
def test_open_gates_keep_their_gradients(gs, dtype, B, T, D):
    rng = np.random.default_rng(T + D)
    x, xv = put(rng.standard_normal((B, T, D)), dtype)
    r, rv = put(rng.uniform(-20, 75, (B, T, D)), dtype)
    i, iv = put(rng.uniform(-20, 75, (B, T, D)), dtype)
    dy, yv = put(rng.standard_normal((B, T, D)), dtype)
    # rates of 1e-3 to 1e-1 in half of the warps, up to 8 and more in the others
    decay, dv = put(np.where(np.arange(D) // 32 % 2 == 0, rng.uniform(-9, -4.5, D), rng.uniform(-4.5, 1, D)))
    (h0, hv), (dh, dhv) = put(rng.standard_normal((B, D))), put(rng.standard_normal((B, D)))
    y, dx, dr, di = (empty((B, T, D), dtype) for _ in range(4))
    dd, dh0 = empty((D,)), empty((B, D))
    states = torch.empty(gs.gs_recurrence_states_size(B, T, D), dtype=torch.uint8, device="cuda")
    ws = torch.empty(gs.gs_recurrence_workspace_size(B, T, D), dtype=torch.uint8, device="cuda")
    gs.gs_recurrence_forward(x, r, i, decay, y, h0=h0, states=states, c=C)
    gs.gs_recurrence_backward(dy, x, r, i, decay, states, dx, dr, di, dd, ws, dh_last=dh, dh0=dh0, c=C)
    exact = layer.recurrence_backward(yv, dhv, xv, rv, iv, dv, hv, None, None, C)
    # the oracle takes 1 - s(v) as a difference: here without
    sr, si = layer.sigmoid(rv), layer.sigmoid(iv)
    for k, v, s in (("dr", rv, sr), ("di", iv, si)):
        shut = 1 - s
        right = 1 / (1 + np.exp(v))
        exact[k] = np.where(shut > 0, exact[k] / np.where(shut > 0, shut, 1), np.nan) * right
    t_di, t_dr = tolerances(xv, rv, iv, dv, hv, yv, dhv)
    for k, got, tol in (("di", di, t_di), ("dr", dr, t_dr)):
        known = np.isfinite(exact[k])   # from about 37 on the oracle's difference is zero
        e = np.where(known, exact[k], 0)
        assert known.mean() > 0.5
        close(np.where(known, got.double().cpu().numpy(), 0), e, bounds.stored(e, tol, dtype), k)

"""The norms around a block on the GPU against the fp64 oracle."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention  # noqa: E402
from tests import attention_bounds as bounds  # noqa: E402
from tests import layer_bounds  # noqa: E402
from tests.test_gpu_attention import close, gs, host  # noqa: E402, F401
from tests.test_gpu_layer import empty, put  # noqa: E402

pytestmark = pytest.mark.gpu


def inputs(rows, cols, dtype, pad, shift, seed, names):
    rng = np.random.default_rng(seed)
    return {n: put(rng.standard_normal((rows, cols)) * (3.0 if n == "gate" else 1.0), dtype, pad, shift) for n in names}


def weights(cols, seed, shift=0):
    return put(1 + 0.2 * np.random.default_rng(seed).standard_normal(cols), "f32", 0, shift)


SHAPES = [(1, 1, 1, 0, 0), (3, 8, 1, 0, 0), (5, 64, 1, 8, 0), (17, 61, 1, 3, 0), (4, 1001, 1, 0, 0), (3, 4099, 1, 0, 1), (33, 256, 4, 0, 0),
          (9, 256, 4, 16, 0), (7, 94, 2, 0, 0), (7, 94, 2, 3, 0), (40, 60, 60, 0, 0), (2, 1024, 8, 0, 3), (300, 128, 1, 0, 0), (2, 16384, 1, 0, 0),
          (1, 12001, 1, 0, 0), (3, 32768, 4, 0, 0), (700, 48, 3, 0, 0)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,groups,pad,shift", SHAPES)
@pytest.mark.parametrize("name", ["silu", "sigmoid", "none"])
def test_forward_backward(gs, rows, cols, groups, pad, shift, name, dtype):
    follow, eps, scale = groups == 1, 1e-5, 0.7
    t = inputs(rows, cols, dtype, pad, shift, rows + cols, ("x", "gate", "residual", "dy", "dz"))
    (x, xv), (gate, gv), (res, rv), (dy, dyv), (dz, dzv) = t.values()
    if name == "none":
        gate, gv = None, None
    w, wv = weights(cols, 1)
    w2, w2v = weights(cols, 2) if follow else (None, None)
    y, rstd = empty((rows, cols), dtype, pad, shift), empty((rows, groups))
    z, r2 = (empty((rows, cols), dtype, pad, shift), empty((rows,))) if follow else (None, None)
    gs.gs_gated_norm(x, w, y, rstd, gate=gate, residual=res, next_weight=w2, z=z, next_rstd=r2, groups=groups, activation=name,
                     scale=scale, eps=eps)
    a = (xv, wv, gv, rv, w2v, groups, name, np.float32(scale), np.float32(eps))
    want, tol = attention.gated_norm(*a), bounds.gated_norm(*a)
    close(y, want[0], layer_bounds.stored(want[0], tol[0], dtype), "y")
    close(rstd, want[1], tol[1] * want[1], "rstd")
    if follow:
        close(z, want[2], layer_bounds.stored(want[2], tol[2], dtype), "z")
        close(r2, want[3], tol[3] * want[3], "next_rstd")
    for with_dy in (True, False) if follow else (True,):
        ws = torch.empty(gs.gs_gated_norm_workspace_size(rows, cols, groups), dtype=torch.uint8, device="cuda").fill_(255)
        out = {n: empty((rows, cols), dtype, pad, shift) for n in ("dx", "dgate", "dresidual")}
        out.update(dweight=empty((cols,)), dnext_weight=empty((cols,)) if follow else None)
        if name == "none":
            out["dgate"] = None
        gs.gs_gated_norm_backward(dy if with_dy else None, x, w, rstd, out["dx"], out["dweight"], ws, gate=gate, dgate=out["dgate"],
                                  dz=dz if follow else None, y=y if follow else None, next_weight=w2, next_rstd=r2,
                                  dresidual=out["dresidual"], dnext_weight=out["dnext_weight"], groups=groups, activation=name, scale=scale)
        a = (dyv if with_dy else None, xv, wv, host(rstd), gv, dzv if follow else None, host(y), w2v, host(r2) if follow else None,
             groups, name, np.float32(scale))
        want, tol = attention.gated_norm_gradients(*a), bounds.gated_norm_gradients(*a)
        for n, got in out.items():
            if got is not None:
                close(got, want[n], layer_bounds.stored(want[n], tol[n], dtype if n in ("dx", "dgate", "dresidual") else "f32"), n)


def test_weights_that_start_anywhere(gs):
    for shift in (1, 2, 3):
        x, xv = put(np.random.default_rng(1).standard_normal((6, 64)), "bf16")
        w, wv = weights(64, 4, shift)
        y, rstd = empty((6, 64), "bf16"), empty((6, 1))
        gs.gs_gated_norm(x, w, y, rstd)
        a = (xv, wv, None, None, None, 1, "none", 1.0, np.float32(1e-6))
        want, tol = attention.gated_norm(*a)[0], bounds.gated_norm(*a)[0]
        close(y, want, layer_bounds.stored(want, tol, "bf16"), "y")


@pytest.mark.parametrize("cols,groups", [(64, 1), (61, 1), (128, 4), (94, 2)])
@pytest.mark.parametrize("over", ["x", "gate", "residual"])
def test_in_place(gs, over, cols, groups):
    t = inputs(50, cols, "bf16", 0, 0, 3, ("x", "gate", "residual"))
    t = {n: v[0] for n, v in t.items()}
    w, _ = weights(cols, 1)
    want, rstd = torch.empty_like(t["x"]), empty((50, groups))
    gs.gs_gated_norm(t["x"], w, want, rstd, gate=t["gate"], residual=t["residual"], groups=groups)
    gs.gs_gated_norm(t["x"], w, t[over], rstd, gate=t["gate"], residual=t["residual"], groups=groups)
    assert torch.equal(t[over], want)


def test_gates_far_open_and_shut(gs):
    u = np.array([0.0, 1e-4, -1e-4, 5, -5, 20, -20, 60, -60, 100, -100, 3e4, -3e4, 1, -1, 2.0])
    x, xv = put(np.ones((1, 16)), "f32")
    gate, gv = put(u[None], "f32")
    w, wv = put(np.ones(16), "f32")
    for name in ("silu", "sigmoid"):
        y, rstd = empty((1, 16)), empty((1, 1))
        gs.gs_gated_norm(x, w, y, rstd, gate=gate, activation=name)
        want, slope = attention.act(name, gv)
        tiny = 2.0 ** -126 * np.maximum(1, np.abs(gv))   # what is below the smallest normal number may be zero
        close(y, want * host(rstd), np.abs(want) * (2 * np.abs(gv) + 60) * layer_bounds.U + tiny, name)
        dx, dg, dw = empty((1, 16)), empty((1, 16)), empty((16,))
        ws = torch.empty(gs.gs_gated_norm_workspace_size(1, 16), dtype=torch.uint8, device="cuda")
        gs.gs_gated_norm_backward(torch.ones_like(x), x, w, rstd, dx, dw, ws, gate=gate, dgate=dg, activation=name)
        s = attention.act("sigmoid", gv)[0]
        size = s * (1 + np.abs(gv) * (1 - s)) if name == "silu" else slope
        close(dg, slope * host(rstd), np.abs(size) * (6 * np.abs(gv) + 120) * layer_bounds.U + tiny, "slope of " + name)


def test_no_rows(gs):
    x, w = torch.empty(0, 64, device="cuda"), torch.ones(64, device="cuda")
    gs.gs_gated_norm(x, w, torch.empty_like(x), torch.empty(0, 1, device="cuda"))
    dw, dn = torch.full((64,), 5.0, device="cuda"), torch.full((64,), 5.0, device="cuda")
    ws = torch.empty(gs.gs_gated_norm_workspace_size(0, 64), dtype=torch.uint8, device="cuda")
    gs.gs_gated_norm_backward(None, x, w, torch.empty(0, 1, device="cuda"), None, dw, ws, dz=x, y=x, next_weight=w,
                              next_rstd=torch.empty(0, device="cuda"), dnext_weight=dn)
    assert not dw.any() and not dn.any()

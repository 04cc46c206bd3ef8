"""fp32 gates of the norms around a block are as exact far from zero as near it."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention  # noqa: E402
from tests.layer_bounds import U  # noqa: E402
from tests.test_gpu_attention import close, gs, host  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["silu", "sigmoid"])
def test_gates(gs, name):
    """In units of 2^-24, relative: e^-u 2 (a unit in the last place), 1 + e^-u and its reciprocal 1 each: s is off by 4, the gate by 5
    with its product; y by 7 with those of rstd and x. 1 - s = e^-u s is off by 2 + 4 + 1, the slope a (1 - s) + s by 5 + 7 + 1
    of its larger terms, s (1 - s) by 12, and dgate by 4 more for rstd, x, weight and dy. Doubled for nothing: second order is far below,
    and is given a hundredth."""
    rows, cols = 64, 256
    u = np.concatenate((np.linspace(-86, 86, rows * cols // 2), np.random.default_rng(0).standard_normal(rows * cols // 2) * 6))
    u = u.reshape(rows, cols).astype(np.float32)
    x, gate, w = torch.ones(rows, cols, device="cuda"), torch.from_numpy(u).cuda(), torch.ones(cols, device="cuda")
    y, rstd = torch.empty_like(x), torch.empty(rows, 1, device="cuda")
    gs.gs_gated_norm(x, w, y, rstd, gate=gate, activation=name)
    a, slope = attention.act(name, u.astype(np.float64))
    tiny = 2.0 ** -126   # a stored value below the smallest normal number has fewer digits
    close(y, a * host(rstd), 1.01 * 7 * U * np.abs(a) + tiny, name)
    dx, dgate, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(gs.gs_gated_norm_workspace_size(rows, cols), dtype=torch.uint8, device="cuda")
    gs.gs_gated_norm_backward(torch.ones_like(x), x, w, rstd, dx, dw, ws, gate=gate, dgate=dgate, activation=name)
    s, rest = attention.act("sigmoid", u.astype(np.float64))[0], attention.act("sigmoid", -u.astype(np.float64))[0]
    size = np.abs(a) * rest + s if name == "silu" else slope
    close(dgate, slope * host(rstd), 1.01 * 17 * U * size + tiny * np.maximum(1, np.abs(u)), "slope of " + name)


def test_beyond_all_digits(gs):
    u = torch.tensor([[-3e38, -1e4, -104.0, -89.0, 89.0, 104.0, 1e4, 3e38]], device="cuda")
    x, w = torch.ones_like(u), torch.ones(8, device="cuda")
    for name, low, high in (("silu", torch.zeros(4), u[0, 4:].cpu()), ("sigmoid", torch.zeros(4), torch.ones(4))):
        y, rstd, dx, dgate, dw = torch.empty_like(x), torch.empty(1, 1, device="cuda"), torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
        ws = torch.empty(gs.gs_gated_norm_workspace_size(1, 8), dtype=torch.uint8, device="cuda")
        gs.gs_gated_norm(x, w, y, rstd, gate=u, activation=name, eps=0.0)
        gs.gs_gated_norm_backward(x, x, w, rstd, dx, dw, ws, gate=u, dgate=dgate, activation=name)
        y, dgate = y[0].cpu(), dgate[0].cpu()
        assert (y[:4] - low).abs().max() < 1e-36 and torch.equal(y[4:], high), (name, y)
        assert (dgate[:4]).abs().max() < 1e-36 and (dgate[4:] - (1.0 if name == "silu" else 0.0)).abs().max() < 1e-36, (name, dgate)

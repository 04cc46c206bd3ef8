"""A decay that is not a number shows in its head's results, and in no other's."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_attention import DT, gs, place  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,D", [(1, 64), (300, 64), (300, 128), (2600, 64), (90, 47)])
def test_nan(gs, T, D, dtype):
    rng = np.random.default_rng(0)
    q, k, v, do = (place((1, T, 3, D), dtype, "dense", rng=rng) for _ in range(4))
    s0 = torch.from_numpy(rng.standard_normal((1, 3, D, D))).to("cuda", torch.float32)
    seen = []
    for g in ([-0.1, float("nan"), -0.01], [-0.1, -0.05, -0.01]):
        g = torch.tensor(g, device="cuda")
        o, dq, dk, dv = (torch.empty_like(t) for t in (v, q, k, v))
        last, ds0 = torch.empty_like(s0), torch.empty_like(s0)
        ws = torch.empty(gs.gs_linear_attention_workspace_size(1, T, 3, 3, D, D, DT[dtype], backward=True), dtype=torch.uint8, device="cuda")
        gs.gs_linear_attention_forward(q, k, v, g, o, ws, s0=s0, s_last=last)
        gs.gs_linear_attention_backward(do, q, k, v, g, dq, dk, dv, ws, s0=s0, ds_last=s0, ds0=ds0)
        state, step = s0.clone(), torch.empty_like(v[:, 0])
        gs.gs_linear_attention_step(q[:, 0], k[:, 0], v[:, 0], g, state, step)
        seen.append([o, dq, dk, dv, step[:, None], last[:, None], ds0[:, None], state[:, None]])
    for n, (a, b) in enumerate(zip(*seen)):
        assert torch.equal(a[:, :, 0::2], b[:, :, 0::2]) and torch.isfinite(b).all()
        # a token's decay comes after it for dk and dv: their last token has none
        assert a[:, :(-1 if n in (2, 3) else None), 1].isnan().all()

"""The factors between two products are sums of two parts of the type, each rounded to nearest: a value just above the middle of
two stored ones is stored as the upper one, wherever it comes from."""

import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_attention import DT, gs  # noqa: E402, F401

pytestmark = pytest.mark.gpu

# just above the middle of 1 and the next value of the type, by less than a first part that is cut off leaves room for
# (bf16: 2^-8 has steps of 2^-15 there, and the distance is three quarters of 2^-16)
ABOVE = {"bf16": 1 + 2.0 ** -8 + 1.5 * 2.0 ** -17, "f16": 1 + 2.0 ** -11 + 2.0 ** -20}
UPPER = {"bf16": 1 + 2.0 ** -7, "f16": 1 + 2.0 ** -10}
T, H, C = 300, 2, 3


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 128), (64, 128), (128, 64)])
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("size", [1.0, -4.0])
def test_nearest(gs, size, state, Dk, Dv, dtype):
    x, up = ABOVE[dtype], size * UPPER[dtype]
    g = torch.zeros(H, device="cuda")
    zeros = lambda d: torch.zeros(1, T, H, d, dtype=DT[dtype], device="cuda")   # noqa: E731
    last = torch.empty(1, H, Dk, Dv, device="cuda") if state else None
    ws = torch.empty(gs.gs_linear_attention_workspace_size(1, T, H, H, Dk, Dv, DT[dtype], backward=True), dtype=torch.uint8, device="cuda")

    # from the state that a call starts with
    q, k, v, o = zeros(Dk), zeros(Dk), zeros(Dv), zeros(Dv)
    q[..., C] = 1
    s0 = torch.full((1, H, Dk, Dv), size * x, device="cuda")
    gs.gs_linear_attention_forward(q, k, v, g, o, ws, s0=s0, s_last=last)
    assert (o == up).all()

    # from scores, and from the state that a block leaves
    q[..., C + 1], q[..., C + 2] = x - 1 - 2.0 ** -9, 2.0 ** -9
    rest = x - 1 - (q[0, 0, 0, C + 1].double() + q[0, 0, 0, C + 2].double()).item()
    q[..., C + 3] = rest
    assert q[0, 0, 0].double().sum().item() == x
    k[:, 0, :, C:C + 4] = 1
    v[:, 0] = size
    gs.gs_linear_attention_forward(q, k, v, g, o, ws, s_last=last)
    assert (o == up).all()

    # from weighted keys: the gradients' scale
    q, do, k, v = zeros(Dk), zeros(Dv), zeros(Dk), zeros(Dv)
    q[:, -1, :, C] = 1
    do[:, -1] = size
    k[..., C] = 1
    v[..., C] = 1
    dq, dk, dv = zeros(Dk), zeros(Dk), zeros(Dv)
    gs.gs_linear_attention_backward(do, q, k, v, g, dq, dk, dv, ws, ds0=last, scale=x)
    assert (dv == up).all() and (dk[..., C] == up).all()
    if state:
        assert (last[:, :, C] == torch.tensor(size * x, device="cuda")).all()

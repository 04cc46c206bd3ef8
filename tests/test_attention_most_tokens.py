"""Linear attention of as many tokens as a call takes."""

import ctypes

import pytest

torch = pytest.importorskip("torch")

MOST = (1 << 31) - (1 << 10)


@pytest.fixture(scope="module")
def gs():
    import os

    import paper_2108_06004_gb300 as lib
    if not os.path.exists(lib.LIB_PATH):
        from paper_2108_06004_gb300 import _build
        _build.build()
    lib.load_library()
    return lib


def test_refusals(gs):
    lib, size = gs.load_library(), ctypes.c_size_t()
    A = 1 << 12
    t = ctypes.byref(gs.GsHeads(A, 1 << 32, 1, 1))
    u = ctypes.byref(gs.GsHeads(A + (1 << 40), 1 << 32, 1, 1))
    for T in (MOST + 1, (1 << 31) - 1):
        for packed in (0, 1):
            assert lib.gs_linear_attention_workspace_size(1, T, 1, 1, 1, 1, gs.GS_F32, 0, packed, ctypes.byref(size)) == gs.GS_ERR_INVALID_ARG
            assert b"T must be at most" in lib.gs_last_error()
        assert lib.gs_linear_attention_forward(t, t, t, A, None, None, None, u, None, 1, T, 1, 1, 1, 1, gs.GS_F32, 1.0, A, 1 << 40,
                                               None) == gs.GS_ERR_INVALID_ARG
        assert b"T must be at most" in lib.gs_last_error()
    for dtype in (gs.GS_F32, gs.GS_BF16):
        assert lib.gs_linear_attention_workspace_size(1, MOST, 1, 1, 1, 1, dtype, 1, 0, ctypes.byref(size)) == gs.GS_OK


@pytest.mark.gpu
def test_most_tokens(gs):
    """With a decay of one a token, what is more than sixty tokens away is below an fp32 rounding: both ends are known."""
    n, gen = 96, torch.Generator(device="cuda").manual_seed(1)
    q, k, v, do = (torch.randn(1, MOST, 1, 1, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    g = torch.tensor([-1.0], device="cuda")
    one = torch.ones(1, 1, 1, 1, device="cuda")
    o, dq, dk, dv = (torch.full_like(t, float("nan")) for t in (v, q, k, v))
    last, ds0 = torch.full_like(one, float("nan")), torch.full_like(one, float("nan"))
    for back in (False, True):
        ws = torch.empty(gs.gs_linear_attention_workspace_size(1, MOST, 1, 1, 1, 1, torch.bfloat16, backward=back), dtype=torch.uint8,
                         device="cuda").fill_(255)
        if back:
            gs.gs_linear_attention_backward(do, q, k, v, g, dq, dk, dv, ws, s0=one, ds_last=one, ds0=ds0, scale=0.5)
        else:
            gs.gs_linear_attention_forward(q, k, v, g, o, ws, s0=one, s_last=last, scale=0.5)
    i = torch.arange(n, device="cuda", dtype=torch.float64)
    w = torch.exp(-(i[:, None] - i[None]).clamp(min=0)).tril()
    for at in (slice(0, n), slice(MOST - n, MOST)):
        Q, K, V, DO = (t[0, at, 0, 0].double() for t in (q, k, v, do))
        first = torch.exp(-(i + 1)) if at.start == 0 else 0 * i          # of the state before
        after = torch.exp(-(n - 1 - i)) if at.start != 0 else 0 * i      # of the gradient behind
        S, R = w @ (K * V) + first, 0.5 * (w.t() @ (Q * DO)) + after
        inner = slice(None) if at.start == 0 else slice(60, None)
        outer = slice(None) if at.start != 0 else slice(0, n - 60)
        # a stored bf16 is off by 2^-8 of its value, of a sum by 2^-20 of its terms'
        for got, want, where in ((o, 0.5 * Q * S, inner), (dq, 0.5 * DO * S, inner), (dk, R * V, outer), (dv, R * K, outer)):
            x, y = got[0, at, 0, 0].double()[where], want[where]
            assert ((x - y).abs() <= 2.0 ** -8 * y.abs() + 2.0 ** -14).all()
        if at.start == 0:
            assert abs(float(ds0) - float(R[0] * torch.exp(-i[1]))) < 1e-5
        else:
            assert abs(float(last) - float(S[-1])) < 1e-5
    # nothing in between was left out
    assert all(torch.isfinite(t).all() for t in (o, dq, dk, dv))

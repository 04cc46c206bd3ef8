"""The linear attention layer's entry points refuse bad arguments on the host, before any device work, and their
fp64 oracle holds against definitions worked out in other ways."""

import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention  # noqa: E402


@pytest.fixture(scope="module")
def gs():
    import os

    import paper_2108_06004_gb300 as lib
    if not os.path.exists(lib.LIB_PATH):
        from paper_2108_06004_gb300 import _build
        _build.build()
    lib.load_library()
    return lib


A = 1 << 12   # an aligned address that is never touched


def heads(gs, data=A, b=4 * 2 * 8, t=2 * 8, h=8):
    return ctypes.byref(gs.GsHeads(data, b, t, h))


def test_rotary_refusals(gs):
    lib, bad, ok = gs.load_library(), gs.GS_ERR_INVALID_ARG, heads(gs)

    def call(x=ok, out=ok, f=A, pos=None, B=2, T=4, H=2, D=8, R=8, dtype=0, m=1.0):
        return lib.gs_rotary(x, out, f, pos, 0, B, T, H, D, R, dtype, 0, 0, m, None)

    for kw in ({"x": None}, {"out": None}, {"x": heads(gs, None)}, {"out": heads(gs, A + 2)}, {"f": None}, {"f": A + 4}, {"pos": A + 2},
               {"B": -1}, {"T": -1}, {"H": -1}, {"D": 0}, {"D": 513}, {"R": 7}, {"R": 10}, {"R": -2}, {"dtype": 3}, {"m": float("nan")},
               {"m": float("inf")}, {"out": heads(gs, h=7)}, {"out": heads(gs, t=8)}, {"out": heads(gs, b=48)}, {"x": heads(gs, h=-1)},
               {"out": heads(gs, b=200)}, {"B": 1 << 20, "T": 1 << 12}, {"H": 1 << 25}):
        assert call(**kw) == bad, kw
    assert call(B=0) == call(T=0, x=heads(gs, None)) == call(H=0) == call(R=0, f=None) == gs.GS_OK
    call(R=7)
    assert b"R must be even" in lib.gs_last_error()


def test_frequencies(gs):
    for kw in ({"R": -2}, {"R": 3}, {"R": 514}, {"base": 0.0}, {"base": float("inf")}, {"factor": 0.5}, {"factor": float("nan")}, {"original": -1.0},
               {"low": -1.0}, {"low": 32.0}, {"high": float("inf")}):
        with pytest.raises(gs.GsError):
            gs.gs_rotary_frequencies(**{"R": 8, **kw})
    assert gs.gs_rotary_frequencies(0).numel() == 0
    for kw in ({}, {"base": 5e5}, {"factor": 4.0}, {"factor": 16.0, "original": 8192.0}, {"factor": 2.0, "original": 100.0, "low": 0.5, "high": 4.0}):
        for R in (2, 20, 128):
            assert np.allclose(gs.gs_rotary_frequencies(R, **kw).numpy(), attention.frequencies(R, **kw), rtol=1e-14, atol=0)


def test_attention_refusals(gs):
    lib, bad, ok = gs.load_library(), gs.GS_ERR_INVALID_ARG, heads(gs)

    def call(q=ok, k=ok, v=ok, g=A, s0=None, lengths=None, offsets=None, o=ok, last=None, B=2, T=4, H=2, K=2, Dk=8, Dv=8, dtype=0, scale=1.0,
             ws=A, n=1 << 30):
        return lib.gs_linear_attention_forward(q, k, v, g, s0, lengths, offsets, o, last, B, T, H, K, Dk, Dv, dtype, scale, ws, n, None)

    wrong = ({"q": None}, {"k": None}, {"v": None}, {"q": heads(gs, None)}, {"k": heads(gs, None)}, {"v": heads(gs, None)}, {"g": None},
             {"g": A + 2}, {"s0": A + 2}, {"lengths": A + 2}, {"offsets": A + 2}, {"lengths": A, "offsets": A}, {"q": heads(gs, A + 1)},
             {"B": -1}, {"T": -1}, {"H": -2}, {"K": 0}, {"H": 3, "K": 2}, {"H": 2, "K": 4}, {"Dk": 0}, {"Dv": 0}, {"Dk": 257}, {"Dv": 257},
             {"dtype": 3}, {"scale": float("nan")}, {"scale": float("inf")}, {"ws": None}, {"ws": A + 16}, {"n": 16}, {"T": 1 << 31},
             {"B": 1 << 20, "T": 1 << 20}, {"B": 1 << 24, "T": 1, "H": 1 << 10, "K": 1})
    for kw in wrong + ({"o": None}, {"o": heads(gs, None)}, {"o": heads(gs, h=4)}, {"o": heads(gs, t=8)}, {"last": A + 2}):
        assert call(**kw) == bad, kw
    assert call(B=0) == call(H=0) == gs.GS_OK
    size = ctypes.c_size_t()
    f = lib.gs_linear_attention_workspace_size
    assert f(1, 1, 1, 1, 8, 8, 0, 0, 0, None) == bad and f(1, -1, 1, 1, 8, 8, 0, 0, 0, ctypes.byref(size)) == bad
    assert f(1, 1, 1, 1, 8, 8, 5, 0, 0, ctypes.byref(size)) == bad
    assert f(1, 100000, 2, 1, 64, 64, 2, 1, 0, ctypes.byref(size)) == gs.GS_OK and size.value >= 100000 * 2 * 64 * 4

    def back(do=ok, q=ok, dq=ok, dk=ok, dv=ok, s0=None, ds=None, ds0=None, **kw):
        a = {"k": ok, "v": ok, "g": A, "lengths": None, "offsets": None, "B": 2, "T": 4, "H": 2, "K": 2, "Dk": 8, "Dv": 8, "dtype": 0, "scale": 1.0,
             "ws": A, "n": 1 << 30, **kw}
        return lib.gs_linear_attention_backward(do, q, a["k"], a["v"], a["g"], s0, ds, a["lengths"], a["offsets"], dq, dk, dv, ds0, a["B"],
                                                a["T"], a["H"], a["K"], a["Dk"], a["Dv"], a["dtype"], a["scale"], a["ws"], a["n"], None)

    for kw in wrong + ({"do": None}, {"do": heads(gs, None)}, {"dq": None}, {"dk": heads(gs, None)}, {"dv": heads(gs, t=8)}, {"ds": A + 1},
                       {"ds0": A + 2}, {"ds0": A, "s0": A}, {"ds0": A, "ds": A}):
        assert back(**kw) == bad, kw

    def step(q=ok, k=ok, v=ok, o=ok, g=A, state=A, stride=2 * 64, n=2, slots=None, B=2, H=2, K=2, Dk=8, Dv=8, scale=1.0):
        return lib.gs_linear_attention_step(q, k, v, g, state, stride, n, slots, o, B, H, K, Dk, Dv, 0, scale, None)

    for kw in ({"q": None}, {"k": heads(gs, None)}, {"v": None}, {"o": None}, {"o": heads(gs, h=4)}, {"g": None}, {"state": None}, {"state": A + 2},
               {"stride": 127}, {"n": 1}, {"n": -1}, {"slots": A + 2}, {"K": 0}, {"Dk": 300}, {"scale": float("nan")}, {"B": 1 << 28, "H": 64, "n": 1, "slots": A}):
        assert step(**kw) == bad, kw
    assert step(B=0) == gs.GS_OK


def test_gated_norm_refusals(gs):
    lib, bad = gs.load_library(), gs.GS_ERR_INVALID_ARG

    def call(x=A, gate=A, res=None, w=A, w2=A, y=A, ys=8, z=A, zs=8, r=A, r2=A, rows=4, cols=8, groups=1, dtype=0, act=2, scale=1.0, eps=1e-6):
        return lib.gs_gated_norm(x, 8, gate, 8, res, 8, w, w2, y, ys, z, zs, r, r2, rows, cols, groups, dtype, act, scale, eps, None)

    for kw in ({"x": None}, {"gate": None}, {"act": 0}, {"act": 3}, {"act": -1}, {"w": None}, {"w": A + 2}, {"y": None}, {"z": None}, {"r": None},
               {"r2": None}, {"w2": None}, {"groups": 0}, {"groups": 3}, {"groups": 2}, {"cols": 0}, {"cols": 16385}, {"rows": -1}, {"dtype": 9},
               {"scale": float("inf")}, {"eps": -1.0}, {"eps": float("nan")}, {"ys": 7}, {"zs": 7}, {"res": A + 2},
               {"cols": 1 << 21, "groups": 1 << 21, "w2": None, "z": None, "r2": None}, {"rows": 1 << 30, "groups": 4, "w2": None, "z": None, "r2": None}):
        assert call(**kw) == bad, kw
    assert call(rows=0, x=None, gate=None, y=None, z=None, r=None, r2=None) == gs.GS_OK
    size = ctypes.c_size_t()
    assert lib.gs_gated_norm_workspace_size(4, 8, 3, ctypes.byref(size)) == bad and lib.gs_gated_norm_workspace_size(4, 8, 1, None) == bad

    def back(dy=A, dz=2 * A, x=3 * A, gate=4 * A, y=5 * A, w=A, w2=A, r=A, r2=A, dx=6 * A, dxs=8, dgate=7 * A, dres=8 * A, dw=A, dw2=A, groups=1, act=2, ws=A, n=1 << 30):
        return lib.gs_gated_norm_backward(dy, 8, dz, 8, x, 8, gate, 8, y, 8, w, w2, r, r2, dx, dxs, dgate, 8, dres, 8, dw, dw2, 4, 8, groups, 0, act, 1.0,
                                          ws, n, None)

    for kw in ({"dz": None}, {"x": None}, {"gate": None}, {"y": None}, {"w": None}, {"w2": None}, {"r": None}, {"r2": None}, {"dw": None}, {"dw2": None},
               {"dxs": 7}, {"groups": 2}, {"act": 0}, {"ws": None}, {"ws": A + 8}, {"n": 8}, {"dx": A}, {"dgate": 4 * A}, {"dres": 2 * A},
               {"w2": None, "dz": None, "y": None, "r2": None, "dw2": None, "dy": None}):
        assert back(**kw) == bad, kw


def test_binding_refusals(gs):
    x, g, w = torch.zeros(2, 4, 2, 8), torch.zeros(2), torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(gs.GsError, match="CUDA device"):
        gs.gs_linear_attention_forward(x, x, x, g, x, w)
    with pytest.raises(gs.GsError, match="CUDA device"):
        gs.gs_rotary(x, x, torch.zeros(4, dtype=torch.float64))
    with pytest.raises(gs.GsError, match="none of float32"):
        gs.gs_linear_attention_step(x[:, 0].double(), x, x, g, x, x)
    with pytest.raises(gs.GsError, match="dimensions"):
        gs.gs_linear_attention_forward(x, x[0], x, g, x, w)
    with pytest.raises(gs.GsError, match="one row"):
        gs.gs_linear_attention_forward(x, x, x, g, x, w, offsets=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(gs.GsError, match="is missing"):
        gs.gs_linear_attention_backward(x, x, None, x, g, x, x, x, w)
    with pytest.raises(gs.GsError, match="is none of"):
        gs.gs_gated_norm(x, g, x, g, gate=x, activation="tanh")
    with pytest.raises(gs.GsError, match="none of float32"):
        gs.gs_linear_attention_workspace_size(1, 1, 1, 1, 8, 8, torch.int32)
    m = torch.empty(2, 4, 2, 8, device="meta")
    for bad in (m.transpose(2, 3), m[:1], m.half()):
        with pytest.raises(gs.GsError):
            gs._heads("f", "t", bad, m.shape, m.dtype, m.device)


def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(0)
    n, H, K, Dk, Dv = 9, 4, 2, 5, 3
    args = [rng.standard_normal(s) for s in ((n, H, Dk), (n, K, Dk), (n, K, Dv), (H, Dk, Dv))]
    g, do, ds = -np.exp(rng.uniform(-3, 0, H)), rng.standard_normal((n, H, Dv)), rng.standard_normal((H, Dk, Dv))

    def value(q, k, v, s0):
        o, last = attention.sequence(q, k, v, g, 0.3, s0)
        return (o * do).sum() + (last * ds).sum()

    for i, grad in enumerate(attention.sequence_gradients(do, *args[:3], g, 0.3, args[3], ds)):
        d = rng.standard_normal(args[i].shape)
        ends = [value(*[a + (h * d if m == i else 0) for m, a in enumerate(args)]) for h in (1e-6, -1e-6)]
        assert abs((ends[0] - ends[1]) / 2e-6 - (grad * d).sum()) < 1e-7


def test_oracle_attention_is_masked_attention():
    """The recurrence equals the sum over earlier tokens with their weights."""
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal((12, 1, 4)) for _ in range(3))
    o, last = attention.sequence(q, k, v, np.array([-0.2]), 0.5, np.zeros((1, 4, 4)))
    i = np.arange(12)
    w = np.tril(np.exp(-0.2 * (i[:, None] - i[None])))
    assert np.allclose(o[:, 0], 0.5 * (q[:, 0] @ k[:, 0].T * w) @ v[:, 0])
    assert np.allclose(last[0], (k[:, 0] * w[-1][:, None]).T @ v[:, 0])


def test_oracle_norm_gradients_against_differences():
    rng = np.random.default_rng(2)
    x, gate, res = (rng.standard_normal((4, 6)) for _ in range(3))
    w, w2, dy, dz = rng.standard_normal(6), rng.standard_normal(6), rng.standard_normal((4, 6)), rng.standard_normal((4, 6))
    for name in ("silu", "sigmoid"):
        def value(x, gate, res, w, w2):
            y, _, z, _ = attention.gated_norm(x, w, gate, res, w2, 1, name, 0.7, 1e-3)
            return (y * dy).sum() + (z * dz).sum()

        y, r, _, r2 = attention.gated_norm(x, w, gate, res, w2, 1, name, 0.7, 1e-3)
        got = attention.gated_norm_gradients(dy, x, w, r, gate, dz, y, w2, r2, 1, name, 0.7)
        args = [x, gate, res, w, w2]
        for i, n in enumerate(("dx", "dgate", "dresidual", "dweight", "dnext_weight")):
            d = rng.standard_normal(args[i].shape)
            ends = [value(*[a + (h * d if m == i else 0) for m, a in enumerate(args)]) for h in (1e-6, -1e-6)]
            assert abs((ends[0] - ends[1]) / 2e-6 - (got[n] * d).sum()) < 1e-6


def test_oracle_rotary_keeps_products():
    """Turning queries and keys leaves products that depend on the distance alone."""
    rng = np.random.default_rng(3)
    q, k, f = rng.standard_normal((1, 1, 1, 8)), rng.standard_normal((1, 1, 1, 8)), attention.frequencies(8)
    at = lambda x, p, inter: attention.rotary(x, f, np.array([[p]]), inter, False, 1.0)   # noqa: E731
    for inter in (False, True):
        assert np.isclose((at(q, 17, inter) * at(k, 5, inter)).sum(), (at(q, 1012, inter) * at(k, 1000, inter)).sum())
    one = attention.rotary(np.array([1.0, 0.0]).reshape(1, 1, 1, 2), np.array([np.pi / 2]), np.array([[1]]), True, False, 2.0)
    assert np.allclose(one.ravel(), [0, 2])


def test_outputs_over_inputs(gs):
    """Attention's outputs, a second norm's and the gradients are no input and not one another: other CTAs read those meanwhile."""
    lib, n = gs.load_library(), 1 << 16
    at = [heads(gs, A + i * n) for i in range(8)]
    sizes = (2, 4, 2, 2, 8, 8, gs.GS_F32, 1.0)
    for o in range(3):
        assert lib.gs_linear_attention_forward(*at[:3], A, None, None, None, at[o], None, *sizes, A, n, None) == gs.GS_ERR_INVALID_ARG
        assert b"o may not be an input" in lib.gs_last_error()
        assert lib.gs_linear_attention_step(*at[:3], A, A, 128, 2, None, at[o], 2, 2, 2, 8, 8, gs.GS_F32, 1.0, None) == gs.GS_ERR_INVALID_ARG
        assert b"o may not be an input" in lib.gs_last_error()
    for place in range(3):
        for other in range(4 + place):   # the inputs, and the gradients ahead of this one
            to = at[4:7]
            to[place] = at[other]
            assert lib.gs_linear_attention_backward(*at[:4], A, None, None, None, None, *to, None, *sizes, A, n, None) == gs.GS_ERR_INVALID_ARG
            assert b"dq, dk and dv may not be" in lib.gs_last_error()
    x, g, r, y = (A + i * n for i in range(4))
    for z in (x, g, r, y):
        assert lib.gs_gated_norm(x, 8, g, 8, r, 8, A, A, y, 8, z, 8, A, A, 4, 8, 1, gs.GS_F32, gs.GS_GATE_SILU, 1.0, 1e-6, None) == gs.GS_ERR_INVALID_ARG
        assert b"z may not be an input" in lib.gs_last_error()
    for y in (x, g, r):
        assert lib.gs_gated_norm(x, 8, g, 8, r, 8, A, None, y, 16, None, 0, A, None, 4, 8, 1, gs.GS_F32, gs.GS_GATE_SILU, 1.0, 1e-6,
                                 None) == gs.GS_ERR_INVALID_ARG
        assert b"same stride" in lib.gs_last_error()
    for dx, dgate in ((g, None), (r, r)):   # dy is x here
        assert lib.gs_gated_norm_backward(x, 8, None, 0, x, 8, g, 8, None, 0, A, None, A, None, dx, 8, dgate, 8, None, 0, A, None, 4, 8, 1, gs.GS_F32,
                                          gs.GS_GATE_SILU, 1.0, A, n, None) == gs.GS_ERR_INVALID_ARG
        assert b"dx, dgate and dresidual may not be" in lib.gs_last_error()

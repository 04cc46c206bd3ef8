"""The recurrent layer's entry points refuse bad arguments on the host, before any device work."""

import ctypes

import pytest

torch = pytest.importorskip("torch")


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


def test_dropout_refusals(gs):
    lib, bad = gs.load_library(), gs.GS_ERR_INVALID_ARG

    def call(x=A, xs=8, res=None, rs=0, out=2 * A, os_=8, rows=4, cols=8, dtype=gs.GS_BF16, p=0.1):
        return lib.gs_dropout(x, xs, res, rs, out, os_, rows, cols, dtype, p, 1, 2, None)

    for kw in ({"x": None}, {"out": None}, {"x": A + 1}, {"out": A + 1}, {"res": A + 1, "rs": 8}, {"dtype": 3}, {"dtype": -1},
               {"p": -0.1}, {"p": 1.1}, {"p": float("nan")}, {"rows": -1}, {"cols": -1}, {"os_": 7}, {"xs": -1},
               {"rows": 1 << 31}, {"rows": 1 << 30, "cols": 1 << 11}):
        assert call(**kw) == bad, kw
    assert call(rows=0, x=None, out=None) == gs.GS_OK and call(cols=0, x=None, out=None) == gs.GS_OK
    assert lib.gs_dropout_backward(None, 8, A, 8, 4, 8, 0, 0.1, 1, 2, None) == bad
    call(p=2.0)
    assert b"p must lie" in lib.gs_last_error()


def test_add_norm_refusals(gs):
    lib, bad = gs.load_library(), gs.GS_ERR_INVALID_ARG

    def call(x=A, res=A, w=A, y=A, ys=8, z=A, zs=8, rstd=A, rows=4, cols=8, dtype=0, p=0.1, eps=1e-6):
        return lib.gs_dropout_add_norm(x, 8, res, 8, w, y, ys, z, zs, rstd, rows, cols, dtype, p, 1, 2, eps, None)

    for kw in ({"x": None}, {"res": None}, {"w": None}, {"y": None}, {"z": None}, {"rstd": None}, {"w": A + 2}, {"cols": 0},
               {"cols": gs.GS_NORM_MAX_COLS + 1}, {"eps": -1.0}, {"eps": float("nan")}, {"ys": 7}, {"zs": 0}, {"dtype": 9},
               {"p": -1.0}):
        assert call(**kw) == bad, kw
    sz = ctypes.c_size_t()
    assert lib.gs_dropout_add_norm_workspace_size(4, 0, ctypes.byref(sz)) == bad
    assert lib.gs_dropout_add_norm_workspace_size(4, 8, None) == bad
    assert lib.gs_dropout_add_norm_workspace_size(1000, 1024, ctypes.byref(sz)) == gs.GS_OK and sz.value >= 4096

    def back(ws=A, n=1 << 30, dz=A, y=A, dw=A, rstd=A, dxs=8):
        return lib.gs_dropout_add_norm_backward(dz, 8, None, 0, y, 8, A, rstd, A, dxs, None, 0, dw, 4, 8, 0, 0.1, 1, 2, ws, n,
                                                None)

    for kw in ({"ws": None}, {"ws": A + 16}, {"n": 16}, {"dz": None}, {"y": None}, {"dw": None}, {"rstd": None}, {"dxs": 5}):
        assert back(**kw) == bad, kw


def test_recurrence_refusals(gs):
    lib, bad = gs.load_library(), gs.GS_ERR_INVALID_ARG
    good = gs.GsSeq(A, 4 * 8, 8)
    ok = ctypes.byref(good)

    def seq(data=A, b=32, t=8):
        return ctypes.byref(gs.GsSeq(data, b, t))

    def call(x=ok, r=ok, i=ok, decay=A, y=ok, states=None, B=2, T=4, D=8, dtype=0, c=8.0, lengths=None):
        return lib.gs_recurrence_forward(x, r, i, decay, None, None, lengths, y, None, states, B, T, D, dtype, c, None)

    for kw in ({"x": None}, {"r": None}, {"i": None}, {"y": None}, {"x": seq(None)}, {"y": seq(None)}, {"decay": None},
               {"x": seq(A + 1)}, {"y": seq(t=7)}, {"y": seq(b=0)}, {"y": seq(b=31)}, {"x": seq(b=-1)}, {"states": A + 16},
               {"B": -1}, {"T": -1}, {"D": -1}, {"T": 1 << 31}, {"B": 1 << 20, "T": 1 << 20, "D": 1 << 10}, {"dtype": 3},
               {"c": 0.0}, {"c": float("inf")}, {"c": float("nan")}, {"lengths": A + 2}, {"B": 1 << 28, "T": 1, "D": 1}):
        assert call(**kw) == bad, kw
    assert call(B=0) == gs.GS_OK
    sz = ctypes.c_size_t()
    for f in (lib.gs_recurrence_states_size, lib.gs_recurrence_workspace_size):
        assert f(2, -1, 8, ctypes.byref(sz)) == bad and f(2, 4, 8, None) == bad
        assert f(2, 1000, 70, ctypes.byref(sz)) == gs.GS_OK and sz.value >= 2 * 70 * 4

    def back(dy=ok, dx=ok, states=A, dd=A, ws=A, n=1 << 30):
        return lib.gs_recurrence_backward(dy, None, ok, ok, ok, A, None, None, states, dx, ok, ok, dd, None, 2, 4, 8, 0, 8.0, ws,
                                          n, None)

    for kw in ({"dy": None}, {"dx": None}, {"dx": seq(None)}, {"states": None}, {"states": A + 4}, {"dd": None}, {"ws": None},
               {"n": 4}):
        assert back(**kw) == bad, kw

    def step(x=A, state=A, ss=8, n=4, slots=A, y=A, ys=8, decay=A, c=8.0):
        return lib.gs_recurrence_step(x, 8, A, 8, A, 8, decay, state, ss, n, slots, y, ys, 4, 8, 0, c, None)

    for kw in ({"x": None}, {"state": None}, {"ss": 7}, {"n": -1}, {"slots": None, "n": 3}, {"slots": A + 1}, {"y": None},
               {"ys": 4}, {"decay": None}, {"c": -1.0}):
        assert step(**kw) == bad, kw


def test_binding_refusals(gs):
    """What the C ABI cannot see of a tensor is checked by the binding."""
    x = torch.zeros(2, 4, 8)
    d = torch.zeros(8)
    with pytest.raises(gs.GsError, match="CUDA device"):
        gs.gs_recurrence_forward(x, x, x, d, x)
    with pytest.raises(gs.GsError, match="CUDA device"):
        gs.gs_dropout(x, x, 0.1, 1, 2)
    with pytest.raises(gs.GsError, match="none of float32"):
        gs.gs_dropout(x.double(), x, 0.1, 1, 2)
    with pytest.raises(gs.GsError, match="dimensions"):
        gs.gs_recurrence_forward(d, d, d, d, d)
    m = torch.device("meta")

    def check(f, *a):
        with pytest.raises(gs.GsError) as e:
            f("f", *a)
        assert e.value.status == gs.GS_ERR_INVALID_ARG

    t = torch.empty(4, 8, device=m)
    check(gs._matrix, "t", t, (4, 9), t.dtype, t.device)
    check(gs._matrix, "t", t, t.shape, torch.float16, t.device)
    check(gs._matrix, "t", t, t.shape, t.dtype, torch.device("cpu"))
    check(gs._matrix, "t", t.t(), (8, 4), t.dtype, t.device)
    odd = torch.empty(3, 4, 16, device=m)[:, ::2, :8]
    check(gs._matrix, "t", torch.empty(3, 5, 8, device=m)[:, :4], (3, 4, 8), t.dtype, t.device)
    assert gs._matrix("f", "t", odd, odd.shape, odd.dtype, odd.device)[1] == 32
    assert gs._matrix("f", "t", t.expand(5, 4, 8)[:, :1], (5, 1, 8), t.dtype, t.device)[1] == 0
    check(gs._dense, "t", t.t(), (8, 4), t.dtype, t.device)
    check(gs._seq, "t", torch.empty(2, 8, 4, device=m).transpose(1, 2), (2, 4, 8), torch.float32, m)
    check(gs._whole, "lengths", torch.empty(2, dtype=torch.int64, device=m), (2,), m)
    check(gs._states_fit, torch.empty(8, dtype=torch.uint8), 2, 1000, 64)

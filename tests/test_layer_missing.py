"""Tensors that a call of the recurrent layer's operators lacks: refused by name with the library's error,
but for those that it can do without."""

import pytest

torch = pytest.importorskip("torch")

DEV = torch.device("meta")


@pytest.fixture
def gs(monkeypatch):
    import os

    import paper_2108_06004_gb300 as lib
    if not os.path.exists(lib.LIB_PATH):
        from paper_2108_06004_gb300 import _build
        _build.build()
    lib.load_library()
    monkeypatch.setattr(lib, "_launch_stream", lambda func, t, stream: 0)
    # an address for what a meta tensor has none of; nothing is launched, since every call here lacks something
    # that the library refuses on the host
    for name in ("_dense", "_matrix", "_seq"):
        real = getattr(lib, name)

        def with_address(func, what, t, *a, _real=real, _name=name):
            out = _real(func, what, t, *a)
            if t is None:
                return out
            return {"_dense": lambda: 4096, "_matrix": lambda: (4096, out[1]),
                    "_seq": lambda: lib.GsSeq(4096, out.batch_stride, out.token_stride)}[_name]()
        monkeypatch.setattr(lib, name, with_address)
    address = lib._ptr
    monkeypatch.setattr(lib, "_ptr", lambda t: 4096 if torch.is_tensor(t) else address(t))
    return lib


def meta(*shape):
    return torch.empty(shape, device=DEV)


def room(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


def refused(gs, match, f, *a, **kw):
    with pytest.raises(gs.GsError, match=match) as e:
        f(*a, **kw)
    assert e.value.status == gs.GS_ERR_INVALID_ARG


@pytest.mark.parametrize("missing,match", [(0, "first tensor|x is NULL"), (1, "r is NULL"), (2, "i is NULL"), (3, "decay is NULL"),
                                           (4, "y is NULL")])
def test_recurrence_forward(gs, missing, match):
    a = [meta(2, 5, 8), meta(2, 5, 8), meta(2, 5, 8), meta(8), meta(2, 5, 8)]
    a[missing] = None
    refused(gs, match, gs.gs_recurrence_forward, *a)


@pytest.mark.parametrize("missing,match", [(0, "dy is NULL"), (1, "first tensor|x is NULL"), (2, "r is NULL"), (3, "i is NULL"),
                                           (4, "decay is NULL"), (5, "states is NULL"), (6, "dx is NULL"), (7, "dr is NULL"),
                                           (8, "di is NULL"), (9, "ddecay is NULL"), (10, "workspace is NULL")])
def test_recurrence_backward(gs, missing, match):
    x = meta(2, 5, 8)
    a = [x, x, x, x, meta(8), room(gs.gs_recurrence_states_size(2, 5, 8)), x, x, x, meta(8), 4096]
    a[missing] = None
    refused(gs, match, gs.gs_recurrence_backward, *a,
            workspace_bytes=gs.gs_recurrence_workspace_size(2, 5, 8))


def test_others(gs):
    x, w = meta(4, 8), meta(8)
    refused(gs, "first tensor|x is NULL", gs.gs_dropout, None, x, 0.1, 1, 2)
    refused(gs, "out is NULL", gs.gs_dropout, x, None, 0.1, 1, 2)
    refused(gs, "residual is NULL", gs.gs_dropout_add_norm, x, None, w, x, x, meta(4), 0.1, 1, 2)
    refused(gs, "weight is NULL", gs.gs_dropout_add_norm, x, x, None, x, x, meta(4), 0.1, 1, 2)
    refused(gs, "workspace is NULL", gs.gs_dropout_add_norm_backward, x, None, x, w, meta(4), x, x, w, 0.1, 1, 2, None)
    refused(gs, "state must", gs.gs_recurrence_step, x, x, x, w, None, x)
    refused(gs, "decay is NULL", gs.gs_recurrence_step, x, x, x, None, x, x)


def test_a_backward_pass_over_no_tokens_needs_no_states(gs, monkeypatch):
    real, passed = gs.load_library(), []

    class Library:
        def __getattr__(self, name):
            if name == "gs_recurrence_backward":
                return lambda *a: passed.append(a) or gs.GS_OK
            return getattr(real, name)

    monkeypatch.setattr(gs, "load_library", lambda: Library())
    e = meta(3, 0, 8)
    gs.gs_recurrence_backward(e, e, e, e, meta(8), None, e, e, e, meta(8), 4096,
                              workspace_bytes=gs.gs_recurrence_workspace_size(3, 0, 8))
    assert passed[0][8] is None

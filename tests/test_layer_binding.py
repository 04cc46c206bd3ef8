"""What the binding of the recurrent layer's operators has to refuse before the library is called, with
the library's launching functions replaced, so that nothing is launched whatever the binding lets through."""

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
    real = lib.load_library()

    class Library:
        reached = []

        def __getattr__(self, name):
            if name.endswith("_size") or name == "gs_last_error":
                return getattr(real, name)
            return lambda *a: self.reached.append((name, a)) or lib.GS_OK

    fake = Library()
    fake.reached.clear()
    monkeypatch.setattr(lib, "load_library", lambda: fake)
    monkeypatch.setattr(lib, "_launch_stream", lambda func, t, stream: 0)
    monkeypatch.setattr(lib, "reached", fake.reached, raising=False)
    return lib


B, T, D = 2, 40, 16


def meta(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device=DEV)


def room(n, device=DEV):
    return torch.empty(n, dtype=torch.uint8, device=device)


def forward(gs, states, **kw):
    x = meta(B, T, D)
    gs.gs_recurrence_forward(x, x, x, meta(D), x, states=states, **kw)


def backward(gs, states, workspace, **kw):
    x = meta(B, T, D)
    gs.gs_recurrence_backward(x, x, x, x, meta(D), states, x, x, x, meta(D), workspace, **kw)


def norm_backward(gs, workspace, **kw):
    x = meta(T, D)
    gs.gs_dropout_add_norm_backward(x, None, x, meta(D), meta(T), x, x, meta(D), 0.1, 1, 2, workspace, **kw)


def refused(gs, match, f, *a, **kw):
    with pytest.raises(gs.GsError, match=match) as e:
        f(gs, *a, **kw)
    assert e.value.status == gs.GS_ERR_INVALID_ARG and not gs.reached


def test_states_and_workspaces_have_to_be_on_the_tensors_device(gs):
    """A kernel would write through the address of another device's memory, or of the host's."""
    ns, nw = gs.gs_recurrence_states_size(B, T, D), gs.gs_recurrence_workspace_size(B, T, D)
    nn = gs.gs_dropout_add_norm_workspace_size(T, D)
    refused(gs, "states is on cpu", forward, room(ns, "cpu"))
    refused(gs, "states is on cpu", backward, room(ns, "cpu"), room(nw))
    refused(gs, "workspace is on cpu", backward, room(ns), room(nw, "cpu"))
    refused(gs, "workspace is on cpu", norm_backward, room(nn, "cpu"))
    forward(gs, room(ns))
    backward(gs, room(ns), room(nw))
    norm_backward(gs, room(nn))
    assert [name for name, _ in gs.reached] == ["gs_recurrence_forward", "gs_recurrence_backward",
                                                "gs_dropout_add_norm_backward"]


def test_workspaces_hold_what_is_said_of_them(gs):
    ns, nw = gs.gs_recurrence_states_size(B, T, D), gs.gs_recurrence_workspace_size(B, T, D)
    nn = gs.gs_dropout_add_norm_workspace_size(T, D)
    refused(gs, "bytes, not", backward, room(ns), room(16), workspace_bytes=nw)
    refused(gs, "bytes, not", norm_backward, room(16), workspace_bytes=nn)
    refused(gs, "contiguous", backward, room(ns), room(2 * nw)[::2])
    refused(gs, "contiguous", norm_backward, room(2 * nn)[::2])
    backward(gs, room(ns), room(nw + 9), workspace_bytes=nw)
    norm_backward(gs, 4096, workspace_bytes=nn)
    (_, a), (_, b) = gs.reached
    assert a[-2] == nw and b[-3:-1] == (4096, nn)

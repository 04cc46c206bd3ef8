"""Waits of the recurrence's sequence kernels that run out: whatever has to do with what did not come is
NaN, whatever is not NaN is right, and the next call is as if nothing had been."""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def gs():
    import paper_2108_06004_gb300 as lib
    lib.load_library()
    torch.cuda.set_device(0)
    return lib


@pytest.fixture(autouse=True)
def whole_waits(gs):
    yield
    gs.gs_recurrence_wait_tries()


def inputs(B, T, D, dtype, reset, lengths):
    gen = torch.Generator(device="cuda").manual_seed(T + D)

    def rand(*shape, dt=DT[dtype]):
        return torch.randn(shape, dtype=dt, device="cuda", generator=gen)

    s = {k: rand(B, T, D) for k in ("x", "r", "i", "dy")}
    f32 = torch.float32
    s.update(decay=rand(D, dt=f32) - 4, h0=rand(B, D, dt=f32), dh=rand(B, D, dt=f32), reset=None, lengths=None)
    if reset:
        s["reset"] = (torch.rand(B, T, device="cuda", generator=gen) < 0.02).to(torch.uint8)
    if lengths:
        n = torch.randint(1, T + 1, (B,), device="cuda", generator=gen, dtype=torch.int32)
        n[0], n[-1] = T, (0 if B > 1 else T)
        s["lengths"] = n
    return s


def forward(gs, s):
    B, T, D = s["x"].shape
    out = {"y": torch.full_like(s["x"], 7.0), "h_last": torch.full_like(s["h0"], 7.0)}
    states = torch.full((gs.gs_recurrence_states_size(B, T, D),), 1, dtype=torch.uint8, device="cuda")
    gs.gs_recurrence_forward(s["x"], s["r"], s["i"], s["decay"], out["y"], h0=s["h0"], reset=s["reset"], lengths=s["lengths"],
                             h_last=out["h_last"], states=states)
    return out, states


def backward(gs, s, states):
    B, T, D = s["x"].shape
    out = {k: torch.full_like(s["x"], 7.0) for k in ("dx", "dr", "di")}
    out.update(ddecay=torch.full_like(s["decay"], 7.0), dh0=torch.full_like(s["h0"], 7.0))
    ws = torch.empty(gs.gs_recurrence_workspace_size(B, T, D), dtype=torch.uint8, device="cuda")
    gs.gs_recurrence_backward(s["dy"], s["x"], s["r"], s["i"], s["decay"], states, out["dx"], out["dr"], out["di"], out["ddecay"],
                              ws, dh_last=s["dh"], reset=s["reset"], lengths=s["lengths"], dh0=out["dh0"])
    return out


def live(s):
    B, T, _ = s["x"].shape
    n = torch.full((B,), T, device="cuda") if s["lengths"] is None else s["lengths"]
    return (torch.arange(T, device="cuda")[None] < n[:, None])[..., None].expand_as(s["x"]), (n > 0)[:, None].expand_as(s["h0"])


def same(a, b):
    return all(torch.equal(a[k], b[k]) for k in b)


# columns that share time in clusters (with 16-byte rows), and enough columns to need none
TILED = [(1, 9000, 40), (3, 2500, 96), (57, 300, 512)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,D", TILED)
@pytest.mark.parametrize("masks", [False, True])
def test_tiles_that_do_not_come(gs, dtype, B, T, D, masks):
    s = inputs(B, T, D, dtype, masks, masks)
    want, states = forward(gs, s)
    want_back = backward(gs, s, states)
    gs.gs_recurrence_wait_tries(tiles=0)
    got, none = forward(gs, s)
    back = backward(gs, s, states)
    gs.gs_recurrence_wait_tries()
    token, row = live(s)
    assert got["y"][token].isnan().all() and not got["y"][~token].any()
    assert got["h_last"][row].isnan().all() and torch.equal(got["h_last"][~row], s["h0"][~row])
    for k in ("dx", "dr", "di"):
        assert back[k][token].isnan().all() and not back[k][~token].any(), k
    assert back["ddecay"].isnan().all()
    assert back["dh0"][row].isnan().all() and torch.equal(back["dh0"][~row], s["dh"][~row])
    # what such a forward pass kept does not pass for states
    after = backward(gs, s, none)
    assert after["ddecay"].isnan().all()
    again, states = forward(gs, s)
    assert same(again, want) and same(backward(gs, s, states), want_back)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,D", [(1, 9000, 40), (1, 9000, 33), (3, 2500, 96)])
@pytest.mark.parametrize("masks", [False, True])
def test_messages_that_do_not_come(gs, dtype, B, T, D, masks):
    s = inputs(B, T, D, dtype, masks, masks)
    want, states = forward(gs, s)
    want_back = backward(gs, s, states)
    gs.gs_recurrence_wait_tries(messages=0)
    got, _ = forward(gs, s)
    back = backward(gs, s, states)
    gs.gs_recurrence_wait_tries()
    token, row = live(s)
    for k, w in {**want, **want_back}.items():
        g = got[k] if k in got else back[k]
        assert (g.isnan() | (g == w)).all(), f"{k}: neither NaN nor right"
        if not masks:
            assert g.isnan().all(), k
    for g in (got["y"], back["dx"]):
        assert g[token].isnan().any() and not g[~token].any()
    assert got["h_last"][row].isnan().all() and back["dh0"][row].isnan().all() and back["ddecay"].isnan().all()
    again, states = forward(gs, s)
    assert same(again, want) and same(backward(gs, s, states), want_back)

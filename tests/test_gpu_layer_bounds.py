"""The recurrent layer's operators write nothing beside their outputs: margins, the space between
rows and the channels past a row's end keep what they held."""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
MARGIN = 256     # elements before and after
MARK = 12288.0   # exact in every type


@pytest.fixture(scope="module")
def gs():
    import paper_2108_06004_gb300 as lib
    lib.load_library()
    torch.cuda.set_device(0)
    return lib


class Guarded:
    """An output inside a larger buffer of a value that no result has."""

    def __init__(self, shape, dtype="f32", pad=0, shift=0):
        n = 1
        for s in shape[:-1]:
            n *= s
        self.flat = torch.full((2 * MARGIN + n * (shape[-1] + pad) + shift,), MARK, dtype=DT[dtype], device="cuda")
        inner = self.flat[MARGIN + shift:MARGIN + shift + n * (shape[-1] + pad)]
        self.t = inner.view(*shape[:-1], shape[-1] + pad)[..., :shape[-1]]

    def check(self, what):
        assert not (self.t == MARK).any(), f"{what}: not all written"
        self.t.fill_(MARK)
        assert (self.flat == MARK).all(), f"{what}: something beside it was written"


CASES = [(72, 8, 0), (72, 0, 0), (200, 56, 0), (66, 2, 0), (1001, 0, 0), (1001, 7, 0), (33, 3, 1), (8, 8, 0), (1, 0, 0), (128, 0, 4)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D,pad,shift", CASES)
@pytest.mark.parametrize("B,T,lengths", [(2, 37, None), (3, 300, [300, 0, 129]), (1, 2100, None)])
def test_recurrence_writes_its_outputs_alone(gs, dtype, D, pad, shift, B, T, lengths):
    gen = torch.Generator(device="cuda").manual_seed(D + T)

    def rand(*shape, dt=DT[dtype]):
        return torch.randn(shape, dtype=dt, device="cuda", generator=gen)

    x, r, i, dy = (rand(B, T, D) for _ in range(4))
    decay, h0, dh = rand(D, dt=torch.float32) - 3, rand(B, D, dt=torch.float32), rand(B, D, dt=torch.float32)
    length = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    reset = (torch.rand(B, T, device="cuda", generator=gen) < 0.02).to(torch.uint8)
    out = {k: Guarded((B, T, D), dtype, pad, shift) for k in ("y", "dx", "dr", "di")}
    out.update(h_last=Guarded((B, D)), ddecay=Guarded((D,)), dh0=Guarded((B, D)))

    def room(n):    # a workspace with a margin after it
        return torch.full((n + 1024,), 7, dtype=torch.uint8, device="cuda")

    ns, nw = gs.gs_recurrence_states_size(B, T, D), gs.gs_recurrence_workspace_size(B, T, D)
    states, ws = room(ns), room(nw)
    gs.gs_recurrence_forward(x, r, i, decay, out["y"].t, h0=h0, reset=reset, lengths=length, h_last=out["h_last"].t,
                             states=states)
    gs.gs_recurrence_backward(dy, x, r, i, decay, states, out["dx"].t, out["dr"].t, out["di"].t, out["ddecay"].t, ws,
                              dh_last=dh, reset=reset, lengths=length, dh0=out["dh0"].t, workspace_bytes=nw)
    for k, g in out.items():
        g.check(k)
    assert (states[ns:] == 7).all() and (ws[nw:] == 7).all()
    y, state = Guarded((B, D), dtype, pad, shift), Guarded((B + 2, D), "f32", pad, shift)
    state.t.zero_()
    gs.gs_recurrence_step(x[:, 0], r[:, 0], i[:, 0], decay, state.t, y.t)
    y.check("step y")
    state.check("state")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols,pad,shift", CASES + [(4099, 0, 0), (2048, 8, 0)])
@pytest.mark.parametrize("rows", [1, 3, 40])
def test_rows_write_their_outputs_alone(gs, dtype, cols, pad, shift, rows):
    gen = torch.Generator(device="cuda").manual_seed(cols + rows)

    def rand(*shape, dt=DT[dtype]):
        return torch.randn(shape, dtype=dt, device="cuda", generator=gen)

    x, res = rand(rows, cols), rand(rows, cols)
    out = Guarded((rows, cols), dtype, pad, shift)
    gs.gs_dropout(x, out.t, 0.3, 1, 2, residual=res)
    out.check("dropout")
    w = rand(cols, dt=torch.float32)
    y, z, rstd = Guarded((rows, cols), dtype, pad, shift), Guarded((rows, cols), dtype, pad, shift), Guarded((rows,))
    gs.gs_dropout_add_norm(x, res, w, y.t, z.t, rstd.t, 0.3, 1, 2)
    stream, scale = y.t.clone(), rstd.t.clone()
    for k, g in (("y", y), ("z", z), ("rstd", rstd)):
        g.check(k)
    dx, dres, dw = Guarded((rows, cols), dtype, pad, shift), Guarded((rows, cols), dtype, pad, shift), Guarded((cols,))
    n = gs.gs_dropout_add_norm_workspace_size(rows, cols)
    ws = torch.full((n + 1024,), 7, dtype=torch.uint8, device="cuda")
    gs.gs_dropout_add_norm_backward(x, res, stream, w, scale, dx.t, dres.t, dw.t, 0.3, 1, 2, ws, workspace_bytes=n)
    for k, g in (("dx", dx), ("dresidual", dres), ("dweight", dw)):
        g.check(k)
    assert (ws[n:] == 7).all()

"""Linear attention with a decay for each head on the GPU against its fp64 oracle, within the bounds of
tests/attention_bounds.py, at the sizes, head layouts, strides and masks where it can go wrong."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention  # noqa: E402
from tests import attention_bounds as bounds  # noqa: E402
from tests import layer_bounds  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def gs():
    import paper_2108_06004_gb300 as lib
    lib.load_library()
    torch.cuda.set_device(0)
    return lib


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, exact, tol, what):
    got = host(got) if torch.is_tensor(got) else got
    bad = ~(np.abs(got - exact) <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} outside, first at {np.argwhere(bad)[0]}: "
                           f"{got[bad][0]!r} for {exact[bad][0]!r} +- {np.broadcast_to(tol, got.shape)[bad][0]!r}")


def place(shape, dtype, how, fill=None, rng=None, scale=1.0):
    """A [B][T][H][D] tensor in one of several layouts; what lies between its rows is NaN."""
    B, T, H, D = shape
    nan = float("nan")
    if how == "heads first":     # [B][H][T][D]
        t = torch.full((B, H, T, D), nan, dtype=DT[dtype], device="cuda").transpose(1, 2)
    elif how == "wide":          # rows of a wider product, every row at a 16-byte boundary
        t = torch.full((B, T, H, -(-D // 8) * 8 + 8), nan, dtype=DT[dtype], device="cuda")[..., :D]
    elif how == "odd":           # rows at odd elements
        t = torch.full((B * T * H * (D + 1) + 1,), nan, dtype=DT[dtype], device="cuda")[1:].view(B, T, H, D + 1)[..., :D]
    else:
        t = torch.full(shape, nan, dtype=DT[dtype], device="cuda")
    if fill is not None:
        t.fill_(fill)
    if rng is not None:
        t.copy_(torch.from_numpy(rng.standard_normal(shape) * scale))
    return t


class Case:
    """Inputs, the library's results and their exact values with bounds."""

    def __init__(self, gs, B, T, H, K, Dk, Dv, dtype, lengths=None, offsets=None, how="dense", seed=0, state=True, g=None, size=1.0):
        rng = np.random.default_rng(seed + 1000 * T + 10 * Dk + Dv)
        self.sizes, self.dtype, self.scale = (B, T, H, K, Dk, Dv), dtype, 0.37
        rows = 1 if offsets is not None else B
        self.rows, self.lengths, self.offsets = rows, lengths, offsets
        self.q, self.k, self.v, self.do = (place((rows, T, h, d), dtype, how, rng=rng, scale=size)
                                           for h, d in ((H, Dk), (K, Dk), (K, Dv), (H, Dv)))
        self.g = np.float32(-np.exp(rng.uniform(-6, 0, H))) if g is None else np.float32(g)
        real = np.clip(self.g.astype(np.float64), -8192, 0)
        put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", torch.float32)   # noqa: E731
        self.s0 = put(rng.standard_normal((B, H, Dk, Dv))) if state else None
        self.ds = put(rng.standard_normal((B, H, Dk, Dv))) if state else None
        whole = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
        more = {"lengths": whole(lengths), "offsets": whole(offsets), "scale": self.scale}
        self.o, self.dq, self.dk, self.dv = (place((rows, T, h, d), dtype, how, fill=7.0)
                                             for h, d in ((H, Dv), (H, Dk), (K, Dk), (K, Dv)))
        self.last, self.ds0 = (torch.full((B, H, Dk, Dv), float("nan"), device="cuda") for _ in range(2))
        G = put(self.g)
        ws = torch.empty(gs.gs_linear_attention_workspace_size(*self.sizes, DT[dtype], packed=offsets is not None),
                         dtype=torch.uint8, device="cuda").fill_(255)
        gs.gs_linear_attention_forward(self.q, self.k, self.v, G, self.o, ws, s0=self.s0, s_last=self.last, **more)
        ws = torch.empty(gs.gs_linear_attention_workspace_size(*self.sizes, DT[dtype], backward=True, packed=offsets is not None),
                         dtype=torch.uint8, device="cuda").fill_(255)
        gs.gs_linear_attention_backward(self.do, self.q, self.k, self.v, G, self.dq, self.dk, self.dv, ws, s0=self.s0,
                                        ds_last=self.ds, ds0=self.ds0, **more)
        self.decay = real

    def check(self):
        B, T, H, K, Dk, Dv = self.sizes
        share, sc = H // K, self.scale
        q, k, v, do = (host(t) for t in (self.q, self.k, self.v, self.do))
        zero = np.zeros((B, H, Dk, Dv))
        s0, ds = (zero if t is None else host(t) for t in (self.s0, self.ds))
        want = {n: np.full((self.rows, T, h, d), 7.0) for n, h, d in (("o", H, Dv), ("dq", H, Dk), ("dk", K, Dk), ("dv", K, Dv))}
        tol = {n: np.zeros(x.shape) for n, x in want.items()}
        for b, (row, start, n) in enumerate(attention.spans(B, T, self.lengths, self.offsets)):
            at = slice(start, start + n)
            if self.offsets is None:
                for x in want.values():
                    x[row, n:] = 0.0
            qs, ks, vs, dos = q[row, at], k[row, at], v[row, at], do[row, at]
            o, last = attention.sequence(qs, ks, vs, self.decay, sc, s0[b])
            dq, dk, dv, ds0 = attention.sequence_gradients(dos, qs, ks, vs, self.decay, sc, s0[b], ds[b])
            for name, x in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
                want[name][row, at] = x
            e = {name: np.zeros(x.shape) for name, x in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv))}
            elast, eds0 = np.zeros((H, Dk, Dv)), np.zeros((H, Dk, Dv))
            for h in range(H):
                g, f = self.decay[h], h // share
                a = (self.dtype,)
                e["o"][:, h], elast[h] = (x * y for x, y in zip(bounds.walk(qs[:, h], ks[:, f], vs[:, f], g, s0[b, h], *a, 1), (sc, 1)))
                e["dq"][:, h] = sc * bounds.walk(dos[:, h], vs[:, f], ks[:, f], g, s0[b, h].T, *a, 1)[0]
                back = lambda x: x[::-1]   # noqa: E731
                y = bounds.walk(back(vs[:, f]), back(sc * dos[:, h]), back(qs[:, h]), g, ds[b, h].T, *a, 0)[0]
                e["dk"][:, f] += back(y)
                y, eds0[h] = bounds.walk(back(ks[:, f]), back(sc * qs[:, h]), back(dos[:, h]), g, ds[b, h], *a, 0)
                e["dv"][:, f] += back(y)
            for name, x in e.items():
                tol[name][row, at] = layer_bounds.stored(want[name][row, at], x * (1 + share * layer_bounds.U), self.dtype)
            close(self.last[b], last, layer_bounds.stored(last, elast, "f32"), f"s_last {b}")
            close(self.ds0[b], ds0, layer_bounds.stored(ds0, eds0, "f32"), f"ds0 {b}")
        for name, x in want.items():
            close(getattr(self, name), x, tol[name], name)


TYPES = ["bf16", "f16", "f32"]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 257, 700])
def test_lengths(gs, T, dtype):
    Case(gs, 2, T, 2, 2, 64, 64, dtype).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,K,Dk,Dv", [(1, 1, 1, 1), (2, 2, 16, 16), (3, 3, 40, 72), (2, 2, 47, 33), (4, 2, 64, 64), (2, 1, 128, 128),
                                       (6, 2, 64, 128), (2, 2, 128, 64), (1, 1, 80, 96), (1, 1, 160, 256), (1, 1, 256, 8), (1, 1, 8, 256),
                                       (1, 1, 65, 129)])
def test_heads(gs, H, K, Dk, Dv, dtype):
    Case(gs, 1, 150, H, K, Dk, Dv, dtype).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 128), (40, 24)])
def test_ragged(gs, Dk, Dv, dtype):
    Case(gs, 7, 260, 4, 2, Dk, Dv, dtype, lengths=[260, 0, 1, 64, 129, 300, -5]).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 128), (40, 24)])
def test_packed(gs, Dk, Dv, dtype):
    """Documents of all lengths, empty ones, and tokens of none at both ends, which stay as they were."""
    Case(gs, 9, 600, 4, 2, Dk, Dv, dtype, offsets=[3, 3, 4, 68, 68, 200, 329, 330, 590, 590]).check()


def test_many_packed(gs):
    cuts = np.concatenate(([0], np.cumsum(np.random.default_rng(3).integers(0, 12, 150))))
    Case(gs, 150, int(cuts[-1]) + 1, 1, 1, 16, 16, "bf16", offsets=cuts.tolist()).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("how", ["heads first", "wide", "odd"])
def test_strides(gs, how, dtype):
    Case(gs, 2, 140, 4, 2, 64, 64, dtype, lengths=[140, 77], how=how).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_decays(gs, dtype):
    """No decay at all, one that forgets at once, the limits of what is taken, and all in between."""
    Case(gs, 1, 400, 8, 8, 64, 64, dtype, g=[0.0, -1e-6, -0.01, -0.49, -0.51, -5.0, -100.0, -1e9]).check()
    Case(gs, 1, 90, 2, 2, 64, 64, dtype, g=[3.0, -float("inf")], state=False).check()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", [1e-3, 30.0])
def test_magnitudes(gs, dtype, size):
    """Small inputs keep their digits and scores and states beyond a half's range do no harm."""
    case = Case(gs, 1, 200, 2, 2, 64, 64, dtype, size=size, state=False)
    if size > 1 and dtype == "f16":
        assert float(case.last.abs().max()) > 20000
        return check_finite(case)
    case.check()


def check_finite(case):
    """Where results leave the type's range they are infinite, and exact elsewhere."""
    exact = attention.sequence(host(case.q)[0], host(case.k)[0], host(case.v)[0], case.decay, case.scale, np.zeros((2, 64, 64)))
    got = host(case.o)[0]
    inside = np.abs(exact[0]) < 65000
    assert np.isfinite(got[inside]).all()
    tol = np.stack([case.scale * bounds.walk(host(case.q)[0, :, h], host(case.k)[0, :, h], host(case.v)[0, :, h], case.decay[h],
                                             np.zeros((64, 64)), "f16", 1)[0] for h in range(2)], axis=1)
    close(got[inside], exact[0][inside], layer_bounds.stored(exact[0], tol, "f16")[inside], "o")


@pytest.mark.parametrize("B,T,H,D", [(1, 5000, 2, 64), (1, 3000, 1, 128)])
def test_long(gs, B, T, H, D):
    """Enough tokens of few heads that their time is cut into pieces."""
    Case(gs, B, T, H, H, D, D, "bf16", lengths=[T - 3]).check()


def test_nothing(gs):
    """No tokens: the states pass through."""
    case = Case(gs, 2, 0, 2, 1, 16, 24, "bf16")
    case.check()
    assert torch.equal(case.last, case.s0) and torch.equal(case.ds0, case.ds)


def test_in_place_state(gs):
    """s_last may be s0 itself, with and without pieces."""
    for T in (100, 3000):
        a = Case(gs, 1, T, 2, 2, 64, 64, "bf16")
        s = a.s0.clone()
        ws = torch.empty(gs.gs_linear_attention_workspace_size(*a.sizes, DT["bf16"]), dtype=torch.uint8, device="cuda")
        o = torch.empty_like(a.o)
        gs.gs_linear_attention_forward(a.q, a.k, a.v, torch.from_numpy(a.g).cuda(), o, ws, s0=s, s_last=s, scale=a.scale)
        assert torch.equal(s, a.last) and torch.equal(o, a.o)


def test_masked_tokens_have_no_influence(gs):
    """What is behind a row's end may be anything."""
    rng = np.random.default_rng(5)
    x = [place((2, 200, 2, 64), "bf16", "dense", rng=rng) for _ in range(4)]
    g = torch.tensor([-0.1, -0.01], device="cuda")
    lengths = torch.tensor([130, 0], dtype=torch.int32, device="cuda")
    ws = torch.empty(gs.gs_linear_attention_workspace_size(2, 200, 2, 2, 64, 64, torch.bfloat16, backward=True), dtype=torch.uint8,
                     device="cuda")

    def run():
        out = [torch.full_like(x[0], 5.0) for _ in range(4)]
        s = [torch.empty(2, 2, 64, 64, device="cuda") for _ in range(2)]
        gs.gs_linear_attention_forward(*x[:3], g, out[0], ws, lengths=lengths, s_last=s[0])
        gs.gs_linear_attention_backward(x[3], *x[:3], g, *out[1:], ws, lengths=lengths, ds0=s[1])
        return out + s

    want = run()
    for t in x:
        t[0, 130:] = float("nan")
        t[1] = float("inf")
    for a, b in zip(run(), want):
        assert torch.equal(a, b)


def test_gradients_against_differences(gs):
    """Directional derivatives of a random function of o and s_last."""
    rng = np.random.default_rng(9)
    B, T, H, K, Dk, Dv = 2, 50, 4, 2, 16, 24
    case = Case(gs, B, T, H, K, Dk, Dv, "f32", lengths=[50, 31])
    do, ds = host(case.do), host(case.ds)

    def value(q, k, v, s0):
        total = 0.0
        for b, (row, _, n) in enumerate(attention.spans(B, T, case.lengths)):
            o, last = attention.sequence(q[row, :n], k[row, :n], v[row, :n], case.decay, case.scale, s0[b])
            total += (o * do[row, :n]).sum() + (last * ds[b]).sum()
        return total

    args = [host(t) for t in (case.q, case.k, case.v, case.s0)]
    for n, grad in enumerate((case.dq, case.dk, case.dv, case.ds0)):
        step = rng.standard_normal(args[n].shape)
        ends = [value(*[a + (h * step if m == n else 0) for m, a in enumerate(args)]) for h in (1e-6, -1e-6)]
        slope = (ends[0] - ends[1]) / 2e-6
        # the function is linear in each argument: the difference is exact to 2^-53 of its value over the step
        assert abs(slope - (host(grad) * step).sum()) < 1e-4 * np.sqrt((host(grad) ** 2).sum() * (step ** 2).sum())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,K,Dk,Dv", [(16, 16, 64, 64), (2, 1, 128, 128), (3, 3, 47, 33), (1, 1, 1, 1), (2, 2, 256, 256), (1, 1, 40, 72)])
@pytest.mark.parametrize("slots", [False, True])
def test_step(gs, H, K, Dk, Dv, slots, dtype):
    rng = np.random.default_rng(Dk)
    B, N = 5, 7
    q, k, v = (place((B, 1, h, d), dtype, "odd" if slots else "dense", rng=rng)[:, 0] for h, d in ((H, Dk), (K, Dk), (K, Dv)))
    state = torch.from_numpy(rng.standard_normal((N, H, Dk, Dv))).to("cuda", torch.float32)
    before, g = state.clone(), torch.from_numpy(np.float32(-np.exp(rng.uniform(-6, 1, H)))).cuda()
    at = [6, -1, 0, 99, 3] if slots else list(range(B))
    o = torch.full((B, H, Dv), float("nan"), dtype=DT[dtype], device="cuda")
    gs.gs_linear_attention_step(q, k, v, g, state, o, slots=torch.tensor(at, dtype=torch.int32, device="cuda") if slots else None, scale=0.5)
    touched = [a for a in at if 0 <= a < N]
    for n in range(N):
        if n not in touched:
            assert torch.equal(state[n], before[n])
    U = layer_bounds.U
    for b, a in enumerate(at):
        if not 0 <= a < N:
            assert not o[b].any()
            continue
        qs, ks, vs, s = host(q[b]), host(k[b]), host(v[b]), host(before[a])
        want, S = attention.sequence(qs[None], ks[None], vs[None], host(g), 0.5, s)
        big = np.exp(host(g))[:, None, None] * np.abs(s) + np.repeat(np.abs(ks[:, :, None] * vs[:, None]), H // K, axis=0)
        # the decay (4u and its exponent's |g| u), its product and the sum: each of a part of what is old or new
        e = (6 + np.abs(host(g)))[:, None, None] * U * (np.abs(s) * np.maximum(np.exp(host(g)), 2.0 ** -20)[:, None, None] + big)
        close(state[a], S, 2 * e, "state")
        eo = 0.5 * np.einsum("hd,hde->he", np.abs(qs), 2 * e + (Dk + 6) * U * big)
        close(o[b], want[0], layer_bounds.stored(want[0], 2 * eo, dtype), "o")


def test_steps_continue_a_prompt(gs):
    """A prompt and single tokens after it give what one pass over all tokens gives."""
    rng = np.random.default_rng(2)
    B, T, H, D = 3, 140, 4, 64
    q, k, v = (place((B, T, H, D), "bf16", "dense", rng=rng) for _ in range(3))
    g = torch.tensor([-0.3, -0.05, -0.01, -0.002], device="cuda")
    ws = torch.empty(gs.gs_linear_attention_workspace_size(B, T, H, H, D, D, torch.bfloat16), dtype=torch.uint8, device="cuda")
    whole, part = torch.empty_like(v), torch.empty_like(v)
    state, last = (torch.empty(B, H, D, D, device="cuda") for _ in range(2))
    gs.gs_linear_attention_forward(q, k, v, g, whole, ws, s_last=last)
    n = 130
    gs.gs_linear_attention_forward(q[:, :n], k[:, :n], v[:, :n], g, part[:, :n], ws, s_last=state)
    for t in range(n, T):
        gs.gs_linear_attention_step(q[:, t], k[:, t], v[:, t], g, state, part[:, t])
    tol = np.stack([np.stack([2 * bounds.walk(host(q)[b, :, h], host(k)[b, :, h], host(v)[b, :, h], float(g[h]), np.zeros((D, D)), "bf16", 1)[0]
                              for h in range(H)], axis=1) for b in range(B)])
    exact = host(whole)
    close(part, exact, layer_bounds.stored(exact, tol, "bf16") + 2.0 ** -8 * np.abs(exact), "o")
    assert float((state - last).norm() / last.norm()) < 2e-6


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
def test_every_multiprocessor_is_shared(gs, D, dtype):
    """More heads than CTAs that run at once."""
    Case(gs, 4, 300, 80, 80, D, D, dtype).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,H,D,lengths", [(10, 1000, 4, 64, None), (6, 900, 3, 128, [900, 0, 257, 513, 128, 1]), (2, 190, 2, 40, [190, 65])])
def test_few_pieces(gs, B, T, H, D, lengths, dtype):
    """Rows of so few pieces that each adds up the ones before it, and the same with s_last in the place of s0."""
    case = Case(gs, B, T, H, H, D, D, dtype, lengths=lengths)
    case.check()
    s, o = case.s0.clone(), torch.empty_like(case.o)
    ws = torch.empty(gs.gs_linear_attention_workspace_size(*case.sizes, DT[dtype]), dtype=torch.uint8, device="cuda")
    whole = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    gs.gs_linear_attention_forward(case.q, case.k, case.v, torch.from_numpy(case.g).cuda(), o, ws, s0=s, s_last=s, lengths=whole, scale=case.scale)
    assert torch.equal(s, case.last) and torch.equal(o, case.o)


def test_few_pieces_packed(gs):
    Case(gs, 3, 1500, 8, 4, 64, 64, "bf16", offsets=[0, 900, 901, 1500]).check()

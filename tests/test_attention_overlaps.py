"""Outputs that share elements with inputs or with one another are refused wherever they start; those that lie between
the rows of another tensor are not."""

import ctypes
import itertools
import random

import pytest

torch = pytest.importorskip("torch")

A = 1 << 20   # an aligned address that is never touched


@pytest.fixture(scope="module")
def gs():
    import os

    import paper_2108_06004_gb300 as lib
    if not os.path.exists(lib.LIB_PATH):
        from paper_2108_06004_gb300 import _build
        _build.build()
    lib.load_library()
    return lib


def elements(start, strides, sizes, D):
    return {start + sum(i * s for i, s in zip(at, strides)) + d for at in itertools.product(*map(range, sizes)) for d in range(D)}


def forward(gs, tensors, B, T, H, K, Dk, Dv, dtype=0, item=4, packed=False):
    """Whether the call is refused for its tensors: it has no workspace, which is found last."""
    h = [ctypes.byref(gs.GsHeads(A + item * start, *strides)) for start, strides in tensors]
    lib = gs.load_library()
    assert lib.gs_linear_attention_forward(*h[:3], A, None, None, A if packed else None, h[3], None, B, T, H, K, Dk, Dv, dtype, 1.0, None, 0,
                                           None) == gs.GS_ERR_INVALID_ARG
    said = lib.gs_last_error()
    assert b"workspace" in said or b"o may not be an input, nor overlap one" in said, said
    return b"workspace" not in said


def test_slices_of_one_buffer(gs):
    B, T, H, D = 2, 5, 4, 8
    row = 4 * H * D
    strides = (T * row, row, D)
    part = [(i * H * D, strides) for i in range(4)]
    assert not forward(gs, part, B, T, H, H, D, D)
    taken = set().union(*(elements(start, strides, (B, T, H), D) for start, _ in part[:3]))
    for at in (H * D - 1, 2 * H * D + 1, 3 * H * D - 1, 3 * H * D, 3 * H * D + 1, row + 5, (T - 1) * row + H * D, 2 * T * row - 1):
        expected = bool(taken & elements(at, strides, (B, T, H), D))
        assert forward(gs, part[:3] + [(at, strides)], B, T, H, H, D, D) == expected, at
    assert not forward(gs, part[:3] + [(B * T * row - H * D, strides)], B, T, H, H, D, D)   # past all of them
    # half a tensor behind its own start
    dense = (T * H * D, H * D, D)
    other = [((i + 2) << 16, dense) for i in range(3)]
    for k, at in itertools.product(range(3), (1, D, H * D, T * H * D, B * T * H * D - 1, -1, 1 - B * T * H * D)):
        assert forward(gs, other + [(other[k][0] + at, dense)], B, T, H, H, D, D)
    for k in range(3):
        assert not forward(gs, other + [(other[k][0] + B * T * H * D, dense)], B, T, H, H, D, D)
        assert not forward(gs, other + [(other[k][0] - B * T * H * D, dense)], B, T, H, H, D, D)


def test_any_layouts(gs):
    """Against the sets of elements, in layouts of any order, with space between rows and broadcast inputs."""
    rng, seen = random.Random(5), [0, 0]
    for _ in range(3000):
        B, T, K, share, Dk, Dv = (rng.randint(1, 4) for _ in range(6))
        H, tensors, sets = K * share, [], []
        for n, (heads, D) in enumerate(((H, Dk), (K, Dk), (K, Dv), (H, Dv))):
            sizes, strides, span = (B, T, heads), [0, 0, 0], D
            for k in rng.sample(range(3), 3):
                span += rng.choice((0, 0, 1, 3, 8))
                strides[k] = span
                span *= sizes[k]
            if n < 3 and rng.random() < 0.2:
                strides[rng.randrange(3)] = 0
            start = rng.randrange(0, 300) if n < 3 else rng.randrange(0, 600)
            tensors.append((start, tuple(strides)))
            sets.append(elements(start, strides, sizes, D))
        expected = any(sets[3] & s for s in sets[:3])
        seen[expected] += 1
        assert forward(gs, tensors, B, T, H, K, Dk, Dv) == expected, (tensors, B, T, H, K, Dk, Dv)
    assert min(seen) > 300, seen


def test_large_strides(gs):
    """Distances past 64 bits do not wrap."""
    far = (1 << 45, 1 << 45, 1 << 45)
    o = (0, (1 << 20, 1 << 10, 8))
    assert forward(gs, [(0, far)] * 3 + [o], 1 << 10, 1 << 9, 1 << 6, 1 << 6, 8, 8)
    assert not forward(gs, [(1 << 40, far)] * 3 + [o], 1 << 10, 1 << 9, 1 << 6, 1 << 6, 8, 8)


def test_other_calls(gs):
    lib, bad = gs.load_library(), gs.GS_ERR_INVALID_ARG
    B, T, H, D = 2, 4, 2, 8
    size = B * T * H * D * 4

    def h(at):
        return ctypes.byref(gs.GsHeads(A + at, T * H * D, H * D, D))

    def token(at):
        return ctypes.byref(gs.GsHeads(A + at, H * D, 0, D))

    for at in (4, 32, size - 4, -4, 4 - size):
        assert lib.gs_rotary(h(0), h(at), A, None, 0, B, T, H, D, D, gs.GS_F32, 0, 0, 1.0, None) == bad and b"overlap" in lib.gs_last_error()
        for n in range(3):
            out = [h((8 + i) * size) for i in range(3)]
            for other in list(range(4)) + [8 + i for i in range(3) if i != n]:
                out[n] = h(other * size + at)
                # an offset may reach the tensor before, too: any refusal for an overlap will do
                assert lib.gs_linear_attention_backward(*(h(i * size) for i in range(4)), A, None, None, None, None, *out, None, B, T, H, H, D, D,
                                                        gs.GS_F32, 1.0, None, 0, None) == bad
                assert b"overlap" in lib.gs_last_error()
    one = B * H * D * 4
    for at, n in itertools.product((4, 32, one - 4, -4, 4 - one), range(3)):
        assert lib.gs_linear_attention_step(*(token(i * one) for i in range(3)), A, A, H * D * D, B, None, token(n * one + at), B, H, H, D, D, gs.GS_F32,
                                            1.0, None) == bad
        assert b"overlap" in lib.gs_last_error()
    out = [h((8 + i) * size) for i in range(3)]
    state = B * H * D * D * 4
    assert lib.gs_linear_attention_backward(*(h(i * size) for i in range(4)), A, None, None, None, None, *out, None, B, T, H, H, D, D, gs.GS_F32, 1.0,
                                            None, 0, None) == bad and b"workspace" in lib.gs_last_error()
    S = A + (1 << 24)
    for to, said in ((S, b"workspace"), (S + 4, b"overlap"), (S - state + 4, b"overlap"), (S + state, b"workspace"), (S - state, b"workspace")):
        assert lib.gs_linear_attention_forward(h(0), h(size), h(2 * size), A, S, None, None, h(3 * size), to, B, T, H, H, D, D, gs.GS_F32, 1.0, None, 0,
                                               None) == bad and said in lib.gs_last_error()
        said = b"overlap" if to == S else said
        for s0, ds in ((S, None), (None, S)):
            assert lib.gs_linear_attention_backward(*(h(i * size) for i in range(4)), A, s0, ds, None, None, *out, to, B, T, H, H, D, D, gs.GS_F32, 1.0,
                                                    None, 0, None) == bad and said in lib.gs_last_error()

    rows, cols = 4, 8
    n = rows * cols * 4
    x, gate, res, y, z = (A + i * n for i in range(5))

    def norm(y, z, ys=8):
        return lib.gs_gated_norm(x, 8, gate, 8, res, 8, A, A, y, ys, z, 8, A, A, rows, cols, 1, gs.GS_F32, gs.GS_GATE_SILU, 1.0, 1e-6, None)

    def back(dx, dgate, dres):
        return lib.gs_gated_norm_backward(x, 8, None, 0, gate, 8, res, 8, None, 0, A, None, A, None, dx, 8, dgate, 8, dres, 8, A, None, rows, cols, 1,
                                          gs.GS_F32, gs.GS_GATE_SILU, 1.0, None, 0, None)

    for off in (4, 32, n - 4):
        for t in (x, gate, res, y):
            assert norm(y, t + off) == bad and b"overlap" in lib.gs_last_error()
        for t in (x, gate, res):
            assert norm(t + off, A + 9 * n) == bad and b"overlap" in lib.gs_last_error()
            for k in range(3):
                to = [A + (6 + 2 * i) * n for i in range(3)]
                to[k] = t + off
                assert back(*to) == bad and b"overlap" in lib.gs_last_error()
        assert back(A + 6 * n, A + 6 * n + off, None) == bad and b"overlap" in lib.gs_last_error()
    assert back(A + 6 * n, A + 7 * n, A + 8 * n) == bad and b"workspace" in lib.gs_last_error()


@pytest.mark.gpu
def test_rows_between_rows(gs):
    """Every tensor of a call in one buffer, side by side, gives what tensors of their own give."""
    B, T, H, D = 2, 150, 3, 64
    torch.manual_seed(0)
    for dtype in (torch.bfloat16, torch.float32):
        whole = torch.randn(B, T, 8 * H, D, device="cuda").to(dtype)
        part = [whole[:, :, i * H:(i + 1) * H] for i in range(8)]
        own = [p.clone() for p in part]
        g = torch.tensor([-0.3, -0.02, -0.001], device="cuda")
        ws = torch.empty(gs.gs_linear_attention_workspace_size(B, T, H, H, D, D, dtype, backward=True), dtype=torch.uint8, device="cuda")
        for t in (part, own):
            gs.gs_linear_attention_forward(*t[:3], g, t[4], ws)
            gs.gs_linear_attention_backward(t[3], *t[:3], g, *t[5:], ws)
        assert all(torch.equal(a, b) for a, b in zip(part, own))
        side = torch.randn(200, 5 * 96, device="cuda").to(dtype)
        part = [side[:, i * 96:(i + 1) * 96] for i in range(5)]
        own = [p.clone() for p in part]
        w, rstd, r2 = torch.ones(96, device="cuda"), torch.empty(200, 1, device="cuda"), torch.empty(200, device="cuda")
        for t in (part, own):
            gs.gs_gated_norm(t[0], w, t[3], rstd, gate=t[1], residual=t[2], next_weight=w, z=t[4], next_rstd=r2)
        assert all(torch.equal(a, b) for a, b in zip(part, own))

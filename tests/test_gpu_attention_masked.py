"""What lies behind a sequence's end, or in the next packed one, may hold anything: no output of a sequence depends on
it, whichever products its last block, cut short after whole ones, goes through."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_attention import DT, gs, place  # noqa: E402, F401

pytestmark = pytest.mark.gpu

SIZES = [(64, 64), (128, 128), (64, 128), (128, 64), (40, 72), (104, 24)]


def run(gs, x, g, state, **mask):
    """Outputs of both passes; state: with the last state and the first one's gradient."""
    q, k, v, do = x
    T, H, Dk, (K, Dv) = q.shape[1], q.shape[2], q.shape[3], v.shape[2:]
    B = q.shape[0] if "offsets" not in mask else mask["offsets"].numel() - 1
    o, dq, dk, dv = torch.full_like(do, 5.0), torch.full_like(q, 5.0), torch.full_like(k, 5.0), torch.full_like(v, 5.0)
    s = [torch.empty(B, H, Dk, Dv, device="cuda") if state else None for _ in range(2)]
    for back in (False, True):
        ws = torch.empty(gs.gs_linear_attention_workspace_size(B, T, H, K, Dk, Dv, q.dtype, backward=back, packed="offsets" in mask),
                         dtype=torch.uint8, device="cuda").fill_(255)
        if back:
            gs.gs_linear_attention_backward(do, q, k, v, g, dq, dk, dv, ws, ds0=s[1], **mask)
        else:
            gs.gs_linear_attention_forward(q, k, v, g, o, ws, s_last=s[0], **mask)
    return [o, dq, dk, dv] + (s if state else [])


def inputs(rows, T, H, K, Dk, Dv, dtype):
    rng = np.random.default_rng(Dk + Dv + T)
    return [place((rows, T, h, d), dtype, "dense", rng=rng) for h, d in ((H, Dk), (K, Dk), (K, Dv), (H, Dv))]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("Dk,Dv", SIZES)
@pytest.mark.parametrize("K", [1, 2])
@pytest.mark.parametrize("state", [False, True])
def test_behind_the_end(gs, state, K, Dk, Dv, dtype):
    lengths = [300, 130, 257, 128, 1, 0, 383, 129]
    x, g = inputs(len(lengths), 400, 2, K, Dk, Dv, dtype), torch.tensor([-0.2, -0.004], device="cuda")
    mask = {"lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda")}
    for t in x:
        for b, n in enumerate(lengths):
            t[b, n:] = 0
    want = run(gs, x, g, state, **mask)
    for what in (float("nan"), float("inf")):
        for t in x:
            for b, n in enumerate(lengths):
                t[b, n:] = what
        for _ in range(5):
            assert all(torch.equal(a, b) for a, b in zip(run(gs, x, g, state, **mask), want))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("Dk,Dv", SIZES)
@pytest.mark.parametrize("K", [1, 2])
@pytest.mark.parametrize("state", [False, True])
def test_next_document(gs, state, K, Dk, Dv, dtype):
    cuts = [0, 130, 261, 262, 647, 900, 1157, 1158, 1500]
    x, g = inputs(1, cuts[-1], 2, K, Dk, Dv, dtype), torch.tensor([-0.2, -0.004], device="cuda")
    mask = {"offsets": torch.tensor(cuts, dtype=torch.int32, device="cuda")}
    want = run(gs, x, g, state, **mask)
    for bad in (range(1, 8, 2), range(0, 8, 2)):
        y = [t.clone() for t in x]
        for t in y:
            for n in bad:
                t[:, cuts[n]:cuts[n + 1]] = float("nan")
        for _ in range(5):
            got = run(gs, y, g, state, **mask)
            for n in set(range(8)) - set(bad):
                for a, b in zip(got[:4], want[:4]):
                    assert torch.equal(a[:, cuts[n]:cuts[n + 1]], b[:, cuts[n]:cuts[n + 1]])
                for a, b in zip(got[4:], want[4:]):
                    assert torch.equal(a[n], b[n])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("Dk,Dv", [(128, 128), (64, 128), (128, 64)])
def test_keys_that_come_late(gs, Dk, Dv, dtype):
    """More heads than fit the device at once, whose blocks' keys, read from memory, come at any time: the same bits each time."""
    x, g = inputs(8, 700, 40, 40, Dk, Dv, dtype), torch.full((40,), -0.01, device="cuda")
    mask = {"lengths": torch.tensor([700, 640, 513, 257, 699, 5, 385, 600], dtype=torch.int32, device="cuda")}
    beside = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    want = run(gs, x, g, False, **mask)
    for _ in range(10):
        beside.fill_(1)
        assert all(torch.equal(a, b) for a, b in zip(run(gs, x, g, False, **mask), want))

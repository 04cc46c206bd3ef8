"""Waits of the tensor core walks that run out, in threads that do not store anything themselves: what has to do with them is NaN,
in memory that the call may not touch nothing changes, and the next call is as if nothing had been."""

import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_attention import DT, gs, place  # noqa: E402, F401

import numpy as np  # noqa: E402

NAN = float("nan")


@pytest.fixture(autouse=True)
def whole_waits():
    yield
    import paper_2108_06004_gb300 as lib
    lib.gs_linear_attention_wait_tries()


def test_refusals():
    import os

    import paper_2108_06004_gb300 as lib
    if not os.path.exists(lib.LIB_PATH):
        from paper_2108_06004_gb300 import _build
        _build.build()
    for k in range(3):
        for bad in (-1, (1 << 20) + 1):
            with pytest.raises(lib.GsError, match="tries must lie"):
                lib.gs_linear_attention_wait_tries(*(bad if i == k else 1 for i in range(3)))
    lib.gs_linear_attention_wait_tries(0, 0, 0)


def run(gs, x, g, s0, lengths, state):
    q, k, v, do = x
    (B, T, H, Dk), (K, Dv) = q.shape, v.shape[2:]
    out = {"o": torch.full_like(do, 5.0), "dq": torch.full_like(q, 5.0), "dk": torch.full_like(k, 5.0), "dv": torch.full_like(v, 5.0)}
    if state:
        out.update(last=torch.full_like(s0, 5.0), ds0=torch.full_like(s0, 5.0))
    sizes = (B, T, H, K, Dk, Dv, q.dtype)
    ws = torch.empty(max(gs.gs_linear_attention_workspace_size(*sizes, backward=b) for b in (False, True)), dtype=torch.uint8, device="cuda")
    gs.gs_linear_attention_forward(q, k, v, g, out["o"], ws, s0=s0, s_last=out.get("last"), lengths=lengths)
    gs.gs_linear_attention_backward(do, q, k, v, g, out["dq"], out["dk"], out["dv"], ws, s0=s0, ds_last=s0, ds0=out.get("ds0"), lengths=lengths)
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,who", [("bf16", "issue"), ("f16", "issue"), ("f16", "find")])   # only fp16 has its largest values found
@pytest.mark.parametrize("B,T,Dk,Dv", [(4, 300, 64, 64), (4, 300, 128, 128), (4, 300, 64, 128), (1, 2600, 128, 64), (1, 2600, 64, 64)])
@pytest.mark.parametrize("state", [False, True])
def test_waits_that_run_out(gs, state, B, T, Dk, Dv, dtype, who):
    rng = np.random.default_rng(1)
    x = [place((B, T, 2, d), dtype, "dense", rng=rng) for d in (Dk, Dk, Dv, Dv)]
    g, s0 = torch.tensor([-0.2, -0.01], device="cuda"), torch.from_numpy(rng.standard_normal((B, 2, Dk, Dv))).to("cuda", torch.float32)
    lengths = torch.tensor([T, 200, 0, 128][:B], dtype=torch.int32, device="cuda")
    want = run(gs, x, g, s0, lengths, state)
    # the others wait for a millisecond at most
    gs.gs_linear_attention_wait_tries(**({"issue": 0, "find": 1000, "work": 1000} if who == "issue" else {"find": 0, "issue": 1000, "work": 1000}))
    got = run(gs, x, g, s0, lengths, state)
    gs.gs_linear_attention_wait_tries()
    counts = (torch.arange(T, device="cuda")[None] < lengths[:, None])
    for name in ("o", "dq", "dk", "dv"):
        assert got[name][counts].isnan().all() and not got[name][~counts].any(), name
    for name in ("last", "ds0") if state else ():
        assert got[name][lengths > 0].isnan().all(), name
        assert torch.equal(got[name][lengths == 0], s0[lengths == 0]), name
    again = run(gs, x, g, s0, lengths, state)
    assert all(torch.equal(again[n], want[n]) for n in want)

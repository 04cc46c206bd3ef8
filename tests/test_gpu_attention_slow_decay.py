"""States that decay slowly, which thousands of tokens make up, keep fp32's digits."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_attention import DT, gs, host  # noqa: E402, F401

pytestmark = pytest.mark.gpu

G = -0.0009


@pytest.mark.parametrize("dtype,Dk,Dv", [("f32", 16, 32), ("f32", 64, 64), ("f32", 128, 40), ("f32", 160, 32), ("bf16", 160, 32), ("f16", 136, 33),
                                         ("bf16", 64, 64), ("f16", 128, 128)])
def test_last_state(gs, dtype, Dk, Dv):
    """A sum that is rounded to nearest is off by at most 2^-24 of its size and, the roundings of random terms being
    independent, by 2^-24 / sqrt(3) of it in the mean square. A state that takes one rounding a block of 16 tokens remembers
    1 / (1 - e^(32 g)) = 35 of them, in the mean square: sqrt(35) 2^-24 / sqrt(3) = 2.0e-7 of it, and half as much again is allowed for the
    blocks' own sums and decays. (One rounding a token makes it four times as much, 8.1e-7.)"""
    rng = np.random.default_rng(Dk + Dv)
    T = 4096
    # so many heads that rows are not cut into pieces, whose states are summed apart; all read one key, at a stride of zero,
    # which no tile describes
    many = 512
    k, v = (torch.from_numpy(rng.standard_normal((1, T, 1, d))).to("cuda", DT[dtype]).expand(1, T, many, d) for d in (Dk, Dv))
    g = torch.full((many,), G, device="cuda")
    o, last = torch.empty(1, T, many, Dv, dtype=DT[dtype], device="cuda"), torch.empty(1, many, Dk, Dv, device="cuda")
    ws = torch.empty(gs.gs_linear_attention_workspace_size(1, T, many, many, Dk, Dv, DT[dtype]), dtype=torch.uint8, device="cuda")
    gs.gs_linear_attention_forward(k, k, v, g, o, ws, s_last=last)
    w = np.exp(np.float64(np.float32(G)) * (T - 1 - np.arange(T)))
    want = (host(k)[0, :, 0] * w[:, None]).T @ host(v)[0, :, 0]
    for h in (0, many // 2, many - 1):
        off = np.linalg.norm(host(last)[0, h] - want) / np.linalg.norm(want)
        assert off < 3e-7, off


@pytest.mark.parametrize("dtype,Dk,Dv", [("bf16", 64, 64), ("bf16", 128, 128), ("f16", 64, 128), ("f16", 128, 64)])
def test_last_state_in_tiles(gs, dtype, Dk, Dv):
    """The same on the tensor cores, whose blocks of 128 tokens take an eighth as many roundings; keys are parts of 2^-23 or better."""
    rng, T, many = np.random.default_rng(Dk + Dv), 4096, 512
    k, v = (torch.from_numpy(rng.standard_normal((1, T, 1, d))).to("cuda", DT[dtype]) for d in (Dk, Dv))
    q, g = torch.zeros(1, T, many, Dk, dtype=DT[dtype], device="cuda"), torch.full((many,), G, device="cuda")
    o, last = torch.empty(1, T, many, Dv, dtype=DT[dtype], device="cuda"), torch.empty(1, many, Dk, Dv, device="cuda")
    ws = torch.empty(gs.gs_linear_attention_workspace_size(1, T, many, 1, Dk, Dv, DT[dtype]), dtype=torch.uint8, device="cuda")
    gs.gs_linear_attention_forward(q, k, v, g, o, ws, s_last=last)
    w = np.exp(np.float64(np.float32(G)) * (T - 1 - np.arange(T)))
    want = (host(k)[0, :, 0] * w[:, None]).T @ host(v)[0, :, 0]
    assert not o.any()
    for h in (0, many // 2, many - 1):
        off = np.linalg.norm(host(last)[0, h] - want) / np.linalg.norm(want)
        assert off < 3e-7, off

"""Sines and cosines of fp32 rotary positions, read from pairs (1, 0) that are turned."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention  # noqa: E402
from tests.test_gpu_attention import gs, host  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_angles(gs, inverse, interleaved):
    """An angle is within an eighth of a turn of its quarter: as an fp32 number it is off by 2^-25 of an eighth's binade (an
    eighth is 2^29 of 2^32 parts, of which 2^29 2^-25 = 2^4 are 2^-28 turns), and by one of the 2^32 parts that cut it off. The sine
    and cosine of at most 1 are right to a unit in the last place, 2^-24 of [1/2, 1). The frequency's 53 bits give 2^-53 of
    the turns, twice (its own and that of 1 / 2 pi)."""
    rng, T, R = np.random.default_rng(0), 4000, 64
    freq = np.concatenate((rng.uniform(0, 3, 24), 10.0 ** -rng.uniform(0, 6, 8)))
    x = torch.zeros(1, T, 1, R, device="cuda")
    x[..., 0::2 if interleaved else 1][..., :R // 2] = 1
    if not interleaved:
        x[..., R // 2:] = 0
    at = rng.integers(-2 ** 20, 2 ** 20, (1, T))
    out = torch.empty_like(x)
    gs.gs_rotary(x, out, torch.from_numpy(freq).cuda(), positions=torch.from_numpy(at.astype(np.int32)).cuda(), interleaved=interleaved,
                 inverse=inverse)
    want = attention.rotary(host(x), freq, at, interleaved, inverse, 1.0)
    off = np.abs(host(out) - want)
    tol = 2 * np.pi * (2.0 ** -28 + 2.0 ** -32) + 2.0 ** -24 + 2 * 2.0 ** -53 * 2 ** 20 * 3
    assert off.max() <= tol, (off.max(), tol)


def test_quarters(gs):
    """At whole quarters of a turn sines and cosines are 0 and 1 in magnitude, to the 2^-32 turns that cut the angle off."""
    x = torch.tensor([1.0, 0.0], device="cuda").view(1, 1, 1, 2).expand(1, 8, 1, 2).contiguous()
    out = torch.empty_like(x)
    gs.gs_rotary(x, out, torch.tensor([np.pi / 2], dtype=torch.float64, device="cuda"), first=-3, interleaved=True)
    want = torch.tensor([[0.0, 1], [-1, 0], [0, -1], [1, 0]] * 2, device="cuda")
    assert float((out[0, :, 0] - want).abs().max()) <= 2 * np.pi * 2.0 ** -32

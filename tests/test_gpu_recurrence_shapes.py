"""The sequence kernels' ways through a call, against the fp64 oracle: thread blocks of 64 channels and of 32,
time dealt to one block or to a cluster, enough steps that every buffer is used again, and channels whose
decay rates take each of the forms of the gates' arithmetic."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_recurrence_range import check, gs  # noqa: E402,F401

pytestmark = pytest.mark.gpu

# B * ceil(D / 64) of 456 and more takes 64 channels a block; few columns over a long time take clusters
MANY = [(60, 200, 512), (40, 150, 769)]
LONG = [(1, 9000, 40), (1, 9000, 33)]
FEW = [(12, 700, 256)]   # 32 channels, no cluster, several steps


def run(gs, dtype, B, T, D, masks, mixed):  # noqa: F811
    rng = np.random.default_rng(B + T + D + masks)
    if mixed:   # groups of 16 channels: slow, medium and very fast decays, alone and side by side in a warp
        kind = (np.arange(D) // 16 + np.arange(D) // 48) % 3
        decay = np.choose(kind, [rng.uniform(-9, -4, D), rng.uniform(-3, 2, D), np.full(D, 1e13)])
    else:
        kind, decay = np.zeros(D, dtype=int), rng.uniform(-9, -4.5, D)
    r = rng.standard_normal((B, T, D))
    r[..., kind == 2] = -32 + 3 * r[..., kind == 2]   # 8e13 times the gate of -32 is about 1
    reset = lengths = None
    if masks:
        reset = (rng.random((B, T)) < 0.01).astype(np.uint8)
        lengths = rng.integers(T // 2, T + 1, B).astype(np.int32)
        lengths[0] = T
        if B > 2:
            lengths[1], lengths[2] = 0, 1
    check(gs, dtype, 8.0, decay, rng.standard_normal((B, T, D)), r, 2 * rng.standard_normal((B, T, D)),
          rng.standard_normal((B, T, D)), rng.standard_normal((B, D)), rng.standard_normal((B, D)), reset, lengths)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,T,D", MANY + LONG)
@pytest.mark.parametrize("masks", [False, True])
def test_shapes(gs, dtype, B, T, D, masks):  # noqa: F811
    run(gs, dtype, B, T, D, masks, mixed=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,D", FEW + MANY[:1] + LONG)
@pytest.mark.parametrize("masks", [False, True])
def test_rates_of_every_kind(gs, dtype, B, T, D, masks):  # noqa: F811
    run(gs, dtype, B, T, D, masks, mixed=True)

"""Rotary positions on the GPU against the fp64 oracle."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention  # noqa: E402
from tests import attention_bounds as bounds  # noqa: E402
from tests import layer_bounds  # noqa: E402
from tests.test_gpu_attention import DT, close, gs, host, place  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def check(gs, shape, R, dtype, how="dense", interleaved=False, inverse=False, inplace=False, positions=None, first=0, magnitude=1.0,
          factor=1.0, base=10000.0):
    B, T, H, D = shape
    x = place(shape, dtype, how, rng=np.random.default_rng(T + D))
    xv = host(x)
    freq = gs.gs_rotary_frequencies(R, base=base, factor=factor, original=4096.0 if factor > 1 else 0.0)
    assert np.allclose(freq.numpy(), attention.frequencies(R, base, factor, 4096.0 if factor > 1 else 0.0), rtol=1e-14, atol=0)
    out = x if inplace else place(shape, dtype, "dense", fill=float("nan"))
    at = None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda").expand(B, T).contiguous()
    gs.gs_rotary(x, out, freq.cuda(), positions=at, first=first, interleaved=interleaved, inverse=inverse, magnitude=magnitude)
    where = np.broadcast_to(first + np.arange(T), (B, T)) if at is None else at.cpu().numpy().astype(np.int64)
    want = attention.rotary(xv, freq.numpy(), where, interleaved, inverse, magnitude)
    err = bounds.rotary(xv, freq.numpy(), where, interleaved, magnitude)
    close(out[..., :R], want[..., :R], layer_bounds.stored(want, err, dtype)[..., :R], "turned")
    assert np.array_equal(host(out)[..., R:], xv[..., R:])
    if not inplace:
        assert np.array_equal(host(x), xv)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R", [(2, 2), (16, 16), (64, 64), (128, 128), (128, 64), (96, 48), (47, 46), (47, 20), (256, 256), (512, 512), (7, 0),
                                 (72, 64), (68, 64)])
def test_heads(gs, D, R, interleaved, dtype):
    for inplace in (False, True):
        check(gs, (2, 5, 3, D), R, dtype, interleaved=interleaved, inplace=inplace, inverse=inplace)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["heads first", "wide", "odd"])
@pytest.mark.parametrize("T,H", [(1, 1), (1, 40), (9, 8), (333, 1), (1500, 5)])
def test_strides_and_sizes(gs, T, H, how, dtype):
    check(gs, (2, T, H, 64), 64, dtype, how=how, inplace=True)
    check(gs, (2, T, H, 64), 32, dtype, how=how, interleaved=True)


@pytest.mark.parametrize("first", [0, 1, 131071, 10_000_019, 2 ** 31 - 40, -7, -2 ** 31])
def test_far_positions(gs, first):
    check(gs, (1, 33, 2, 64), 64, "f32", first=first)


def test_positions_and_scaling(gs):
    check(gs, (3, 4, 2, 64), 64, "f32", positions=[0, 2 ** 31 - 1, -2 ** 31, 77], magnitude=1.2)
    check(gs, (3, 4, 2, 128), 128, "f32", positions=[0, 5, 1000, 32767], factor=8.0, magnitude=0.1 * np.log(8.0) + 1)
    check(gs, (3, 4, 2, 64), 64, "bf16", positions=[[3], [1 << 20], [9]], factor=4.0, base=500000.0)


def test_inverse_undoes(gs):
    x = torch.randn(2, 100, 4, 64, device="cuda")
    y, z, f = torch.empty_like(x), torch.empty_like(x), gs.gs_rotary_frequencies(64).cuda()
    gs.gs_rotary(x, y, f, first=5000)
    gs.gs_rotary(y, z, f, first=5000, inverse=True)
    assert float((z - x).abs().max()) < 40 * 2.0 ** -24 * float(x.abs().max())
    # the gradient: <turn(x), d> = <x, turn back(d)>
    d = torch.randn_like(x)
    back = torch.empty_like(x)
    gs.gs_rotary(d, back, f, first=5000, inverse=True)
    a, b = (y.double() * d.double()).sum(), (x.double() * back.double()).sum()
    assert abs(float(a - b)) < 1e-5 * float(x.norm() * d.norm())


def test_frequencies_as_given(gs):
    """Any finite frequencies, negative and above a turn a token too."""
    f = torch.tensor([0.0, -0.5, 7.0, -123.25, 1e-9, 6.283185307179586, 3e8, 1.0], dtype=torch.float64)
    x = place((1, 50, 1, 16), "f32", "dense", rng=np.random.default_rng(1))
    out = torch.empty_like(x)
    gs.gs_rotary(x, out, f.cuda(), first=3)
    at = np.arange(3, 53)[None]
    want = attention.rotary(host(x), f.numpy(), at, False, False, 1.0)
    close(out, want, layer_bounds.stored(want, bounds.rotary(host(x), f.numpy(), at, False, 1.0), "f32"), "turned")

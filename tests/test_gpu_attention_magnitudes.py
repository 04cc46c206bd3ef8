"""Large inputs whose results are well inside the type's range, at every decay."""

import pytest

pytest.importorskip("torch")

from tests.test_gpu_attention import Case, gs  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 128), (64, 128), (128, 64), (47, 33)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e9, 1e-9])
def test_magnitudes(gs, size, dtype, Dk, Dv):
    """128 g from 1 to 40: outputs of about 1e29 and 1e-25."""
    Case(gs, 1, 300, 8, 8, Dk, Dv, dtype, size=size, state=False, g=[-0.008, -0.03, -0.0624, -0.0626, -0.1, -0.2, -0.24, -0.3]).check()

"""Rows are cut into pieces, whose sums a workspace holds, where fewer of them than three eighths of a full device are to be walked."""

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def gs():
    import os

    import paper_2108_06004_gb300 as lib
    if not os.path.exists(lib.LIB_PATH):
        from paper_2108_06004_gb300 import _build
        _build.build()
    lib.load_library()
    return lib


@pytest.mark.parametrize("D,dtype,cut,whole", [(128, torch.bfloat16, 3, 4), (64, torch.bfloat16, 7, 8), (32, torch.float32, 14, 15), (128, torch.float32, 1, 2)])
def test_cut(gs, D, dtype, cut, whole):
    size = lambda B: gs.gs_linear_attention_workspace_size(B, 2048, 16, 16, D, D, dtype)   # noqa: E731
    assert size(whole) == 256 and size(cut) >= 2 * cut * 16 * D * D * 4

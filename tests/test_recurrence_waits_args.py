"""The limits of the recurrence's waits are checked on the host."""

import pytest

pytest.importorskip("torch")


def test_wait_tries_refusals():
    import os

    import paper_2108_06004_gb300 as gs
    if not os.path.exists(gs.LIB_PATH):
        from paper_2108_06004_gb300 import _build
        _build.build()
    for bad in ((-1, 1), (1, -1), ((1 << 20) + 1, 1), (1, (1 << 20) + 1)):
        with pytest.raises(gs.GsError, match="tries must lie"):
            gs.gs_recurrence_wait_tries(*bad)
    gs.gs_recurrence_wait_tries(0, 0)
    gs.gs_recurrence_wait_tries()

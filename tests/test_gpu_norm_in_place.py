"""gs_dropout_add_norm with y in the place of x or of the residual, and gs_dropout with out in theirs: the same
bits as out of place, at widths and strides where groups straddle rows."""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def gs():
    import paper_2108_06004_gb300 as lib
    lib.load_library()
    torch.cuda.set_device(0)
    return lib


def place(values, pad, shift):
    """These values in a wider buffer, `shift` elements past an aligned address."""
    rows, cols = values.shape
    flat = torch.full((rows * (cols + pad) + shift,), 7.0, dtype=values.dtype, device="cuda")
    t = flat[shift:].view(rows, cols + pad)[:, :cols]
    t.copy_(values)
    return t, flat


CASES = [(64, 0, 0), (1001, 0, 0), (1001, 7, 0), (33, 3, 1), (4099, 0, 1), (4097, 5, 0), (12, 1, 3), (7, 0, 0), (9000, 0, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols,pad,shift", CASES)
@pytest.mark.parametrize("rows", [1, 2, 37])
@pytest.mark.parametrize("into", ["x", "residual"])
def test_in_place(gs, dtype, cols, pad, shift, rows, into):
    gen = torch.Generator(device="cuda").manual_seed(cols + rows)
    xv, rv = (torch.randn(rows, cols, dtype=DT[dtype], device="cuda", generator=gen) for _ in range(2))
    w = torch.randn(cols, device="cuda", generator=gen)

    def buffers():
        return place(xv, pad, shift), place(rv, pad, shift)

    def beside(flat):
        return flat[:shift], flat[shift:].view(rows, cols + pad)[:, cols:]

    (x, _), (res, _) = buffers()
    y, z, rstd = place(xv, pad, shift)[0], place(xv, pad, shift)[0], torch.empty(rows, device="cuda")
    gs.gs_dropout_add_norm(x, res, w, y, z, rstd, 0.3, 5, 6)
    (x2, xf), (res2, rf) = buffers()
    y2, flat = (x2, xf) if into == "x" else (res2, rf)
    z2, rstd2 = place(xv, pad, shift)[0], torch.empty(rows, device="cuda")
    gs.gs_dropout_add_norm(x2, res2, w, y2, z2, rstd2, 0.3, 5, 6)
    assert torch.equal(y2, y) and torch.equal(z2, z) and torch.equal(rstd2, rstd)
    assert torch.equal(res2 if into == "x" else x2, rv if into == "x" else xv)
    assert all((b == 7).all() for b in beside(flat))

    out = place(xv, pad, shift)[0]
    gs.gs_dropout(x, out, 0.3, 5, 6, residual=res)
    (x3, xf), (res3, rf) = buffers()
    out3, flat = (x3, xf) if into == "x" else (res3, rf)
    gs.gs_dropout(x3, out3, 0.3, 5, 6, residual=res3)
    assert torch.equal(out3, out)
    assert all((b == 7).all() for b in beside(flat))

"""Matrices of the floating-point head whose rows lie at odd addresses: the same bits as with aligned
rows, and nothing written beside the matrix."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu
SIZES = [(1, 1), (3, 31), (31, 17), (33, 32), (64, 785), (129, 250), (257, 513), (700, 96)]
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _in(t, pad, shift):
    """t at column `shift` of a buffer that is `pad` columns wider."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan") if t.is_floating_point() else 99, device="cuda").to(t.dtype)
    wide[:, shift: shift + t.shape[1]] = t
    return wide[:, shift: shift + t.shape[1]]


def _out(rows, cols, dtype, pad, shift):
    wide = torch.full((rows, cols + pad), -77.0, device="cuda", dtype=dtype)
    return wide, wide[:, shift: shift + cols]


def _beside_is_clean(wide, shift, cols):
    assert (wide[:, :shift] == -77).all() and (wide[:, shift + cols:] == -77).all()


def _places(cols):
    # aligned, then odd strides, odd offsets, and 4- and 8-byte alignment only
    return ((-cols) % 16, 0), ((-cols) % 16 + 1, 0), ((-cols) % 16 + 3, 1), ((-cols) % 16 + 2, 2), ((-cols) % 16 + 4, 4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, cols", SIZES + [(5000, 1003)])
def test_store(rows, cols, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=g, device="cuda").to(DT[dtype])
    nq, ns = nb.mx4_bytes(rows, cols)
    first = None
    for pad, shift in _places(cols):
        q, sc = (torch.full((n,), 0xEE, dtype=torch.uint8, device="cuda") for n in (nq, ns))
        nb.mx4_quantize(_in(x, pad, shift), q, sc)
        wide, y = _out(rows, cols, DT[dtype], pad, shift)
        scales = torch.full((rows, -(-cols // 32)), -1.0, device="cuda")
        nb.mx4_dequantize(q, sc, y, scales)
        _beside_is_clean(wide, shift, cols)
        got = q, sc, y.clone(), scales
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, cols", SIZES)
def test_linear(rows, cols, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    x = torch.randn(rows, 200, generator=g, device="cuda").to(DT[dtype])
    w = torch.randn(cols, 200, generator=g, device="cuda")
    nq, ns = nb.mx4_bytes(cols, 200)
    q, sc = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in (nq, ns))
    nb.mx4_quantize(w, q, sc)
    h = nb.Mx4Linear(rows, 200, cols)
    first = None
    for pad, shift in _places(cols):
        wide, y = _out(rows, cols, DT[dtype], pad, shift)
        h.run(_in(x, 16 + pad % 4, shift), q, sc, y)
        _beside_is_clean(wide, shift, cols)
        first = y.clone() if first is None else first
        assert torch.equal(y, first)
    h.close()


@pytest.mark.parametrize("rows, features", SIZES + [(2, 40), (12, 70)])
def test_xent(rows, features):
    classes = 333
    g = torch.Generator(device="cuda").manual_seed(rows + features)
    x = torch.randn(rows, features, generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn(classes, features, generator=g, device="cuda") / features ** 0.5).to(torch.bfloat16)
    labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    h = nb.SoftmaxXent(rows, features, classes)
    first = None
    for pad, shift in _places(features):
        xs, ws = _in(x, pad, shift), _in(w, pad, shift)
        loss, lse = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
        h.forward(xs, ws, labels, loss, lse)
        if first is not None:       # few rows are summed in another order at odd addresses
            assert (lse - first[0]).abs().max() <= 2.0 ** -18 * (1 + first[0].abs().max())
        lse = lse if first is None else first[0]
        wide_x, dx = _out(rows, features, torch.bfloat16, pad, shift)
        wide_w, dw = _out(classes, features, torch.bfloat16, pad, shift)
        h.backward(xs, ws, labels, lse, None, dx, dw)
        _beside_is_clean(wide_x, shift, features)
        _beside_is_clean(wide_w, shift, features)
        first = first or (lse, dx.clone(), dw.clone())
        assert torch.equal(dx, first[1]) and torch.equal(dw, first[2])
    assert h.status() == nb.NITRO_OK
    h.close()


@pytest.mark.parametrize("rows, cols", [(31, 17), (129, 250), (257, 513), (700, 150), (150, 6000)])
def test_orth(rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    m = torch.randn(rows, cols, generator=g, device="cuda").to(torch.bfloat16)
    h = nb.Orthogonalizer(1, rows, cols)
    first = None
    for pad, shift in _places(cols):
        wide, out = _out(rows, cols, torch.bfloat16, pad, shift)
        h.run(_in(m, pad, shift), out)
        _beside_is_clean(wide, shift, cols)
        first = out.clone() if first is None else first
        # (the norm's partial sums are taken in another order)
        assert (out.float() - first.float()).abs().max() <= 2.0 ** -8 * first.float().abs().max()
    h.close()

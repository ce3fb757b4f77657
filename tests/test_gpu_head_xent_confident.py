"""Gradients of rows whose label has nearly all of the softmax, against the formulas in 64 bits.

Logits are exact (small integers' sums times the scale), so what is off is the exponential: scale log2 e, the
log-sum and the exponent are rounded a few times each, together less than 2^-20 (1 + |z| + |lse|) of an entry
of the softmax, and so is the label's entry if it is the sum of the others.  (As the label's own
exponential less one it is off by 2^-24 |lse| of one, which is many times a small loss.)  Then u = 2^-8 (u^2 up to 32
rows) for G in bf16, u for the result, and the 32-bit sums of the products."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


def _data(rows, features, classes, offset, xt, seed):
    """x_i = c_i w_label (c = 5 to 12), w = -1 or 1: the label's logit leads by 10 to 24, times 2 / features a unit."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randint(0, 2, (classes, features), generator=g, device="cuda") * 2 - 1
    labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    c = torch.randint(5, 13, (rows, 1), generator=g, device="cuda")
    x = w[labels.long()] * c
    if offset:                              # the same large term in every logit
        x[:, 0], w[:, 0] = 64, 128
    return x.to(torch.int8 if xt == "i8" else torch.bfloat16), w.to(torch.bfloat16), labels, 2.0 / features


def _check(x, w, labels, scale, dx, dw, loss, gout=1.0, chunk=4096):
    rows, features = x.shape
    scale = float(torch.tensor(scale, dtype=torch.float32))
    ug = U * U if rows <= 32 else U
    wd = w.double()
    want_w, bound_w = torch.zeros(2, w.shape[0], features, device="cuda", dtype=torch.float64)
    for r in range(0, rows, chunk):
        s = slice(r, min(r + chunk, rows))
        xd, lab = x[s].double(), labels[s].long()
        live = lab >= 0
        at = lab.clamp(min=0)[:, None]
        z = scale * (xd @ wd.t())
        lse = torch.logsumexp(z, 1)
        e = 2.0 ** -20 * (1 + z.abs().amax(1) + lse.abs())
        G = torch.exp(z - lse[:, None])
        G.scatter_(1, at, 0.0)
        rest = G.sum(1)                     # 1 - the label's entry, without its cancellation
        G.scatter_(1, at, -rest[:, None])
        G[~live] = 0.0
        if loss is not None:
            eloss = torch.where(live, -torch.log1p(-rest), torch.zeros_like(rest))
            assert ((loss[s].double() - eloss).abs() <= 2.0 ** -19 * (1 + eloss)).all()
        G *= scale * gout
        tol = (ug + e)[:, None] * G.abs()
        if dx is not None:
            want, mag = G @ wd, G.abs() @ wd.abs()
            k = (-(-w.shape[0] // 16) + 8) * 2.0 ** -23 * mag
            assert ((dx[s].double() - want).abs() <= 1.02 * (U * want.abs() + tol @ wd.abs() + k) + 1e-38).all()
        want_w += G.t() @ xd
        bound_w += (tol + (-(-rows // 16) + 8) * 2.0 ** -23 * G.abs()).t() @ xd.abs()
    if dw is not None:
        assert ((dw.double() - want_w).abs() <= 1.02 * (U * want_w.abs() + bound_w) + 1e-38).all()


def _run(x, w, labels, scale, dx, dw, gout=None):
    rows = x.shape[0]
    h = nb.SoftmaxXent(rows, x.shape[1], w.shape[0])
    loss, lse = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
    h.forward(x, w, labels, loss, lse, scale=scale)
    h.backward(x, w, labels, lse, gout, dx, dw, scale=scale)
    assert h.status() == nb.NITRO_OK
    h.close()
    return loss


def _nan(*shape):
    return torch.full(shape, float("nan"), device="cuda", dtype=torch.bfloat16)


@pytest.mark.parametrize("xt", ["bf16", "i8"])
@pytest.mark.parametrize("offset", [False, True])
@pytest.mark.parametrize("rows, features, classes", [
    (1, 64, 100), (8, 64, 1000), (3, 2304, 50), (32, 64, 257), (40, 64, 100), (64, 4096, 1000), (129, 72, 2), (300, 64, 3000),
    (1000, 40, 700)])
def test_gradients(rows, features, classes, offset, xt):
    x, w, labels, scale = _data(rows, features, classes, offset, xt, rows + features)
    if rows > 8:
        labels[::6] = -1
    dx, dw = _nan(rows, features), _nan(classes, features)
    loss = _run(x, w, labels, scale, dx, dw)
    _check(x, w, labels, scale, dx, dw, loss)


@pytest.mark.parametrize("rows", [2, 50])
def test_a_lone_class_has_no_gradient(rows):
    x, w, labels, scale = _data(rows, 64, 1, True, "bf16", 3)
    dx, dw = _nan(rows, 64), _nan(1, 64)
    _run(x, w, labels, scale, dx, dw)
    assert (dx == 0).all() and (dw == 0).all()


# more than the 2^31 elements of G that a handle holds: the classes go in pieces
@pytest.mark.parametrize("features, xt, pad, want", [(24, "bf16", 0, "both"), (17, "i8", 3, "both"), (40, "bf16", 1, "dx"), (24, "i8", 0, "dw")])
def test_several_pieces_of_the_classes(features, xt, pad, want):
    rows, classes = 36000, 60001
    assert rows * classes > 1 << 31
    x, w, labels, scale = _data(rows, features, classes, False, xt, features)
    labels[::7] = -1
    # half of the rows are not confident at all
    labels[::2] = torch.where(labels[::2] >= 0, (labels[::2] + 11) % classes, labels[::2])
    wide = torch.zeros(classes, features + pad, device="cuda", dtype=torch.bfloat16)
    wide[:, :features] = w
    gx, gw = torch.full((rows, features + pad), 7.0, device="cuda", dtype=torch.bfloat16), torch.full_like(wide, 7.0)
    dx, dw = (gx[:, :features] if want != "dw" else None), (gw[:, :features] if want != "dx" else None)
    gout = torch.full((rows,), 0.125, device="cuda")
    loss = _run(x, wide[:, :features], labels, scale, dx, dw, gout)
    assert (gx[:, features:] == 7).all() and (gw[:, features:] == 7).all()
    _check(x, w, labels, scale, dx, dw, None, gout=0.125, chunk=3000)
    assert loss.isfinite().all()

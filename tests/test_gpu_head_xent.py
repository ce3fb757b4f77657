"""Softmax cross entropy of a linear head against its formulas in 64 bits, and its
gradients against differences of its own losses as well.

Tolerances.  A logit is a sum of exact products on the tensor cores, which add 16 at a
time and drop what 32 bits do not hold: each of ceil(F / 16) additions loses less than
2^-23 of the sum of magnitudes S, the factors and the exponential a few 2^-24 more.  bf16
rounds by at most u = 2^-8 of a value.  dx: G is rounded once (u of each |G_ij|, u^2 where
both halves are kept), the result once more; dw likewise, and x gout_i / ref, which is not
exact under unequal gout, by another u."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


def _inputs(rows, features, classes, xt, seed, pad=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, features + pad, generator=g, device="cuda")
    x = (x * 40).round().clamp(-127, 127).to(torch.int8) if xt == "i8" else x.to(torch.bfloat16)
    w = (torch.randn(classes, features + pad, generator=g, device="cuda") * spread / features ** 0.5).to(torch.bfloat16)
    labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    return x[:, :features], w[:, :features], labels, g


def _formula(x, w, labels, scale, gout):
    x, w, classes = x.double(), w.double(), w.shape[0]
    live = (labels >= 0) & (labels < classes)
    z = scale * (x @ w.t())
    lse = torch.logsumexp(z, 1)
    at = labels.clamp(0, classes - 1).long()
    loss = torch.where(live, lse - z.gather(1, at[:, None])[:, 0], torch.zeros_like(lse))
    G = torch.softmax(z, 1)
    G[torch.arange(len(at), device=x.device), at] -= 1.0
    G[~live] = 0.0
    gi = torch.where(live, gout.double() * scale, torch.zeros_like(lse))
    xl = torch.where(live[:, None], x, torch.zeros_like(x))
    return loss, lse, G, gi, xl


def _check(x, w, labels, scale, gout, loss, lse, dx, dw):
    rows, features = x.shape
    eloss, else_, G, gi, xl = _formula(x, w, labels, scale, torch.ones(rows, device="cuda") if gout is None else gout)
    S = scale * (x.double().abs() @ w.double().abs().t()).amax(1)
    ez = (-(-features // 16) + 8) * 2.0 ** -23 * S
    tol = 2 * ez + 2.0 ** -20 * (1 + else_.abs())
    assert ((loss.double() - eloss).abs() <= tol).all()
    assert ((lse.double() - else_).abs() <= tol).all()
    eg = (2 * tol).expm1()[:, None] * (G.abs() + 1e-30)          # what an error of z and lse does to the softmax
    ug = U * U if rows <= 32 else U
    if dx is not None:
        want = (G @ w.double()) * gi[:, None]
        bound = ((ug * G.abs() + eg) @ w.double().abs()) * gi.abs()[:, None]
        k = (-(-w.shape[0] // 16) + 8) * 2.0 ** -23 * (G.abs() @ w.double().abs()) * gi.abs()[:, None]
        assert ((dx.double() - want).abs() <= 1.02 * (U * want.abs() + bound + k) + 1e-30).all()
    if dw is not None:
        Gg = G * gi[:, None]
        want = Gg.t() @ xl
        ux = 0.0 if gout is None or (gout == gout[0]).all() else U
        bound = ((ug + ux) * Gg.abs() + eg * gi.abs()[:, None]).t() @ xl.abs()
        k = (-(-rows // 16) + 8) * 2.0 ** -23 * (Gg.abs().t() @ xl.abs())
        assert ((dw.double() - want).abs() <= 1.02 * (U * want.abs() + bound + k) + 1e-30).all()


def _run(x, w, labels, scale=1.0, gout=None, want_dx=True, want_dw=True, max_rows=None, stream=None):
    rows, features = x.shape
    h = nb.SoftmaxXent(max_rows or rows, features, w.shape[0])
    loss, lse = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
    dx = torch.full((rows, features), float("nan"), device="cuda", dtype=torch.bfloat16) if want_dx else None
    dw = torch.full((w.shape[0], features), float("nan"), device="cuda", dtype=torch.bfloat16) if want_dw else None
    h.forward(x, w, labels, loss, lse, scale=scale, stream=stream)
    h.backward(x, w, labels, lse, gout, dx, dw, scale=scale, stream=stream)
    st = h.status()
    h.close()
    return st, loss, lse, dx, dw


@pytest.mark.parametrize("xt", ["bf16", "i8"])
@pytest.mark.parametrize("rows, features, classes, pad", [
    (1, 1, 1, 0), (1, 64, 257, 0), (2, 7, 31, 0), (3, 8, 1000, 3), (32, 130, 64, 8), (33, 65, 2, 0), (64, 1024, 100, 0),
    (128, 72, 300, 1), (129, 64, 129, 0), (257, 40, 1300, 0), (300, 2056, 513, 8), (1000, 24, 33, 0), (40, 4096, 48, 0)])
def test_against_the_formulas(rows, features, classes, pad, xt):
    x, w, labels, g = _inputs(rows, features, classes, xt, rows + features, pad, spread=3.0)
    labels[torch.rand(rows, generator=g, device="cuda") < 0.2] = -1
    scale = 1 / 32 if xt == "i8" else 1.0
    gout = torch.full((rows,), 1 / 7, device="cuda")
    st, *out = _run(x, w, labels, scale, gout)
    assert st == nb.NITRO_OK
    _check(x, w, labels, scale, gout, *out)


@pytest.mark.parametrize("gout", ["none", "uneven", "some_zero", "first_zero"])
def test_row_gradients(gout):
    x, w, labels, g = _inputs(70, 96, 200, "bf16", 5)
    go = None if gout == "none" else torch.rand(70, generator=g, device="cuda") * 3 - 1
    if gout == "some_zero":
        go[::3] = 0.0
    if gout == "first_zero":
        go[:9] = 0.0
        go[20] = 0.0
    st, *out = _run(x, w, labels, 1.0, go)
    assert st == nb.NITRO_OK
    _check(x, w, labels, 1.0, go, *out)


def test_wide_logits():
    # logits of some hundreds: the row's maximum matters, most of the softmax underflows
    x, w, labels, _ = _inputs(50, 256, 700, "bf16", 8, spread=60.0)
    st, *out = _run(x, w, labels)
    assert st == nb.NITRO_OK
    _check(x, w, labels, 1.0, None, *out)


def test_several_pieces_of_the_classes():
    # G of 70000 x 2500 does not fit its workspace at once: dx adds over two pieces
    x, w, labels, _ = _inputs(70000, 16, 2500, "bf16", 9, spread=2.0)
    gout = torch.full((70000,), 1 / 70000, device="cuda")
    st, *out = _run(x, w, labels, 1.0, gout)
    assert st == nb.NITRO_OK
    _check(x, w, labels, 1.0, gout, *out)


def test_either_gradient_alone():
    x, w, labels, _ = _inputs(90, 64, 150, "bf16", 10)
    both = _run(x, w, labels)
    only_x = _run(x, w, labels, want_dw=False)
    only_w = _run(x, w, labels, want_dx=False)
    assert torch.equal(both[3], only_x[3]) and torch.equal(both[4], only_w[4])


def test_rows_that_are_left_out():
    x, w, labels, _ = _inputs(60, 80, 90, "bf16", 11)
    labels[10:20] = -1
    clean = _run(x, w, labels)
    x[10, 3], x[12, 5] = float("nan"), float("inf")           # inside rows that are left out
    st, loss, lse, dx, dw = _run(x, w, labels)
    assert st == nb.NITRO_OK
    assert (loss[10:20] == 0).all() and (dx[10:20] == 0).all()
    assert torch.equal(dw, clean[4]) and torch.equal(dx, clean[3])
    labels[:] = -1
    st, loss, lse, dx, dw = _run(x, w, labels)
    assert st == nb.NITRO_OK and (loss == 0).all() and (dx == 0).all() and (dw == 0).all()


def test_a_label_out_of_range_is_latched_and_left_out():
    x, w, labels, _ = _inputs(40, 64, 50, "bf16", 12)
    bad = labels.clone()
    bad[7], bad[9] = 50, -2
    labels[7] = labels[9] = -1
    good = _run(x, w, labels)
    st, *out = _run(x, w, bad)
    assert st == nb.NITRO_ERR_ARG and good[0] == nb.NITRO_OK
    for a, b in zip(out, good[1:]):
        assert torch.equal(a, b)


def test_a_nan_stays_in_its_row():
    x, w, labels, _ = _inputs(40, 64, 50, "bf16", 13)
    clean = _run(x, w, labels, want_dw=False)
    x[5, 1] = float("nan")
    _, loss, lse, dx, _ = _run(x, w, labels, want_dw=False)
    assert loss[5].isnan() and lse[5].isnan() and dx[5].isnan().all()
    keep = torch.arange(40, device="cuda") != 5
    assert torch.equal(loss[keep], clean[1][keep]) and torch.equal(dx[keep], clean[3][keep])


def test_empty_batch():
    _, w, _, _ = _inputs(4, 64, 50, "bf16", 14)
    h = nb.SoftmaxXent(4, 64, 50)
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    labels = torch.empty(0, dtype=torch.int32, device="cuda")
    none = torch.empty(0, device="cuda")
    dw = torch.ones(50, 70, dtype=torch.bfloat16, device="cuda")
    h.forward(x, w, labels, none, none)
    h.backward(x, w, labels, none, None, None, dw[:, :64])
    assert (dw[:, :64] == 0).all() and (dw[:, 64:] == 1).all() and h.status() == nb.NITRO_OK
    h.close()


def test_gradients_against_differences():
    """(loss(x + h v) - loss(x - h v)) / 2h of the calls' own losses, summed over the rows, on points that bf16
    holds.  Off by at most h^2 / 6 times the third derivative, a third central moment of v w_j under
    the softmax and so at most the cube of its range R, and by the losses' own error over h."""
    g = torch.Generator(device="cuda").manual_seed(15)
    rows, features, classes, h = 48, 32, 60, 0.125
    x = torch.randint(-16, 17, (rows, features), generator=g, device="cuda") / 8
    w = torch.randint(-16, 17, (classes, features), generator=g, device="cuda") / 64
    labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    op = nb.SoftmaxXent(rows, features, classes)

    def loss(x, w):
        out, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        op.forward(x.to(torch.bfloat16), w.to(torch.bfloat16), labels, out, lse)
        return out.double(), lse

    _, lse = loss(x, w)
    dx = torch.empty(rows, features, dtype=torch.bfloat16, device="cuda")
    dw = torch.empty(classes, features, dtype=torch.bfloat16, device="cuda")
    op.backward(x.to(torch.bfloat16), w.to(torch.bfloat16), labels, lse, None, dx, dw)
    v = torch.randint(-1, 2, (rows, features), generator=g, device="cuda").float()
    diff = (loss(x + h * v, w)[0] - loss(x - h * v, w)[0]) / (2 * h)
    R = ((v @ w.t()).amax(1) - (v @ w.t()).amin(1)).double()
    got = (dx.double() * v).sum(1)
    tol = h * h / 6 * R ** 3 + 1e-5 / h + 2 * U * (dx.double().abs() * v.abs()).sum(1) + 2 * U * (w.double().abs() @ v.double().abs().t()).amax(0)
    assert ((got - diff).abs() <= tol).all()
    hw = 1 / 64
    vw = torch.randint(-1, 2, (classes, features), generator=g, device="cuda").float()
    diff = ((loss(x, w + hw * vw)[0] - loss(x, w - hw * vw)[0]) / (2 * hw)).sum()
    R = ((x @ vw.t()).amax(1) - (x @ vw.t()).amin(1)).double()
    tol = (hw * hw / 6 * R ** 3).sum() + rows * 1e-5 / hw + 2 * U * (dw.double().abs() * vw.abs()).sum()
    assert ((dw.double() * vw).sum() - diff).abs() <= tol + U * (x.abs() @ vw.abs().t()).amax(1).sum()
    op.close()


def test_same_bits_twice_on_another_stream_and_in_a_graph():
    x, w, labels, _ = _inputs(200, 128, 3000, "bf16", 16, spread=2.0)
    first = _run(x, w, labels)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = _run(x, w, labels)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first[1:], second[1:]):
        assert torch.equal(a, b)
    h = nb.SoftmaxXent(300, 128, 3000)                         # more rows than used
    loss, lse = torch.empty(200, device="cuda"), torch.empty(200, device="cuda")
    dx, dw = torch.empty_like(first[3]), torch.empty_like(first[4])

    def step():
        h.forward(x, w, labels, loss, lse)
        h.backward(x, w, labels, lse, None, dx, dw)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (loss, lse, dx, dw):
        t.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip((loss, lse, dx, dw), first[1:]):
        assert torch.equal(a, b)
    h.close()


def test_refusals():
    x, w, labels, _ = _inputs(8, 64, 50, "bf16", 17)
    h = nb.SoftmaxXent(4, 64, 50)
    out = torch.empty(8, device="cuda")
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(nb.NitroError):
            h.forward(x[:4], w, labels[:4], out[:4], out[4:], scale=scale)
    with pytest.raises(nb.NitroError):
        h.forward(x, w, labels, out, out)                      # more rows than the handle's
    with pytest.raises(ValueError):
        h.forward(x[:4].float(), w, labels[:4], out[:4], out[4:])
    with pytest.raises(ValueError):
        h.forward(x[:4], w[:49], labels[:4], out[:4], out[4:])
    with pytest.raises(ValueError):
        h.forward(x[:4], w, labels[:4].long(), out[:4], out[4:])
    with pytest.raises(ValueError):
        h.forward(x[:4, :32].t(), w, labels[:4], out[:4], out[4:])
    with pytest.raises(ValueError):
        h.backward(x[:4], w, labels[:4], out[:4], None, torch.empty(4, 64, device="cuda"))
    h.close()

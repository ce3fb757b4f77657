"""Classes that are masked by a weight of bf16's lowest value on a feature that is one (or two: their logits are then
infinite): they have no part in the loss or the gradients, in any form."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


@pytest.mark.parametrize("bias", [1.0, 2.0])
@pytest.mark.parametrize("scale", [0.5, 1.0])
@pytest.mark.parametrize("rows", [1, 2, 4, 7, 12, 40, 200])
def test_masked_classes(rows, bias, scale):
    """Tolerances: as for logits of a few units, sums of 41 products; G and the results rounded to bf16."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    classes, features = 700, 41
    x = torch.randn(rows, features, generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn(classes, features, generator=g, device="cuda") / features ** 0.5).to(torch.bfloat16)
    x[:, 0], w[:, 0] = bias, 0.0
    masked = torch.rand(classes, generator=g, device="cuda") < 0.3
    masked[512:] = True                     # whole tiles among them
    masked[5] = False
    open_ = (~masked).nonzero()[:, 0]
    labels = open_[torch.randint(0, len(open_), (rows,), generator=g, device="cuda")].to(torch.int32)
    w[masked, 0] = torch.finfo(torch.bfloat16).min
    h = nb.SoftmaxXent(rows, features, classes)
    loss, lse = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
    dx = torch.full((rows, features), float("nan"), device="cuda", dtype=torch.bfloat16)
    dw = torch.full((classes, features), float("nan"), device="cuda", dtype=torch.bfloat16)
    h.forward(x, w, labels, loss, lse, scale=scale)
    h.backward(x, w, labels, lse, None, dx, dw, scale=scale)
    assert h.status() == nb.NITRO_OK
    h.close()
    xd, wd = x.double(), w.double()
    z = scale * (xd @ wd[open_].t())
    want = torch.logsumexp(z, 1)
    at = torch.searchsorted(open_, labels.long())
    hit = z.gather(1, at[:, None])[:, 0]
    assert ((lse.double() - want).abs() <= 2.0 ** -18 * (1 + want.abs())).all()
    assert ((loss.double() - (want - hit)).abs() <= 2.0 ** -18 * (1 + want.abs())).all()
    G = torch.softmax(z, 1)
    G[torch.arange(rows, device="cuda"), at] -= 1.0
    G *= scale
    wo = wd[open_]
    assert ((dx.double() - G @ wo).abs() <= 2.2 * U * (G.abs() @ wo.abs()) + 1e-30).all()
    assert (dw[masked] == 0).all()
    assert ((dw[open_].double() - G.t() @ xd).abs() <= 2.2 * U * (G.abs().t() @ xd.abs()) + 1e-30).all()

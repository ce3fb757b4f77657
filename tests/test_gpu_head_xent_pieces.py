"""The backward over several pieces of the classes, the last one shorter, against its formulas in
64 bits."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


@pytest.mark.parametrize("rows, features, classes", [(150000, 24, 2500), (150000, 17, 1793), (40000, 64, 20000)])
def test_against_the_formulas(rows, features, classes):
    """Tolerances: G and the result are rounded to bf16 once each, u of the magnitudes that are summed; logits and 32-bit
    sums add less than u / 8 to that."""
    assert rows * classes > 256 << 20           # more than a piece's G holds
    g = torch.Generator(device="cuda").manual_seed(classes)
    x = torch.randn(rows, features, generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn(classes, features, generator=g, device="cuda") * 2 / features ** 0.5).to(torch.bfloat16)
    labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    labels[::7] = -1
    gout = torch.full((rows,), 1.0 / rows, device="cuda")
    h = nb.SoftmaxXent(rows, features, classes)
    loss, lse = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
    dx = torch.full((rows, features), float("nan"), device="cuda", dtype=torch.bfloat16)
    dw = torch.full((classes, features), float("nan"), device="cuda", dtype=torch.bfloat16)
    h.forward(x, w, labels, loss, lse)
    h.backward(x, w, labels, lse, gout, dx, dw)
    assert h.status() == nb.NITRO_OK
    h.close()
    xd, wd = x.double(), w.double()
    want_w, mag_w = torch.zeros(2, classes, features, device="cuda", dtype=torch.float64)
    for r in range(0, rows, 10000):
        s = slice(r, min(r + 10000, rows))
        z = xd[s] @ wd.t()
        G = torch.softmax(z, 1)
        live = labels[s] >= 0
        G[torch.arange(len(live), device="cuda"), labels[s].clamp(min=0).long()] -= 1.0
        G[~live] = 0.0
        G /= rows
        want = torch.logsumexp(z, 1)
        S = (xd[s].abs() @ wd.abs().t()).amax(1)
        assert ((lse[s].double() - want).abs() <= (-(-features // 16) + 8) * 2.0 ** -23 * S + 2.0 ** -20 * (1 + want.abs())).all()
        want, mag = G @ wd, G.abs() @ wd.abs()
        assert ((dx[s].double() - want).abs() <= U * want.abs() + 1.2 * U * mag).all()
        want_w += G.t() @ xd[s]
        mag_w += G.abs().t() @ xd[s].abs()
    assert ((dw.double() - want_w).abs() <= U * want_w.abs() + 1.2 * U * mag_w).all()

"""The forward of a few rows, which runs on the CUDA cores, and small losses in every form.

Tolerances.  A lane adds ceil(F / 32) products of its own with one rounding each, 2^-24 of the
sum of magnitudes S at most, then 5 additions over the lanes and up to 7 over the warps; scale log2 e
and the exponent are rounded to 2^-24 a few times.  exp2f and log2f are within 2^-22."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu


def _forward(x, w, labels, scale, stream=None):
    rows = x.shape[0]
    h = nb.SoftmaxXent(rows, x.shape[1], w.shape[0])
    loss, lse = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
    h.forward(x, w, labels, loss, lse, scale=scale, stream=stream)
    st = h.status()
    h.close()
    return st, loss.double(), lse.double()


def _exact(x, w, labels, scale):
    z = scale * (x.double() @ w.double().t())
    lse = torch.logsumexp(z, 1)
    hit = z.gather(1, labels.clamp(min=0).long()[:, None])[:, 0]
    return torch.where(labels >= 0, lse - hit, torch.zeros_like(lse)), lse


@pytest.mark.parametrize("xt", ["bf16", "i8"])
@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 7, 8])
@pytest.mark.parametrize("features, classes", [
    (1, 1), (1, 70000), (7, 2), (255, 33), (256, 4), (257, 1001), (520, 9731), (2049, 10), (2048, 4864), (4100, 300),
    (70000, 3)])
def test_against_the_formula(rows, features, classes, pad, xt):
    g = torch.Generator(device="cuda").manual_seed(rows * 1000 + features)
    x = torch.randn(rows, features + pad, generator=g, device="cuda")
    x = (x * 40).round().clamp(-128, 127).to(torch.int8) if xt == "i8" else x.to(torch.bfloat16)
    w = (torch.randn(classes, features + pad, generator=g, device="cuda") * 2 / features ** 0.5).to(torch.bfloat16)
    x, w = x[:, :features], w[:, :features]
    labels = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    labels[torch.rand(rows, generator=g, device="cuda") < 0.2] = -1
    scale = 1 / 32 if xt == "i8" else 1.0
    st, loss, lse = _forward(x, w, labels, scale)
    assert st == nb.NITRO_OK
    eloss, else_ = _exact(x, w, labels, scale)
    S = scale * (x.double().abs() @ w.double().abs().t()).amax(1)
    ez = (-(-features // 32) + 16) * 2.0 ** -24 * S
    assert ((lse - else_).abs() <= 2 * ez + 2.0 ** -20 * (1 + else_.abs())).all()
    assert ((loss - eloss).abs() <= 4 * ez + 2.0 ** -20 * (1 + eloss)).all()


@pytest.mark.parametrize("rows, features, classes", [(1, 40, 10), (4, 300, 100), (8, 40, 10), (40, 300, 100), (300, 64, 2000)])
def test_small_losses_beside_large_logits(rows, features, classes):
    """Logits of some hundreds, small integers' exact sums, whose distance to the label's is a few: the loss is
    not off by the rounding of its log-sum (2^-16 at 256)."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randint(-2, 3, (rows, features), generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randint(-2, 3, (classes, features), generator=g, device="cuda").to(torch.bfloat16)
    x[:, 0], w[:, 0] = 128.0, 64.0              # 8192 in every logit
    labels = (x.double() @ w.double().t()).argmax(1).to(torch.int32)
    scale = 0.0371
    st, loss, lse = _forward(x, w, labels, scale)
    eloss, else_ = _exact(x, w, labels, float(torch.tensor(scale, dtype=torch.float32)))
    assert st == nb.NITRO_OK
    assert ((lse - else_).abs() <= 2.0 ** -21 * else_).all()
    assert ((loss - eloss).abs() <= 2.0 ** -19 * (1 + eloss)).all()


@pytest.mark.parametrize("rows", [1, 3, 8])
def test_rows_do_not_reach_one_another(rows):
    """A NaN in a row stays in that row."""
    x = torch.ones(rows, 300, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(50, 300, device="cuda").to(torch.bfloat16)
    labels = torch.full((rows,), 7, device="cuda", dtype=torch.int32)
    _, want, _ = _forward(x, w, labels, 0.05)
    x[rows - 1, 299] = float("nan")
    _, got, lse = _forward(x, w, labels, 0.05)
    assert torch.equal(got[: rows - 1], want[: rows - 1])
    assert got[rows - 1].isnan() and lse[rows - 1].isnan()


def test_calls_repeat_bit_by_bit_and_on_other_streams():
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(4, 520, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn(9000, 520, generator=g, device="cuda").to(torch.bfloat16)
    labels = torch.randint(0, 9000, (4,), generator=g, device="cuda", dtype=torch.int32)
    h = nb.SoftmaxXent(4, 520, 9000)
    outs = []
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for k in range(6):
        loss, lse = (torch.full((4,), float("nan"), device="cuda") for _ in range(2))
        torch.cuda.synchronize()
        h.forward(x, w, labels, loss, lse, scale=0.1, stream=side if k & 1 else None)
        torch.cuda.synchronize()
        outs.append((loss, lse))
    assert h.status() == nb.NITRO_OK
    h.close()
    for loss, lse in outs[1:]:
        assert torch.equal(loss, outs[0][0]) and torch.equal(lse, outs[0][1])


def test_labels_out_of_range_are_told():
    x = torch.ones(2, 8, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(5, 8, device="cuda", dtype=torch.bfloat16)
    st, loss, _ = _forward(x, w, torch.tensor([5, 1], device="cuda", dtype=torch.int32), 1.0)
    assert st == nb.NITRO_ERR_ARG
    assert loss[0] == 0.0

"""Group norm where a sample is shared out over many CTAs, and where a thread has thousands of values.

A thread's values go in runs of 32, its runs are added up, then 256 / (vectors of a pixel) threads' sums, 16 at a time, lanes', and the
CTAs'.  `chain` counts the longest of these sums together; the sums of the checks here are off by at most that many times 2^-24 of their
absolute terms, by half of it where all terms are equal (a partial sum's rounding is of what it holds by then)."""
import pytest
import torch

import test_gpu_head_gnorm as gn
from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def parts(pixels, channels, samples=1):
    """Values of a thread's run, its runs, and what joins threads, lanes and CTAs."""
    v = 8 if channels % 8 == 0 else 4 if channels % 4 == 0 else 1
    vecs = -(-channels // v)
    vecs = -(-vecs // -(-vecs // 256))
    rows = 256 // vecs
    # four CTAs an SM of single channels, two at least of vectors, 152 SMs
    ctas = max(1, min((600 if v == 1 else 300) // samples, -(-pixels // (8 * rows))))
    steps = -(-pixels // (ctas * rows))
    return min(32, steps), -(-steps // 32), min(16, rows) + -(-rows // 16) + 5 + 608 // 32 + 5


def chain(*shape):
    return sum(parts(*shape))


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("x, pad", [("bf16", 0), ("f32", 0), ("bf16", 3)])
@pytest.mark.parametrize("n, p, c, groups", [(3, 70001, 100, 5), (1, 40000, 1000, 10), (2, 90001, 64, 2)])
def test_gradients_with_a_mean(n, p, c, groups, x, pad, act, monkeypatch):
    xx, _, gamma, beta = gn.inputs(n, p, c, x, "f32", pad, seed=p)
    # dy with a mean, and along h: both group means are a large part of dx
    v = xx.float().reshape(n, p, groups, -1)
    h = ((v - v.mean(dim=(1, 3), keepdim=True)) / v.std(dim=(1, 3), keepdim=True)).reshape(n, p, c)
    g = torch.Generator(device="cuda").manual_seed(1)
    dy = gn.view(0.5 + 0.3 * h + 0.2 * torch.randn(n, p, c, generator=g, device="cuda"), pad)
    monkeypatch.setattr(gn, "steps", lambda p, c: chain(p, c, n))
    out = gn.run(xx, dy, gamma, beta, groups, 1e-5, act, pad=pad)
    gn.check(xx, dy, gamma, beta, groups, 1e-5, act, *out)


@pytest.mark.parametrize("b", [1.1, 1.2345678, 1.37])
def test_statistics_of_one_long_channel(b):
    pixels = 1 << 28
    g = torch.Generator(device="cuda").manual_seed(2)
    ones = torch.randint(0, 2, (pixels,), generator=g, device="cuda", dtype=torch.int8)
    share = ones.sum().item() / pixels
    x = (ones * torch.tensor(b, device="cuda")).view(1, pixels, 1)
    b = torch.tensor(b).double().item()
    mean, var = share * b, share * (1 - share) * b * b
    op = nb.GroupNorm(1, pixels, 1, 1)
    m, r = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    y = torch.empty(1, pixels, 1, dtype=torch.bfloat16, device="cuda")
    op.forward(x, None, None, y, m, r, eps=1e-6)
    op.close()
    run, runs, rest = parts(pixels, 1)
    # A thread's distances to its first value are b or 0, half of each: its squares' sum S and its sum's square over the count, S / 2, are
    # off by (run + runs + 2) / 2 and twice that of themselves, and their difference, S / 2, by four times (run + runs + 2) / 2;
    # threads' alike sums by rest / 2 more.  rstd is off by half of the variance's.
    want = (var + 1e-6) ** -0.5
    assert abs(m.item() - mean) <= 0.5 * (run + runs + rest + 4) * E * b
    assert abs(r.item() - want) <= (run + runs + 2 + 0.25 * rest + 16) * E * want


@pytest.mark.parametrize("c", [1.37, 1.2345678, 1.1, 0.3])
def test_gradients_all_alike(c):
    pixels = 1 << 28
    x = torch.randint(-50, 50, (1, pixels, 1), device="cuda", dtype=torch.int8)
    dy = torch.full((1, pixels, 1), c, device="cuda")
    op = nb.GroupNorm(1, pixels, 1, 1)
    mean, rstd = torch.zeros(1, device="cuda"), torch.ones(1, device="cuda")
    db = torch.empty(1, device="cuda")
    op.backward(x, None, None, mean, rstd, dy, None, None, db)
    op.close()
    want = dy[0, 0, 0].double().item() * pixels
    assert abs(db.item() - want) <= 0.5 * chain(pixels, 1) * E * want

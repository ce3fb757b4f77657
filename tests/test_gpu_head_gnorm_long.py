"""Group norm where a sample is shared out over many CTAs, and where a thread has thousands of values.

A thread's values go in runs of 32, its runs are added up, then 256 / (vectors of a pixel) threads' sums, 16 at a time, lanes', and the
CTAs'.  `chain` counts the longest of these sums together; the sums of the checks here are off by at most that many times 2^-24 of their
absolute terms, by half of it where all terms are equal (a partial sum's rounding is of what it holds by then)."""
import pytest
import torch

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

"""The norm over many values a thread, by each way that values are reached.

Every value here is the same, so that all roundings of a sum may fall one way.  k equal terms in one run are off by 2^-24 of every partial
sum at most, (k + 1) / 2 of them of the whole: 8.5 for runs of 16 squares, one more for a run's two halves.  What joins runs keeps its roundings.  Outside
the squares' own range the joins over lanes, warps and CTAs round some 20 times.  A norm is off by half of that: 15 2^-24 < 2^-20."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def norm_of(ts):
    op = nb.GradClip(ts)
    norm = torch.empty((), device="cuda")
    op.run(norm)
    assert op.status() == nb.NITRO_OK
    op.close()
    return norm.item()


def value(t, c):
    return torch.tensor(c, dtype=t).double().item()


@pytest.mark.parametrize("t, c", [(BF, 1.1484375), (BF, 1.9), (F32, 1.2345678), (F32, 1.37)])
@pytest.mark.parametrize("cols, ld, start", [(4001, 4101, 1),       # rows far apart that start anywhere: single values
                                             (7, 64, 0)])           # rows without a whole vector of bf16, or with more values after it
def test_single_values(cols, ld, start, t, c):
    rows, times = 16000000 // ld, 8 if cols == 4001 else 40
    buf = torch.full((rows, ld), c, dtype=t, device="cuda")
    m = buf[:, start: start + cols]
    # (matrices that are not written may be the same one)
    want = value(t, c) * (times * rows * cols) ** 0.5
    assert abs(norm_of([m] * times) - want) <= 2.0 ** -20 * want


@pytest.mark.parametrize("t, c", [(BF, 1.1484375), (F32, 1.2345678), (F32, 1.37)])
@pytest.mark.parametrize("start", [0, 1])
@pytest.mark.parametrize("n, times", [(8000000, 1), (8000000, 2), (16000000, 60)])
def test_vectors(n, times, start, t, c):
    m = torch.full((n + 1,), c, dtype=t, device="cuda")[start: start + n]
    want = value(t, c) * (times * n) ** 0.5
    assert abs(norm_of([m] * times) - want) <= 2.0 ** -20 * want


@pytest.mark.parametrize("c", [1.2345678e-30, 1.37e-25, 1.2345678e30, 1.37e25])
@pytest.mark.parametrize("times", [1, 60])
def test_vectors_past_the_squares(times, c):
    n = 16000000
    m = torch.full((n,), c, dtype=F32, device="cuda")
    want = value(F32, c) * (times * n) ** 0.5
    assert abs(norm_of([m] * times) - want) <= 2.0 ** -20 * want


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("start", [0, 1])
@pytest.mark.parametrize("n", [50, 5000000, 60000000])
def test_a_value_that_is_not_finite(n, start, bad):
    m = torch.ones(n + 1, device="cuda")[start:]
    m[n // 3] = bad
    got = norm_of([m])
    assert got == float("inf") if bad == bad else got != got

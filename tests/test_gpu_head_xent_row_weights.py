"""Weight gradients under row gradients of very different size, against the formulas in 64 bits.
Tolerances: those of test_gpu_head_xent.py; rows whose gradient is far below the largest one may be left with
nothing, which is less than one rounding of the others."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb
from test_gpu_head_xent import _check, _inputs, _run

pytestmark = pytest.mark.gpu


def _step(rows, gout, seed=1, xt="bf16"):
    x, w, labels, g = _inputs(rows, 72, 90, xt, seed)
    labels[1::5] = -1                       # the largest and smallest gradients stand in other rows
    if x.dtype == torch.bfloat16:
        x = x * 4
    scale = 1 / 32 if xt == "i8" else 0.25
    st, *out = _run(x, w, labels, scale, gout)
    assert st == nb.NITRO_OK
    assert out[2].isfinite().all() and out[3].isfinite().all()
    _check(x, w, labels, scale, gout, *out)
    return out[3]


@pytest.mark.parametrize("rows", [3, 40, 1500, 5003])
@pytest.mark.parametrize("tiny", [1e-20, 1e-30, 1e-38, 1e-39, 1e-45])
@pytest.mark.parametrize("first", [True, False])
def test_one_tiny_gradient(rows, tiny, first):
    gout = torch.ones(rows, device="cuda")
    gout[0 if first else -1] = tiny
    _step(rows, gout)


@pytest.mark.parametrize("rows", [2, 33, 2000])
@pytest.mark.parametrize("xt", ["bf16", "i8"])
def test_one_large_gradient(rows, xt):
    # all but one row tiny, the large one last
    gout = torch.full((rows,), 1e-39, device="cuda")
    gout[-1] = 2.0
    labels_of_last = (rows - 1) % 5
    if labels_of_last == 1:                 # that row is left out
        gout[0] = 2.0
    _step(rows, gout, xt=xt)


@pytest.mark.parametrize("rows", [20, 700, 4100])
@pytest.mark.parametrize("backwards", [False, True])
def test_weights_of_exponential_range(rows, backwards):
    s = torch.linspace(0, 100, rows, device="cuda")
    gout = torch.exp(-s)
    _step(rows, gout.flip(0).contiguous() if backwards else gout)


@pytest.mark.parametrize("rows", [20, 700, 4100])
def test_a_large_gradient_of_a_row_that_is_left_out(rows):
    gout = torch.linspace(-1, 1, rows, device="cuda")
    gout[1::5] = 1e38                       # rows without a label
    gout[6] = float("nan")
    _step(rows, gout)


@pytest.mark.parametrize("rows", [20, 700, 4100])
def test_equal_gradients_scale_exactly(rows):
    one = _step(rows, None)
    assert torch.equal(_step(rows, torch.full((rows,), 0.25, device="cuda")), one * 0.25)

"""Matrices whose squares do not fit 32 bits: the norm, and with it the update, is right over the whole range of the
types.  Tolerance: see test_gpu_head_orth.py."""
import pytest
import torch

from test_gpu_head_orth import DT, _check, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("steps", [0, 2, 5])
@pytest.mark.parametrize("rows, cols", [(20, 33), (140, 150), (50, 700), (700, 50), (130, 400)])
@pytest.mark.parametrize("factor", [1e17, 1e20, 1e30, 4e37])
def test_large_values(rows, cols, dtype, steps, factor):
    g = torch.Generator(device="cuda").manual_seed(rows)
    m = (torch.randn(3, rows, cols, generator=g, device="cuda").clamp(-4, 4).double() * factor).to(DT[dtype])
    m[1] = m[1] * 1e-25                     # an ordinary one beside them
    assert m.isfinite().all()
    _check(m, _run(m, steps=steps), steps)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, cols", [(1, 1), (20, 33), (140, 150)])
def test_the_largest_value(rows, cols, dtype):
    m = torch.full((1, rows, cols), torch.finfo(DT[dtype]).max, dtype=DT[dtype], device="cuda")
    m[:, ::2, ::3] *= -1
    _check(m, _run(m))
    m = torch.zeros_like(m)
    m[0, 0, 0] = torch.finfo(DT[dtype]).max
    _check(m, _run(m))


@pytest.mark.parametrize("rows, cols", [(20, 33), (140, 150)])
def test_an_infinity_is_no_large_value(rows, cols):
    m = torch.full((2, rows, cols), 1e30, device="cuda")
    m[0, 1, 2] = float("inf")
    out = _run(m)
    assert out[0].isnan().any() and out[1].isfinite().all()

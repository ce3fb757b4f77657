"""Clipping by factors of any size: limits far below the norm, norms past the type, limits next to the smallest numbers.

The norm is off by 2^-20 of itself at most, the factor and each value by a rounding of 32 bits, and an output by half a step of its
type: of itself, or of the type's smallest numbers (2^-133 in bf16, 2^-149 in fp32)."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def clip(ts, outs, limit):
    op = nb.GradClip(ts, outs)
    norm = torch.empty((), device="cuda")
    op.run(norm, limit)
    assert op.status() == nb.NITRO_OK
    op.close()
    return norm.item()


def check(ts, outs, f):
    for t, o in zip(ts, outs):
        if o is None:
            continue
        w = t.double() * f
        step = 2.0 ** -133 if t.dtype == BF else 2.0 ** -149
        assert ((o.double() - w).abs() <= (torch.finfo(t.dtype).eps / 2 + 2.0 ** -19) * w.abs() + step).all()


def norm(ts):
    return sum(t.double().square().sum().item() for t in ts) ** 0.5


# (a limit is what fp32 holds of it)
def as_f32(v):
    return torch.tensor(v, dtype=F32).item()


@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("shape, ld", [((300, 50), 50), ((300, 50), 57), ((40, 333), 1000)])
@pytest.mark.parametrize("size, limit", [(1e37, 1.0), (1e37, 1e-3), (1e37, 1e-8), (1e37, 1e-20), (1e36, 1e-37), (3e36, 1e-44), (1e25, 1e-13), (1e18, 1e-20),
                                         (1e9, 1e-30), (1.0, 1e-38), (1.0, 1e-42), (1e-12, 1e-38), (1e-12, 1e-43), (1e-30, 1e-40), (1e-36, 1e-44)])
def test_limits_far_below(size, limit, shape, ld, t):
    g = torch.Generator().manual_seed(5)
    wide = (torch.randn(shape[0], ld, generator=g) * size).to(t).cuda()
    ts = [wide[:, : shape[1]], (torch.randn(77, generator=g) * size).to(F32).cuda()]
    outs = [torch.full(shape, 9.0, dtype=t, device="cuda"), torch.full((77,), 9.0, device="cuda")]
    clip(ts, outs, limit)
    check(ts, outs, as_f32(limit) / norm(ts))
    # in place, as runs without gaps, whose sums go in another order
    place = [x.clone() for x in ts]
    clip(place, place, limit)
    check(ts, place, as_f32(limit) / norm(ts))


def test_small_values_beside_large_ones():
    # values of every size under one factor
    g = torch.Generator().manual_seed(6)
    for size, limit in ((1e37, 1e-3), (1e37, 1e30), (1e20, 1e-25), (1e-5, 1e-40)):
        e = torch.rand(5000, generator=g) * 36
        ts = [(torch.randn(5000, generator=g) * size * 10.0 ** -e).cuda(), torch.full((3,), size, device="cuda")]
        outs = [torch.empty_like(x) for x in ts]
        clip(ts, outs, limit)
        check(ts, outs, as_f32(limit) / norm(ts))

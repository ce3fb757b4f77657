"""A norm over more of the largest numbers than fp32 has room for even of their scaled squares: it is not infinite, and scales."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("times", [20, 300])
def test_billions_of_the_largest(times):
    n, big = 1 << 24, 3.3e38
    many = torch.full((n,), big, dtype=torch.bfloat16, device="cuda")
    some = torch.linspace(1e25, 1e30, 1000, device="cuda")
    ts, outs = [many] * times + [some], [None] * times + [torch.zeros_like(some)]
    op = nb.GradClip(ts, outs)
    norm = torch.empty((), device="cuda")
    op.run(norm, 1e38)
    op.close()
    assert norm.item() == float("inf")
    true = many[0].double().item() * (times * n) ** 0.5
    w = some.double() * (torch.tensor(1e38).item() / true)
    # the norm 2^-20, the factor and the product a rounding each
    assert ((outs[-1].double() - w).abs() <= 2.0 ** -19 * w).all()

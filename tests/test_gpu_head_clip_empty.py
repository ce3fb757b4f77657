"""Clipping where there is nothing to clip: no gradients, or empty ones, under a limit."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shapes", [[], [(0,)], [(0, 5), (3, 0)]])
@pytest.mark.parametrize("place", [False, True])
def test_nothing(shapes, place):
    ts = [torch.empty(s, device="cuda", dtype=torch.bfloat16) for s in shapes]
    op = nb.GradClip(ts, ts if place else [torch.empty_like(t) for t in ts])
    norm = torch.full((), 3.0, device="cuda")
    op.run(norm, 0.5)
    assert norm.item() == 0.0
    op.close()


def test_values_and_none_is_written():
    ts = [torch.ones(5, device="cuda"), torch.empty(0, device="cuda")]
    op = nb.GradClip(ts, [None, ts[1]])
    with pytest.raises(nb.NitroError):
        op.run(torch.empty((), device="cuda"), 0.5)
    op.close()

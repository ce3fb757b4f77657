"""How far a step of the gated head takes an entry of its matrices.

The update of a matrix is orthogonal (the gate and the up matrix by themselves), rows x cols: its entries' mean square is
1 / max(rows, cols) times the singular values', which the update's five steps take to between 0.6 and 1.3."""
import math

import pytest
import torch

from paper_2407_11698_gb300.many_class import GatedHead

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pixels, channels, hidden, classes", [(4, 16, 256, 300), (4, 16, 48, 300), (16, 24, 72, 40), (4, 16, 64, 64)])
def test_entries_move_by_the_rate(pixels, channels, hidden, classes):
    rate = 0.01
    head = GatedHead(pixels, channels, 4, hidden, classes, 128, lr=rate)
    g = torch.Generator().manual_seed(hidden)
    x = (torch.randn(128, pixels, channels, generator=g) * 30).round().clamp(-127, 127).to(torch.int8).cuda()
    labels = torch.randint(0, classes, (128,), generator=g).to(torch.int32).cuda()
    before = [m.clone() for m in head.masters]
    head.step(x, labels)
    features = pixels * channels
    for old, new, u, longest in zip(before, head.masters, head.updates, (max(hidden, features), max(classes, hidden))):
        moved, want = (old - new).double(), u.double() * (rate * math.sqrt(longest))
        # the difference of two fp32 values up to 2^3, and the product's rounding
        assert ((moved - want).abs() <= 2.0 ** -20 + 2.0 ** -22 * want.abs()).all()
        assert moved.square().mean().sqrt().item() <= 1.3 * rate
    head.close()

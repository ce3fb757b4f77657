"""A cross-entropy handle takes no more device memory than its header states: copies of x and W, G, the row
statistics and the 32-bit sums."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows, features, classes", [(4, 512, 10000), (40, 8, 1 << 24), (20, 64, 1 << 22), (8192, 64, 64000), (1 << 20, 8, 5000)])
def test_stated_bytes(rows, features, classes):
    nb.SoftmaxXent(4, 8, 8).close()
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    h = nb.SoftmaxXent(rows, features, classes)
    used = before - torch.cuda.mem_get_info()[0]
    h.close()
    up = lambda v, to: -(-v // to) * to
    copies = 2 * (2 * rows + classes) * up(features, 8)
    g = min(4 << 30, 2 * max(rows, 2 * min(rows, 32)) * up(classes, 64))
    stats = max(8 * rows * up(classes, 128) // 32, 1 << 15) + 8 * (rows + 1)
    sums = max(64 << 20, 4 * rows * up(features, 32))
    assert used <= copies + g + stats + sums + (16 << 20)       # allocations are in whole pages

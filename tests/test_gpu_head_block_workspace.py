"""Handles of group norm, the gated block and clipping take no more device memory than their headers state."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu

PAGES = 16 << 20        # allocations are in whole pages


def up(v, to):
    return -(-v // to) * to


def used(make):
    make().close()
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    h = make()
    n = before - torch.cuda.mem_get_info()[0]
    h.close()
    return n


@pytest.mark.parametrize("samples, pixels, channels, groups", [(1, 64, 8, 1), (65535, 64, 8192, 8192), (64, 1 << 20, 2048, 32), (3, 1 << 27, 256, 256)])
def test_group_norm(samples, pixels, channels, groups):
    stated = 8192 * (channels + groups) + min(samples, 1024) * (16 * groups + 4)
    assert used(lambda: nb.GroupNorm(samples, pixels, channels, groups)) <= stated + PAGES


@pytest.mark.parametrize("rows, features, hidden", [(1, 8, 8), (8192, 2048, 8192), (40, 4096, 1 << 18), (1 << 20, 64, 512), (33, 1 << 17, 100)])
def test_gated_block(rows, features, hidden):
    copies = 2 * (rows + 2 * hidden) * up(features, 8)
    d = 2 * max(rows, 2 * min(rows, 32)) * up(2 * hidden, 8)
    sums = min(64 << 20, 64 * rows * up(features, 32))
    assert used(lambda: nb.GatedLinear(rows, features, hidden)) <= copies + d + sums + PAGES


@pytest.mark.parametrize("count, n", [(1, 100), (1, 1 << 30), (100000, 256)])
def test_clipping(count, n):
    buf = torch.zeros(n + 64, dtype=torch.bfloat16, device="cuda")
    ts = [buf[:n]] * count
    assert used(lambda: nb.GradClip(ts)) <= 64 * count + (1 << 20) + PAGES

"""Forms that only larger sizes take: tiles of 256 columns, CTAs that take several tiles, sums in two accumulators.
Tolerances: those of the operators' own test files."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb
import test_gpu_head_mx4 as mx4
import test_gpu_head_orth as orth
import test_gpu_head_xent as xent

pytestmark = pytest.mark.gpu


# symmetric products in pairs of 256 x 256 (the first four sizes, up to 1.8 tiles a pair), of 256 x 128 and alone; the
# update in 256-wide tiles, alone and in pairs, up to four a CTA
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("count, rows, cols", [
    (1, 2500, 2500), (1, 2400, 2304), (1, 2304, 2401), (1, 4100, 4096), (1, 1500, 5000), (1, 5000, 1500), (1, 3100, 3000), (1, 3000, 3100),
    (20, 300, 1200), (20, 1200, 300), (8, 256, 2304), (8, 512, 2304)])
def test_orth(count, rows, cols, dtype):
    m = orth._matrix(count, rows, cols, dtype, rows + cols, rank=64 if rows == 2500 else 0)
    out = orth._run(m)
    orth._check(m, out)
    assert torch.equal(out, orth._run(m))


# more tiles than SMs: columns of up to 32 rows (quantised in the product), of up to 64, and pairs
@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("rows, k, n", [(1, 300, 20000), (9, 700, 40001), (32, 64, 20000), (32, 1111, 39000), (50, 300, 20001), (64, 1000, 40000),
                                        (130, 2000, 20000), (3000, 520, 5001)])
def test_mx4_product(rows, k, n, y):
    g = torch.Generator(device="cuda").manual_seed(rows + k)
    x = torch.randn(rows, k, generator=g, device="cuda").to(mx4.DT["bf16" if rows % 2 else "f32"])
    w = torch.randn(n, k, generator=g, device="cuda") / k ** 0.5
    q, s = mx4._quantize(w)
    wv = torch.empty(n, k, device="cuda")
    nb.mx4_dequantize(q, s, wv)             # exact: see test_gpu_head_mx4.py
    first = mx4._linear(x, q, s, n, y)
    mx4._check(x, first, wv.double().cpu().numpy())
    assert torch.equal(first, mx4._linear(x, q, s, n, y))


@pytest.mark.parametrize("rows, features, classes", [(1500, 2500, 10000), (200, 2304, 20000), (1000, 2100, 12001)])
def test_xent(rows, features, classes):
    x, w, labels, _ = xent._inputs(rows, features, classes, "bf16", 6, spread=3.0)
    labels[::9] = -1
    gout = torch.full((rows,), 1 / rows, device="cuda")
    st, *out = xent._run(x, w, labels, 1.0, gout)
    assert st == nb.NITRO_OK
    xent._check(x, w, labels, 1.0, gout, *out)
    st, *again = xent._run(x, w, labels, 1.0, gout)
    assert all(torch.equal(a, b) for a, b in zip(out, again))

"""Newton-Schulz orthogonalisation against its formula in 64 bits.

Tolerance on the 2-norm of the difference, relative: bf16 rounds each output by at most
u = 2^-8 of it.  The last two of the steps round X, A and B to fp16 (2^-11 of a value each);
what a step adds is multiplied by at most a = 3.4445 in each one after it, so 3 2^-11 (1 +
3.4445), and earlier steps keep 22 bits.  Other coefficients: a with theirs."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu
DEFAULT = (3.4445, -4.7750, 2.0315)
DT = {"bf16": torch.bfloat16, "f32": torch.float32, "i64": torch.int64}


def _formula(m, steps, coef):
    x = m.double()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    tall = x.shape[1] > x.shape[2]
    x = x.mT if tall else x
    for _ in range(steps):
        a = x @ x.mT
        x = coef[0] * x + (coef[1] * a + coef[2] * (a @ a)) @ x
    return x.mT if tall else x


def _tol(coef):
    return 2.0 ** -8 + 3 * 2.0 ** -11 * (1 + abs(coef[0]))


def _check(m, out, steps=5, coef=DEFAULT):
    want = _formula(m, steps, coef)
    for k in range(m.shape[0]):
        d = (out[k].double() - want[k]).norm()
        assert d <= _tol(coef) * want[k].norm(), (k, float(d / want[k].norm()))


def _matrix(count, rows, cols, dtype, seed, rank=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if rank:
        m = torch.randn(count, rows, rank, generator=g, device="cuda") @ torch.randn(count, rank, cols, generator=g, device="cuda")
    else:
        m = torch.randn(count, rows, cols, generator=g, device="cuda")
    return (m * 1e6).round().to(torch.int64) if dtype == "i64" else m.to(DT[dtype])


def _run(m, steps=5, coef=None, out=None):
    count, rows, cols = m.shape
    h = nb.Orthogonalizer(count, rows, cols)
    out = torch.full((count, rows, cols), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    h.run(m, out, steps=steps, coef=coef)
    assert h.status() == nb.NITRO_OK
    h.close()
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32", "i64"])
@pytest.mark.parametrize("count, rows, cols", [
    (1, 1, 1), (1, 1, 5), (2, 7, 3), (1, 32, 32), (3, 33, 257), (1, 128, 256), (1, 128, 513), (2, 700, 128), (1, 96, 2048),
    (1, 2048, 40), (1, 40, 2049), (1, 129, 40), (2, 130, 130), (1, 130, 2050), (1, 300, 200), (5, 256, 320), (1, 1000, 520)])
def test_against_the_formula(count, rows, cols, dtype):
    m = _matrix(count, rows, cols, dtype, rows + cols)
    _check(m, _run(m))


@pytest.mark.parametrize("rows, cols", [(64, 300), (200, 500), (500, 200)])
@pytest.mark.parametrize("rank", [1, 5])
@pytest.mark.parametrize("dtype", ["bf16", "f32", "i64"])
def test_low_rank(rows, cols, rank, dtype):
    # the gradient of a small batch: what rounding puts outside its rank must not grow
    m = _matrix(1, rows, cols, dtype, 3, rank)
    if dtype == "bf16":
        m = (torch.randint(-8, 9, (1, rows, rank), device="cuda").float() @ torch.randint(-3, 4, (1, rank, cols), device="cuda").float()).to(torch.bfloat16)
        if rank == 5:
            m = _matrix(1, rows, cols, "bf16", 4, 5)
    _check(m, _run(m))


@pytest.mark.parametrize("rows, cols", [(40, 70), (150, 260)])
@pytest.mark.parametrize("steps", [0, 1, 2, 3, 8])
def test_steps(rows, cols, steps):
    m = _matrix(2, rows, cols, "f32", steps)
    _check(m, _run(m, steps=steps), steps)


@pytest.mark.parametrize("rows, cols", [(40, 70), (150, 260)])
@pytest.mark.parametrize("coef", [(1.875, -1.25, 0.375), (1.5, -0.5, 0.0), (2.0, -1.5, 0.5)])
def test_coefficients(rows, cols, coef):
    m = _matrix(1, rows, cols, "bf16", 7)
    _check(m, _run(m, coef=coef), coef=coef)


@pytest.mark.parametrize("rows, cols", [(20, 33), (140, 150)])
def test_zeros_and_a_nan(rows, cols):
    m = _matrix(3, rows, cols, "f32", 8)
    clean = _run(m)
    m[0] = 0
    m[1, 2, 3] = float("nan")
    out = _run(m)
    assert (out[0] == 0).all() and out[1].isnan().any() and torch.equal(out[2], clean[2])


@pytest.mark.parametrize("rows, cols", [(20, 33), (140, 150)])
def test_large_and_small_values(rows, cols):
    m = _matrix(1, rows, cols, "f32", 9)
    for f in (1e-12, 1e15):
        _check(m * f, _run(m * f))
    big = (m.double() * 2.0 ** 59).to(torch.int64)
    _check(big, _run(big))
    _check(_matrix(1, rows, cols, "i64", 10) // 1000000, _run(_matrix(1, rows, cols, "i64", 10) // 1000000))


@pytest.mark.parametrize("rows, cols", [(20, 35), (140, 150), (150, 60)])
@pytest.mark.parametrize("dtype", ["bf16", "f32", "i64"])
@pytest.mark.parametrize("pad", [1, 8])
def test_strides(rows, cols, dtype, pad):
    wide = _matrix(2, rows + 2, cols + pad, dtype, 11)
    m = wide[:, :rows, :cols]
    keep = torch.full((2, rows + 3, cols + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    out = _run(m, out=keep[:, :rows, :cols])
    assert torch.equal(out, _run(m.contiguous()))
    assert (keep[:, rows:] == 7).all() and (keep[:, :, cols:] == 7).all()


@pytest.mark.parametrize("rows, cols", [(60, 500), (300, 260)])
def test_same_bits_on_another_stream_and_in_a_graph(rows, cols):
    m = _matrix(2, rows, cols, "bf16", 12)
    first = _run(m)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = _run(m)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, second)
    h = nb.Orthogonalizer(3, rows, cols)                       # more matrices than used
    out = torch.empty_like(first)
    h.run(m, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.run(m, out)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, out)
    h.close()


def test_a_lone_matrix_and_no_matrix():
    m = _matrix(1, 30, 50, "bf16", 13)
    h = nb.Orthogonalizer(2, 30, 50)
    out = torch.empty(30, 50, dtype=torch.bfloat16, device="cuda")
    h.run(m[0], out)
    assert torch.equal(out, _run(m)[0])
    h.run(m[:0], out.unsqueeze(0)[:0])
    assert h.status() == nb.NITRO_OK
    h.close()


def test_refusals():
    m = _matrix(2, 30, 50, "bf16", 14)
    out = torch.empty_like(m)
    h = nb.Orthogonalizer(1, 30, 50)
    for bad in (lambda: h.run(m, out),                                        # more matrices than the handle's
                lambda: h.run(m[0], out[0], steps=-1), lambda: h.run(m[0], out[0], steps=101),
                lambda: h.run(m[0], out[0], coef=(9.0, 0.0, 0.0)),            # a singular value would pass 8
                lambda: h.run(m[0], out[0], coef=(float("nan"), 0.0, 0.0))):
        with pytest.raises(nb.NitroError):
            bad()
    for bad in (lambda: h.run(m[0].half(), out[0]), lambda: h.run(m[0].t(), out[0].t()), lambda: h.run(m[0], out[0].float()),
                lambda: h.run(m[0, :29], out[0, :29]), lambda: h.run(m[0].t().contiguous().t(), out[0])):
        with pytest.raises(ValueError):
            bad()
    assert h.status() == nb.NITRO_OK
    h.close()

"""Microscaled 4-bit floating point: quantisation against its definition (exact), and the
product against 64 bits.

Product tolerance: products and scales are exact, the tensor cores add 64 at a time and
drop what 32 bits do not hold, each of ceil(K / 64) additions less than 2^-22 of the sum of
magnitudes, splits of K some more; bf16 rounds by at most 2^-8."""
import numpy as np
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu
VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _define(x):
    """(values, scales) of x [rows x cols] by the definition, in 64 bits."""
    x = x.double().cpu().numpy()
    rows, cols = x.shape
    blocks = -(-cols // 32)
    b = np.zeros((rows, blocks * 32))
    b[:, :cols] = x
    b = b.reshape(rows, blocks, 32)
    bad = ~np.isfinite(b).all(2)
    top = np.where(bad, 1.0, np.abs(np.where(np.isfinite(b), b, 0)).max(2))
    e = np.where(top > 0, np.frexp(np.where(top > 0, top, 1.0))[1] - 1 - 2, -127).clip(-127, 127)
    scale = np.ldexp(1.0, e)
    u = np.minimum(np.abs(np.where(np.isfinite(b), b, 0)) / scale[..., None], 6.0)
    d = np.abs(u[..., None] - VALUES)
    best = d.min(-1, keepdims=True)
    # of two codes as near, the even one
    code = np.where(d == best, np.arange(8) % 2 * 8 + np.arange(8), 99).min(-1) % 8
    v = np.copysign(VALUES[code], b) * scale[..., None]
    v[bad] = np.nan
    scale[bad] = np.nan
    return v.reshape(rows, -1)[:, :cols], scale


def _quantize(x):
    rows, cols = x.shape
    nq, ns = nb.mx4_bytes(rows, cols)
    q = torch.full((nq,), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full((ns,), 0xA5, dtype=torch.uint8, device="cuda")
    return nb.mx4_quantize(x, q, s)


def _round_trip(x, out="f32"):
    rows, cols = x.shape
    q, s = _quantize(x)
    v = torch.full((rows, cols), 9.0, dtype=DT[out], device="cuda")
    sv = torch.full((rows, -(-cols // 32)), 9.0, device="cuda")
    nb.mx4_dequantize(q, s, v, sv)
    return v, sv, q, s


def _same(a, b):
    return np.array_equal(a.double().cpu().numpy(), b, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, cols, pad", [(1, 1, 0), (1, 32, 0), (3, 31, 0), (2, 33, 0), (128, 128, 0), (129, 130, 8), (40, 1000, 3),
                                             (300, 64, 1), (17, 4100, 0)])
def test_round_trip(rows, cols, pad, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    x = torch.randn(rows, cols + pad, generator=g, device="cuda")
    x = (x * torch.exp2(torch.randint(-20, 20, (rows, 1), generator=g, device="cuda").float())).to(DT[dtype])[:, :cols]
    v, sv, q, s = _round_trip(x)
    want, scales = _define(x)
    assert _same(v, want) and _same(sv, scales)
    assert _same(_round_trip(x, "bf16")[0], want)
    # places past the last row, block and column hold zero
    blocks = -(-cols // 32)
    rt, bt = -(-rows // 128), -(-blocks // 4)
    t = s.view(rt, bt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, bt * 4)
    assert (t[rows:] == 0).all() and (t[:, blocks:] == 0).all()
    codes = torch.stack((q & 15, q >> 4), 1).view(rows, blocks * 32)
    assert (codes[:, cols:] == 0).all()


def test_ties_and_every_code():
    # with 6 in the block the scale is 1: the fifteen values, every tie, and what lies next to one
    ticks = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    vals = list(VALUES) + ticks + [t + d for t in ticks for d in (-2.0 ** -9, 2.0 ** -9)] + [6.0]
    x = torch.zeros(2, 64, device="cuda")
    x[0, : len(vals)] = torch.tensor(vals, device="cuda")
    x[0, 31] = x[0, 63] = 6.0
    x[1] = -x[0]
    v, sv, _, _ = _round_trip(x)
    want, scales = _define(x)
    assert (sv == 1.0).all() and _same(v, want) and _same(sv, scales)


def test_extreme_blocks():
    x = torch.zeros(9, 32, device="cuda")
    x[1] = 2.0 ** -149                              # the smallest subnormal
    x[2, 5] = 2.0 ** -126
    x[3] = 3.0e38                                   # values that saturate
    x[3, 0] = torch.finfo(torch.float32).max
    x[4, 3] = float("inf")
    x[5, 3] = float("nan")
    x[6, 3] = -float("inf")
    x[7, 0], x[7, 1] = 7.99, 1e-6                   # above 6 times the scale; far below it
    x[8] = -0.0
    v, sv, _, _ = _round_trip(x)
    want, scales = _define(x)
    assert _same(v, want) and _same(sv, scales)
    assert v[4:7].isnan().all() and not v[:4].isnan().any()


def _weights(n, k, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randn(n, k, generator=g, device="cuda") / k ** 0.5
    return _quantize(w), _define(w)[0]


def _linear(x, q, s, n, y="f32", out=None, h=None):
    own = h is None
    h = h or nb.Mx4Linear(x.shape[0], x.shape[1], n)
    out = torch.full((x.shape[0], n), float("nan"), dtype=DT[y], device="cuda") if out is None else out
    h.run(x, q, s, out)
    assert h.status() == nb.NITRO_OK
    if own:
        h.close()
    return out


def _check(x, y, wv):
    xv = torch.from_numpy(_define(x)[0]).cuda()
    wv = torch.from_numpy(wv).cuda()
    want, mag = xv @ wv.t(), xv.abs() @ wv.abs().t()
    tol = (-(-x.shape[1] // 64) + 16) * 2.0 ** -22 * mag + (2.0 ** -8 * want.abs() if y.dtype == torch.bfloat16 else 0)
    assert ((y.double() - want).abs() <= 1.01 * tol + 1e-30).all()


@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("rows, k, n", [(1, 1, 1), (1, 32, 127), (1, 4096, 1000), (2, 33, 129), (31, 64, 40), (33, 300, 257), (64, 1000, 128),
                                        (65, 1000, 130), (130, 96, 1000), (300, 2080, 513), (700, 544, 700), (1500, 256, 1300)])
def test_product(rows, k, n, y):
    g = torch.Generator(device="cuda").manual_seed(rows + k + n)
    x = torch.randn(rows, k, generator=g, device="cuda")
    x = (x * torch.exp(torch.randn(1, k, generator=g, device="cuda"))).to(DT["bf16" if rows % 2 else "f32"])
    (q, s), wv = _weights(n, k, 5)
    _check(x, _linear(x, q, s, n, y), wv)


@pytest.mark.parametrize("rows", [3, 50, 200])
@pytest.mark.parametrize("pad", [1, 8])
def test_strides(rows, pad):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, 200 + pad, generator=g, device="cuda").to(torch.bfloat16)[:, :200]
    (q, s), wv = _weights(150, 200, 6)
    for dt in ("bf16", "f32"):
        keep = torch.full((rows, 150 + pad), 7.0, dtype=DT[dt], device="cuda")
        out = _linear(x, q, s, 150, out=keep[:, :150])
        assert torch.equal(out, _linear(x.contiguous(), q, s, 150, dt)) and (keep[:, 150:] == 7).all()
    _check(x, out, wv)


@pytest.mark.parametrize("rows", [5, 100, 300])
def test_a_nan_stays_in_its_row_and_column(rows):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, 160, generator=g, device="cuda")
    w = torch.randn(140, 160, generator=g, device="cuda")
    clean = _linear(x, *_quantize(w), 140)
    x[3, 7] = float("inf")
    w[139, 40] = float("nan")
    y = _linear(x, *_quantize(w), 140)
    assert y[3].isnan().all() and y[:, 139].isnan().all()
    rest = torch.arange(rows, device="cuda") != 3
    assert torch.equal(y[rest, :139], clean[rest, :139])


def test_handle_kept_over_batches_streams_and_graphs():
    g = torch.Generator(device="cuda").manual_seed(9)
    (q, s), wv = _weights(600, 512, 7)
    h = nb.Mx4Linear(300, 512, 600)
    xs = [torch.randn(n, 512, generator=g, device="cuda") for n in (300, 1, 64, 150, 300)]
    first = [_linear(x, q, s, 600, h=h) for x in xs]
    for x, y in zip(xs, first):
        _check(x, y, wv)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = [_linear(x, q, s, 600, h=h) for x in xs]
    torch.cuda.current_stream().wait_stream(side)
    out = torch.empty(300, 600, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.run(xs[0], q, s, out)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(first + [first[0]], second + [out]):
        assert torch.equal(a, b)
    empty = torch.empty(0, 512, device="cuda")
    h.run(empty, q, s, torch.empty(0, 600, device="cuda"))
    assert h.status() == nb.NITRO_OK
    h.close()


def test_refusals():
    x = torch.zeros(4, 64, device="cuda")
    q, s = _quantize(x)
    h = nb.Mx4Linear(2, 64, 4)
    y = torch.empty(4, 4, device="cuda")
    with pytest.raises(nb.NitroError):
        h.run(x, q, s, y)                                       # more rows than the handle's
    for bad in (lambda: nb.mx4_quantize(x.half(), q, s), lambda: nb.mx4_quantize(x, q[:-1], s), lambda: nb.mx4_quantize(x, q, s[1:]),
                lambda: nb.mx4_quantize(x.t(), q, s), lambda: nb.mx4_dequantize(q, s, x.to(torch.int8)),
                lambda: h.run(x[:2], q, s, y[:2].half()), lambda: h.run(x[:2, :32], q, s, y[:2]), lambda: h.run(x[:2], q, s, y[:2, :3])):
        with pytest.raises(ValueError):
            bad()
    odd = torch.empty(q.numel() + 8, dtype=torch.uint8, device="cuda")[8:]
    with pytest.raises(nb.NitroError):
        nb.mx4_quantize(x, odd, s)                              # codes not 16-byte aligned
    h.close()


def test_extreme_blocks_in_bf16():
    x = torch.zeros(6, 32, dtype=torch.bfloat16, device="cuda")
    x[1] = 2.0 ** -133                              # the smallest subnormal
    x[2, 5], x[2, 6] = 2.0 ** -126, -2.0 ** -128
    x[3] = 3.0e38
    x[4, 3] = float("inf")
    x[5, 3] = float("nan")
    v, sv, _, _ = _round_trip(x)
    want, scales = _define(x)
    assert _same(v, want) and _same(sv, scales)
    # values down to 2^-128 are multiples of bf16's smallest
    assert _same(_round_trip(x, "bf16")[0], want)


@pytest.mark.parametrize("rows", [1, 2, 17, 32])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k, pad", [(40, 0), (255, 3), (513, 8), (3000, 1)])
def test_few_rows(rows, dtype, k, pad):
    # quantised inside the product: the same bits as quantised before it
    g = torch.Generator(device="cuda").manual_seed(rows + k)
    x = (torch.randn(rows, k + pad, generator=g, device="cuda") * 5).to(DT[dtype])[:, :k]
    (q, s), wv = _weights(300, k, 8)
    _check(x, _linear(x, q, s, 300), wv)

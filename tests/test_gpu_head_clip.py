"""The norm over many gradients, and clipping, against 64 bits.

Tolerances: a thread adds at most some thousand squares in 32 bits, (its count) 2^-24 of the sum at worst, under the root half of
it; the tests' threads add 4096 at most, so 2^-13 is the worst of a norm and 2^-20 what roundings that fall either
way leave of it with room (the root of the count); one of those more for the factor, and half a step of the type for each value."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu

BF, F32, I64 = torch.bfloat16, torch.float32, torch.int64


def grads(shapes, seed=0, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(*s, generator=g) * size).to(t).cuda() for s, t in shapes]


def true_norm(ts):
    return sum((t.double() ** 2).sum().item() for t in ts) ** 0.5


def check(ts, outs, norm, limit):
    want = true_norm(ts)
    assert abs(norm.item() - want) <= 2.0 ** -20 * want
    f = min(1.0, limit / want) if want > 0 else 1.0
    for t, o in zip(ts, outs):
        w = t.double() * f
        assert ((o.double() - w).abs() <= (torch.finfo(t.dtype).eps / 2 + 2.0 ** -20) * w.abs()).all()


def run(ts, limit, outs=None):
    outs = [torch.full_like(t, 9) for t in ts] if outs is None else outs
    op = nb.GradClip(ts, outs)
    norm = torch.empty((), device="cuda")
    op.run(norm, limit)
    assert op.status() == nb.NITRO_OK
    op.close()
    return outs, norm


SETS = [
    [((1,), F32)], [((1,), BF)], [((7, 3), BF), ((5,), F32)], [((1000, 1000), BF)], [((333, 1001), F32), ((1001,), BF), ((2, 3, 4, 5), F32)],
    [((k,), (BF, F32)[k % 2]) for k in range(1, 90)], [((3000, 1700), F32), ((4096, 3001), BF), ((256,), F32)],
]


@pytest.mark.parametrize("shapes", SETS)
@pytest.mark.parametrize("limit", [0.3, 1e6])
def test_sets(shapes, limit):
    ts = grads(shapes, seed=len(shapes))
    outs, norm = run(ts, limit)
    check(ts, outs, norm, limit)
    if limit > norm.item():
        assert all(torch.equal(t, o) for t, o in zip(ts, outs))
    again, norm2 = run(ts, limit)
    assert torch.equal(norm, norm2) and all(torch.equal(a, b) for a, b in zip(outs, again))
    place = [t.clone() for t in ts]
    run(place, limit, place)
    assert all(torch.equal(a, b) for a, b in zip(outs, place))


def test_norm_alone_of_every_type():
    ts = grads([((100, 30), BF), ((77,), F32)], size=1e3) + [torch.arange(-5000, 5001, device="cuda") * 1000003]
    op = nb.GradClip(ts)
    norm = torch.empty(1, device="cuda")
    op.run(norm)
    assert abs(norm.item() - true_norm(ts)) <= 2.0 ** -20 * true_norm(ts)
    with pytest.raises(nb.NitroError):
        op.run(norm, 1.0)          # none is written
    op.close()


def test_some_are_counted_and_not_written():
    ts = grads([((100, 30), BF), ((77,), F32), ((64, 64), F32)]) + [torch.arange(50, device="cuda")]
    outs = [torch.empty_like(ts[0]), None, torch.empty_like(ts[2]), None]
    _, norm = run(ts, 1.0, outs)
    f = 1.0 / true_norm(ts)
    for k in (0, 2):
        assert ((outs[k].double() - ts[k].double() * f).abs() <= (torch.finfo(ts[k].dtype).eps / 2 + 2.0 ** -20) * (ts[k].double() * f).abs()).all()


@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("rows, cols, ld", [(40, 33, 40), (5, 5000, 5003), (3000, 3, 8), (9, 64, 72), (1, 7, 9), (700, 1, 5), (2000, 1000, 1003), (3, 400001, 400009),
                                            (50000, 7, 9), (300, 129, 1000), (20000, 5, 6), (777, 2048, 2049)])
def test_matrices_in_wider_buffers(rows, cols, ld, t):
    src, dst = grads([((rows, ld), t), ((rows, ld + 3), t)], seed=rows)
    keep = dst.clone()
    outs, norm = run([src[:, 1: 1 + cols]], 0.5, [dst[:, 2: 2 + cols]])
    check([src[:, 1: 1 + cols]], outs, norm, 0.5)
    keep[:, 2: 2 + cols] = dst[:, 2: 2 + cols]
    assert torch.equal(keep, dst)          # what lies between the rows stays as it was
    # in place, and into one without gaps
    place, flat = src.clone(), torch.empty(rows, cols, dtype=t, device="cuda")
    run([place[:, 1: 1 + cols]], 0.5, [place[:, 1: 1 + cols]])
    run([src[:, 1: 1 + cols]], 0.5, [flat])
    assert torch.equal(place[:, 1: 1 + cols], outs[0]) and torch.equal(flat, outs[0])
    place[:, 1: 1 + cols] = src[:, 1: 1 + cols]
    assert torch.equal(place, src)


def test_columns_of_one_buffer():
    buf = grads([((50, 64), F32)])[0]
    want = buf.double() * (0.7 / true_norm([buf]))
    parts = [buf[:, :10], buf[:, 10:11], buf[:, 11:40], buf[:, 40:]]
    run(parts, 0.7, parts)
    assert ((buf.double() - want).abs() <= 2.0 ** -20 * want.abs()).all()


@pytest.mark.parametrize("offset", [1, 3])
def test_buffers_that_start_anywhere(offset):
    a, b = grads([((70001,), BF), ((70001,), BF)])
    outs, norm = run([a[offset:]], 0.5, [b[: 70001 - offset]])
    check([a[offset:]], outs, norm, 0.5)


def test_no_gradients_and_empty_ones():
    norm = torch.full((), 3.0, device="cuda")
    for ts in ([], [torch.empty(0, 5, device="cuda"), torch.empty(0, device="cuda", dtype=BF)]):
        op = nb.GradClip(ts, ts)
        op.run(norm)
        assert norm.item() == 0.0
        op.close()
    ts = [torch.zeros(100, device="cuda")]
    outs, norm = run(ts, 0.5)
    assert norm.item() == 0.0 and (outs[0] == 0).all()


@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e-19, 1e18, 1e25, 1e37])
def test_ranges_past_the_squares(size, t):
    ts = grads([((300, 50), t), ((33,), F32)], size=size)
    limit = 0.25 * size
    outs, norm = run(ts, limit)
    want = true_norm(ts)
    if want < 3e38:
        assert abs(norm.item() - want) <= 2.0 ** -20 * want
    else:
        assert norm.item() == float("inf")
    f = limit / want
    for a, o in zip(ts, outs):
        w = a.double() * f
        # (values below 2^-126 are spaced 2^-149 in fp32 and 2^-133 in bf16)
        tiny = 2.0 ** -133 if t == BF else 2.0 ** -149
        assert ((o.double() - w).abs() <= (torch.finfo(a.dtype).eps / 2 + 2.0 ** -20) * w.abs() + tiny).all()


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_not_finite(bad):
    ts = grads([((300, 50), F32), ((33,), BF)])
    ts[0][3, 4] = bad
    outs, norm = run(ts, 0.5)
    assert not norm.isfinite().item()
    assert all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(ts, outs))


def test_values_change_between_runs_and_replays():
    ts = grads([((300, 500), F32), ((33, 7), BF)])
    outs = [torch.empty_like(t) for t in ts]
    op = nb.GradClip(ts, outs)
    norm = torch.empty((), device="cuda")
    for k in (1.0, 5.0, 0.01):
        ts[0].mul_(k)
        op.run(norm, 0.5)
        check(ts, outs, norm, 0.5)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        op.run(norm, 0.25)
    for k in (100.0, 0.5, 1e-4):
        ts[1].mul_(k)
        graph.replay()
        torch.cuda.synchronize()
        check(ts, outs, norm, 0.25)
    op.close()


def test_captured_first():
    ts = grads([((300, 500), F32)])
    outs = [torch.empty_like(ts[0])]
    op = nb.GradClip(ts, outs)
    norm = torch.empty((), device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        op.run(norm, 0.25)
    op.run(norm, 0.5)
    check(ts, outs, norm, 0.5)
    graph.replay()
    torch.cuda.synchronize()
    check(ts, outs, norm, 0.25)
    op.close()


def test_refusals():
    a, b = grads([((8, 8), F32), ((8, 8), F32)])
    for ins, outs in (([a, a], [a, None]), ([a, b], [b, a]), ([a[:4], a[3:]], [a[:4], a[3:]]), ([a[:4]], [a[1:5]]),
                      ([a.expand(8, 8)[:, :1].expand(8, 8)[:, :1].t().expand(8, 8)], None)):
        with pytest.raises((nb.NitroError, ValueError)):
            nb.GradClip(ins, outs)
    for ins, outs in (([a.to(torch.float16)], None), ([a], [b.to(BF)]), ([a], [b[:4]]), ([a.t()[:, ::2]], None), ([a], [a, b])):
        with pytest.raises(ValueError):
            nb.GradClip(ins, outs)
    op = nb.GradClip([a], [b])
    norm = torch.empty((), device="cuda")
    for limit in (0.0, -1.0, float("nan")):
        with pytest.raises(ValueError):
            op.run(norm, limit)
    op.close()

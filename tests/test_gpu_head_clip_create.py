"""Clipping handles made while the default stream is busy: creation does not wait for it, and the handle runs at once on another."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu


def make(count, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ts = [torch.randn(1 + 977 * k, generator=g, device="cuda").to((torch.bfloat16, torch.float32)[k % 2]) for k in range(count)]
    want = sum(t.double().square().sum().item() for t in ts) ** 0.5
    return ts, [torch.empty_like(t) for t in ts], torch.empty((), device="cuda"), want


def check(ts, outs, norm, want, limit):
    assert abs(norm.item() - want) <= 2.0 ** -20 * want
    for t, o in zip(ts, outs):
        w = t.double() * min(1.0, limit / want)
        assert ((o.double() - w).abs() <= (torch.finfo(t.dtype).eps / 2 + 2.0 ** -20) * w.abs()).all()


@pytest.mark.parametrize("count", [1, 40, 3000])
def test_made_beside_a_busy_stream(count):
    ts, outs, norm, want = make(count if count < 100 else 100, count)
    if count > 100:           # many pieces: a table of some hundred kilobytes
        cut = [(i, i + 50) for i in range(0, 50 * (count - 100), 50)]
        big = torch.zeros(cut[-1][1], device="cuda")
        ts, outs = ts + [big[a:b] for a, b in cut], outs + [torch.empty(b - a, device="cuda") for a, b in cut]
    side = torch.cuda.Stream()
    op = nb.GradClip(ts, outs)            # (the first launch of a process loads the kernel, which may wait)
    op.run(norm, 0.25, stream=side)
    op.close()
    torch.cuda.synchronize()
    torch.cuda._sleep(1 << 30)            # half a second, on the default stream
    op = nb.GradClip(ts, outs)
    assert not torch.cuda.default_stream().query()
    op.run(norm, 0.25, stream=side)
    op.run(norm, 0.5, stream=side)
    side.synchronize()                    # (a grid of all SMs waits for the one that is busy)
    check(ts, outs, norm, want, 0.5)
    op.run(norm, 0.25)
    check(ts, outs, norm, want, 0.25)
    op.close()


def test_captured_first_and_replayed_around_other_runs():
    ts, outs, norm, want = make(30, 1)
    op = nb.GradClip(ts, outs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for limit in (0.25, 0.125):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            op.run(norm, limit)
    for graph, limit in ((graphs[1], 0.125), (graphs[0], 0.25)):
        graph.replay()
        torch.cuda.synchronize()
        check(ts, outs, norm, want, limit)
    op.run(norm, 0.5)
    check(ts, outs, norm, want, 0.5)
    for graph, limit in ((graphs[0], 0.25), (graphs[1], 0.125), (graphs[0], 0.25)):
        graph.replay()
        torch.cuda.synchronize()
        check(ts, outs, norm, want, limit)
    assert op.status() == nb.NITRO_OK
    op.close()

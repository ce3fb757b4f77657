"""Group norm, the gated block, cross entropy, clipping and the orthogonal update together, as a head on a block's maps.

Tolerance of a gradient, in norm: the maps' y, the block's h, the cross entropy's G, the block's D and dh are rounded to bf16, each by
at most 2^-8 of itself, and so is the gradient: six of those, 0.024.  The reference takes no rounding but the weights'."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb
from paper_2407_11698_gb300.many_class import GatedHead, demo

pytestmark = pytest.mark.gpu

N, P, C, G, H, V = 37, 16, 24, 4, 72, 301


def _data(n=N, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, P, C, generator=g) * 30 * torch.exp(0.3 * torch.randn(C, generator=g))).round().clamp(-127, 127).to(torch.int8)
    labels = torch.randint(0, V, (n,), generator=g).to(torch.int32)
    labels[::7] = -1
    return x.cuda(), labels.cuda()


def _reference(head, x, labels):
    leaves = [t.double().requires_grad_() for t in (head.w[0], head.w[1], head.gamma, head.beta)]
    w1, w2, gamma, beta = leaves
    n = x.shape[0]
    v = x.double().view(n, P, G, C // G)
    v = v - v.mean(dim=(1, 3), keepdim=True)
    v = (v / (v.square().mean(dim=(1, 3), keepdim=True) + 1e-5).sqrt()).view(n, P, C)
    u = gamma * v + beta
    y = (u * torch.sigmoid(u)).view(n, P * C)
    z = y @ w1.t()
    h = z[:, :H] * torch.sigmoid(z[:, :H]) * z[:, H:]
    live = labels >= 0
    loss = torch.logsumexp(h @ w2.t(), dim=1) - (h @ w2.t())[torch.arange(n), labels.clamp(min=0).long()]
    loss = loss * live
    return loss.detach(), torch.autograd.grad(loss.sum() / live.sum(), leaves)


def _close(a, b, tol):
    return (a.double() - b).norm() <= tol * b.norm()


def test_gradients_of_the_whole():
    head = GatedHead(P, C, G, H, V, N)
    head.gamma.copy_(1 + 0.1 * torch.randn(C, device="cuda"))
    head.beta.copy_(0.1 * torch.randn(C, device="cuda"))
    x, labels = _data()
    loss, _ = head.gradients(x, labels)
    want, grads = _reference(head, x, labels)
    assert ((loss.double() - want).abs() <= 0.024 * want.abs().max()).all()
    for got, ref in zip(head.dw + [head.dgamma, head.dbeta], grads):
        assert _close(got, ref, 0.024)
    assert head.status() == nb.NITRO_OK
    head.close()


@pytest.mark.parametrize("max_norm", [0.05, 1e4])
def test_step_clips_all_gradients_together(max_norm):
    head = GatedHead(P, C, G, H, V, N, max_norm=max_norm)
    x, labels = _data(seed=1)
    head.gradients(x, labels)
    before = [t.clone() for t in head.dw + [head.dgamma, head.dbeta]]
    norm = sum(t.double().square().sum() for t in before).sqrt()
    assert max_norm == 1e4 or norm > max_norm
    head.step(x, labels)
    assert abs(head.norm.item() - norm) <= 2.0 ** -20 * norm
    f = min(1.0, max_norm / norm.item())
    for t, b in zip(head.dw + [head.dgamma, head.dbeta], before):
        assert ((t.double() - b.double() * f).abs() <= (torch.finfo(t.dtype).eps / 2 + 2.0 ** -20) * f * b.double().abs()).all()
    assert head.status() == nb.NITRO_OK
    head.close()


def test_batches_of_all_sizes_and_serving():
    head = GatedHead(P, C, G, H, V, N)
    for n in (N, 1, 3, 20):
        x, labels = _data(n, seed=n)
        labels[0] = 5
        loss = head.step(x, labels)
        assert loss.isfinite().item()
        # what is served is the product of the same hidden values in 4 bits
        h = head._hidden(x, False)[0]
        served = head.serve(x)
        got = torch.empty_like(served)
        head.serve_op.run(h, head.q, head.s, got)
        assert torch.equal(got, served) and served.shape == head.logits(x).shape
    assert head.status() == nb.NITRO_OK
    head.close()


def test_a_step_captured_and_replayed():
    a, b = GatedHead(P, C, G, H, V, N, seed=4), GatedHead(P, C, G, H, V, N, seed=4)
    x, labels = _data(seed=2)
    for _ in range(4):
        a.step(x, labels)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.step(x, labels)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step(x, labels)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for t, u in zip(a.masters + [a.gamma, a.beta, a.norm], b.masters + [b.gamma, b.beta, b.norm]):
        assert torch.equal(t, u)
    a.close()
    b.close()


def test_demo_runs():
    first, last, acc, acc4 = demo(steps=6, batch=32, classes=100, log=lambda *_: None, gated=True)
    assert all(abs(v) < float("inf") for v in (first, last, acc, acc4))

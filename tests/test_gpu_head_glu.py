"""The gated block against its definition in 64 bits.

Tolerances.  A sum of K products is off by (K / 8 + 16) 2^-23 of the sum A of its terms' sizes: the tensor cores add 16
products at a time and cut off, twice at most; the CUDA cores round, less often.  z is a sum over the features.  |act'| and |act''| are below 1.2, so
out = act(a) b is off by 1.2 |b| dz + |act(a)| dz and 2^-20 of its terms for the activation's own roundings, D accordingly; D is rounded
to bf16, 2^-8 of it (2^-16 where it is kept as two halves), and each output by 2^-8 of itself."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb
from test_gpu_head_gnorm import ACT, smooth

pytestmark = pytest.mark.gpu


def view(t, pad):
    wide = torch.full((t.shape[0], t.shape[1] + pad), 77, dtype=t.dtype, device=t.device)
    wide[:, : t.shape[1]] = t
    return wide[:, : t.shape[1]]


def inputs(n, f, h, x="bf16", pad=0, seed=0):
    g = torch.Generator().manual_seed(seed)
    v = torch.randn(n, f, generator=g)
    scale = 1.0
    if x == "i8":
        v, scale = (v * 32).round().clamp(-127, 127).to(torch.int8), 1 / 32
    else:
        v = v.to(torch.bfloat16)
    w = (torch.randn(2 * h, f, generator=g) * 1.5 / f ** 0.5).to(torch.bfloat16)
    dout = (torch.randn(n, h, generator=g) * 1e-2).to(torch.bfloat16)
    return view(v.cuda(), pad), view(w.cuda(), pad), view(dout.cuda(), pad), scale


def run(x, w, dout, scale, act, op=None, grads=(True, True), pad=0):
    n, f, h = x.shape[0], x.shape[1], dout.shape[1]
    own = op is None
    op = nb.GatedLinear(max(1, n), f, h) if own else op
    bf = dict(dtype=torch.bfloat16, device="cuda")
    out = view(torch.full((n, h), 5, **bf), pad)
    saved = torch.full((n, 2 * h), 5.0, device="cuda")
    dx = view(torch.full((n, f), 5, **bf), pad) if grads[0] else None
    dw = view(torch.full((2 * h, f), 5, **bf), pad) if grads[1] else None
    op.forward(x, w, out, saved, act=ACT[act], scale=scale)
    op.backward(x, w, saved, dout, dx, dw, act=ACT[act], scale=scale)
    assert op.status() == nb.NITRO_OK
    if own:
        op.close()
    return out, saved, dx, dw


def unfold(saved, n, h):
    """z from saved: lines of 16 gates and their ups for each row, by blocks of 16 units, then what is left of the units."""
    whole = h // 16 * 16
    a = saved[: n * 2 * whole].view(h // 16, n, 2, 16).permute(1, 2, 0, 3).reshape(n, 2, whole)
    b = saved[n * 2 * whole:].view(n, 2, h - whole)
    return torch.cat((a, b), dim=2).reshape(n, 2 * h)


def check(x, w, dout, scale, act, out, saved, dx, dw):
    n, h = dout.shape
    xd, wd, g = x.double(), w.double(), dout.double()
    err = lambda k: (k / 8 + 16) * 2.0 ** -23
    half = 2.0 ** -8
    z = (xd @ wd.t() * scale).requires_grad_()
    ref = smooth(z[:, :h], act) * z[:, h:]
    D = torch.autograd.grad(ref, z, g)[0] if n else z.detach()
    with torch.no_grad():
        z = z.detach()
        dz = err(x.shape[1]) * (xd.abs() @ wd.abs().t() * scale) + 2.0 ** -23 * z.abs()
        a, b, da, db = z[:, :h], z[:, h:], dz[:, :h], dz[:, h:]
        ok = lambda got, want, tol: ((got.double() - want).abs() <= tol).all()
        assert ok(unfold(saved.reshape(-1), n, h), z, dz)
        assert ok(out, ref, half * ref.abs() + 1.2 * b.abs() * da + (a.abs() + 0.1) * db + 2.0 ** -20 * (a * b).abs())
        low = half if n > 32 else half * half
        dD = torch.cat((g, g), dim=1).abs() * torch.cat((1.2 * (b.abs() * da + db) + 2.0 ** -20 * b.abs(), 1.2 * da + 2.0 ** -20 * a.abs()), dim=1)
        if act == "relu":      # a gate within its error of the slope's jump may take either side of it
            dD[:, :h] += g.abs() * b.abs() * (a.abs() <= da)
        dD = dD + low * D.abs()
        if dx is not None:
            t = D @ wd * scale
            assert ok(dx, t, half * t.abs() + scale * ((dD + err(2 * h) * D.abs()) @ wd.abs()))
        if dw is not None:
            t = D.t() @ xd * scale
            assert ok(dw, t, half * t.abs() + scale * ((dD + err(n) * D.abs()).t() @ xd.abs()))


# one row and few (CUDA cores), up to and past 32 (halves of D), tiles that end anywhere, several splits and tiles a CTA
SIZES = [(1, 1, 1), (6, 257, 50), (16, 1000, 301), (10, 2049, 33), (1, 4096, 300), (2, 33, 7), (3, 1000, 1501), (4, 600, 24), (5, 600, 24), (13, 1000, 501), (32, 72, 40), (33, 72, 40), (64, 4096, 100),
         (129, 65, 130), (300, 200, 1366), (1000, 24, 16), (257, 2500, 90), (700, 520, 2000)]


@pytest.mark.parametrize("x", ["bf16", "i8"])
@pytest.mark.parametrize("act", ["silu", "gelu", "none"])
@pytest.mark.parametrize("n, f, h", SIZES)
def test_sizes(n, f, h, act, x):
    t = inputs(n, f, h, x, seed=n + f + h)
    out = run(*t, act)
    check(*t, act, *out)
    assert all(torch.equal(a, b) for a, b in zip(out, run(*t, act)))


@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("pad", [3, 4, 8])
@pytest.mark.parametrize("n, f, h", [(3, 40, 9), (20, 41, 36), (70, 104, 33)])
def test_strides(n, f, h, pad, act):
    t = inputs(n, f, h, "i8" if pad == 4 else "bf16", pad, seed=7 + pad)
    out = run(*t, act, pad=pad)
    check(*t, act, *out)
    for o in (out[0], out[2], out[3]):      # what lies between the rows stays as it was
        assert (o.as_strided((o.shape[0], pad), o.stride(), o.storage_offset() + o.shape[1]) == 77).all()


@pytest.mark.parametrize("offset", [1, 4])
@pytest.mark.parametrize("n", [2, 50])
def test_buffers_that_start_anywhere(n, offset):
    t = list(inputs(n, 64, 48, seed=5))
    for i in range(3):
        buf = torch.zeros(t[i].numel() + offset, dtype=t[i].dtype, device="cuda")
        buf[offset:] = t[i].reshape(-1)
        t[i] = buf[offset:].view(t[i].shape)
    check(*t, "silu", *run(*t, "silu"))


@pytest.mark.parametrize("grads", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("n", [3, 40])
def test_gradients_that_are_not_wanted(n, grads):
    t = inputs(n, 100, 60, "i8", seed=3)
    check(*t, "silu", *run(*t, "silu", grads=grads))


@pytest.mark.parametrize("n", [1, 4, 30, 200])
def test_forward_without_saved(n):
    x, w, dout, scale = inputs(n, 300, 77, seed=3)
    want = run(x, w, dout, scale, "silu")[0]
    op = nb.GatedLinear(n, 300, 77)
    out = torch.empty_like(want)
    op.forward(x, w, out, act=nb.NITRO_ACT_SILU, scale=scale)
    assert torch.equal(out, want)
    op.close()


def test_empty_batch_and_smaller_ones():
    x, w, dout, scale = inputs(90, 72, 40, seed=3)
    op = nb.GatedLinear(90, 72, 40)
    for pad in (0, 3):
        out, saved, dx, dw = run(x[:0], w, dout[:0], scale, "silu", op, pad=pad)
        assert (dw == 0).all()
    for n in (90, 1, 17, 50):
        check(x[:n], w, dout[:n], scale, "silu", *run(x[:n], w, dout[:n], scale, "silu", op))
    op.close()


def test_far_arguments():
    """Gates of any size: act(a) is a or 0 far from 0, and no exponential's range makes a NaN."""
    n, f, h = 64, 16, 32
    for rows in (2, 64):
        x, w, dout, scale = inputs(n, f, h, seed=4)
        x = x[:rows] * torch.logspace(-3, 4, rows, device="cuda").to(torch.bfloat16)[:, None]
        for act in ("silu", "gelu"):
            out = run(x, w, dout[:rows], scale, act)
            check(x, w, dout[:rows], scale, act, *out)


def test_nan_stays_in_its_row():
    x, w, dout, scale = inputs(40, 64, 32, seed=4)
    want = list(run(x, w, dout, scale, "silu"))
    x[7, 3] = float("nan")
    got = run(x, w, dout, scale, "silu")
    for t in (want, got):
        t[1].copy_(unfold(t[1].reshape(-1), 40, 32))
    for i in (0, 1, 2):
        assert got[i][7].isnan().all() and torch.equal(got[i][:7], want[i][:7]) and torch.equal(got[i][8:], want[i][8:])
    assert got[3].isnan().all()


def test_gradients_against_differences():
    n, f, h = 3, 8, 4
    x, w, dout, scale = inputs(n, f, h, seed=1)
    out, saved, dx, dw = run(x, w, dout, scale, "gelu")
    xd, wd = x.double().cpu(), w.double().cpu()

    def loss(x, w):
        z = x @ w.t()
        return (smooth(z[:, :h], "gelu") * z[:, h:] * dout.double().cpu()).sum().item()

    step = 1e-4
    for t, grad, pos in ((0, dx, (1, 3)), (0, dx, (2, 7)), (1, dw, (1, 2)), (1, dw, (6, 5))):
        v = []
        for s in (step, -step):
            args = [xd.clone(), wd.clone()]
            args[t][pos] += s
            v.append(loss(*args))
        want = (v[0] - v[1]) / (2 * step)
        # bf16 of the result, and its sums' terms (eight of 1e-2 times a few)
        assert abs(want - grad[pos].item()) < 2.0 ** -8 * abs(want) + 1e-6


@pytest.mark.parametrize("n", [1, 100])
def test_captured_and_replayed_on_another_stream(n):
    x, w, dout, scale = inputs(n, 200, 64, "i8", seed=5)
    want = run(x, w, dout, scale, "silu")
    op = nb.GatedLinear(n, 200, 64)
    got = [torch.empty_like(t) for t in want]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        op.forward(x, w, got[0], got[1], scale=scale)
        op.backward(x, w, got[1], dout, got[2], got[3], scale=scale)
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    op.close()


def test_refusals():
    x, w, dout, scale = inputs(4, 16, 8)
    op = nb.GatedLinear(3, 16, 8)
    out, saved = torch.empty_like(dout), torch.empty(4, 16, device="cuda")
    for bad in (lambda: op.forward(x, w, out), lambda: op.forward(x[:2], w, out[:2], act=4), lambda: op.forward(x[:2], w, out[:2], act=-1),
                lambda: op.forward(x[:2], w, out[:2], scale=0.0), lambda: op.forward(x[:2], w, out[:2], scale=float("nan")),
                lambda: op.forward(x[:2], w, out[:2], scale=2e30), lambda: op.backward(x, w, saved, dout, x, w)):
        with pytest.raises(nb.NitroError):
            bad()
    for bad in (lambda: op.forward(x[:2].float(), w, out[:2]), lambda: op.forward(x[:2], w[:8], out[:2]), lambda: op.forward(x[:2], w, out[:2].float()),
                lambda: op.forward(x[:2], w.float(), out[:2]), lambda: op.forward(x[:2], w, out[:2], saved), lambda: op.forward(x[:2, :8], w, out[:2]),
                lambda: op.backward(x[:2], w, saved[:2], dout[:2].float(), x[:2], w),
                lambda: op.backward(x[:2], w, saved[:2].to(torch.bfloat16), dout[:2], x[:2], w)):
        with pytest.raises(ValueError):
            bad()
    op.close()

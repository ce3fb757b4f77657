"""Group norm with an activation against its definition in 64 bits.

Tolerances.  e = 2^-24.  A thread's sums run over at most n of its values, CTAs' parts are joined in trees, so mean and
variance are off by (n + 32) e of the mean distance to a thread's first value: of the spread, times up to 4 for normal
values.  x - m is rounded where |m| is many times the spread: h is off by K e (4 + |m| r) (1 + |h|) with K = n + 64, which
holds the roundings of u and of the activation (its exponential's argument is rounded: |u| e) as well; |act'| and |act''| are
below 1.2.  An output's rounding is half a step of its type.  Sums over values add (n + 64) e of the sum of absolute
terms."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
DT = {"i8": torch.int8, "bf16": torch.bfloat16, "f32": torch.float32}
ACT = {"none": nb.NITRO_ACT_NONE, "relu": nb.NITRO_ACT_RELU, "silu": nb.NITRO_ACT_SILU, "gelu": nb.NITRO_ACT_GELU}


def smooth(u, act):
    if act == "relu":
        return torch.clamp(u, min=0)
    if act == "silu":
        return u * torch.sigmoid(u)
    if act == "gelu":
        return u * torch.special.ndtr(u)
    return u


def view(t, pad):
    wide = torch.full((*t.shape[:-1], t.shape[-1] + pad), 77, dtype=t.dtype, device=t.device)
    wide[..., : t.shape[-1]] = t
    return wide[..., : t.shape[-1]]


def inputs(n, p, c, x="bf16", y="bf16", pad=0, seed=0, level=0.7):
    g = torch.Generator().manual_seed(seed)
    v = torch.randn(n, p, c, generator=g) * torch.exp(0.4 * torch.randn(c, generator=g)) + level * torch.randn(c, generator=g)
    if x == "i8":
        v = (v * 30).round().clamp(-127, 127)
    dy = torch.randn(n, p, c, generator=g) * 1e-2
    gamma, beta = 1 + 0.2 * torch.randn(c, generator=g), 0.2 * torch.randn(c, generator=g)
    return view(v.to(DT[x]).cuda(), pad), view(dy.to(DT[y]).cuda(), pad), gamma.cuda(), beta.cuda()


def run(x, dy, gamma, beta, groups, eps, act, h=None, grads=(True, True, True), pad=0):
    n, p, c = x.shape
    own = h is None
    h = nb.GroupNorm(max(1, n), p, c, groups) if own else h
    y = view(torch.full(dy.shape, 5, dtype=dy.dtype, device="cuda"), pad)
    dx = view(torch.full(dy.shape, 5, dtype=dy.dtype, device="cuda"), pad) if grads[0] else None
    mean, rstd = torch.empty(n, groups, device="cuda"), torch.empty(n, groups, device="cuda")
    dg, db = (torch.full((c,), 3.0, device="cuda") if k else None for k in grads[1:])
    h.forward(x, gamma, beta, y, mean, rstd, eps=eps, act=ACT[act])
    h.backward(x, gamma, beta, mean, rstd, dy, dx, dg, db, act=ACT[act])
    assert h.status() == nb.NITRO_OK
    if own:
        h.close()
    return y, mean, rstd, dx, dg, db


def steps(p, c):
    """The most values of a channel that one thread adds up: threads take vectors of one to eight channels, a CTA of
    256 threads eight steps at least, one of 1216 CTAs' share at most."""
    vecs = min(256, c)
    rows = 256 // vecs
    return max(8, p // rows) + 8


def check(x, dy, gamma, beta, groups, eps, act, y, mean, rstd, dx, dg, db):
    n, p, c = x.shape
    xd = x.double().requires_grad_()
    gd = (torch.ones(c, device="cuda") if gamma is None else gamma).double().requires_grad_()
    bd = (torch.zeros(c, device="cuda") if beta is None else beta).double().requires_grad_()
    v = xd.reshape(n, p, groups, -1)
    m = v.mean(dim=(1, 3), keepdim=True)
    r = ((v - m) ** 2).mean(dim=(1, 3), keepdim=True).add(eps).rsqrt()
    hh = ((v - m) * r).reshape(n, p, c)
    u = gd * hh + bd
    ref = smooth(u, act)
    rx, rg, rb = torch.autograd.grad(ref, (xd, gd, bd), dy.double())
    with torch.no_grad():
        K = steps(p, c) + 64
        lean = (4 + (m.abs() * r)).expand(n, p, groups, c // groups).reshape(n, p, c)
        dh = K * E * lean * (1 + hh.abs())                    # of h
        du = dh * gd.abs() + 8 * E * (u.abs() + bd.abs())     # of u
        half = torch.finfo(dy.dtype).eps / 2
        ok = lambda got, want, tol: ((got.double() - want).abs() <= tol).all()
        assert ok(mean, m.reshape(n, groups), (K * E * (4 / r + m.abs())).reshape(n, groups))
        assert ok(rstd, r.reshape(n, groups), (K * E * 8 * r).reshape(n, groups))
        assert ok(y, ref, half * ref.abs() + 1.2 * du + 16 * E * u.abs())
        t = 1.2 * dy.double().abs()                            # bounds du dy and what it is off by
        td = dy.double().abs() * (1.2 * du + 16 * E)
        if act == "relu":      # a u within its error of the slope's jump may take either side of it
            td = td + dy.double().abs() * (u.abs() <= du)
        terms = (K + 64) * E * (t * (1 + hh.abs())).sum(dim=(0, 1))
        if db is not None:
            assert ok(db, rb, terms + td.sum(dim=(0, 1)))
        if dg is not None:
            assert ok(dg, rg, terms + (td * hh.abs() + t * dh).sum(dim=(0, 1)))
        if dx is not None:
            grp = lambda a: a.reshape(n, p, groups, -1).mean(dim=(1, 3), keepdim=True).expand(n, p, groups, c // groups).reshape(n, p, c)
            ga = gd.abs()
            e1 = grp(ga * td) + (K + 64) * E * grp(ga * t)
            e2 = grp(ga * (td * hh.abs() + t * dh)) + (K + 64) * E * grp(ga * t * hh.abs())
            rr = r.expand(n, p, groups, c // groups).reshape(n, p, c)
            whole = ga * t + grp(ga * t) + hh.abs() * grp(ga * t * hh.abs())
            tol = half * rx.abs() + rr * (ga * td + e1 + hh.abs() * e2 + dh * grp(ga * t * hh.abs()) + 8 * K * E * whole)
            assert ok(dx, rx, tol)


# vectors of eight, of four, and single channels; groups of one channel, of some, of all; more channels than a CTA takes
# at once; one pixel; chunks of odd lengths
SIZES = [(1, 64, 256, 32), (3, 7, 8, 8), (2, 1, 64, 2), (5, 33, 100, 5), (1, 1000, 36, 4), (2, 50, 33, 11), (1, 17, 1, 1), (2, 9, 2056, 4),
         (1, 5, 2050, 2), (1, 20, 4100, 1), (70, 20, 16, 16), (1, 9001, 24, 3), (1, 3, 8192, 8)]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("x, y", [("i8", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("i8", "f32")])
@pytest.mark.parametrize("n, p, c, groups", SIZES)
def test_sizes_and_types(n, p, c, groups, x, y, act):
    t = inputs(n, p, c, x, y, seed=p + c)
    out = run(*t, groups, 1e-5, act)
    check(*t, groups, 1e-5, act, *out)
    again = run(*t, groups, 1e-5, act)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("pad", [3, 4, 8])
@pytest.mark.parametrize("n, p, c, groups", [(2, 30, 40, 5), (3, 11, 52, 4)])
def test_strides(n, p, c, groups, pad, act):
    t = inputs(n, p, c, pad=pad, seed=12 + pad)
    out = run(*t, groups, 1e-3, act, pad=pad)
    check(*t, groups, 1e-3, act, *out)
    for o in (out[0], out[3]):          # what lies between the rows stays as it was
        rest = o.as_strided((n, p, pad), o.stride(), o.storage_offset() + c)
        assert (rest == 77).all()


@pytest.mark.parametrize("offset", [1, 2, 4])
def test_buffers_that_start_anywhere(offset):
    n, p, c, groups = 2, 21, 32, 4
    t = list(inputs(n, p, c, seed=5))
    for i in (0, 1):
        buf = torch.zeros(t[i].numel() + offset, dtype=t[i].dtype, device="cuda")
        buf[offset:] = t[i].reshape(-1)
        t[i] = buf[offset:].view(n, p, c)
    check(*t, groups, 1e-5, "silu", *run(*t, groups, 1e-5, "silu"))


# vectors of eight and of four values in rows that start anywhere: in one pass and in two, groups of whole vectors and of parts of
# them, the last row at the buffer's end, and outputs that are aligned although the inputs are not
@pytest.mark.parametrize("out_pad", [0, 1])
@pytest.mark.parametrize("pad", [1, 2, 5])
@pytest.mark.parametrize("x, y", [("i8", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("i8", "f32")])
@pytest.mark.parametrize("n, p, c, groups", [(3, 50, 64, 8), (2, 33, 48, 4), (1, 1, 8, 1), (1, 900, 1024, 1), (40, 3000, 16, 1),
                                             (3, 50, 60, 6), (2, 33, 52, 4), (1, 1, 4, 2), (1, 900, 1028, 1), (30, 3000, 20, 1)])
def test_vectors_that_start_anywhere(n, p, c, groups, x, y, pad, out_pad):
    t = list(inputs(n, p, c, x, y, seed=pad + c))
    for i in (0, 1):
        ld = c + pad
        buf = torch.full((pad + (n * p - 1) * ld + c,), 77, dtype=t[i].dtype, device="cuda")
        v = buf.as_strided((n, p, c), (p * ld, ld, 1), pad)
        v.copy_(t[i])
        t[i] = v
    out = run(*t, groups, 1e-5, "silu", pad=out_pad * pad)
    check(*t, groups, 1e-5, "silu", *out)
    if out_pad:
        for o in (out[0], out[3]):
            assert (o.as_strided((n, p, pad), o.stride(), o.storage_offset() + c) == 77).all()
    assert all(torch.equal(a, b) for a, b in zip(out, run(*t, groups, 1e-5, "silu", pad=out_pad * pad)))


def test_samples_apart_and_a_part_of_the_pixels():
    n, p, c, groups = 3, 40, 24, 3
    x, dy, gamma, beta = inputs(n, p, c, seed=8)
    x, dy = x[:, 5:29], dy[:, 7:31]
    check(x, dy, gamma, beta, groups, 1e-5, "silu", *run(x, dy, gamma, beta, groups, 1e-5, "silu"))


@pytest.mark.parametrize("which", [(True, False, False), (False, True, False), (False, False, True), (False, True, True), (True, True, True)])
@pytest.mark.parametrize("params", [(True, True), (False, True), (True, False), (False, False)])
def test_gradients_that_are_not_wanted(which, params):
    x, dy, gamma, beta = inputs(2, 50, 48, "i8", seed=3)
    gamma, beta = gamma if params[0] else None, beta if params[1] else None
    check(x, dy, gamma, beta, 6, 1e-5, "silu", *run(x, dy, gamma, beta, 6, 1e-5, "silu", grads=which))


def test_forward_without_statistics():
    x, dy, gamma, beta = inputs(4, 50, 48, "i8", seed=3)
    want = run(x, dy, gamma, beta, 6, 1e-5, "silu")[0]
    h = nb.GroupNorm(9, 70, 48, 6)
    y = torch.empty_like(want)
    h.forward(x, gamma, beta, y, eps=1e-5, act=nb.NITRO_ACT_SILU)
    assert torch.equal(y, want)
    h.close()


@pytest.mark.parametrize("p", [80, 30000])
def test_in_place(p):
    x, dy, gamma, beta = inputs(3, p, 64, seed=9)
    want = run(x, dy, gamma, beta, 8, 1e-5, "gelu")
    h = nb.GroupNorm(3, p, 64, 8)
    a, b = x.clone(), dy.clone()
    mean, rstd = torch.empty(3, 8, device="cuda"), torch.empty(3, 8, device="cuda")
    h.backward(x, gamma, beta, want[1], want[2], b, b, act=nb.NITRO_ACT_GELU)
    h.forward(a, gamma, beta, a, mean, rstd, act=nb.NITRO_ACT_GELU)
    assert torch.equal(a, want[0]) and torch.equal(b, want[3]) and torch.equal(mean, want[1]) and torch.equal(rstd, want[2])
    h.close()


@pytest.mark.parametrize("level", [100.0, 3000.0])
@pytest.mark.parametrize("p", [64, 5000])
def test_means_far_from_zero(p, level):
    t = inputs(2, p, 32, "f32", "f32", seed=4, level=level)
    check(*t, 32, 1e-5, "none", *run(*t, 32, 1e-5, "none"))


def test_an_outlier_first_and_constant_groups():
    x, dy, gamma, beta = inputs(2, 600, 16, "f32", "f32", seed=4)
    x[0, 0, :4] = 1e4
    check(x, dy, gamma, beta, 4, 1e-5, "silu", *run(x, dy, gamma, beta, 4, 1e-5, "silu"))
    x[:] = 2.5                                  # no spread: h is 0 and y = act(beta)
    y, mean, rstd, dx, dg, db = run(x, dy, gamma, beta, 4, 1e-5, "silu")
    check(x, dy, gamma, beta, 4, 1e-5, "silu", y, mean, rstd, dx, dg, db)
    assert (mean == 2.5).all() and (dg == 0).all()


def test_nan_and_infinity_stay_in_their_groups():
    x, dy, gamma, beta = inputs(2, 300, 32, "bf16", "f32", seed=6)
    want = run(x, dy, gamma, beta, 4, 1e-5, "silu")
    x[0, 17, 3] = float("nan")
    x[1, 200, 30] = float("inf")
    got = run(x, dy, gamma, beta, 4, 1e-5, "silu")
    for i in (0, 3):
        assert got[i][0, :, :8].isnan().all() and got[i][1, :, 24:].isnan().all()
        assert torch.equal(got[i][0, :, 8:], want[i][0, :, 8:]) and torch.equal(got[i][1, :, :24], want[i][1, :, :24])


def test_empty_batch_and_a_smaller_one():
    x, dy, gamma, beta = inputs(6, 30, 40, seed=2)
    h = nb.GroupNorm(6, 64, 40, 5)
    y, mean, rstd, dx, dg, db = run(x[:0], dy[:0], gamma, beta, 5, 1e-5, "silu", h)
    assert (dg == 0).all() and (db == 0).all()
    for n in (6, 1, 4):
        check(x[:n], dy[:n], gamma, beta, 5, 1e-5, "silu", *run(x[:n], dy[:n], gamma, beta, 5, 1e-5, "silu", h))
    h.close()


# more than a launch's samples; slabs that no cluster holds, of one sample and of so many that CTAs take several; groups
# of more channels than a warp's lanes take, and than a CTA's; the same without vectors; sums of more CTAs than are kept
@pytest.mark.parametrize("n, p, c, groups, x, pad", [
    (2500, 6, 16, 4, "i8", 0), (20, 5000, 128, 8, "bf16", 0), (3, 70001, 100, 5, "bf16", 0), (1, 70001, 33, 3, "bf16", 0), (40, 15000, 16, 1, "f32", 0),
    (90, 15000, 16, 2, "i8", 0), (2, 900, 1024, 1, "bf16", 0), (1, 900, 2048, 2, "i8", 0), (1, 250, 4096, 1, "bf16", 0), (1, 900, 600, 2, "bf16", 3),
    (2, 9000, 64, 1, "bf16", 3), (1, 40000, 1000, 250, "bf16", 0), (9, 50000, 8, 8, "f32", 0)])
def test_batches(n, p, c, groups, x, pad):
    t = inputs(n, p, c, x, "f32" if x == "f32" else "bf16", pad=pad, seed=21)
    out = run(*t, groups, 1e-5, "silu", pad=pad)
    check(*t, groups, 1e-5, "silu", *out)
    assert all(torch.equal(a, b) for a, b in zip(out, run(*t, groups, 1e-5, "silu", pad=pad)))


def test_gradients_against_differences():
    n, p, c, groups = 1, 6, 8, 2
    x, dy, gamma, beta = inputs(n, p, c, "f32", "f32", seed=1)
    dx, dg, db = run(x, dy, gamma, beta, groups, 1e-5, "gelu")[3:]
    f = lambda x, g, b: (run(x, dy, g, b, groups, 1e-5, "gelu")[0].double() * dy.double()).sum().item()
    step = 2.0 ** -7
    for t, grad, pos in ((0, dx, (0, 3, 2)), (0, dx, (0, 5, 7)), (1, dg, (4,)), (2, db, (1,))):
        v = []
        for s in (step, -step):
            args = [x.clone(), gamma.clone(), beta.clone()]
            args[t][pos] += s
            v.append(f(*args))
        # values of f are off by 1e-7 of a sum of absolute terms near 0.4, over twice the step; the third derivative's part is
        # step^2 times a few gradients' size (1e-2)
        assert abs((v[0] - v[1]) / (2 * step) - grad[pos].item()) < 2e-7 * 0.5 / step + step ** 2 * 0.1


@pytest.mark.parametrize("p", [3000, 40000])
def test_captured_and_replayed_on_another_stream(p):
    x, dy, gamma, beta = inputs(2, p, 64, seed=5)
    want = run(x, dy, gamma, beta, 8, 1e-5, "silu")
    h = nb.GroupNorm(2, p, 64, 8)
    y, dx = torch.empty_like(dy), torch.empty_like(dy)
    mean, rstd = torch.empty(2, 8, device="cuda"), torch.empty(2, 8, device="cuda")
    dg, db = torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        h.forward(x, gamma, beta, y, mean, rstd, act=nb.NITRO_ACT_SILU)
        h.backward(x, gamma, beta, mean, rstd, dy, dx, dg, db, act=nb.NITRO_ACT_SILU)
    for _ in range(3):
        for t in (y, mean, rstd, dx, dg, db):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, mean, rstd, dx, dg, db), want))
    h.close()


def test_refusals():
    x, dy, gamma, beta = inputs(2, 10, 16)
    h = nb.GroupNorm(2, 10, 16, 4)
    mean, rstd = torch.empty(2, 4, device="cuda"), torch.empty(2, 4, device="cuda")
    y = torch.empty_like(dy)
    big = inputs(3, 11, 16)
    for bad in (lambda: h.forward(big[0][:, :10], gamma, beta, big[1][:, :10]), lambda: h.forward(big[0][:2], gamma, beta, big[1][:2]),
                lambda: h.forward(x, gamma, beta, y, eps=0.0), lambda: h.forward(x, gamma, beta, y, eps=float("nan")),
                lambda: h.forward(x, gamma, beta, y, eps=float("inf")), lambda: h.forward(x, gamma, beta, y, act=4),
                lambda: h.forward(x, gamma, beta, y, act=-1), lambda: h.forward(x, gamma, beta, y, mean),
                lambda: h.forward(x[:1].expand(2, 10, 16), gamma, beta, y), lambda: h.forward(x[:, :0], gamma, beta, y[:, :0]),
                lambda: h.backward(x, gamma, beta, None, None, dy, y)):
        with pytest.raises(nb.NitroError):
            bad()
    p = lambda t, off=0: t.data_ptr() + off
    for gam, mu, dga in ((p(gamma, 2), p(mean), p(beta)), (p(gamma), p(mean, 1), p(beta)), (p(gamma), p(mean), p(beta, 2))):
        assert nb.lib().nitro_gnorm_backward(h.h, p(x), 0, 16, 160, 2, 10, gam, None, mu, p(rstd), 0, p(dy), 0, 16, 160, None, 16, 160, dga,
                                             None, None) == nb.NITRO_ERR_ARG
    assert nb.lib().nitro_gnorm_forward(h.h, p(x, 1), 0, 16, 160, 2, 10, None, None, 1e-5, 0, p(y), 0, 16, 160, None, None, None) == nb.NITRO_ERR_ARG
    for bad in (lambda: h.forward(x.to(torch.float16), gamma, beta, y), lambda: h.forward(x, gamma, beta, y.to(torch.int8)),
                lambda: h.forward(x[..., :8], gamma, beta, y[..., :8]), lambda: h.forward(x, gamma[:8], beta, y),
                lambda: h.forward(x, gamma.to(torch.bfloat16), beta, y), lambda: h.forward(x, gamma, beta, y[:1]),
                lambda: h.forward(x.transpose(1, 2), gamma, beta, y), lambda: h.forward(x, gamma, beta, y, mean[:1], rstd),
                lambda: h.backward(x, gamma, beta, mean, rstd, dy, y.float())):
        with pytest.raises((ValueError, IndexError)):
            bad()
    h.close()

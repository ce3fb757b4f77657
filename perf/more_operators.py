"""Performance cases of the operators around the floating-point head: what stands between the
integer blocks' maps and the class matrix, and between the gradients and the update.

* ``gnorm``: group norm with an activation on channels-last maps, x [samples x pixels x
  channels]; u = gamma (x - mean) / sqrt(var + eps) + beta, y = act(u), mean and variance
  over the pixels and channels of a group; for a training step the gradients of x, gamma
  and beta as well.
* ``glu``: a gated feed-forward block, out = act(scale x Wg^T) * (scale x Wu^T) with both
  weights in one matrix (gate rows first); for a training step the gradients of x and of
  the weights.
* ``clip``: the norm over many gradients, and the gradients scaled where it is above a
  limit.

``run`` is one pass: with ``own`` the calls of the public binding, without it the
operators' definition in elementary torch operations, in 32 bits and rounded once.
"""
import math
import random

import torch

own = False

EPS = 1e-5
BF16, F32 = torch.bfloat16, torch.float32
DT = {"bf16": BF16, "f32": F32, "i8": torch.int8}
SIZE = {"bf16": 2, "f32": 4, "i8": 1}
MOST_PRODUCTS = 8192 * 2048 * 8192          # rows x features x hidden of a glu
MOST_VALUES = 128 * 4096 * 256              # of a map
MOST_BYTES = 4 << 30                        # of a set of gradients


# ------------------------------------------------------------------ the cases
def gnorm(name, samples, pixels, channels, groups, x="i8", y="bf16", act="silu", train=True, pad=0):
    return {"name": name, "kind": "gnorm", "samples": samples, "pixels": pixels, "channels": channels, "groups": groups, "x": x,
            "y": y, "act": act, "train": train, "pad": pad}


def glu(name, rows, features, hidden, x="bf16", act="silu", train=True, pad=0):
    return {"name": name, "kind": "glu", "rows": rows, "features": features, "hidden": hidden, "x": x, "act": act,
            "train": train, "pad": pad}


def clip(name, count, lo, hi, m="mixed", above=True, pad=0, pick=0):
    return {"name": name, "kind": "clip", "count": count, "lo": lo, "hi": hi, "m": m, "above": above, "pad": pad, "pick": pick}


def listed():
    return [
        # one image's 8 x 8 map as a server normalises it: latency
        gnorm("gnorm_answer", 1, 64, 256, 32, train=False),
        # a step at the paper's batch on the int8 maps of a VGG stage
        gnorm("gnorm_step_batch64", 64, 256, 256, 32),
        # few large maps of odd sizes, a view of wider buffers: a group's values are many
        gnorm("gnorm_step_maps", 3, 301 * 257, 100, 5, x="bf16", act="gelu", pad=12),
        # the largest step: maps beyond what the chip's caches hold
        gnorm("gnorm_step_large", 128, 4096, 256, 32, x="bf16"),
        # one sample's features, as a server answers: the weights' bytes
        glu("glu_answer", 1, 4096, 4096, train=False),
        # a few samples on int8 activations, odd sizes
        glu("glu_answer_few", 13, 1000, 1501, x="i8", act="gelu", train=False, pad=3),
        # a step at the paper's batch on the int8 activations of a VGG's learning layer (d^lr = 4096)
        glu("glu_step_batch64", 64, 4096, 1024, x="i8"),
        # an ordinary step: sizes that no tile divides, a view of wider buffers
        glu("glu_step_ragged", 1000, 1000, 1366, act="gelu", pad=24),
        # the largest step: a big batch and a wide block
        glu("glu_step_large", 8192, 2048, 8192),
        # the gradients of a small head (class matrix, gated block, scales and shifts): latency
        clip("clip_head", 6, 256, 1 << 20),
        # all layers of a deep network, from single values up, none above the limit
        clip("clip_many", 300, 1, 300000, m="f32", above=False),
        # a large model's gradients: bandwidth
        clip("clip_large", 48, 1 << 22, 1 << 26),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Over the range's logarithm, half of them multiples of 8."""
    v = _log(rng, lo, hi)
    return max(lo, v // 8 * 8) if rng.random() < 0.5 else v


def draw(rng):
    kind = rng.choice(["gnorm", "gnorm", "glu", "glu", "glu", "clip"])
    pad = rng.choice([0, 0, 8, 3])
    act = rng.choice(["silu", "silu", "gelu", "none"])
    if kind == "gnorm":
        per = rng.choice([1, 2, 4, 6, 8, 16, 20, 32, 64])
        groups = _log(rng, 1, 1024 // per)
        pixels = _log(rng, max(1, -(-64 // per)), 1 << 17)
        c = per * groups
        while pixels * c > MOST_VALUES:
            pixels //= 2
        case = gnorm("", _log(rng, 1, min(512, MOST_VALUES // (pixels * c))), pixels, c, groups, x=rng.choice(["i8", "bf16", "f32"]),
                     y=rng.choice(["bf16", "bf16", "f32"]), act=act, train=rng.random() < 0.6, pad=pad)
    elif kind == "glu":
        f, h = _size(rng, 32, 4096), _size(rng, 16, 8192)
        case = glu("", _log(rng, 1, min(8192, MOST_PRODUCTS // (f * h))), f, h, x=rng.choice(["bf16", "bf16", "i8"]), act=act,
                   train=rng.random() < 0.6, pad=pad)
    else:
        count = _log(rng, 1, 400)
        hi = _log(rng, 64, min(1 << 26, MOST_BYTES // 8 // count))
        case = clip("", count, max(1, hi // rng.choice([1, 16, 4096])), hi, m=rng.choice(["bf16", "f32", "mixed"]),
                    above=rng.random() < 0.7, pad=pad, pick=rng.randrange(1 << 20))
    del case["name"]
    return case


def _shapes(case):
    """The gradients' types, rows and columns, which are the case's alone."""
    rng = random.Random(case["pick"])
    out = []
    for i in range(case["count"]):
        n = _log(rng, case["lo"], case["hi"])
        cols = _log(rng, 1, min(n, 8192)) if rng.random() < 0.7 else n
        if case["pad"] and cols > 8192:
            cols = 4097
        m = case["m"] if case["m"] != "mixed" else ("f32" if rng.random() < 0.3 else "bf16")
        out.append((m, n // cols, cols))
    return out


# ------------------------------------------------------------------ inputs
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=F32)


def _view(t, pad):
    """t as the left part of a buffer whose last dimension is `pad` wider."""
    if not pad:
        return t.contiguous()
    wide = torch.zeros(*t.shape[:-1], t.shape[-1] + pad, dtype=t.dtype, device=t.device)
    wide[..., : t.shape[-1]] = t
    return wide[..., : t.shape[-1]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "gnorm":
        n, p, c = case["samples"], case["pixels"], case["channels"]
        # channels of different level and spread, samples of different contrast
        x = _normal(g, n, p, c)
        x *= torch.exp(0.4 * _normal(g, c)) * torch.exp(0.3 * _normal(g, n, 1, 1))
        x += 0.7 * _normal(g, c)
        if case["x"] == "i8":  # block activations: within [-127, 127]
            x = x.mul_(30).round_().clamp_(-127, 127)
        s["x"] = _view(x.to(DT[case["x"]]), case["pad"])
        s["gamma"] = 1.0 + 0.2 * _normal(g, c)
        s["beta"] = 0.2 * _normal(g, c)
        if case["train"]:
            s["dy"] = _view((_normal(g, n, p, c) * 1e-3).to(DT[case["y"]]), case["pad"])
        return s
    if case["kind"] == "glu":
        n, f, h = case["rows"], case["features"], case["hidden"]
        x = _normal(g, n, f)
        s["scale"] = 1.0
        if case["x"] == "i8":
            x = (x * 32).round().clamp_(-127, 127)
            s["scale"] = 1.0 / 32
        s["x"] = _view(x.to(DT[case["x"]]), case["pad"])
        s["w"] = _view((_normal(g, 2 * h, f) * (1.5 / math.sqrt(f))).to(BF16), case["pad"])
        if case["train"]:
            s["dout"] = _view((_normal(g, n, h) * 1e-3).to(BF16), case["pad"])
        return s
    # tensors of different size of entries; their norm is then 1, and the limit below or above it
    grads, total = [], 0.0
    for m, rows, cols in _shapes(case):
        t = _normal(g, rows, cols) * (10.0 ** torch.rand(1, generator=g, device="cuda"))
        total += t.square().sum().double()
        grads.append(t)
    s["grads"] = [_view((t / total.sqrt()).to(DT[m]), case["pad"]) for t, (m, _, _) in zip(grads, _shapes(case))]
    s["limit"] = 0.3 if case["above"] else 4.0
    return s


def _flat(case, like=None):
    """A buffer for each type with room for its gradients one after another, and the views of it that hold
    them: as a program keeps many small tensors (starts at multiples of 8 values)."""
    ends, at = {}, []
    for m, rows, cols in _shapes(case):
        at.append((m, ends.get(m, 0), rows, cols))
        ends[m] = at[-1][1] + -(-rows * cols // 8) * 8
    buf = {m: torch.zeros(n, dtype=like or DT[m], device="cuda") for m, n in ends.items()}
    return buf, [buf[m][i: i + rows * cols].view(rows, cols) for m, i, rows, cols in at]


# ------------------------------------------------------------------ the plain forms
def _act(u, act):
    """(act(u), its derivative)"""
    if act == "none":
        return u, torch.ones_like(u)
    if act == "silu":
        t = 1.0 / (1.0 + torch.exp(-u))
        return u * t, t * (1.0 + u * (1.0 - t))
    t = 0.5 * torch.erfc(u * -math.sqrt(0.5))
    return u * t, t + u * torch.exp(-0.5 * u * u) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_gnorm(s):
    case, x = s["case"], s["x"].to(F32)
    n, p, c, gr = case["samples"], case["pixels"], case["channels"], case["groups"]
    x = x.reshape(n, p, gr, c // gr)
    x = x - x.mean(dim=(1, 3), keepdim=True)
    rstd = 1.0 / torch.sqrt((x * x).mean(dim=(1, 3), keepdim=True) + EPS)
    h = (x * rstd).reshape(n, p, c)
    y, slope = _act(s["gamma"] * h + s["beta"], case["act"])
    y = y.to(DT[case["y"]])
    if not case["train"]:
        return {"y": y}
    du = s["dy"].to(F32) * slope
    del slope
    dgamma, dbeta = (du * h).sum(dim=(0, 1)), du.sum(dim=(0, 1))
    t = (du * s["gamma"]).reshape(n, p, gr, c // gr)
    h = h.reshape(n, p, gr, c // gr)
    dx = rstd * (t - t.mean(dim=(1, 3), keepdim=True) - h * (t * h).mean(dim=(1, 3), keepdim=True))
    return {"y": y, "dx": dx.reshape(n, p, c).to(DT[case["y"]]), "dgamma": dgamma, "dbeta": dbeta}


def _plain_glu(s):
    case, x, w, scale, h = s["case"], s["x"].to(F32), s["w"].to(F32), s["scale"], s["case"]["hidden"]
    z = (x @ w.t()) * scale
    a, b = z[:, :h], z[:, h:]
    v, slope = _act(a, case["act"])
    out = (v * b).to(BF16)
    if not case["train"]:
        return {"out": out}
    dout = s["dout"].to(F32)
    d = torch.cat((dout * b * slope, dout * v), dim=1)
    return {"out": out, "dx": ((d @ w) * scale).to(BF16), "dw": ((d.t() @ x) * scale).to(BF16)}


def _plain_clip(s):
    total = sum(t.to(F32).square().sum(dtype=torch.float64) for t in s["grads"])
    norm = total.sqrt()
    f = torch.where(norm > s["limit"], s["limit"] / norm, torch.ones_like(norm)).to(F32)
    out, views = _flat(s["case"])
    for t, v in zip(s["grads"], views):
        v.copy_(t.to(F32) * f)
    return {"norm": norm.to(F32), **out}


# ------------------------------------------------------------------ the framework's calls
_handles = {}  # a program makes the handle of a shape once and keeps it


def _handle(kind, *shape):
    from paper_2407_11698_gb300 import binding as nb
    key = (kind,) + shape
    if key not in _handles:
        _handles[key] = getattr(nb, kind)(*shape)
    return nb, _handles[key]


def _act_code(nb, act):
    return {"none": nb.NITRO_ACT_NONE, "silu": nb.NITRO_ACT_SILU, "gelu": nb.NITRO_ACT_GELU}[act]


def _own_gnorm(s):
    case = s["case"]
    n, p, c, gr = case["samples"], case["pixels"], case["channels"], case["groups"]
    nb, h = _handle("GroupNorm", n, p, c, gr)
    act = _act_code(nb, case["act"])
    y = torch.empty(n, p, c, dtype=DT[case["y"]], device="cuda")
    if not case["train"]:
        h.forward(s["x"], s["gamma"], s["beta"], y, eps=EPS, act=act)
        return {"y": y}
    mean, rstd = torch.empty(n, gr, device="cuda"), torch.empty(n, gr, device="cuda")
    h.forward(s["x"], s["gamma"], s["beta"], y, mean, rstd, eps=EPS, act=act)
    dx = torch.empty(n, p, c, dtype=DT[case["y"]], device="cuda")
    dgamma, dbeta = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    h.backward(s["x"], s["gamma"], s["beta"], mean, rstd, s["dy"], dx, dgamma, dbeta, act=act)
    return {"y": y, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _own_glu(s):
    case = s["case"]
    n, f, hid = case["rows"], case["features"], case["hidden"]
    nb, h = _handle("GatedLinear", n, f, hid)
    act = _act_code(nb, case["act"])
    out = torch.empty(n, hid, dtype=BF16, device="cuda")
    if not case["train"]:
        h.forward(s["x"], s["w"], out, act=act, scale=s["scale"])
        return {"out": out}
    saved = torch.empty(n, 2 * hid, device="cuda")
    h.forward(s["x"], s["w"], out, saved, act=act, scale=s["scale"])
    dx = torch.empty(n, f, dtype=BF16, device="cuda")
    dw = torch.empty(2 * hid, f, dtype=BF16, device="cuda")
    h.backward(s["x"], s["w"], saved, s["dout"], dx, dw, act=act, scale=s["scale"])
    return {"out": out, "dx": dx, "dw": dw}


def _own_clip(s):
    if "plan" not in s:  # a program's gradients stay where they are from step to step
        from paper_2407_11698_gb300 import binding as nb
        s["out"], views = _flat(s["case"])
        s["norm"] = torch.empty((), device="cuda")
        s["plan"] = nb.GradClip(s["grads"], views)
    s["plan"].run(s["norm"], s["limit"])
    return {"norm": s["norm"], **s["out"]}


PLAIN = {"gnorm": _plain_gnorm, "glu": _plain_glu, "clip": _plain_clip}
OWN = {"gnorm": _own_gnorm, "glu": _own_glu, "clip": _own_clip}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["kind"]](state)


# ------------------------------------------------------------------ work
def work(case):
    if case["kind"] == "gnorm":
        v, c = case["samples"] * case["pixels"] * case["channels"], case["channels"]
        fwd = (SIZE[case["x"]] + SIZE[case["y"]]) * v + 8 * c
        return {"bytes": fwd + (2 * SIZE[case["y"]] * v + 8 * c if case["train"] else 0), "flops": 0}
    if case["kind"] == "glu":
        n, f, h = case["rows"], case["features"], case["hidden"]
        fwd = SIZE[case["x"]] * n * f + 4 * h * f + 2 * n * h
        if not case["train"]:
            return {"bytes": fwd, "flops": 4 * n * f * h}
        return {"bytes": fwd + 2 * n * h + 2 * n * f + 4 * h * f, "flops": 12 * n * f * h}
    return {"bytes": sum(2 * SIZE[m] * r * c for m, r, c in _shapes(case)), "flops": 0}


# ------------------------------------------------------------------ in 64 bits
def _smooth(u, act):
    if act == "silu":
        return u * torch.sigmoid(u)
    if act == "gelu":
        return u * torch.special.ndtr(u)
    return u


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "gnorm":
        leaves = [s[k].double().requires_grad_(case["train"]) for k in ("x", "gamma", "beta")]
        x, gamma, beta = leaves
        u = x.unflatten(2, (case["groups"], -1)).transpose(1, 2).flatten(2)      # a group's values in a row
        m = u.sum(dim=2, keepdim=True) / u.shape[2]
        v = ((u - m) ** 2).sum(dim=2, keepdim=True) / u.shape[2]
        u = ((u - m) * (v + EPS) ** -0.5).unflatten(2, (case["pixels"], -1)).transpose(1, 2).flatten(2)
        y = _smooth(gamma * u + beta, case["act"])
        if not case["train"]:
            return {"y": y}
        dx, dgamma, dbeta = torch.autograd.grad(y, leaves, s["dy"].double())
        return {"y": y.detach(), "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if case["kind"] == "glu":
        if work(case)["flops"] > 4e12:
            return None
        x, w = (s[k].double().requires_grad_(case["train"]) for k in ("x", "w"))
        z = torch.mm(x, w.mT).mul(s["scale"])
        a, b = z.unflatten(1, (2, -1)).unbind(1)
        out = _smooth(a, case["act"]) * b
        if not case["train"]:
            return {"out": out}
        dx, dw = torch.autograd.grad(out, (x, w), s["dout"].double())
        return {"out": out.detach(), "dx": dx, "dw": dw}
    flat = [t.double() for t in s["grads"]]
    norm = torch.stack([torch.linalg.vector_norm(t) for t in flat]).norm()
    out, views = _flat(case, torch.float64)
    for t, v in zip(flat, views):
        torch.mul(t, s["limit"] / torch.clamp(norm, min=s["limit"]), out=v)
    return {"norm": norm, **out}

"""Performance cases of the floating-point head: the operators that train and serve a
classifier over many classes on top of the integer blocks' activations.

* ``xent``: softmax cross entropy of a linear head, z = scale x W^T, with int8 block
  activations or bf16 features x; the loss of every row, and for a training step the
  gradients of x and W.  Rows with label -1 are left out.
* ``orth``: the update made orthogonal by Newton-Schulz steps, X <- a X + (b A + c A^2) X
  with A = X X^T, of one matrix or of several of one shape (bf16, fp32, or the int64
  weight gradients of the blocks).
* ``mx4``: microscaled 4-bit floating point, e2m1 values that share a power of two in
  blocks of 32 along a row: the product of quantised features with 4-bit weights
  (``linear``), and the round trip through 4 bits (``store``).

``run`` is one pass: with ``own`` the calls of the public binding, without it the
operators' definition in elementary torch operations, in 32 bits and rounded once.
"""
import math

import torch

own = False

STEPS, COEF = 5, (3.4445, -4.7750, 2.0315)
NORM_EPS = 1e-7
BF16, F32 = torch.bfloat16, torch.float32
DT = {"bf16": BF16, "f32": F32, "i64": torch.int64, "i8": torch.int8}


# ------------------------------------------------------------------ the cases
def xent(name, rows, features, classes, x="bf16", train=True, ignored=0.0, pad=0):
    return {"name": name, "kind": "xent", "rows": rows, "features": features, "classes": classes, "x": x, "train": train,
            "ignored": ignored, "pad": pad}


def orth(name, rows, cols, count=1, m="bf16", rank=0):
    return {"name": name, "kind": "orth", "rows": rows, "cols": cols, "count": count, "m": m, "rank": rank}


def linear(name, rows, k, n, x="bf16", y="bf16", pad=0):
    return {"name": name, "kind": "linear", "rows": rows, "in": k, "out": n, "x": x, "y": y, "pad": pad}


def store(name, rows, cols, x="bf16", pad=0):
    return {"name": name, "kind": "store", "rows": rows, "cols": cols, "x": x, "pad": pad}


def listed():
    return [
        # a few samples scored against ten thousand classes, as a server answers: latency
        xent("xent_score_few", 4, 512, 10000, train=False),
        # a step at the paper's batch on the int8 activations of a VGG's learning layer (d^lr = 4096)
        xent("xent_step_batch64", 64, 4096, 1000, x="i8"),
        # an ordinary step: sizes that no tile divides, some rows without a label, a view of a wider buffer
        xent("xent_step_ragged", 1000, 1000, 20011, ignored=0.15, pad=24),
        # the largest step: a big batch against a vocabulary whose logits would take 2 GB
        xent("xent_step_large", 8192, 2048, 64000),
        # one hidden layer of the smallest network (100 -> 50): latency
        orth("orth_small", 50, 100),
        # the eight conv layers of a stage at once, int64 gradients as a backward at batch 64 leaves them
        orth("orth_conv_stage", 256, 2304, count=8, m="i64", rank=64),
        # the weights of a large head
        orth("orth_large", 4096, 8192),
        # one sample against 4-bit weights, as a server answers: the weights' bytes
        linear("linear_token", 1, 4096, 10000),
        # an evaluation batch, odd sizes: the last block of a row is short (3000 = 93 * 32 + 24)
        linear("linear_ragged", 77, 3000, 1001, x="f32", y="f32", pad=5),
        # a large batch: the 4-bit tensor rate
        linear("linear_large", 8192, 8192, 8192),
        # a small activation kept in 4 bits: latency
        store("store_small", 64, 784, x="f32"),
        # a layer's activations kept in 4 bits and brought back: bandwidth
        store("store_large", 16384, 4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Over the range's logarithm, half of them multiples of 8."""
    v = _log(rng, lo, hi)
    return max(lo, v // 8 * 8) if rng.random() < 0.5 else v


def draw(rng):
    kind = rng.choice(["xent", "xent", "orth", "orth", "linear", "linear", "store"])
    if kind == "xent":
        f, c = _size(rng, 64, 4096), _size(rng, 10, 64000)
        most = min(8192, 8192 * 2048 * 64000 // (f * c))
        case = xent("", _log(rng, 1, most), f, c, x=rng.choice(["bf16", "bf16", "i8"]), train=rng.random() < 0.7,
                    ignored=rng.choice([0.0, 0.1, 0.5]), pad=rng.choice([0, 0, 8, 3]))
    elif kind == "orth":
        while True:
            r, c, n = _size(rng, 16, 8192), _size(rng, 16, 8192), rng.choice([1, 1, 2, 3, 8])
            if n * min(r, c) ** 2 * (3 * max(r, c) + min(r, c)) <= 4096 ** 2 * (3 * 8192 + 4096):
                break
        case = orth("", r, c, count=n, m=rng.choice(["bf16", "f32", "i64"]), rank=rng.choice([0, 0, 64, 5]))
    elif kind == "linear":
        k, n = _size(rng, 64, 8192), _size(rng, 64, 16384)
        case = linear("", _log(rng, 1, min(8192, 8192 ** 3 // (k * n))), k, n, x=rng.choice(["bf16", "f32"]),
                      y=rng.choice(["bf16", "f32"]), pad=rng.choice([0, 0, 8, 3]))
    else:
        cols = _size(rng, 32, 8192)
        case = store("", _log(rng, 1, min(32768, 16384 * 4096 // cols)), cols, x=rng.choice(["bf16", "f32"]), pad=rng.choice([0, 0, 8, 3]))
    del case["name"]
    return case


# ------------------------------------------------------------------ inputs
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=F32)


def _view(t, pad):
    """t as the left part of a buffer that is `pad` columns wider."""
    if not pad:
        return t.contiguous()
    wide = torch.zeros(t.shape[0], t.shape[1] + pad, dtype=t.dtype, device=t.device)
    wide[:, : t.shape[1]] = t
    return wide[:, : t.shape[1]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "xent":
        n, d, c = case["rows"], case["features"], case["classes"]
        labels = torch.randint(0, c, (n,), generator=g, device="cuda")
        w = _normal(g, c, d) / math.sqrt(d)
        # features that lean towards their class, as a head some way into its training sees them
        x = _normal(g, n, d) * 1.5
        x += w[labels] * (6.0 * torch.rand(n, 1, generator=g, device="cuda"))
        if case["x"] == "i8":  # block activations: centred on 0, within [-127, 127]
            x = (x * 32).round().clamp_(-127, 127)
            s["scale"] = 1.0 / 32
        else:
            s["scale"] = 1.0
        labels[torch.rand(n, generator=g, device="cuda") < case["ignored"]] = -1
        s["x"] = _view(x.to(DT[case["x"]]), case["pad"])
        s["w"] = _view(w.to(BF16), case["pad"])
        s["labels"] = labels.to(torch.int32)
        # what the mean over the rows with a label hands back to each row
        s["gout"] = torch.full((n,), 1.0 / max(1, int((labels >= 0).sum())), device="cuda")
        return s
    if case["kind"] == "orth":
        k, r, c = case["count"], case["rows"], case["cols"]
        if case["rank"]:  # the gradient of one batch, and what momentum has kept of many before it
            q = min(case["rank"], r, c)
            m = _normal(g, k, r, q) @ _normal(g, k, q, c) / math.sqrt(q) + 0.02 * _normal(g, k, r, c)
        else:
            m = _normal(g, k, r, c)
        m *= 2e4 if case["m"] == "i64" else 1e-3
        s["m"] = m.round().to(torch.int64) if case["m"] == "i64" else m.to(DT[case["m"]])
        return s
    if case["kind"] == "linear":
        k, n = case["in"], case["out"]
        s["x"] = _view(_normal(g, case["rows"], k).to(DT[case["x"]]), case["pad"])
        # the 4-bit weights as a checkpoint holds them: two codes a byte, scales in tiles of 128 rows x 4 blocks
        codes, exps = _mx4_codes(_normal(g, n, k) / math.sqrt(k))
        s["wq"], s["ws"] = _mx4_pack(codes, exps)
        return s
    x = _normal(g, case["rows"], case["cols"])
    x *= torch.exp(_normal(g, 1, case["cols"]))  # channels of different size
    s["x"] = _view(x.to(DT[case["x"]]), case["pad"])
    return s


# ------------------------------------------------------------------ the plain forms
def _mx4_codes(x):
    """e2m1 codes (0..15) [rows][blocks][32] and the blocks' exponents [rows][blocks] of x (fp32): the
    scale is 2^(floor(log2 max|x|) - 2), values go to the nearest code, ties to the even one, 6 at most."""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    b = torch.zeros(rows, blocks * 32, dtype=F32, device=x.device)
    b[:, :cols] = x
    b = b.view(rows, blocks, 32)
    top = b.abs().amax(dim=2)
    e = (torch.frexp(top)[1] - 3).clamp(-127, 127)
    e = torch.where(top == 0, torch.full_like(e, -127), e)
    y = torch.ldexp(b.abs(), -e.unsqueeze(2))
    code = torch.zeros(y.shape, dtype=torch.uint8, device=x.device)
    for_up = (0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)
    code = sum((y >= t if up else y > t).to(torch.uint8) for t, up in for_up)
    return code + 8 * (b < 0).to(torch.uint8), e


def _mx4_values(codes, exps, cols):
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=F32, device=codes.device)
    v = table[(codes & 7).long()] * (1 - 2 * (codes >> 3).to(F32))
    v = v * torch.exp2(exps.to(F32)).unsqueeze(2)
    return v.flatten(1)[:, :cols]


def _mx4_pack(codes, exps):
    rows, blocks = exps.shape
    q = (codes[..., 0::2] | (codes[..., 1::2] << 4)).flatten(1).contiguous()
    rt, bt = -(-rows // 128), -(-blocks // 4)
    t = torch.zeros(rt * 128, bt * 4, dtype=torch.uint8, device=exps.device)
    t[:rows, :blocks] = (exps + 127).to(torch.uint8)
    # tile (rt, bt) of 512 bytes: row r, block j at (r % 32) 16 + (r / 32) 4 + j
    t = t.view(rt, 4, 32, bt, 4).permute(0, 3, 2, 1, 4).contiguous()
    return q, t.view(-1)


def _mx4_unpack(q, s, rows, cols):
    blocks = -(-cols // 32)
    rt, bt = -(-rows // 128), -(-blocks // 4)
    codes = torch.stack((q & 15, q >> 4), dim=2).view(rows, blocks, 32)
    e = s.view(rt, bt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, bt * 4)[:rows, :blocks]
    return _mx4_values(codes, e.to(torch.int32) - 127, cols)


def _plain_xent(s):
    case, x, w, scale = s["case"], s["x"].to(F32), s["w"].to(F32), s["scale"]
    labels = s["labels"].long()
    live = labels >= 0
    at = labels.clamp(min=0).unsqueeze(1)
    z = (x @ w.t()) * scale
    top = z.amax(dim=1, keepdim=True)
    p = torch.exp(z - top)
    total = p.sum(dim=1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(1)
    loss = torch.where(live, lse - z.gather(1, at).squeeze(1), torch.zeros_like(lse))
    if not case["train"]:
        return {"loss": loss, "lse": lse}
    del z
    p /= total
    p.scatter_add_(1, at, torch.full_like(total, -1.0))
    p *= torch.where(live, s["gout"] * scale, torch.zeros_like(lse)).unsqueeze(1)
    return {"loss": loss, "lse": lse, "dx": (p @ w).to(BF16), "dw": (p.t() @ x).to(BF16)}


def _plain_orth(s):
    x = s["m"].to(F32)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    x = x / (x.square().sum(dim=(1, 2), keepdim=True).sqrt() + NORM_EPS)
    a, b, c = COEF
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return {"out": (x.transpose(1, 2) if tall else x).to(BF16).contiguous()}


def _plain_linear(s):
    case = s["case"]
    codes, exps = _mx4_codes(s["x"].to(F32))
    xv = _mx4_values(codes, exps, case["in"])
    wv = _mx4_unpack(s["wq"], s["ws"], case["out"], case["in"])
    return {"y": (xv @ wv.t()).to(DT[case["y"]])}


def _plain_store(s):
    codes, exps = _mx4_codes(s["x"].to(F32))
    return {"values": _mx4_values(codes, exps, s["case"]["cols"]).to(BF16), "scales": torch.exp2(exps.to(F32))}


# ------------------------------------------------------------------ the framework's calls
_handles = {}  # a program makes the handle of a shape once and keeps it


def _handle(kind, *shape):
    from paper_2407_11698_gb300 import binding as nb
    key = (kind,) + shape
    if key not in _handles:
        _handles[key] = getattr(nb, kind)(*shape)
    return nb, _handles[key]


def _own_xent(s):
    case = s["case"]
    n, d, c = case["rows"], case["features"], case["classes"]
    _, h = _handle("SoftmaxXent", n, d, c)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    h.forward(s["x"], s["w"], s["labels"], loss, lse, scale=s["scale"])
    if not case["train"]:
        return {"loss": loss, "lse": lse}
    dx = torch.empty(n, d, dtype=BF16, device="cuda")
    dw = torch.empty(c, d, dtype=BF16, device="cuda")
    h.backward(s["x"], s["w"], s["labels"], lse, s["gout"], dx, dw, scale=s["scale"])
    return {"loss": loss, "lse": lse, "dx": dx, "dw": dw}


def _own_orth(s):
    case = s["case"]
    _, h = _handle("Orthogonalizer", case["count"], case["rows"], case["cols"])
    out = torch.empty(case["count"], case["rows"], case["cols"], dtype=BF16, device="cuda")
    h.run(s["m"], out, steps=STEPS, coef=COEF)
    return {"out": out}


def _own_linear(s):
    case = s["case"]
    _, h = _handle("Mx4Linear", case["rows"], case["in"], case["out"])
    y = torch.empty(case["rows"], case["out"], dtype=DT[case["y"]], device="cuda")
    h.run(s["x"], s["wq"], s["ws"], y)
    return {"y": y}


def _own_store(s):
    from paper_2407_11698_gb300 import binding as nb
    rows, cols = s["case"]["rows"], s["case"]["cols"]
    nq, ns = nb.mx4_bytes(rows, cols)
    q = torch.empty(nq, dtype=torch.uint8, device="cuda")
    sc = torch.empty(ns, dtype=torch.uint8, device="cuda")
    nb.mx4_quantize(s["x"], q, sc)
    values = torch.empty(rows, cols, dtype=BF16, device="cuda")
    scales = torch.empty(rows, -(-cols // 32), device="cuda")
    nb.mx4_dequantize(q, sc, values, scales)
    return {"values": values, "scales": scales}


PLAIN = {"xent": _plain_xent, "orth": _plain_orth, "linear": _plain_linear, "store": _plain_store}
OWN = {"xent": _own_xent, "orth": _own_orth, "linear": _own_linear, "store": _own_store}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["kind"]](state)


# ------------------------------------------------------------------ work
def work(case):
    size = {"bf16": 2, "f32": 4, "i64": 8, "i8": 1}
    if case["kind"] == "xent":
        n, d, c = case["rows"], case["features"], case["classes"]
        x = size[case["x"]] * n * d
        if not case["train"]:
            return {"bytes": x + 2 * c * d + 12 * n, "flops": 2 * n * d * c}
        return {"bytes": x + 2 * c * d + 16 * n + 2 * n * d + 2 * c * d, "flops": 6 * n * d * c}
    if case["kind"] == "orth":
        m, n = sorted((case["rows"], case["cols"]))
        # the two symmetric products by halves
        return {"bytes": (size[case["m"]] + 2) * case["count"] * m * n, "flops": case["count"] * STEPS * (3 * m * m * n + m ** 3)}
    if case["kind"] == "linear":
        r, k, n = case["rows"], case["in"], case["out"]
        return {"bytes": size[case["x"]] * r * k + n * (-(-k // 32)) * 17 + size[case["y"]] * r * n, "flops": 2 * r * k * n}
    r, c = case["rows"], case["cols"]
    return {"bytes": (size[case["x"]] + 2) * r * c + 4 * r * (-(-c // 32)), "flops": 0}


# ------------------------------------------------------------------ in 64 bits
def _exact_mx4(x):
    """(values, scales) of x in 64 bits: the nearest of the fifteen values, of two the one whose code is even."""
    x = x.double()
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % 32)).unflatten(1, (-1, 32))
    big = x.abs().max(dim=2, keepdim=True).values
    e = torch.where(big > 0, torch.floor(torch.log2(big.clamp(min=2.0 ** -140))), torch.full_like(big, -127.0))
    e = torch.where(big >= 2.0 ** (e + 1), e + 1, torch.where((big < 2.0 ** e) & (big > 0), e - 1, e))
    scale = 2.0 ** torch.where(big > 0, e - 2, e).clamp(-127, 127)
    u = x / scale
    # within [2^j, 2^(j+1)) the values lie 2^(j-1) apart, below 1 they lie 1/2 apart; torch rounds halves to even,
    # which is the even code
    step = torch.where(u.abs() < 2, 0.5, torch.where(u.abs() < 4, 1.0, 2.0))
    v = (torch.round(u / step) * step).clamp(-6, 6)
    return (v * scale).flatten(1)[:, :cols], scale.squeeze(2)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "xent":
        if work(case)["flops"] > 1.2e13:
            return None
        x, w, live = s["x"].double(), s["w"].double(), s["labels"] >= 0
        z = x @ w.mT * s["scale"]
        lse = torch.logsumexp(z, dim=1)
        hot = torch.zeros_like(z)
        hot[live, s["labels"][live].long()] = 1.0
        loss = torch.where(live, lse - (z * hot).sum(dim=1), 0.0)
        if not case["train"]:
            return {"loss": loss, "lse": lse}
        g = torch.exp(z - lse[:, None]).sub_(hot)
        del z, hot
        g *= (s["gout"].double() * s["scale"] * live)[:, None]
        return {"loss": loss, "lse": lse, "dx": g @ w, "dw": g.mT @ x}
    if case["kind"] == "orth":
        x = s["m"].double()
        flip = case["rows"] > case["cols"]
        x = x.mT if flip else x
        x = x / (torch.linalg.matrix_norm(x)[:, None, None] + NORM_EPS)
        for _ in range(STEPS):
            gram = torch.bmm(x, x.mT)
            x = COEF[0] * x + torch.bmm(COEF[1] * gram + COEF[2] * torch.bmm(gram, gram), x)
        return {"out": x.mT.contiguous() if flip else x}
    if case["kind"] == "linear":
        g = torch.Generator(device="cuda").manual_seed(seed)
        _normal(g, case["rows"], case["in"])
        wv = _exact_mx4(_normal(g, case["out"], case["in"]) / math.sqrt(case["in"]))[0]
        return {"y": _exact_mx4(s["x"])[0] @ wv.mT}
    v, sc = _exact_mx4(s["x"])
    return {"values": v, "scales": sc}

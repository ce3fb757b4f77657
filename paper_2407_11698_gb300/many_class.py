"""A head over many classes on the activations of integer blocks.

The paper's output layer holds at most 64 classes.  ``ManyClassHead`` puts a bf16
linear head on the int8 activations of trained blocks: it trains on softmax cross
entropy (``SoftmaxXent``), orthogonalises the momentum of its gradient before every
update (``Orthogonalizer``) and answers with its weights in 4 bits (``Mx4Linear``).

``GatedHead`` puts more between the two: the block's map is normalised by groups of
channels (``GroupNorm``), goes through a gated block (``GatedLinear``), whose outputs the
class matrix takes, and the gradients of all of it are clipped together (``GradClip``).

``python -m paper_2407_11698_gb300.many_class`` trains one integer block and a
``ManyClassHead`` on synthetic images and prints the loss and both forms' accuracy; with
``--gated`` a ``GatedHead``.
"""
import math
import sys

import torch

from . import binding as nb


class ManyClassHead:
    """z = scale x W^T on int8 features x [rows x features], W [classes x features] bf16.

    scale: 1 / 32 suits activations that fill int8 (the logits of W ~ 1 / sqrt(features)
    are then of order 1).  step() takes W by lr sqrt(max(classes, features)) times an
    orthogonal matrix, so an entry moves by about lr."""

    def __init__(self, features, classes, max_rows, lr=0.002, momentum=0.9, scale=1.0 / 32, seed=0, device="cuda"):
        g = torch.Generator(device="cpu").manual_seed(seed)
        w = torch.randn(classes, features, generator=g) / math.sqrt(features)
        self.master = w.to(device)                       # fp32; the calls take the bf16 copy
        self.w = self.master.to(torch.bfloat16)
        self.m = torch.zeros_like(self.master)
        self.dw = torch.empty_like(self.w)
        self.update = torch.empty_like(self.w)
        self.lr, self.momentum, self.scale = lr, momentum, scale
        self.features, self.classes, self.max_rows = features, classes, max_rows
        self.loss_op = nb.SoftmaxXent(max_rows, features, classes)
        self.orth_op = nb.Orthogonalizer(1, classes, features)
        self.serve_op = None
        self.stale = True                                # whether the 4-bit weights are of an older W

    def step(self, x, labels):
        """One training step on x int8 [rows x features], labels int32 (-1: left out); returns
        the mean loss over the rows with a label (a CUDA tensor, not synchronised)."""
        n = x.shape[0]
        loss = torch.empty(n, device=x.device)
        lse = torch.empty(n, device=x.device)
        self.loss_op.forward(x, self.w, labels, loss, lse, scale=self.scale)
        live = (labels >= 0).sum().clamp(min=1).to(torch.float32)
        gout = (1.0 / live).expand(n).contiguous()
        self.loss_op.backward(x, self.w, labels, lse, gout, None, self.dw, scale=self.scale)
        self.m.mul_(self.momentum).add_(self.dw)
        self.orth_op.run(self.m, self.update)
        self.master.add_(self.update, alpha=-self.lr * math.sqrt(max(self.classes, self.features)))
        self.w.copy_(self.master)
        self.stale = True
        return loss.sum() / live

    def logits(self, x):
        """The logits of x in bf16 weights, for comparison (a plain product)."""
        return (x.to(torch.float32) @ self.w.to(torch.float32).t()) * self.scale

    def serve(self, x):
        """The logits of x (int8) from the weights and the features in 4 bits."""
        if self.serve_op is None:
            nq, ns = nb.mx4_bytes(self.classes, self.features)
            self.q = torch.empty(nq, dtype=torch.uint8, device=x.device)
            self.s = torch.empty(ns, dtype=torch.uint8, device=x.device)
            self.serve_op = nb.Mx4Linear(self.max_rows, self.features, self.classes)
        if self.stale:
            nb.mx4_quantize(self.w, self.q, self.s)
            self.stale = False
        y = torch.empty(x.shape[0], self.classes, dtype=torch.float32, device=x.device)
        self.serve_op.run(x.to(torch.bfloat16), self.q, self.s, y)
        return y * self.scale

    def status(self):
        """The first latched status of the head's handles that is not NITRO_OK, or that."""
        for op in (self.loss_op, self.orth_op, self.serve_op):
            st = op.status() if op is not None else nb.NITRO_OK
            if st != nb.NITRO_OK:
                return st
        return nb.NITRO_OK

    def close(self):
        for op in (self.loss_op, self.orth_op, self.serve_op):
            if op is not None:
                op.close()


class GatedHead:
    """logits = (act(n Wg^T) * (n Wu^T)) Wc^T with n = act(group norm of x), on int8 maps x [rows x pixels x channels].

    Wg and Wu are one matrix w1 [2 hidden x features], features = pixels * channels; Wc is w2 [classes x hidden], both bf16
    with an fp32 master.  step() scales all gradients so that their norm together is at most max_norm (gradients whose norm, kept in
    self.norm, is infinite or NaN go on as they are), and takes the matrices by orthogonal updates as ManyClassHead does,
    the gate and the up matrix each by itself, the norm's scales and shifts by lr times their momentum."""

    def __init__(self, pixels, channels, groups, hidden, classes, max_rows, lr=0.002, momentum=0.9, max_norm=1.0, seed=0, device="cuda"):
        g = torch.Generator(device="cpu").manual_seed(seed)
        features = pixels * channels
        self.pixels, self.channels, self.groups, self.features = pixels, channels, groups, features
        self.hidden, self.classes, self.max_rows = hidden, classes, max_rows
        self.lr, self.momentum, self.max_norm = lr, momentum, max_norm
        self.masters = [(torch.randn(2 * hidden, features, generator=g) / math.sqrt(features)).to(device),
                        (torch.randn(classes, hidden, generator=g) / math.sqrt(hidden)).to(device)]
        self.w = [m.to(torch.bfloat16) for m in self.masters]
        self.gamma, self.beta = torch.ones(channels, device=device), torch.zeros(channels, device=device)
        self.dw = [torch.empty_like(w) for w in self.w]
        self.dgamma, self.dbeta = torch.empty_like(self.gamma), torch.empty_like(self.beta)
        self.updates = [torch.empty_like(w) for w in self.w]
        self.m = [torch.zeros_like(m) for m in self.masters] + [torch.zeros_like(self.gamma), torch.zeros_like(self.beta)]
        self.norm = torch.zeros((), device=device)
        self.norm_op = nb.GroupNorm(max_rows, pixels, channels, groups)
        self.gate_op = nb.GatedLinear(max_rows, features, hidden)
        self.loss_op = nb.SoftmaxXent(max_rows, hidden, classes)
        self.orth_ops = [nb.Orthogonalizer(2, hidden, features), nb.Orthogonalizer(1, classes, hidden)]
        grads = self.dw + [self.dgamma, self.dbeta]
        self.clip_op = nb.GradClip(grads, grads)
        self.serve_op = None
        self.stale = True               # the 4-bit class matrix lags behind w[1]

    def _hidden(self, x, train):
        """(block's output, and for a backward what the calls hand on)"""
        n = x.shape[0]
        y = torch.empty(n, self.pixels, self.channels, dtype=torch.bfloat16, device=x.device)
        h = torch.empty(n, self.hidden, dtype=torch.bfloat16, device=x.device)
        mean = rstd = saved = None
        if train:
            mean, rstd = (torch.empty(n, self.groups, device=x.device) for _ in range(2))
            saved = torch.empty(n, 2 * self.hidden, device=x.device)
        self.norm_op.forward(x, self.gamma, self.beta, y, mean, rstd, act=nb.NITRO_ACT_SILU)
        y = y.view(n, self.features)
        self.gate_op.forward(y, self.w[0], h, saved, act=nb.NITRO_ACT_SILU)
        return h, (y, mean, rstd, saved)

    def gradients(self, x, labels):
        """The rows' losses (fp32) for x int8 [rows x pixels x channels] and labels int32 (-1: left out), and the gradients
        of their mean in dw, dgamma and dbeta, as they are."""
        n = x.shape[0]
        h, (y, mean, rstd, saved) = self._hidden(x, True)
        loss, lse = torch.empty(n, device=x.device), torch.empty(n, device=x.device)
        self.loss_op.forward(h, self.w[1], labels, loss, lse)
        gout = (1.0 / (labels >= 0).sum().clamp(min=1).to(torch.float32)).expand(n).contiguous()
        dh, dy = torch.empty_like(h), torch.empty_like(y)
        self.loss_op.backward(h, self.w[1], labels, lse, gout, dh, self.dw[1])
        self.gate_op.backward(y, self.w[0], saved, dh, dy, self.dw[0], act=nb.NITRO_ACT_SILU)
        self.norm_op.backward(x, self.gamma, self.beta, mean, rstd, dy.view(n, self.pixels, self.channels), None, self.dgamma,
                              self.dbeta, act=nb.NITRO_ACT_SILU)
        return loss, gout

    def step(self, x, labels):
        """One training step; returns the mean loss over the rows with a label.  The gradients' norm before clipping is
        in self.norm (CUDA tensors, not synchronised)."""
        loss, gout = self.gradients(x, labels)
        self.clip_op.run(self.norm, self.max_norm)
        for m, d in zip(self.m, self.dw + [self.dgamma, self.dbeta]):
            m.mul_(self.momentum).add_(d)
        pair = lambda t: t.view(2, self.hidden, self.features)      # the gate and the up matrix, each by itself
        self.orth_ops[0].run(pair(self.m[0]), pair(self.updates[0]))
        self.orth_ops[1].run(self.m[1], self.updates[1])
        # an entry of an orthogonal rows x cols matrix is 1 / sqrt(max(rows, cols)) in the mean square: times lr, here
        longest = max(self.hidden, self.features), max(self.classes, self.hidden)
        for master, w, u, n in zip(self.masters, self.w, self.updates, longest):
            master.add_(u, alpha=-self.lr * math.sqrt(n))
            w.copy_(master)
        for p, m in zip((self.gamma, self.beta), self.m[2:]):
            p.add_(m, alpha=-self.lr)
        self.stale = True
        return (loss * gout).sum()

    def logits(self, x):
        """The logits of x with bf16 class weights, for comparison (a plain product)."""
        return self._hidden(x, False)[0].to(torch.float32) @ self.w[1].to(torch.float32).t()

    def serve(self, x):
        """The logits of x with the class matrix and its inputs in 4 bits."""
        if self.serve_op is None:
            nq, ns = nb.mx4_bytes(self.classes, self.hidden)
            self.q = torch.empty(nq, dtype=torch.uint8, device=x.device)
            self.s = torch.empty(ns, dtype=torch.uint8, device=x.device)
            self.serve_op = nb.Mx4Linear(self.max_rows, self.hidden, self.classes)
        if self.stale:
            nb.mx4_quantize(self.w[1], self.q, self.s)
            self.stale = False
        out = torch.empty(x.shape[0], self.classes, dtype=torch.float32, device=x.device)
        return self.serve_op.run(self._hidden(x, False)[0], self.q, self.s, out)

    def _ops(self):
        return [self.norm_op, self.gate_op, self.loss_op, self.clip_op, *self.orth_ops] + ([self.serve_op] if self.serve_op else [])

    def status(self):
        """The first latched status of the head's handles that is not NITRO_OK, or that."""
        return next((st for st in (op.status() for op in self._ops()) if st != nb.NITRO_OK), nb.NITRO_OK)

    def close(self):
        for op in self._ops():
            op.close()


def demo(steps=60, batch=128, classes=1000, seed=3, log=print, gated=False):
    """Images of `classes` prototypes with noise through one integer conv block and the head (with `gated` a GatedHead);
    the block trains on the class modulo 10.  Returns (first loss, last loss, accuracy with bf16 weights,
    accuracy with 4 bits)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    protos = torch.randint(-100, 101, (classes, 8 * 8 * 4), generator=g, device="cuda").to(torch.float32)
    block = nb.Block([(nb.NITRO_CONV3X3, 4, 64, 8, 8, 1)], 8 * 8 * 4, seed=seed, max_batch=batch)
    feats = torch.empty(batch, block.out_features, dtype=torch.int8, device="cuda")
    if gated:
        head, seen = GatedHead(16, 64, 8, 256, classes, batch, seed=seed), feats.view(batch, 16, 64)
    else:
        head, seen = ManyClassHead(block.out_features, classes, batch, seed=seed), feats

    def features(labels):
        noise = torch.randn(batch, protos.shape[1], generator=g, device="cuda") * 10
        x = (protos[labels] + noise).round().clamp(-127, 127).to(torch.int8)
        return x, block.forward(x, feats)

    losses = []
    for _ in range(steps):
        labels = torch.randint(0, classes, (batch,), generator=g, device="cuda")
        x, _ = features(labels)
        block.backward(x, (labels % 10).to(torch.int32), None)
        losses.append(head.step(seen, labels.to(torch.int32)))
        block.sgd()
    labels = torch.randint(0, classes, (batch,), generator=g, device="cuda")
    features(labels)
    acc = [(f(seen).argmax(dim=1) == labels).float().mean().item() for f in (head.logits, head.serve)]
    first, last = losses[0].item(), losses[-1].item()
    if head.status() != nb.NITRO_OK:
        raise nb.NitroError(head.status(), type(head).__name__)
    log("loss %.3f -> %.3f after %d steps; accuracy over %d classes: %.2f, with 4-bit weights and features %.2f"
        % (first, last, steps, classes, acc[0], acc[1]))
    head.close()
    block.close()
    return first, last, acc[0], acc[1]


if __name__ == "__main__":
    demo(gated="--gated" in sys.argv[1:])

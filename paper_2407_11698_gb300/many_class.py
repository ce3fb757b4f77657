"""A head over many classes on the activations of integer blocks.

The paper's output layer holds at most 64 classes.  ``ManyClassHead`` puts a bf16
linear head on the int8 activations of trained blocks: it trains on softmax cross
entropy (``SoftmaxXent``), orthogonalises the momentum of its gradient before every
update (``Orthogonalizer``) and answers with its weights in 4 bits (``Mx4Linear``).

``python -m paper_2407_11698_gb300.many_class`` trains one integer block and such a
head on synthetic images and prints the loss and both forms' accuracy.
"""
import math

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


def demo(steps=60, batch=128, classes=1000, seed=3, log=print):
    """Images of `classes` prototypes with noise through one integer conv block and the head;
    the block trains on the class modulo 10.  Returns (first loss, last loss, accuracy with bf16 weights,
    accuracy with 4 bits)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    protos = torch.randint(-100, 101, (classes, 8 * 8 * 4), generator=g, device="cuda").to(torch.float32)
    block = nb.Block([(nb.NITRO_CONV3X3, 4, 64, 8, 8, 1)], 8 * 8 * 4, seed=seed, max_batch=batch)
    head = ManyClassHead(block.out_features, classes, batch, seed=seed)
    feats = torch.empty(batch, block.out_features, dtype=torch.int8, device="cuda")

    def features(labels):
        noise = torch.randn(batch, protos.shape[1], generator=g, device="cuda") * 10
        x = (protos[labels] + noise).round().clamp(-127, 127).to(torch.int8)
        return x, block.forward(x, feats)

    losses = []
    for _ in range(steps):
        labels = torch.randint(0, classes, (batch,), generator=g, device="cuda")
        x, _ = features(labels)
        block.backward(x, (labels % 10).to(torch.int32), None)
        losses.append(head.step(feats, labels.to(torch.int32)))
        block.sgd()
    labels = torch.randint(0, classes, (batch,), generator=g, device="cuda")
    features(labels)
    acc = [(f(feats).argmax(dim=1) == labels).float().mean().item() for f in (head.logits, head.serve)]
    first, last = losses[0].item(), losses[-1].item()
    if head.status() != nb.NITRO_OK:
        raise nb.NitroError(head.status(), "ManyClassHead")
    log("loss %.3f -> %.3f after %d steps; accuracy over %d classes: %.2f, with 4-bit weights and features %.2f"
        % (first, last, steps, classes, acc[0], acc[1]))
    head.close()
    block.close()
    return first, last, acc[0], acc[1]


if __name__ == "__main__":
    demo()

"""The head's operators together: an integer block's activations, a head over a thousand
classes trained on them, and its answers from 4-bit weights."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb
from paper_2407_11698_gb300 import many_class

pytestmark = pytest.mark.gpu


def test_demo_learns():
    first, last, acc, acc4 = many_class.demo(steps=60, batch=256, classes=100, log=lambda s: None)
    assert last < 0.5 * first and acc > 0.8 and acc4 > 0.8


def test_a_step_is_what_its_calls_are():
    g = torch.Generator(device="cuda").manual_seed(1)
    head = many_class.ManyClassHead(200, 70, 64)
    x = torch.randint(-127, 128, (64, 200), generator=g, device="cuda").to(torch.int8)
    labels = torch.randint(-1, 70, (64,), generator=g, device="cuda", dtype=torch.int32)
    w0 = head.master.clone()
    loss = head.step(x, labels)
    z = (x.double() @ w0.to(torch.bfloat16).double().t()) * head.scale
    live = labels >= 0
    want = torch.nn.functional.cross_entropy(z[live], labels[live].long())
    assert (loss.double() - want).abs() < 1e-4 * want
    # every singular value of the update is near 1, so the weights moved by lr sqrt(200) in every direction
    sv = torch.linalg.svdvals((w0 - head.master).double()) / (head.lr * 200 ** 0.5)
    assert sv[:60].min() > 0.6 and sv.max() < 1.3
    assert head.status() == nb.NITRO_OK
    head.close()

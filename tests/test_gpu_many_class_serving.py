"""Training and serving a many-class head in turn: the 4-bit handle lives on, and what it latched is not lost."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb
from paper_2407_11698_gb300 import many_class

pytestmark = pytest.mark.gpu


def _head_and_data():
    g = torch.Generator(device="cuda").manual_seed(2)
    head = many_class.ManyClassHead(200, 70, 64)
    x = torch.randint(-127, 128, (64, 200), generator=g, device="cuda").to(torch.int8)
    labels = torch.randint(0, 70, (64,), generator=g, device="cuda", dtype=torch.int32)
    return head, x, labels


def test_answers_follow_the_weights():
    head, x, labels = _head_and_data()
    before = head.serve(x)
    handle = head.serve_op
    for _ in range(3):
        head.step(x, labels)
        y = head.serve(x)
        assert head.serve_op is handle
        fresh, _, _ = _head_and_data()
        fresh.w = head.w
        assert torch.equal(y, fresh.serve(x)) and not torch.equal(y, before)
        assert torch.equal(y, head.serve(x))            # and again from the same 4-bit weights
        fresh.close()
    assert head.status() == nb.NITRO_OK
    head.close()


def test_a_latched_status_survives_a_step():
    class Latched:
        closed = False

        def status(self, clear=False):
            return nb.NITRO_ERR_TIMEOUT

        def close(self):
            self.closed = True

    head, x, labels = _head_and_data()
    head.serve(x)
    head.serve_op.close()
    head.serve_op = latched = Latched()
    head.step(x, labels)
    assert head.status() == nb.NITRO_ERR_TIMEOUT
    head.close()
    assert latched.closed

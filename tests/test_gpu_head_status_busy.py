"""The status of a handle that was made while the default stream is busy: what its first calls on another stream
latch is not cleared once the default stream comes to it."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2407_11698_gb300 import binding as nb
from test_gpu_head_create_busy import busy, forward, make, still_busy


@pytest.mark.parametrize("rows", [3, 20])
def test_a_bad_label_is_kept(rows):
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x, w, labels, _ = make(rows)
        h = nb.SoftmaxXent(rows, 520, 700)
        forward(h, x, w, labels, side)
        bad = labels.clone()
        bad[rows - 1] = 700
    h.close()
    busy()
    h = nb.SoftmaxXent(rows, 520, 700)
    try:
        still_busy()
        with torch.cuda.stream(side):
            forward(h, x, w, bad, side)
            side.synchronize()
        still_busy()
        assert h.status() == nb.NITRO_ERR_ARG
        assert h.status(clear=True) == nb.NITRO_ERR_ARG and h.status() == nb.NITRO_OK
        with torch.cuda.stream(side):
            forward(h, x, w, bad, side)
        assert h.status() == nb.NITRO_ERR_ARG       # latched again after the clear
    finally:
        h.close()

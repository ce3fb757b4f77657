"""Handles of the floating-point head made while the default stream is busy and used at once on
another stream, and a handle whose first call is captured."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2407_11698_gb300 import binding as nb


def busy():
    torch.cuda.synchronize()
    torch.cuda._sleep(1 << 30)            # half a second, on the default stream


def still_busy():
    if torch.cuda.default_stream().query():
        pytest.skip("making the handle waited for the default stream: the test could not fail")


def make(rows):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, 520, generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn(700, 520, generator=g, device="cuda") / 20).to(torch.bfloat16)
    labels = torch.randint(0, 700, (rows,), generator=g, device="cuda", dtype=torch.int32)
    z = x.double() @ w.double().t()
    want = torch.logsumexp(z, 1)
    return x, w, labels, want


def forward(h, x, w, labels, stream):
    loss, lse = (torch.full((x.shape[0],), float("nan"), device="cuda") for _ in range(2))
    h.forward(x, w, labels, loss, lse, stream=stream)
    return lse


@pytest.mark.parametrize("rows", [3, 20])
def test_xent(rows):
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x, w, labels, want = make(rows)
        h = nb.SoftmaxXent(rows, 520, 700)
        forward(h, x, w, labels, side)
    h.close()
    busy()
    h = nb.SoftmaxXent(rows, 520, 700)
    try:
        still_busy()
        for _ in range(2):                # while the default stream is busy, and after
            with torch.cuda.stream(side):
                lse = forward(h, x, w, labels, side)
                side.synchronize()
                assert ((lse.double() - want).abs() < 1e-4).all()
            torch.cuda.synchronize()
    finally:
        h.close()


@pytest.mark.parametrize("rows", [3, 20])
def test_first_call_captured(rows):
    side = torch.cuda.Stream()
    x, w, labels, want = make(rows)
    h = nb.SoftmaxXent(rows, 520, 700)
    try:
        loss, lse = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                h.forward(x, w, labels, loss, lse, stream=side)
        first = forward(h, x, w, labels, None)
        assert ((first.double() - want).abs() < 1e-4).all()
        for _ in range(2):
            lse.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert ((lse.double() - want).abs() < 1e-4).all()
    finally:
        h.close()

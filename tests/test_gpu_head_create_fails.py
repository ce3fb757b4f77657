"""A handle that does not fit the device's memory: the call says so, and leaves nothing behind that later calls, of the
library or of the program around it, would take for an error of their own."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2407_11698_gb300 import binding as nb


def test_what_follows_is_not_blamed():
    a = torch.randint(-9, 10, (16, 16), device="cuda").to(torch.int8)
    b = torch.randint(-9, 10, (16, 16), dtype=torch.int32, device="cuda")
    c = torch.empty(16, 16, dtype=torch.int64, device="cuda")
    g = nb.IntGemm(16, 16, 16)
    free = torch.cuda.mem_get_info()[0]
    with pytest.raises(nb.NitroError) as e:
        nb.SoftmaxXent(1 << 20, 8, 1 << 23)         # 2 TB of row statistics: refused, not taken
    assert e.value.status == nb.NITRO_ERR_CUDA
    g.run(a, b, c)                                  # a call of the library
    d = torch.ones(100, device="cuda") * 2          # and one beside it
    assert d.sum().item() == 200
    assert torch.equal(c.cpu(), a.long().cpu() @ b.long().cpu().t())
    assert torch.cuda.mem_get_info()[0] >= free - (64 << 20)
    g.close()

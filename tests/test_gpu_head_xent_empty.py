"""The weight gradient of an empty batch into a view with wide rows: one operation on the stream, whatever the classes."""
import ctypes

import pytest
import torch

from paper_2407_11698_gb300 import binding as nb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("classes, features, pad, shift", [(5000, 64, 8, 0), (5000, 63, 2, 1), (1, 40, 3, 0), (3, 1, 0, 0), (70000, 5, 1, 1)])
def test_one_operation(classes, features, pad, shift):
    h = nb.SoftmaxXent(4, features, classes)
    w = torch.zeros(classes, features, dtype=torch.bfloat16, device="cuda")
    x = torch.empty(0, features, dtype=torch.bfloat16, device="cuda")
    labels, lse = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    wide = torch.ones(classes, features + pad, dtype=torch.bfloat16, device="cuda")
    dw = wide[:, shift:shift + features]
    h.backward(x, w, labels, lse, None, None, dw)
    torch.cuda.synchronize()
    assert (dw == 0).all()
    assert (wide[:, :shift] == 1).all() and (wide[:, shift + features:] == 1).all()
    rt = ctypes.CDLL("libcudart.so.13")
    side = torch.cuda.Stream()
    s, graph, n = ctypes.c_void_p(side.cuda_stream), ctypes.c_void_p(), ctypes.c_size_t()
    assert rt.cudaStreamBeginCapture(s, 2) == 0
    h.backward(x, w, labels, lse, None, None, dw, stream=side)
    assert rt.cudaStreamEndCapture(s, ctypes.byref(graph)) == 0
    assert rt.cudaGraphGetNodes(graph, None, ctypes.byref(n)) == 0
    rt.cudaGraphDestroy(graph)
    assert n.value == 1
    assert h.status() == nb.NITRO_OK
    h.close()

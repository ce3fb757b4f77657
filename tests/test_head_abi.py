"""Host-side checks of the floating-point head's calls (no GPU needed): what is refused
before any device call, the sizes of 4-bit matrices, and the binding's own checks."""
import ctypes

import pytest
import torch

from paper_2407_11698_gb300 import binding as nb
from paper_2407_11698_gb300 import build as nbuild


@pytest.fixture(scope="module")
def lib():
    nbuild.build()
    return nb.lib()


def _create(fn, *shape):
    h = ctypes.c_void_p(1)
    st = fn(*shape, ctypes.byref(h))
    return st, h.value


@pytest.mark.parametrize("shape", [(0, 8, 8), (8, 0, 8), (8, 8, 0), (-1, 8, 8), ((1 << 20) + 1, 8, 8), (8, 1 << 18, 8),
                                   (8, 8, (1 << 24) + 1), (1 << 20, 1 << 17, 8)])
def test_xent_sizes_refused(lib, shape):
    assert _create(lib.nitro_xent_create, *shape) == (nb.NITRO_ERR_ARG, None)


@pytest.mark.parametrize("shape", [(0, 8, 8), (1, 0, 8), (1, 8, 0), (4097, 8, 8), (1, 1 << 19, 8), (1, 1 << 16, 1 << 16)])
def test_orth_sizes_refused(lib, shape):
    assert _create(lib.nitro_orth_create, *shape) == (nb.NITRO_ERR_ARG, None)


@pytest.mark.parametrize("shape", [(0, 8, 8), (8, 0, 8), (8, 8, 0), ((1 << 20) + 1, 8, 8), (8, (1 << 20) + 1, 8)])
def test_mx4_sizes_refused(lib, shape):
    assert _create(lib.nitro_mx4_create, *shape) == (nb.NITRO_ERR_ARG, None)


def test_null_handles_and_pointers(lib):
    A = nb.NITRO_ERR_ARG
    for op in ("xent", "orth", "mx4"):
        assert getattr(lib, "nitro_%s_create" % op)(1, 1, 1, None) == A
        assert getattr(lib, "nitro_%s_status" % op)(None, 0) == A
        getattr(lib, "nitro_%s_destroy" % op)(None)
    assert lib.nitro_xent_forward(None, 16, 0, 8, 16, 8, 16, 1, 1.0, 16, 16, None) == A
    assert lib.nitro_xent_backward(None, 16, 0, 8, 16, 8, 16, 1, 1.0, 16, 16, 16, 8, 16, 8, None) == A
    assert lib.nitro_orth_run(None, 16, 0, 8, 64, 1, 5, None, 16, 8, 64, None) == A
    assert lib.nitro_mx4_linear(None, 16, 0, 8, 1, 16, 16, 16, 0, 8, None) == A
    assert lib.nitro_mx4_quantize(None, nb.NITRO_F32, 8, 1, 8, 16, 16, None) == A
    assert lib.nitro_mx4_quantize(16, nb.NITRO_F32, 8, 1, 8, None, 16, None) == A
    assert lib.nitro_mx4_quantize(16, nb.NITRO_F32, 7, 1, 8, 16, 16, None) == A       # stride below the columns
    assert lib.nitro_mx4_quantize(18, nb.NITRO_F32, 8, 1, 8, 16, 16, None) == A       # not aligned
    assert lib.nitro_mx4_quantize(16, nb.NITRO_F32, 8, 1, 8, 24, 16, None) == A
    assert lib.nitro_mx4_quantize(16, nb.NITRO_I8, 8, 1, 8, 16, 16, None) == A        # type
    assert lib.nitro_mx4_quantize(16, nb.NITRO_F32, 8, -1, 8, 16, 16, None) == A
    assert lib.nitro_mx4_dequantize(16, 16, 1, 8, None, nb.NITRO_F32, 8, None, None) == A
    assert lib.nitro_mx4_dequantize(16, 16, 1, 8, 16, nb.NITRO_F32, 8, 18, None) == A
    assert lib.nitro_mx4_bytes(1, 0, ctypes.byref(ctypes.c_size_t()), ctypes.byref(ctypes.c_size_t())) == A
    assert lib.nitro_mx4_bytes(1, 1, None, None) == A


@pytest.mark.parametrize("rows, cols, codes, scales", [(1, 1, 16, 512), (1, 32, 16, 512), (1, 33, 32, 512), (128, 128, 8192, 512),
                                                       (129, 129, 129 * 80, 2 * 2 * 512), (0, 5, 0, 0),
                                                       (77, 3000, 77 * 94 * 16, 24 * 512)])
def test_mx4_bytes(lib, rows, cols, codes, scales):
    q, s = ctypes.c_size_t(), ctypes.c_size_t()
    assert lib.nitro_mx4_bytes(rows, cols, ctypes.byref(q), ctypes.byref(s)) == nb.NITRO_OK
    assert (q.value, s.value) == (codes, scales) == nb.mx4_bytes(rows, cols)


def test_binding_refuses_tensors_that_are_not_on_the_gpu(lib):
    x = torch.zeros(4, 32)
    q, s = (torch.zeros(n, dtype=torch.uint8) for n in nb.mx4_bytes(4, 32))
    with pytest.raises(ValueError):
        nb.mx4_quantize(x, q, s)
    with pytest.raises(ValueError):
        nb.mx4_dequantize(q, s, x)

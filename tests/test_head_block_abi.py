"""Host-side checks of group norm, the gated block and gradient clipping (no GPU needed): what is refused before any
device call, and the binding's own checks."""
import ctypes

import pytest
import torch

from paper_2407_11698_gb300 import binding as nb
from paper_2407_11698_gb300 import build as nbuild

A = nb.NITRO_ERR_ARG


@pytest.fixture(scope="module")
def lib():
    nbuild.build()
    return nb.lib()


def _create(fn, *shape):
    h = ctypes.c_void_p(1)
    return fn(*shape, ctypes.byref(h)), h.value


@pytest.mark.parametrize("shape", [(0, 8, 8, 2), (8, 0, 8, 2), (8, 8, 0, 1), (8, 8, 8, 0), (8, 8, 8, 3), (65536, 8, 8, 2), (8, 8, 8193, 1),
                                   (8, 8, 2, 4), (1, (1 << 30) + 1, 8, 1), (1, 1 << 30, 8192, 1), (65535, 1 << 20, 8192, 1)])
def test_gnorm_sizes_refused(lib, shape):
    assert _create(lib.nitro_gnorm_create, *shape) == (A, None)


@pytest.mark.parametrize("shape", [(0, 8, 8), (8, 0, 8), (8, 8, 0), ((1 << 20) + 1, 8, 8), (8, (1 << 17) + 1, 8), (8, 8, (1 << 20) + 1),
                                   (1 << 20, 1 << 17, 8), (1 << 20, 8, 1 << 20), (8, 1 << 17, 1 << 20)])
def test_glu_sizes_refused(lib, shape):
    assert _create(lib.nitro_glu_create, *shape) == (A, None)


def test_null_handles_and_pointers(lib):
    assert lib.nitro_gnorm_create(1, 1, 1, 1, None) == A
    assert lib.nitro_glu_create(1, 1, 1, None) == A
    assert lib.nitro_clip_create(None, 0, None) == A
    for op in ("gnorm", "glu", "clip"):
        assert getattr(lib, "nitro_%s_status" % op)(None, 0) == A
        getattr(lib, "nitro_%s_destroy" % op)(None)
    assert lib.nitro_gnorm_forward(None, 16, 0, 8, 64, 1, 8, None, None, 1e-5, 0, 16, 0, 8, 64, None, None, None) == A
    assert lib.nitro_gnorm_backward(None, 16, 0, 8, 64, 1, 8, None, None, 16, 16, 0, 16, 0, 8, 64, 16, 8, 64, 16, 16, None) == A
    assert lib.nitro_glu_forward(None, 16, 0, 8, 16, 8, 1, 1.0, 0, 16, 8, None, None) == A
    assert lib.nitro_glu_backward(None, 16, 0, 8, 16, 8, 1, 1.0, 0, 16, 16, 8, 16, 8, 16, 8, None) == A
    assert lib.nitro_clip_run(None, 1.0, 16, None) == A


def _clip(lib, *rows):
    table = (nb.nitro_clip_matrix * max(1, len(rows)))(*[nb.nitro_clip_matrix(*r) for r in rows])
    return _create(lib.nitro_clip_create, table, len(rows))


B, F, L = nb.NITRO_BF16, nb.NITRO_F32, nb.NITRO_I64


@pytest.mark.parametrize("rows", [
    [(None, None, 1, 8, 8, 8, F)],                                             # no matrix
    [(4096, None, 1, 8, 8, 8, nb.NITRO_I8)],                                   # type
    [(4096, None, -1, 8, 8, 8, F)],
    [(4096, None, 1, -8, 8, 8, F)],
    [(4096, None, 2, 8, 7, 8, F)],                                             # stride below the columns
    [(4096, 8192, 2, 8, 8, 7, F)],
    [(4098, None, 1, 8, 8, 8, F)],                                             # not at a multiple of its type
    [(4096, 8193, 1, 8, 8, 8, B)],
    [(4096, 8192, 1, 8, 8, 8, L)],                                             # int64 is not scaled
    [(4096, None, 1 << 30, 1 << 30, 1 << 30, 1, F)],                           # more than 2^40 values
    [(4096, None, 1, 1 << 40, 1, 1, B), (4096, None, 1, 8, 8, 8, F)],
    [(4096, 4100, 1, 8, 8, 8, F)],                                             # out overlaps in, but is not it
    [(4096, 4096, 2, 8, 8, 9, F)],
    [(4096, 4096, 1, 8, 8, 8, F), (4112, 8192, 1, 8, 8, 8, F)],                # and another's in
    [(4096, 8192, 1, 8, 8, 8, F), (4160, 8208, 1, 8, 8, 8, F)],                # two outs
    [(4096, 4096, 1, 8, 8, 8, F), (4096, 4096, 1, 8, 8, 8, F)],                # the same matrix twice
    [(4096, 4096, 4, 8, 16, 16, F), (4124, 4124, 4, 8, 16, 16, F)],            # columns 0..7 and 7..14 of one buffer
    [(4096, 4096, 4, 8, 16, 16, F), (4128, 4128, 4, 8, 15, 15, F)],
    [(4096, 4096, 4, 8, 16, 16, F), (4096 + 4 * 9, 4096 + 4 * 9, 4, 8, 16, 16, F)],   # columns 9..16: into the next row
])
def test_clip_lists_refused(lib, rows):
    assert _clip(lib, *rows) == (A, None)


def test_clip_counts_refused(lib):
    assert _create(lib.nitro_clip_create, None, 1) == (A, None)
    assert _create(lib.nitro_clip_create, None, -1) == (A, None)
    table = (nb.nitro_clip_matrix * 1)()
    assert _create(lib.nitro_clip_create, table, (1 << 20) + 1) == (A, None)


def test_binding_refuses_tensors_that_are_not_on_the_gpu(lib):
    x = torch.zeros(2, 4, 8)
    h = object.__new__(nb.GroupNorm)
    h.channels, h.groups = 8, 2
    with pytest.raises(ValueError):
        h.forward(x, None, None, x)
    with pytest.raises(ValueError):
        h.backward(x, None, None, x, x, x)
    g = object.__new__(nb.GatedLinear)
    g.features, g.hidden = 8, 4
    with pytest.raises(ValueError):
        g.forward(x[0], torch.zeros(8, 8), torch.zeros(4, 4))
    with pytest.raises(ValueError):
        g.backward(x[0], torch.zeros(8, 8), torch.zeros(4, 8), torch.zeros(4, 4))
    with pytest.raises(ValueError):
        nb.GradClip([x])
    with pytest.raises(ValueError):
        nb.GradClip([x], [])

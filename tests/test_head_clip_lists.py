"""Which lists of matrices a clipping handle takes, without a GPU."""
import ctypes

import pytest

from paper_2407_11698_gb300 import binding as nb
from paper_2407_11698_gb300 import build as nbuild

F = nb.NITRO_F32


def _create(*rows):
    nbuild.build()
    table = (nb.nitro_clip_matrix * max(1, len(rows)))(*[nb.nitro_clip_matrix(*r) for r in rows])
    h = ctypes.c_void_p(1)
    st = nb.lib().nitro_clip_create(table, len(rows), ctypes.byref(h))
    if h.value:
        nb.lib().nitro_clip_destroy(h)
    return st


def _m(first, rows, cols, ld, base=1 << 20):
    """Columns from `first` on of a buffer of fp32 rows, scaled in place."""
    at = base + 4 * first
    return (at, at, rows, cols, ld, ld, F)


# columns of one buffer of rows of 64, some of them in its first row, in one in the middle or in its last row alone
@pytest.mark.parametrize("rows", [
    [_m(0, 50, 10, 64), _m(10, 1, 20, 64)],
    [_m(0, 50, 10, 64), _m(20 * 64 + 10, 1, 54, 64)],
    [_m(0, 50, 10, 64), _m(49 * 64 + 10, 1, 30, 64)],
    [_m(10, 50, 54, 64), _m(64, 1, 10, 64)],
    [_m(10, 50, 54, 64), _m(0, 1, 10, 64), _m(64, 1, 10, 64), _m(128, 48, 10, 64)],
    [_m(10, 50, 54, 64), _m(64 + 4, 1, 6, 6), _m(64, 2, 2, 2)],
])
def test_rows_beside_columns_are_taken(rows):
    assert _create(*rows) != nb.NITRO_ERR_ARG
    assert _create(*rows[::-1]) != nb.NITRO_ERR_ARG


@pytest.mark.parametrize("rows", [
    [_m(0, 50, 10, 64), _m(9, 1, 20, 64)],
    [_m(0, 50, 10, 64), _m(20 * 64 + 10, 1, 55, 64)],          # into the next row
    [_m(0, 50, 10, 64), _m(20 * 64 + 10, 1, 200, 64)],
    [_m(0, 50, 10, 64), _m(49 * 64 + 9, 1, 30, 64)],
    [_m(10, 50, 54, 64), _m(64, 1, 11, 64)],
    [_m(10, 50, 54, 64), _m(63, 1, 2, 64)],
    [_m(10, 50, 54, 64), _m(0, 1, 64 * 50, 64)],
])
def test_rows_across_columns_are_refused(rows):
    assert _create(*rows) == nb.NITRO_ERR_ARG
    assert _create(*rows[::-1]) == nb.NITRO_ERR_ARG

"""Calls of the layer normalisation and clipping entry points that are refused before anything is launched (no
GPU needed)."""
import ctypes as C

import pytest

from paper_2402_11857_b200 import liec
from test_operator_arguments import desc, lib  # noqa: F401  (fixture)


def test_outputs_that_overlap(lib):
    """2 workers, 8 rows of 64 binary32 (256 bytes a row): y, dx within x or dy; dweight within dbias."""
    at = 1 << 20
    forward = lambda d, x, y: lib.liec_layer_norm_forward(C.byref(d), x, None, None, y, 256, 256, None)
    backward = lambda d, dy=at, x=2 * at, dx=3 * at, dw=4 * at, db=5 * at: lib.liec_layer_norm_backward(
        C.byref(d), dy, x, 256, 256, None, dx, dw, db, 6 * at, 1 << 20, None)
    one_row_on = lambda p: p + 256
    slices = dict(x_row_stride=100, y_row_stride=100, dx_row_stride=100, x_group_stride=800, y_group_stride=800, dx_group_stride=800)
    for d, y in ((desc(), one_row_on(at)), (desc(), at + 4), (desc(), at - 256), (desc(), at + 2 * 512 * 4 - 4), (desc(**slices), at + 63 * 4),
                 (desc(**slices), at + 400 * 7), (desc(x_row_stride=0, x_group_stride=0), at - 512 * 4)):
        assert forward(d, at, y) == 1 and b"overlap" in lib.liec_last_error(None)
    for kw in (dict(dx=one_row_on(at)), dict(dx=one_row_on(2 * at)), dict(dx=2 * at - 4 * 512 * 2 + 4)):
        assert backward(desc(), **kw) == 1 and b"dx overlaps" in lib.liec_last_error(None)
    for kw in (dict(db=4 * at), dict(db=4 * at + 63 * 4), dict(db=4 * at - 63 * 4), dict(db=4 * at + 200 * 4 + 32), dict(db=4 * at + 137 * 4)):
        assert backward(desc(), **kw) == 1 and b"dweight and dbias" in lib.liec_last_error(None)
    assert backward(desc(groups=1, dweight_stride=0, dbias_stride=0), dw=4 * at, db=4 * at + 4) == 1

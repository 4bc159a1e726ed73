"""Argument checks of the layer normalisation and clipping entry points that need no GPU: a bad call is
refused before any CUDA call, with a message."""
import ctypes as C

import pytest

from paper_2402_11857_b200 import build as cuda_build
from paper_2402_11857_b200 import liec


@pytest.fixture(scope="module")
def lib():
    cuda_build.build()
    return liec.load_library()


def desc(**kw):
    d = liec.liec_layer_norm_desc()
    d.groups, d.rows, d.cols, d.dtype, d.grad_dtype, d.eps = 2, 8, 64, liec.F32, liec.F32, 1e-5
    d.x_row_stride = d.y_row_stride = d.dx_row_stride = 64
    d.x_group_stride = d.y_group_stride = d.dx_group_stride = 512
    d.weight_stride = d.bias_stride = d.dweight_stride = d.dbias_stride = 200
    for k, v in kw.items():
        setattr(d, k, v)
    return d


BAD = [(dict(groups=0), 1), (dict(groups=65536), 2), (dict(rows=-1), 1), (dict(rows=1 << 31), 2), (dict(cols=0), 1), (dict(cols=65537), 2),
       (dict(dtype=2), 1), (dict(grad_dtype=-1), 1), (dict(eps=-1e-9), 1), (dict(eps=float("inf")), 1), (dict(eps=float("nan")), 1),
       (dict(x_row_stride=-64), 1), (dict(weight_stride=-1), 1), (dict(dx_group_stride=1 << 41), 1)]


@pytest.mark.parametrize("change,status", BAD)
def test_bad_descs(lib, change, status):
    d = desc(**change)
    assert lib.liec_layer_norm_workspace_bytes(C.byref(d)) == 0
    assert lib.liec_layer_norm_forward(C.byref(d), 256, 256, 256, 512, 256, 256, None) == status
    assert lib.liec_last_error(None)
    assert lib.liec_layer_norm_backward(C.byref(d), 256, 256, 256, 256, 256, 512, 512, 512, 256, 1 << 30, None) == status


def test_bad_forward_pointers(lib):
    call = lambda d, x=256, w=256, b=256, y=512, m=256, r=256: lib.liec_layer_norm_forward(C.byref(d), x, w, b, y, m, r, None)
    assert lib.liec_layer_norm_forward(None, 256, 256, 256, 512, 256, 256, None) == 1
    assert call(desc(), x=None) == 1 and call(desc(), y=None) == 1 and call(desc(), y=256) == 1
    assert call(desc(), x=258) == 1 and call(desc(), y=513) == 1 and call(desc(), w=257) == 1 and call(desc(), r=254) == 1
    assert call(desc(dtype=liec.BF16), x=257) == 1
    for kw in (dict(y_row_stride=63), dict(y_row_stride=0), dict(y_group_stride=0), dict(y_group_stride=511),
               dict(y_group_stride=64, y_row_stride=127)):
        assert call(desc(**kw)) == 1
        assert b"overlap" in lib.liec_last_error(None)
    assert call(desc(rows=0), x=None, y=None) == 0          # nothing to do


def test_bad_backward_arguments(lib):
    def call(d, dy=256, x=256, m=256, r=256, w=256, dx=512, dw=512, db=512, ws=256, size=1 << 30):
        return lib.liec_layer_norm_backward(C.byref(d), dy, x, m, r, w, dx, dw, db, ws, size, None)
    for kw in (dict(dy=None), dict(x=None), dict(m=None), dict(r=None), dict(dx=256), dict(ws=None), dict(ws=264), dict(dw=514),
               dict(m=258), dict(x=257)):
        assert call(desc(), **kw) == 1, kw
    assert call(desc(dweight_stride=63)) == 1 and call(desc(dbias_stride=0)) == 1 and call(desc(dx_row_stride=32)) == 1
    need = lib.liec_layer_norm_workspace_bytes(C.byref(desc()))
    assert need >= 2 * 2 * 64 * 4
    assert call(desc(), size=0) == 3
    assert call(desc(), dx=None, dw=None, db=None) == 0     # nothing wanted


def test_workspace_grows_with_rows_and_stays_small(lib):
    for rows, cols in ((0, 64), (1, 1), (4096, 768), (1 << 20, 1024)):
        need = lib.liec_layer_norm_workspace_bytes(C.byref(desc(rows=rows, cols=cols, groups=1)))
        assert need <= max(16 << 20, rows * cols // 4)


def test_clipping_without_a_context(lib):
    assert lib.liec_clip_grads(None, 256, 256, 1.0, 0, None, None) == 1
    assert lib.liec_set_tensors(None, 256, 0, None) == 1
    assert lib.liec_gather_grads(None, 256, 1.0, 0, None, None) == 1

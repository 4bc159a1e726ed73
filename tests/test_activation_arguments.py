"""Argument checks of the operators on activations that need no GPU: a bad call is refused before any CUDA call, with a
message; calls with nothing to do succeed."""
import ctypes as C

import pytest

from paper_2402_11857_b200 import liec
from test_operator_arguments import lib  # noqa: F401  (fixture)

AT = 1 << 24   # places far apart


def activation(**kw):
    d = liec.liec_activation_desc()
    d.workers, d.rows, d.cols, d.dtype, d.x_row_stride, d.x_worker_stride = 2, 8, 40, liec.F32, 40, 320
    return change(d, kw)


def group_norm(**kw):
    d = liec.liec_group_norm_desc()
    d.workers, d.samples, d.pixels, d.channels, d.groups = 2, 3, 10, 24, 4
    d.dtype, d.grad_dtype, d.activation, d.eps = liec.F32, liec.F32, 2, 1e-5
    for name in ("x", "y", "dx"):
        for axis, step in (("pixel", 24), ("sample", 240), ("worker", 720)):
            setattr(d, f"{name}_{axis}_stride", step)
    d.weight_stride = d.bias_stride = d.dweight_stride = d.dbias_stride = 100
    return change(d, kw)


def weight_grad(**kw):
    d = liec.liec_weight_grad_desc()
    d.workers, d.rows, d.in_, d.out, d.dtype, d.grad_dtype = 2, 50, 40, 24, liec.F32, liec.F32
    d.dy_row_stride, d.dy_worker_stride, d.dweight_row_stride, d.dweight_worker_stride = 24, 1200, 40, 960
    return change(d, kw)


def change(d, kw):
    for k, v in kw.items():
        setattr(d, k, v)
    return d


BAD_ACTIVATION = [(dict(workers=0), 1), (dict(workers=65536), 2), (dict(rows=-1), 1), (dict(rows=1 << 31), 2), (dict(cols=0), 1), (dict(cols=65537), 2),
                  (dict(dtype=2), 1), (dict(x_row_stride=-1), 1), (dict(x_worker_stride=1 << 41), 1), (dict(workers=60000, rows=1 << 30, cols=65536), 2)]


@pytest.mark.parametrize("kw,status", BAD_ACTIVATION)
def test_bad_activation_descs(lib, kw, status):
    d = C.byref(activation(**kw))
    assert lib.liec_activation_compress(d, AT, 2 * AT, 3 * AT, None) == status and lib.liec_last_error(None)
    assert lib.liec_activation_restore(d, 2 * AT, 3 * AT, AT, None) == status


def test_activation_pointers(lib):
    compress = lambda d, x=AT, q=2 * AT, s=3 * AT: lib.liec_activation_compress(C.byref(d), x, q, s, None)
    restore = lambda d, x=AT, q=2 * AT, s=3 * AT: lib.liec_activation_restore(C.byref(d), q, s, x, None)
    for call in (compress, restore):
        assert call(activation(), x=None) == 1 and call(activation(), q=None) == 1 and call(activation(), s=None) == 1
        assert call(activation(), x=AT + 2) == 1 and call(activation(dtype=liec.BF16), x=AT + 1) == 1
        assert call(activation(), q=2 * AT + 8) == 1 and b"16-byte" in lib.liec_last_error(None)
        assert call(activation(), q=AT) == 1 and b"overlap" in lib.liec_last_error(None)
        assert call(activation(), s=AT + 4 * 639) == 1 and call(activation(), q=AT - 1024 + 16) == 1     # q: 16 rows of 64 bytes
        assert call(activation(rows=0), x=None, q=None, s=None) == 0
        assert lib.liec_activation_compress(None, AT, 2 * AT, 3 * AT, None) == 1
    assert compress(activation(), q=2 * AT, s=2 * AT + 1023) == 1
    for kw in (dict(x_row_stride=39), dict(x_row_stride=0), dict(x_worker_stride=0), dict(x_worker_stride=319)):
        assert restore(activation(**kw)) == 1 and b"overlap" in lib.liec_last_error(None)


def test_padded_columns(lib):
    for cols in (1, 31, 32, 33, 1000, 65536):
        assert lib.liec_activation_cols(cols) == liec.liec_activation_cols(cols) == -(-cols // 32) * 32
    assert lib.liec_activation_cols(0) == lib.liec_activation_cols(65537) == 0


BAD_GROUP_NORM = [(dict(workers=0), 1), (dict(workers=65536), 2), (dict(samples=-1), 1), (dict(pixels=-1), 1), (dict(pixels=1 << 31), 2), (dict(channels=0), 1),
                  (dict(channels=65544, groups=1), 2), (dict(groups=0), 1), (dict(groups=5), 1), (dict(dtype=7), 1), (dict(grad_dtype=-1), 1), (dict(activation=3), 1),
                  (dict(activation=-1), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(x_pixel_stride=-1), 1),
                  (dict(dbias_stride=1 << 41), 1), (dict(samples=1 << 30), 2), (dict(pixels=1 << 30, samples=1000), 2)]


@pytest.mark.parametrize("kw,status", BAD_GROUP_NORM)
def test_bad_group_norm_descs(lib, kw, status):
    d = C.byref(group_norm(**kw))
    assert lib.liec_group_norm_workspace_bytes(d, 0) == lib.liec_group_norm_workspace_bytes(d, 1) == 0
    assert lib.liec_group_norm_forward(d, AT, None, None, 2 * AT, 3 * AT, 4 * AT, None, None, 5 * AT, 1 << 20, None) == status and lib.liec_last_error(None)
    assert lib.liec_group_norm_backward(d, AT, 2 * AT, None, None, 3 * AT, 4 * AT, None, None, 5 * AT, 6 * AT, 7 * AT, 8 * AT, 1 << 20, None) == status


def test_group_norm_forward_pointers(lib):
    def call(d, x=AT, w=2 * AT, b=3 * AT, y=4 * AT, m=5 * AT, r=6 * AT, q=7 * AT, s=8 * AT, ws=9 * AT, size=1 << 24):
        return lib.liec_group_norm_forward(C.byref(d), x, w, b, y, m, r, q, s, ws, size, None)
    for kw in (dict(x=None), dict(y=None), dict(m=None), dict(r=None), dict(q=None), dict(s=None), dict(x=AT + 2), dict(y=4 * AT + 1), dict(w=2 * AT + 2),
               dict(q=7 * AT + 8), dict(y=AT), dict(y=AT + 96), dict(m=AT + 4 * 1439), dict(r=5 * AT + 4 * 23), dict(s=7 * AT + 60 * 32 - 1), dict(y=2 * AT - 4)):
        assert call(group_norm(), **kw) == 1, kw
    for kw in (dict(y_pixel_stride=23), dict(y_pixel_stride=0), dict(y_sample_stride=239), dict(y_worker_stride=719), dict(y_sample_stride=0)):
        assert call(group_norm(**kw)) == 1 and b"rows of y overlap" in lib.liec_last_error(None), kw
    for kw in (dict(samples=0), dict(pixels=0)):
        assert call(group_norm(**kw), x=None, y=None, m=None, r=None, q=None, s=None, ws=None) == 0
    big = group_norm(workers=2, samples=4, pixels=100000, x_sample_stride=2400000, x_worker_stride=9600000, y_sample_stride=2400000, y_worker_stride=9600000)
    far = 1 << 32
    need = lib.liec_group_norm_workspace_bytes(C.byref(big), 0)
    assert need > 0
    at = [far * k for k in range(1, 10)]
    assert lib.liec_group_norm_forward(C.byref(big), at[0], None, None, at[1], at[2], at[3], None, None, None, need, None) == 1
    assert lib.liec_group_norm_forward(C.byref(big), at[0], None, None, at[1], at[2], at[3], None, None, at[4], need - 256, None) == 3


def test_group_norm_backward_pointers(lib):
    def call(d, dy=AT, x=2 * AT, q=None, s=None, m=3 * AT, r=4 * AT, w=5 * AT, b=6 * AT, dx=7 * AT, dw=8 * AT, db=9 * AT, ws=10 * AT, size=1 << 24):
        return lib.liec_group_norm_backward(C.byref(d), dy, x, q, s, m, r, w, b, dx, dw, db, ws, size, None)
    for kw in (dict(dy=None), dict(x=None), dict(m=None), dict(r=None), dict(q=11 * AT, s=12 * AT), dict(x=None, q=11 * AT), dict(dx=AT), dict(dx=2 * AT + 4), dict(dw=9 * AT),
               dict(dw=9 * AT + 4 * 23), dict(dw=5 * AT), dict(ws=None), dict(ws=10 * AT + 8), dict(x=None, q=11 * AT + 8, s=12 * AT), dict(dx=7 * AT + 2), dict(db=2 * AT),
               dict(dx=11 * AT + 32, x=None, q=11 * AT, s=12 * AT)):
        assert call(group_norm(), **kw) == 1, kw
    assert call(group_norm(), size=0) == 3
    assert call(group_norm(dweight_stride=23)) == 1 and call(group_norm(dbias_stride=0)) == 1 and call(group_norm(dx_pixel_stride=12)) == 1
    assert call(group_norm(), dx=None, dw=None, db=None) == 0
    assert call(group_norm(pixels=0), dw=None, db=None) == 0


def test_workspaces_stay_small(lib):
    """Two sums per channel for every part of an image: at most a quarter of the activations, and no more than some MB for one image."""
    for kw in (dict(workers=8, samples=32, pixels=3136, channels=64, groups=32), dict(workers=1, samples=1, pixels=1 << 20, channels=128, groups=32),
               dict(workers=1, samples=1, pixels=64, channels=65536, groups=1), dict(workers=300, samples=7, pixels=9, channels=90, groups=5)):
        d = group_norm(**kw)
        for backward in (0, 1):
            need = lib.liec_group_norm_workspace_bytes(C.byref(d), backward)
            elements = kw["workers"] * kw["samples"] * kw["pixels"] * kw["channels"]
            assert need <= max(elements * 4 // 4, 8 * kw["workers"] * kw["samples"] * (kw["channels"] + kw["groups"]) + 512), (kw, backward, need)


BAD_WEIGHT_GRAD = [(dict(workers=0), 1), (dict(workers=65536), 2), (dict(rows=-1), 1), (dict(rows=1 << 31), 2), (dict(in_=0), 1), (dict(out=0), 1), (dict(in_=65537), 2),
                   (dict(out=65537), 2), (dict(dtype=2), 1), (dict(grad_dtype=-1), 1), (dict(dy_row_stride=-1), 1), (dict(dweight_worker_stride=1 << 41), 1),
                   (dict(workers=1000, in_=60000, out=60000), 2)]


@pytest.mark.parametrize("kw,status", BAD_WEIGHT_GRAD)
def test_bad_weight_grad_descs(lib, kw, status):
    d = C.byref(weight_grad(**kw))
    assert lib.liec_weight_grad_workspace_bytes(d, AT) == 0
    assert lib.liec_weight_grad(d, AT, 2 * AT, 3 * AT, 4 * AT, 5 * AT, 1 << 30, None) == status and lib.liec_last_error(None)


def test_weight_grad_pointers_and_workspace(lib):
    def call(d, dy=AT, q=2 * AT, s=3 * AT, dw=4 * AT, ws=5 * AT, size=1 << 30):
        return lib.liec_weight_grad(C.byref(d), dy, q, s, dw, ws, size, None)
    for kw in (dict(dy=None), dict(q=None), dict(s=None), dict(dw=None), dict(dy=AT + 2), dict(dw=4 * AT + 2), dict(q=2 * AT + 8),
               dict(dw=AT), dict(dw=2 * AT), dict(dw=3 * AT + 4), dict(dw=AT + 4 * 2399)):
        assert call(weight_grad(), **kw) == 1, kw
    for kw in (dict(ws=None), dict(ws=5 * AT + 8)):
        assert call(weight_grad(dy_row_stride=25), **kw) == 1, kw
    assert call(weight_grad(dy_row_stride=25), size=0) == 3
    assert call(weight_grad(dweight_row_stride=39)) == 1 and call(weight_grad(dweight_worker_stride=0)) == 1 and call(weight_grad(dweight_worker_stride=959)) == 1
    need = lambda at=AT, **kw: lib.liec_weight_grad_workspace_bytes(C.byref(weight_grad(**kw)), at)
    # a dy with rows on 16 bytes goes as it is, any other is packed
    bf = dict(dtype=liec.BF16, workers=40)
    assert need(**bf) == 0 and need(at=AT + 2, **bf) >= 40 * 50 * 24 * 2 and need(dy_row_stride=25, **bf) >= 40 * 50 * 24 * 2
    f32 = dict(dtype=liec.F32, workers=40)
    assert need(**f32) == 0 and need(at=AT + 4, **f32) >= 40 * 50 * 24 * 4 and need(dy_row_stride=26, **f32) >= 40 * 50 * 24 * 4
    assert need(rows=0) == 0
    # runs of tokens never take more than a place for each of some 16 x 74 pieces of 256 x 512
    assert need(dtype=liec.BF16, rows=1 << 20, dy_worker_stride=24 << 20) <= 16 * 74 * 256 * 512 * 4


def test_sizes_that_the_descriptor_cannot_hold(lib):
    """Sizes beyond 32 bits are refused, not cut to what is left of them (broadcast tensors reach them without memory)."""
    import torch
    bf16, wide = torch.bfloat16, (1 << 32) + 2
    f32 = torch.float32
    vector = ((8,), (1,), f32)
    for shape in ((wide, 1, 1, 8), (1, wide, 1, 8)):
        images = (shape, (0, 0, 8, 1), bf16)
        with pytest.raises(ValueError, match="2\\^31"):
            liec._gn_desc(images, True, images, None, None, None, None, None, 4, "none", 1e-5)
        with pytest.raises(ValueError, match="2\\^31"):
            liec._gn_desc(images, True, images, images, None, None, vector, vector, 4, "none", 1e-5)
    with pytest.raises(ValueError, match="2\\^31"):
        liec._activation_desc("x", ((3, wide), (0, 1), bf16))
    for dy, dweight, cols in ((((wide, 4, 8), (0, 8, 1), bf16), ((wide, 8, 8), (64, 8, 1), f32), 8),
                              (((2, 4, wide), (0, 0, 1), bf16), ((2, wide, 8), (0, 8, 1), f32), 8),
                              (((2, 4, 8), (32, 8, 1), bf16), ((2, 8, wide), (0, 0, 1), f32), wide)):
        with pytest.raises(ValueError, match="2\\^31"):
            liec._wg_desc(dy, dweight, cols, 0)

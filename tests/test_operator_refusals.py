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


def shared_layouts():
    """x, dy and dx of the backward pass with one weight for three workers: what the forward pass takes as well."""
    import torch
    full = torch.empty(3, 10, 64)
    dense = lambda t: torch.empty_like(t, memory_format=torch.contiguous_format)
    yield "no rows", full[:, :0], dense(full[:, :0])
    yield "the last row of each", full[:, -1:], dense(full[:, -1:])
    yield "the first rows", full[:, :4], dense(full[:, :4])
    yield "every second row", full[:, ::2], dense(full[:, ::2])
    yield "workers inside", full.transpose(0, 1).contiguous().transpose(0, 1), dense(full)
    yield "dy broadcast over rows", full, full[:, :1].expand(3, 10, 64)
    yield "dy broadcast over workers", full, full[:1].expand(3, 10, 64)
    yield "dy broadcast over both", full, full[:1, :1].expand(3, 10, 64)
    yield "one after another", full, dense(full)


@pytest.mark.parametrize("name,x,dy", list(shared_layouts()), ids=lambda v: v if isinstance(v, str) else "")
def test_layouts_with_a_shared_gradient(lib, name, x, dy):
    import torch
    vector, dx = torch.empty(64), torch.empty(x.shape)
    layout = liec._layout
    d, _, need = liec._ln_desc(layout(x), layout(dy), layout(dx), layout(vector), None, layout(vector), layout(vector), 0.0)
    assert d.groups * d.rows == x.shape[0] * x.shape[1] or d.rows == 0
    # every row of the descriptor is the row of the tensors that it stands for, in the same order
    for t, row, group in ((x, d.x_row_stride, d.x_group_stride), (dy, d.y_row_stride, d.y_group_stride), (dx, d.dx_row_stride, d.dx_group_stride)):
        want = [n * t.stride(0) + r * t.stride(1) for n in range(x.shape[0]) for r in range(x.shape[1])]
        assert [g * group + r * row for g in range(d.groups) for r in range(d.rows)] == want
    assert bool(d.shared_grads) == (d.groups > 1)
    assert need >= 0


@pytest.mark.parametrize("shared", [0, 1])
@pytest.mark.parametrize("groups,rows,cols", [(1, 1, 1), (1, 4096, 768), (32, 4096, 768), (1, 1 << 20, 1024), (2, 2_200_000, 1024), (4, 4096, 4096),
                                              (300, 7, 96), (5000, 40, 64), (4, 4096, 16384), (1, 512, 65536), (65535, 1, 8)])
def test_workspace_is_what_the_pieces_need(lib, groups, rows, cols, shared):
    """A piece is two rows of column sums: one per resident CTA (148 SMs, at most 3 each) or per 1024 rows of a CTA of
    at least one row at a time, whichever is more, and one more per worker."""
    d = desc(groups=groups, rows=rows, cols=cols, shared_grads=shared, x_group_stride=rows * 64)
    need = lib.liec_layer_norm_workspace_bytes(C.byref(d))
    pieces = max(3 * 148, -(-groups * rows // 1024)) + 1 + groups
    assert 8 * cols * groups <= need <= 8 * cols * pieces + 256

"""Layer normalisation at the edges of what a call may be given: workspaces, layouts, outputs that do not fit."""
import pytest
import torch

from paper_2402_11857_b200 import liec
from test_gpu_layer_norm import DT, check_backward, draw

pytestmark = pytest.mark.gpu

forward, backward = liec.liec_layer_norm_forward, liec.liec_layer_norm_backward


def test_workspace_that_is_larger_in_name_only():
    """An expanded or strided tensor counts more bytes than lie behind its first one."""
    x, dy, w, b = draw(2, 600, 64, "f32", seed=2)
    _, mean, rstd = forward(x, w, b)
    for bad in (torch.empty(1, device="cuda").expand(1 << 22), torch.empty(1 << 22, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            backward(dy, x, mean, rstd, w, workspace=bad)
    fine = torch.empty(1 << 22, device="cuda")
    check_backward(dy, x, mean, rstd, w, "f32", "f32", *backward(dy, x, mean, rstd, w, workspace=fine))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,rows,h", [(3, 5, 64), (2, 40, 257), (1, 9, 1000), (4, 1, 48)])
def test_slices_of_one_buffer(N, rows, h, dtype):
    """x and y, dy and dx side by side in one buffer, dweight and dbias in one row: they do not overlap."""
    x, dy, w, b = draw(N, rows, h, dtype, seed=6)
    want = forward(x, w, b)
    both = torch.zeros(N, rows, 2 * h + 3, dtype=DT[dtype], device="cuda")
    both[..., :h] = x
    y, mean, rstd = forward(both[..., :h], w, b, y=both[..., h + 3:])
    assert torch.equal(y, want[0]) and torch.equal(both[..., :h], x) and (both[..., h:h + 3] == 0).all()
    inner = torch.zeros(rows, N, 2 * h, dtype=DT[dtype], device="cuda").transpose(0, 1)   # the same with the workers inside
    inner[..., h:] = dy
    grads = torch.zeros(N, 2 * h, device="cuda")
    dx, dw, db = backward(inner[..., h:], x, mean, rstd, w, dx=inner[..., :h], dweight=grads[:, h:], dbias=grads[:, :h])
    check_backward(dy, x, mean, rstd, w, dtype, "f32", dx, dw, db)
    assert torch.equal(inner[..., h:], dy)
    with pytest.raises(liec.LiecError, match="overlap"):
        backward(dy, x, mean, rstd, w, dweight=grads[:, 1:h + 1], dbias=grads[:, :h])
    with pytest.raises(liec.LiecError, match="overlap"):
        forward(both[..., :h], w, b, y=both[..., h - 1:2 * h - 1])


def check_shared(x, dy, w, b, dtype, **given):
    """Forward and backward with one weight for all workers, against the formulas over all rows."""
    N, rows, h = x.shape
    y, mean, rstd = forward(x, w, b)
    dx, dw, db = backward(dy, x, mean, rstd, w, **given)
    assert dx.shape == x.shape and dw.shape == (h,) and db.shape == (h,)
    flat = lambda t: t.reshape(1, N * rows, *t.shape[2:])
    check_backward(flat(dy), flat(x), flat(mean), flat(rstd), w[None], dtype, "f32", flat(dx), dw[None], db[None])
    again = backward(dy, x, mean, rstd, w, **{k: v.clone().fill_(float("nan")) for k, v in given.items()})
    for p, q in zip((dx, dw, db), again):
        assert torch.equal(p, q)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,rows,h", [(3, 10, 64), (2, 33, 255), (5, 12, 768), (300, 7, 768), (3, 300, 1001), (2, 40, 4096), (3, 8, 9000), (2, 3000, 48)])
def test_shared_weight_any_layout(N, rows, h, dtype):
    """One weight for all workers on what the forward pass takes: slices of the activations, workers inside, an incoming
    gradient that is broadcast.  (Its sums over rows add at most 1024 in binary32 and the rest in binary64.)"""
    x, dy, w, b = draw(N, rows, h, dtype, seed=12)
    w, b = w[0].contiguous(), b[0].contiguous()
    inside = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    check_shared(x, dy, w, b, dtype)
    check_shared(x[:, -1:], dy[:, -1:], w, b, dtype)
    check_shared(x[:, :4], dy[:, :4], w, b, dtype)
    check_shared(x[:, ::3], dy[:, ::3].contiguous(), w, b, dtype)
    check_shared(inside(x), dy, w, b, dtype)
    check_shared(x, dy[:, :1].expand(N, rows, h), w, b, dtype)
    check_shared(x, dy[:1].expand(N, rows, h), w, b, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("h", [48, 768, 4096, 9000])
def test_shared_weight_where_shares_meet_groups(h, dtype):
    """Rows dealt so that workers and shares end together in some places and not in others, in a workspace that
    holds NaN: every place of it that is joined was written."""
    for N, rows in ((4, 1184), (8, 296), (37, 64), (296, 8), (3, 1024), (5, 333)):
        x, dy, w, b = draw(N, rows, h if N * rows < 3000 or h < 1000 else 4096, dtype, seed=N)
        check_shared(x, dy[:, :1].expand(x.shape), w[0].contiguous(), b[0].contiguous(), dtype,
                     workspace=torch.full((1 << 24,), float("nan"), device="cuda"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_shared_weight_without_rows_and_in_bfloat16_gradients(dtype):
    x, w = torch.empty(3, 0, 64, dtype=DT[dtype], device="cuda"), torch.ones(64, device="cuda")
    _, mean, rstd = forward(x, w, w)
    dx, dw, db = backward(x, x, mean, rstd, w)
    assert dx.shape == x.shape and (dw == 0).all() and (db == 0).all() and dw.shape == (64,)
    x, dy, w, b = draw(3, 50, 100, dtype, seed=3)
    w = w[0].contiguous()
    _, mean, rstd = forward(x, w)
    grads = torch.full((2, 100), 7.0, dtype=torch.bfloat16, device="cuda")
    cut = slice(0, 30)
    want = backward(dy[:, cut].contiguous(), x[:, cut].contiguous(), mean[:, cut].contiguous(), rstd[:, cut].contiguous(), w)
    dx, dw, db = backward(dy[:, cut], x[:, cut], mean[:, cut].contiguous(), rstd[:, cut].contiguous(), w, dweight=grads[0], dbias=grads[1])
    assert torch.equal(dx, want[0])
    flat = lambda t: t.reshape(1, 90, *t.shape[2:])
    check_backward(flat(dy[:, cut]), flat(x[:, cut]), flat(mean[:, cut]), flat(rstd[:, cut]), w[None], dtype, "bf16", flat(dx), dw[None], db[None])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,rows,h", [(3, 50, 96), (2, 700, 48), (2, 500, 256), (4, 300, 512), (4, 600, 768), (2, 300, 1024), (2, 400, 2048),
                                      (2, 300, 4096), (1, 60, 8192), (1, 70, 16384), (2, 9, 768)])
def test_bits_do_not_depend_on_the_layout(N, rows, h, dtype):
    """The same values on 16 bytes and off them, as rows of a wider buffer and with the workers inside: equal bits of
    everything that the forward and the backward pass return."""
    x, dy, w, b = draw(N, rows, h, dtype, seed=h)

    def elsewhere(t, pad, at, inside):
        shape = (rows, N, h + pad) if inside else (N, rows, h + pad)
        wide = torch.full((shape[0] * shape[1] * shape[2] + at,), float("nan"), dtype=t.dtype, device="cuda")[at:].view(shape)
        cut = (wide.transpose(0, 1) if inside else wide)[..., :h]
        cut.copy_(t)
        return cut

    y, mean, rstd = forward(x, w, b)
    want = (y, mean, rstd) + backward(dy, x, mean, rstd, w)
    for pad, at, inside in ((1, 0, False), (8, 0, True), (5, 3, False), (0, 1, True)):
        xs, ds = elsewhere(x, pad, at, inside), elsewhere(dy, pad, at, inside)
        got = forward(xs, w, b) + backward(ds, xs, mean, rstd, w)
        for name, p, q in zip(("y", "mean", "rstd", "dx", "dweight", "dbias"), got, want):
            assert torch.equal(p, q), (name, pad, at, inside, float((p.float() - q.float()).abs().max()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,rows,h,shared", [(3, 5, 96, False), (2, 700, 768, False), (4, 1500, 1001, False), (700, 20, 48, False), (2, 300, 4096, False),
                                             (2, 40, 9000, False), (1, 9000, 16, False), (3, 5, 96, True), (37, 64, 768, True), (2, 40, 9000, True)])
def test_workspace_of_exactly_the_reported_size(N, rows, h, shared, dtype):
    """Nothing beyond liec_layer_norm_workspace_bytes is written, and half of it is refused."""
    x, dy, w, b = draw(N, rows, h, dtype, seed=N + rows)
    vector = torch.empty(h if shared else N * h, device="cuda").view(*(() if shared else (N,)), h)
    if shared:
        w, b = w[0].contiguous(), b[0].contiguous()
        dy = dy[:, :1].expand(N, rows, h)      # (not foldable into one worker)
    _, mean, rstd = forward(x, w, b)
    layout = liec._layout
    d, _, need = liec._ln_desc(layout(x), layout(dy), layout(x), layout(w), None, layout(vector), layout(vector), 0.0)
    assert need == liec.liec_layer_norm_workspace_bytes(d) and bool(d.shared_grads) == shared
    memory = torch.full((need + (2 << 20),), 77, dtype=torch.uint8, device="cuda")
    inside = memory[1 << 20:][:need]
    dx, dw, db = backward(dy, x, mean, rstd, w, workspace=inside)
    assert (memory[:1 << 20] == 77).all() and (memory[(1 << 20) + need:] == 77).all()
    flat = (lambda t: t.reshape(1, N * rows, *t.shape[2:])) if shared else (lambda t: t)
    one = (lambda t: t[None]) if shared else (lambda t: t)
    check_backward(flat(dy), flat(x), flat(mean), flat(rstd), one(w), dtype, "f32", flat(dx), one(dw), one(db))
    with pytest.raises(liec.LiecError) as err:
        backward(dy, x, mean, rstd, w, workspace=inside[:need // 2])
    assert err.value.status == 3


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("h", [5, 768, 4096, 9000])
def test_rows_whose_squares_leave_binary32(h, dtype):
    """Finite entries beyond 1e19: infinite variance, so r = 0 and y = b; the rows beside them are not touched by it."""
    x, dy, w, b = draw(1, 4, h, dtype, seed=17)
    x, want = x.clone(), forward(x, w, b)
    x[0, 2, h // 2] = -3.0e38      # as a mask value
    y, mean, rstd = forward(x, w, b)
    assert rstd[0, 2] == 0 and torch.isfinite(mean).all() and torch.equal(y[0, 2], b[0].to(DT[dtype]))
    for p, q in zip((y, mean, rstd), want):
        assert torch.equal(p[0, [0, 1, 3]], q[0, [0, 1, 3]])


def test_outputs_have_no_graph():
    x, dy, w, b = draw(2, 8, 64, "f32", seed=1)
    out = forward(x.clone().requires_grad_(), w.clone().requires_grad_(), b)
    assert not any(t.requires_grad for t in out)

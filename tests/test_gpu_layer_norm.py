"""Layer normalisation on the GPU, forward and backward, against the formulas in binary64.

Tolerances are error bounds of the binary32 evaluation, element by element.  u = 2^-24 is one rounding.
A sum over a row passes through at most 40 + h/256 additions on the way of any one term (32 terms per
thread, shuffles, a few joins; the widest rows take h/256 terms per thread), a sum over R rows through
at most 40 + R; one more rounding per product.  Outputs in bfloat16 add 2^-8 of their magnitude.
"""
import numpy as np
import pytest
import torch

from paper_2402_11857_b200 import liec

pytestmark = pytest.mark.gpu

U, U_BF = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(N, rows, h, dtype, seed, pad=0, at=0, loud=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    x = r(N, rows, h) + 0.5 * r(N, rows, 1) + (3.0 if loud else 0.0) * r(h)
    dy = r(N, rows, h) * 0.1
    wide = [torch.full((N, rows, h + pad), float("nan"), dtype=DT[dtype], device="cuda") for _ in range(2)]
    for w, t in zip(wide, (x, dy)):
        w[..., :h] = t.to(DT[dtype])
    params = 1.0 + 0.3 * r(N, at + 2 * h + 3)
    return wide[0][..., :h], wide[1][..., :h], params[:, at:at + h], params[:, at + h:at + 2 * h]


def forward64(x, w, b, eps):
    x = x.double()
    m = x.mean(-1, keepdim=True)
    c = x - m
    v = c.square().mean(-1, keepdim=True)
    r = 1.0 / torch.sqrt(v + eps)
    return c * r * w.double().unsqueeze(-2) + b.double().unsqueeze(-2), m, r, v


def backward64(dy, x, m, r, w):
    dy, m, r = dy.double(), m.double()[..., None], r.double()[..., None]
    xh, t = (x.double() - m) * r, dy * w.double().unsqueeze(-2)
    along, level = (t * xh).mean(-1, keepdim=True), t.mean(-1, keepdim=True)
    return r * (t - level - xh * along), (dy * xh).sum(-2), dy.sum(-2), (xh, t, along, level, r)


def out_bound(t, dtype):
    return (U_BF if dtype == "bf16" else U) * t.abs() + 1e-37


def check(got, want, bound, what):
    got, bad = got.double(), None
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {float(((got - want).abs() / bound).max()):.2f} of the bound"


def check_forward(x, w, b, eps, dtype, y, mean, rstd):
    h = x.shape[-1]
    want, m, r, v = forward64(x, w, b, eps)
    k = 40 + h / 256
    dm = (k + 1) * U * x.double().abs().mean(-1, keepdim=True)
    rel = ((k + 3) * U + dm.square() / (v + eps)) / 2 + 3 * U
    check(mean, m[..., 0], dm[..., 0] + U * m[..., 0].abs(), "mean")
    check(rstd, r[..., 0], (rel * r)[..., 0], "rstd")
    xhw = (x.double() - m).abs() * r * w.double().abs().unsqueeze(-2)
    bound = r * w.double().abs().unsqueeze(-2) * dm * (1 + rel) + xhw * (rel + 4 * U) + 2 * U * (xhw + b.double().abs().unsqueeze(-2))
    check(y, want, bound + out_bound(want, dtype), "y")


def check_backward(dy, x, mean, rstd, w, dtype, gdtype, dx, dw, db, eps=None):
    h, rows = x.shape[-1], x.shape[-2]
    want, ww, wb, (xh, t, along, level, r) = backward64(dy, x, mean, rstd, w)
    k, kr = 40 + h / 256, 40 + rows
    da = (k + 5) * U * (t * xh).abs().mean(-1, keepdim=True)
    dl = (k + 3) * U * t.abs().mean(-1, keepdim=True)
    bound = r * (6 * U * (t.abs() + level.abs() + (xh * along).abs()) + dl + xh.abs() * da)
    check(dx, want, bound + out_bound(want, dtype), "dx")
    check(dw, ww, (kr + 4) * U * (dy.double() * xh).abs().sum(-2) + out_bound(ww, gdtype), "dweight")
    check(db, wb, (kr + 1) * U * dy.double().abs().sum(-2) + out_bound(wb, gdtype), "dbias")


SHAPES = [(1, 1, 1), (3, 4, 2), (2, 5, 7), (1, 1, 32), (4, 33, 31), (2, 9, 64), (3, 17, 255), (2, 40, 256), (5, 6, 257),
          (1, 300, 384), (3, 70, 512), (32, 20, 768), (1, 2500, 768), (2, 31, 1000), (2, 31, 1001), (3, 50, 1024), (2, 7, 1333),
          (1, 40, 1536), (2, 30, 2048), (1, 9, 2049), (1, 20, 3000), (2, 25, 4096), (1, 10, 4099), (1, 17, 5120), (1, 12, 8192),
          (1, 5, 8193), (1, 4, 12288), (2, 3, 16384), (1, 3, 20001), (1, 2, 32768), (1, 2, 65536), (400, 3, 48), (1, 9000, 16)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,rows,h", SHAPES)
def test_forward_and_backward(N, rows, h, dtype):
    x, dy, w, b = draw(N, rows, h, dtype, seed=h + rows)
    y, mean, rstd = liec.liec_layer_norm_forward(x, w, b, 1e-5)
    check_forward(x, w, b, 1e-5, dtype, y, mean, rstd)
    gdtype = "bf16" if (h + rows) % 2 else "f32"
    grads = torch.full((N, 2 * h + 5), 7.0, dtype=DT[gdtype], device="cuda")
    dx, dw, db = liec.liec_layer_norm_backward(dy, x, mean, rstd, w, dweight=grads[:, 2:2 + h], dbias=grads[:, 3 + h:3 + 2 * h])
    check_backward(dy, x, mean, rstd, w, dtype, gdtype, dx, dw, db)
    # what lies beside the two column ranges is left alone
    assert (grads[:, :2] == 7).all() and (grads[:, 2 + h:3 + h] == 7).all() and (grads[:, 3 + 2 * h:] == 7).all()
    # equal calls, equal bits
    again = liec.liec_layer_norm_backward(dy, x, mean, rstd, w)
    if gdtype == "f32":
        assert torch.equal(again[1], dw) and torch.equal(again[2], db)
    assert torch.equal(again[0], dx)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,rows,h,pad,at", [(3, 11, 96, 8, 0), (2, 13, 100, 3, 5), (2, 21, 768, 1, 3), (4, 10, 1024, 16, 8),
                                             (1, 15, 2048, 5, 1), (2, 6, 9000, 4, 2)])
def test_strided_rows_and_odd_places(N, rows, h, pad, at, dtype):
    """Rows that are slices of wider buffers, parameters at any place, workers as the inner axis."""
    x, dy, w, b = draw(N, rows, h, dtype, seed=5, pad=pad, at=at)
    wide = torch.full((N, rows, h + pad), 5.0, dtype=DT[dtype], device="cuda")
    y, mean, rstd = liec.liec_layer_norm_forward(x, w, b, 1e-3, y=wide[..., :h])
    check_forward(x, w, b, 1e-3, dtype, y, mean, rstd)
    assert (wide[..., h:] == 5).all()
    dxw = torch.full((rows, N, h + pad), 5.0, dtype=DT[dtype], device="cuda")
    xt = x.transpose(0, 1).contiguous().transpose(0, 1)          # [N, rows, h] with the workers inside
    dx, dw, db = liec.liec_layer_norm_backward(dy, xt, mean, rstd, w, dx=dxw.transpose(0, 1)[..., :h])
    check_backward(dy, x, mean, rstd, w, dtype, "f32", dx, dw, db)
    assert (dxw[..., h:] == 5).all()
    y2, _, _ = liec.liec_layer_norm_forward(xt, w, b, 1e-3)
    assert torch.equal(y2, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("h", [40, 768, 1001, 4096, 16384])
def test_two_axes_shared_and_missing_parameters(h, dtype):
    x, dy, w, b = draw(3, 10, h, dtype, seed=9)
    ones, zeros = torch.ones(3, h, device="cuda"), torch.zeros(3, h, device="cuda")
    y, mean, rstd = liec.liec_layer_norm_forward(x)
    check_forward(x, ones, zeros, 1e-5, dtype, y, mean, rstd)
    # one vector for all workers; its gradient sums over the workers as well
    y, mean, rstd = liec.liec_layer_norm_forward(x, w[0].contiguous(), b[0].contiguous())
    check_forward(x, w[:1].expand(3, h), b[:1].expand(3, h), 1e-5, dtype, y, mean, rstd)
    dx, dw, db = liec.liec_layer_norm_backward(dy, x, mean, rstd, w[0].contiguous())
    assert dw.shape == (h,) and db.shape == (h,)
    flat = lambda t: t.reshape(1, 30, *t.shape[2:])
    check_backward(flat(dy), flat(x), flat(mean), flat(rstd), w[:1], dtype, "f32", flat(dx), dw[None], db[None])
    # one weight for all workers, a gradient row for each
    rows = torch.zeros(3, h, device="cuda")
    dx2, dw2, db2 = liec.liec_layer_norm_backward(dy, x, mean, rstd, w[0].contiguous(), dweight=rows, dbias=torch.zeros(3, h, device="cuda"))
    check_backward(dy, x, mean, rstd, w[:1].expand(3, h), dtype, "f32", dx2, dw2, db2)
    # [rows, h]: one worker
    y1, m1, r1 = liec.liec_layer_norm_forward(x[1], w[1], b[1])
    check_forward(x[1:2], w[1:2], b[1:2], 1e-5, dtype, y1[None], m1[None], r1[None])
    dx1, dw1, db1 = liec.liec_layer_norm_backward(dy[1], x[1], m1, r1, w[1])
    check_backward(dy[1:2], x[1:2], m1[None], r1[None], w[1:2], dtype, "f32", dx1[None], dw1[None], db1[None])
    # no affine part at all
    dx3, dw3, _ = liec.liec_layer_norm_backward(dy[1], x[1], m1, r1)
    check_backward(dy[1:2], x[1:2], m1[None], r1[None], ones[:1], dtype, "f32", dx3[None], dw3[None], db1[None])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,rows,h", [(2000, 400, 1), (2000, 400, 3), (2000, 400, 5), (2000, 400, 7), (1500, 250, 13), (600, 200, 129),
                                      (4, 9000, 255), (1, 20000, 511), (3, 5000, 767), (2, 6000, 1019), (1, 4000, 2047), (1, 2500, 4095)])
def test_odd_rows_through_every_place_of_the_ring(N, rows, h, dtype):
    """Widths that start each row at another byte of a 16-byte granule (and rows that end in the granule in which
    they start), with so many rows that every place in shared memory holds many of them one after another."""
    x, dy, w, b = draw(N, rows, h, dtype, seed=h)
    y, mean, rstd = liec.liec_layer_norm_forward(x, w, b, 1e-4)
    check_forward(x, w, b, 1e-4, dtype, y, mean, rstd)
    dx, dw, db = liec.liec_layer_norm_backward(dy, x, mean, rstd, w)
    check_backward(dy, x, mean, rstd, w, dtype, "f32", dx, dw, db)


@pytest.mark.parametrize("h", [5, 768, 1001, 2048, 10000])
def test_broadcast_incoming_gradient(h):
    """dy as the gradient of a sum: one value expanded over rows and workers (strides 0)."""
    x, _, w, b = draw(2, 12, h, "f32", seed=4)
    _, mean, rstd = liec.liec_layer_norm_forward(x, w, b)
    dy = torch.randn(1, 1, h, device="cuda").expand(2, 12, h)
    dx, dw, db = liec.liec_layer_norm_backward(dy, x, mean, rstd, w)
    check_backward(dy, x, mean, rstd, w, "f32", "f32", dx, dw, db)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("h", [3, 768, 1001, 4096, 12288])
def test_no_rows(h, dtype):
    x = torch.empty(3, 0, h, dtype=DT[dtype], device="cuda")
    w = torch.ones(3, h, device="cuda")
    y, mean, rstd = liec.liec_layer_norm_forward(x, w, w)
    assert y.shape == x.shape and mean.shape == (3, 0)
    grads = torch.full((3, 2 * h), 7.0, device="cuda")
    dx, dw, db = liec.liec_layer_norm_backward(x, x, mean, rstd, w, dweight=grads[:, :h], dbias=grads[:, h:])
    assert dx.shape == x.shape and (grads == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("h", [1, 8, 768, 1001, 4096, 9000])
def test_constant_far_and_infinite_rows(h, dtype):
    """A constant row gives the bias; a row far from zero keeps its digits (the variance is taken around the
    mean); infinities and NaN stay in their row."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn(1, 6, h, generator=gen, device="cuda")
    x[0, 1] = 1024.0
    x[0, 2] += 4096.0
    x[0, 3, h // 2] = float("inf")
    x[0, 4, h - 1] = float("nan")
    x = x.to(DT[dtype])
    w, b = torch.full((1, h), 1.5, device="cuda"), torch.full((1, h), 0.25, device="cuda")
    y, mean, rstd = liec.liec_layer_norm_forward(x, w, b, 1e-5)
    assert torch.isnan(y[0, 3:5]).all() and torch.isnan(mean[0, 4]) and torch.isinf(mean[0, 3])
    fine = [0, 2, 5] + ([1] if h & (h - 1) == 0 else [])     # (the sum of a constant is exact for these h)
    check_forward(x[:, fine], w, b, 1e-5, dtype, y[:, fine], mean[:, fine], rstd[:, fine])
    if h & (h - 1) == 0:
        assert (y[0, 1].float() == 0.25).all()
    dy = torch.randn(1, 6, h, generator=gen, device="cuda").to(DT[dtype])
    dx, dw, db = liec.liec_layer_norm_backward(dy, x, mean, rstd, w)
    assert torch.isnan(dx[0, 3:5]).all() and torch.isfinite(dx[0, fine].float()).all()
    assert torch.isnan(dw).all() and torch.isfinite(db).all()
    if h == 1:
        assert (dx[0, fine] == 0).all()


@pytest.mark.parametrize("h", [6, 48, 770])
def test_gradient_against_differences(h):
    """L = sum c . LN(x): central differences of the binary64 forward formula along random directions.
    With step s the truncation error is s^2 times third derivatives; s = 1e-4 and unit-size data leave
    1e-6 of the derivative's scale, beside the binary32 bound of the gradient (1e-5 of that scale)."""
    x, _, w, b = draw(2, 4, h, "f32", seed=21, loud=False)
    gen = torch.Generator(device="cuda").manual_seed(3)
    c = torch.randn(2, 4, h, generator=gen, device="cuda")
    _, mean, rstd = liec.liec_layer_norm_forward(x, w, b, 1e-3)
    dx, dw, db = liec.liec_layer_norm_backward(c, x, mean, rstd, w)
    loss = lambda x_, w_, b_: float((c.double() * forward64(x_, w_, b_, 1e-3)[0]).sum())
    s = 1e-4
    x64, w64, b64 = x.double(), w.double(), b.double()
    for trial in range(4):
        vx, vw, vb = (torch.randn(t.shape, generator=gen, device="cuda", dtype=torch.float64) for t in (x, w, b))
        for v, g, plus, minus in ((vx, dx, (x64 + s * vx, w64, b64), (x64 - s * vx, w64, b64)),
                                  (vw, dw, (x64, w64 + s * vw, b64), (x64, w64 - s * vw, b64)),
                                  (vb, db, (x64, w64, b64 + s * vb), (x64, w64, b64 - s * vb))):
            numeric = (loss(*plus) - loss(*minus)) / (2 * s)
            terms = g.double() * v
            assert abs(float(terms.sum()) - numeric) <= 1e-5 * float(terms.abs().sum()) + 1e-6


def test_long_batches_and_far_offsets():
    """More than 2^32 elements: the last rows of the last worker against the formula."""
    free, _ = torch.cuda.mem_get_info()
    N, rows, h = 2, 2_200_000, 1024
    assert free > 30 << 30
    x = torch.empty(N, rows, h, dtype=torch.bfloat16, device="cuda").normal_()
    w, b = 1.0 + 0.1 * torch.randn(N, h, device="cuda"), torch.randn(N, h, device="cuda")
    y, mean, rstd = liec.liec_layer_norm_forward(x, w, b)
    tail = (slice(1, 2), slice(rows - 64, rows))
    check_forward(x[tail], w[1:], b[1:], 1e-5, "bf16", y[tail], mean[tail], rstd[tail])
    dx, dw, db = liec.liec_layer_norm_backward(y, x, mean, rstd, w)
    d64 = backward64(y[tail], x[tail], mean[tail], rstd[tail], w[1:])[0]
    check(dx[tail], d64, out_bound(d64, "bf16") + 1e-4, "dx")
    # sums over 2.2 million rows: piecewise in binary64; every accumulator takes at most a few thousand rows
    for i in range(N):
        sw, sb, aw, ab = (torch.zeros(h, dtype=torch.float64, device="cuda") for _ in range(4))
        for at in range(0, rows, 100_000):
            cut = (slice(i, i + 1), slice(at, at + 100_000))
            g, xh = y[cut].double(), (x[cut].double() - mean[cut].double()[..., None]) * rstd[cut].double()[..., None]
            sw += (g * xh).sum((0, 1)); sb += g.sum((0, 1)); aw += (g * xh).abs().sum((0, 1)); ab += g.abs().sum((0, 1))
        check(dw[i], sw, 3000 * U * aw, "dweight")
        check(db[i], sb, 3000 * U * ab, "dbias")


def test_on_a_side_stream_and_captured():
    x, dy, w, b = draw(2, 64, 768, "bf16", seed=31)
    y0, m0, r0 = liec.liec_layer_norm_forward(x, w, b)
    g0 = liec.liec_layer_norm_backward(dy, x, m0, r0, w)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    y1, m1, r1 = liec.liec_layer_norm_forward(x, w, b, stream=s)
    g1 = liec.liec_layer_norm_backward(dy, x, m1, r1, w, stream=s)
    s.synchronize()
    for p, q in zip((y0, m0, r0) + g0, (y1, m1, r1) + g1):
        assert torch.equal(p, q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y2, m2, r2 = liec.liec_layer_norm_forward(x, w, b)
        g2 = liec.liec_layer_norm_backward(dy, x, m2, r2, w)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for p, q in zip((y0, m0, r0) + g0, (y2, m2, r2) + g2):
        assert torch.equal(p, q)


def test_binding_refusals():
    x, dy, w, b = draw(2, 8, 64, "f32", seed=1)
    y, m, r = liec.liec_layer_norm_forward(x, w, b)
    fwd, bwd = liec.liec_layer_norm_forward, liec.liec_layer_norm_backward
    for call in (lambda: fwd(x.cpu()), lambda: fwd(x.half()), lambda: fwd(x[0, 0]), lambda: fwd(x.transpose(1, 2)),
                 lambda: fwd(x, w[:, :32]), lambda: fwd(x, w.bfloat16()), lambda: fwd(x, w.cpu()), lambda: fwd(x, w[:1]),
                 lambda: fwd(x, y=torch.empty(2, 8, 32, device="cuda")), lambda: fwd(x, y=torch.empty_like(x, dtype=torch.bfloat16)),
                 lambda: bwd(dy.bfloat16(), x, m, r, w), lambda: bwd(dy[:, :4], x, m, r, w), lambda: bwd(dy, x, m[:1], r, w),
                 lambda: bwd(dy, x, m.double(), r, w), lambda: bwd(dy, x, m, r, w, dweight=torch.zeros(64, device="cuda")),
                 lambda: bwd(dy, x, m, r, w, dweight=torch.zeros(2, 64, device="cuda"), dbias=torch.zeros(2, 64, device="cuda").bfloat16()),
                 lambda: bwd(dy, x, m, r, w, dweight=torch.zeros(2, 64, device="cuda").double())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: fwd(x, y=x), lambda: fwd(x, eps=-1.0), lambda: fwd(x, eps=float("nan")),
                 lambda: fwd(x, y=torch.empty(1, 8, 64, device="cuda").expand(2, 8, 64)), lambda: bwd(dy, x, m, r, w, dx=x),
                 lambda: bwd(dy, x, m, r, w, dx=dy), lambda: bwd(dy, x, m, r, w, workspace=torch.empty(0, device="cuda")),
                 lambda: fwd(torch.zeros(1, 65537, device="cuda"))):
        with pytest.raises(liec.LiecError) as err:
            call()
        assert err.value.status in (1, 2, 3)

"""Group normalisation with an activation on the GPU, forward and backward, against the formulas in binary64."""
import pytest
import torch

from activation_helpers import DT, check_group_norm_backward, check_group_norm_forward, restored64
from paper_2402_11857_b200 import liec

pytestmark = pytest.mark.gpu
forward, backward = liec.liec_group_norm_forward, liec.liec_group_norm_backward


def draw(shape, dtype, seed, pad=0, at=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    N, C = shape[0], shape[-1]
    x, dy = r(*shape) + 2.0 * r(C), 0.1 * r(*shape)
    wide = [torch.full(shape[:-1] + (C + pad,), float("nan"), dtype=DT[dtype], device="cuda") for _ in range(2)]
    for w, t in zip(wide, (x, dy)):
        w[..., :C] = t.to(DT[dtype])
    params = 0.3 * r(N, at + 2 * C + 3)
    params[:, at:at + C] += 1.0
    return wide[0][..., :C], wide[1][..., :C], params[:, at:at + C], params[:, at + C:at + 2 * C]


# N, samples, pixels, channels, groups: one of everything, groups of one channel, one group, widths off every grid, wide
# groups, images that one block, a cluster of blocks or only the whole GPU holds
SHAPES = [(1, 1, 1, 1, 1), (1, 2, 1, 8, 2), (2, 3, 5, 6, 3), (2, 1, 49, 32, 32), (1, 3, 64, 64, 8), (3, 2, 77, 36, 9), (2, 2, 100, 90, 5), (1, 2, 196, 150, 1),
          (2, 1, 361, 128, 32), (1, 1, 400, 320, 32), (5, 1, 9, 2048, 32), (1, 1, 30, 4100, 4), (1, 1, 7, 9000, 1), (2, 2, 1024, 48, 6), (1, 1, 3136, 64, 32),
          (1, 1, 9001, 40, 8), (1, 2, 12544, 64, 16), (1, 1, 65536, 32, 4), (300, 2, 4, 16, 4), (2, 40, 16, 512, 32)]
ACTS = ["none", "relu", "silu"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_backward(shape, dtype):
    *shape, groups = shape
    shape, N, C = tuple(shape), shape[0], shape[-1]
    for act in ACTS if shape[2] <= 400 else ACTS[shape[2] % 3:][:1]:
        x, dy, w, b = draw(shape, dtype, seed=C + shape[2])
        y, mean, rstd, q, scales = forward(x, groups, w, b, 1e-5, activation=act, compress=True)
        check_group_norm_forward(x, w, b, groups, 1e-5, act, dtype, y, mean, rstd)
        want = liec.liec_activation_compress(x)
        assert torch.equal(q, want[0]) and torch.equal(scales, want[1])
        plain = forward(x, groups, w, b, 1e-5, activation=act)
        assert all(torch.equal(s, t) for s, t in zip(plain, (y, mean, rstd)))
        gdtype = "bf16" if (C + shape[2]) % 2 else "f32"
        for source, given in ((x, x), ((q, scales), restored64(q, scales, C))):
            grads = torch.full((N, 2 * C + 5), 7.0, dtype=DT[gdtype], device="cuda")
            dx, dw, db = backward(dy, source, mean, rstd, w, b, activation=act, dweight=grads[:, 2:2 + C], dbias=grads[:, 3 + C:3 + 2 * C])
            check_group_norm_backward(dy, given, mean, rstd, w, b, act, dtype, gdtype, dx, dw, db)
            # what lies beside the two column ranges is left alone
            assert (grads[:, :2] == 7).all() and (grads[:, 2 + C:3 + C] == 7).all() and (grads[:, 3 + 2 * C:] == 7).all()
            again = backward(dy, source, mean, rstd, w, b, activation=act)   # equal calls, equal bits
            assert torch.equal(again[0], dx) and (gdtype == "bf16" or (torch.equal(again[1], dw) and torch.equal(again[2], db)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pixels,C,groups,pad,at", [(30, 64, 8, 8, 0), (50, 60, 5, 3, 5), (900, 96, 6, 1, 3), (4000, 40, 4, 5, 1)])
def test_strided_images_and_odd_places(pixels, C, groups, pad, at, dtype):
    """Slices of wider buffers, parameters at any place, samples and workers as inner axes."""
    N, S = 2, 3
    x, dy, w, b = draw((N, S, pixels, C), dtype, seed=5, pad=pad, at=at)
    wide = torch.full((N, S, pixels, C + pad), 5.0, dtype=DT[dtype], device="cuda")
    y, mean, rstd = forward(x, groups, w, b, 1e-3, activation="silu", y=wide[..., :C])
    check_group_norm_forward(x, w, b, groups, 1e-3, "silu", dtype, y, mean, rstd)
    assert (wide[..., C:] == 5).all()
    xt = x.permute(2, 1, 0, 3).contiguous().permute(2, 1, 0, 3)
    dyt = dy.permute(1, 2, 0, 3).contiguous().permute(2, 0, 1, 3)
    dxw = torch.full((S, pixels, N, C + pad), 5.0, dtype=DT[dtype], device="cuda")
    dx, dw, db = backward(dyt, xt, mean, rstd, w, b, activation="silu", dx=dxw.permute(2, 0, 1, 3)[..., :C])
    check_group_norm_backward(dy, x, mean, rstd, w, b, "silu", dtype, "f32", dx, dw, db)
    assert (dxw[..., C:] == 5).all()
    assert torch.equal(forward(xt, groups, w, b, 1e-3, activation="silu")[0], y)
    # repeated rows and images
    flat = x[:, :, :1].expand(N, S, pixels, C)
    check_group_norm_forward(flat, w, b, groups, 1e-3, "relu", dtype, *forward(flat, groups, w, b, 1e-3, activation="relu"))
    check_group_norm_backward(dy[:, :1].expand_as(dy), x, mean, rstd, w, b, "relu", dtype, "f32", *backward(dy[:, :1].expand_as(dy), x, mean, rstd, w, b, "relu"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pixels", [20, 5000])
def test_three_axes_shared_and_missing_parameters(pixels, dtype):
    x, dy, w, b = draw((3, 2, pixels, 48), dtype, seed=9)
    ones, zeros = torch.ones(3, 48, device="cuda"), torch.zeros(3, 48, device="cuda")
    y, mean, rstd = forward(x, 6, activation="silu")
    check_group_norm_forward(x, ones, zeros, 6, 1e-5, "silu", dtype, y, mean, rstd)
    check_group_norm_backward(dy, x, mean, rstd, ones, zeros, "silu", dtype, "f32", *backward(dy, x, mean, rstd, activation="silu"))
    # one vector for all workers: its gradient sums over them
    w1, b1 = w[0].contiguous(), b[0].contiguous()
    check_group_norm_forward(x, w[:1].expand(3, 48), b[:1].expand(3, 48), 6, 1e-5, "relu", dtype, *forward(x, 6, w1, b1, activation="relu"))
    dx, dw, db = backward(dy, x, mean, rstd, w1, b1, activation="relu")
    assert dw.shape == (48,)
    check_group_norm_backward(dy, x, mean, rstd, w[:1].expand(3, 48), b[:1].expand(3, 48), "relu", dtype, "f32", dx, dw, db, shared=True)
    # one worker without the axis (how an image is cut depends on how many there are: the last bits may differ)
    y1, mean1, rstd1 = forward(x[1], 6, w1, b1, activation="relu")
    assert y1.shape == x[1].shape and mean1.shape == (2, 6)
    check_group_norm_forward(x[1:2], w1[None], b1[None], 6, 1e-5, "relu", dtype, y1[None], mean1[None], rstd1[None])
    dx1, dw1, db1 = backward(dy[1], x[1], mean[1].contiguous(), rstd[1].contiguous(), w1, b1, activation="relu")
    assert dx1.shape == x[1].shape and dw1.shape == (48,)
    check_group_norm_backward(dy[1:2], x[1:2], mean[1:2], rstd[1:2], w1[None], b1[None], "relu", dtype, "f32", dx1[None], dw1[None], db1[None])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pixels", [40, 6000])
def test_far_means_constant_images_and_eps(pixels, dtype):
    x, dy, w, b = draw((2, 2, pixels, 32), dtype, seed=11)
    far = (x.float() + 300.0).to(x.dtype)
    check_group_norm_forward(far, w, b, 4, 1e-5, "none", dtype, *forward(far, 4, w, b))
    same = torch.full_like(x, 0.7)
    y, mean, rstd = forward(same, 4, w, b, 1e-4)
    check_group_norm_forward(same, w, b, 4, 1e-4, "none", dtype, y, mean, rstd)
    # every z of a ReLU on the border (d = 0 and b = 0): slope 0
    zero = torch.zeros_like(b)
    dx, dw, db = backward(dy, torch.zeros_like(x), torch.zeros_like(mean), rstd, w, zero, activation="relu")
    assert (dx == 0).all() and (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_relu_decides_as_in_binary64(dtype):
    """x at and next to the root of z: what binary32 rounds away decides."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    C, P = 32, 500
    mean, rstd = torch.randn(1, 1, 4, generator=gen, device="cuda"), torch.rand(1, 1, 4, generator=gen, device="cuda") + 0.5
    w, b = torch.randn(1, C, generator=gen, device="cuda"), torch.randn(1, C, generator=gen, device="cuda")
    root = mean.repeat_interleave(8, -1)[0, 0] - b[0] / (w[0] * rstd.repeat_interleave(8, -1)[0, 0])
    x = root[None, None, None].repeat(1, 1, P, 1).to(DT[dtype])
    bits = x.view(torch.int32 if dtype == "f32" else torch.int16)
    bits += torch.randint(-3, 4, bits.shape, generator=gen, device="cuda").to(bits.dtype)
    dy = torch.rand(1, 1, P, C, generator=gen, device="cuda").to(DT[dtype])
    check_group_norm_backward(dy, x, mean, rstd, w, b, "relu", dtype, "f32", *backward(dy, x, mean, rstd, w, b, activation="relu"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pixels", [30, 7000])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_not_finite_stays_in_its_group(value, pixels, dtype):
    x, dy, w, b = draw((2, 3, pixels, 48), dtype, seed=13)
    clean = forward(x, 6, w, b, activation="silu", compress=True)
    cdx, cdw, cdb = backward(dy, x, clean[1], clean[2], w, b, activation="silu")
    x = x.clone()
    x[1, 2, pixels // 2, 17] = value                                # group 2 of 6, channels 16 to 23
    y, mean, rstd, q, scales = forward(x, 6, w, b, activation="silu", compress=True)
    hit = torch.zeros(2, 3, 1, 48, dtype=torch.bool, device="cuda")
    hit[1, 2, 0, 16:24] = True
    assert y[hit.expand_as(y)].isnan().all() and torch.equal(y[~hit.expand_as(y)], clean[0][~hit.expand_as(y)])
    assert int(mean.isfinite().logical_not().sum()) == 1
    dx, dw, db = backward(dy, x, mean, rstd, w, b, activation="silu")
    assert dx[hit.expand_as(dx)].isnan().all() and torch.equal(dx[~hit.expand_as(dx)], cdx[~hit.expand_as(dx)])
    assert dw[1, 16:24].isnan().all() and torch.equal(dw[0], cdw[0]) and torch.equal(dw[1, :16], cdw[1, :16]) and torch.equal(db[1, 24:], cdb[1, 24:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,S,P", [(2, 0, 5), (2, 3, 0), (1, 0, 0)])
def test_no_images_and_no_pixels(N, S, P, dtype):
    x = torch.empty(N, S, P, 24, dtype=DT[dtype], device="cuda")
    y, mean, rstd, q, scales = forward(x, 3, activation="relu", compress=True)
    assert y.shape == x.shape and mean.shape == (N, S, 3) and q.shape == (N, S, P, 32)
    dx, dw, db = backward(x, x, mean, rstd, dweight=torch.ones(N, 24, device="cuda"), dbias=torch.ones(N, 24, device="cuda"))
    assert dx.shape == x.shape and (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("pixels", [64, 20000])
def test_streams_and_graphs(pixels):
    x, dy, w, b = draw((2, 2, pixels, 64), "bf16", seed=15)
    want = forward(x, 8, w, b, activation="silu", compress=True)
    grads = backward(dy, want[3:], *want[1:3], w, b, activation="silu")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = forward(x, 8, w, b, activation="silu", compress=True, stream=s)
    got_grads = backward(dy, got[3:], *got[1:3], w, b, activation="silu", stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(p, t) for p, t in zip(got + got_grads, want + grads))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = forward(x, 8, w, b, activation="silu", compress=True)
        got_grads = backward(dy, got[3:], *got[1:3], w, b, activation="silu")
    x.copy_(x.flip(2))
    dy.copy_(dy.flip(2))
    graph.replay()
    want = forward(x, 8, w, b, activation="silu", compress=True)
    grads = backward(dy, want[3:], *want[1:3], w, b, activation="silu")
    assert all(torch.equal(p, t) for p, t in zip(got + got_grads, want + grads))


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(act):
    """Central differences of sum(c y) in binary64 around a small case: 2e-5 of step, error 1e-9 and the call's own 2e-6."""
    x, c, w, b = draw((1, 2, 6, 8), "f32", seed=17)

    def loss(x, w, b):
        g = x.unflatten(-1, (2, 4))
        m = g.mean((2, 4), keepdim=True)
        r = 1 / torch.sqrt((g - m).square().mean((2, 4), keepdim=True) + 1e-3)
        z = ((g - m) * r).flatten(-2) * w[:, None, None] + b[:, None, None]
        y = z.clamp(min=0) if act == "relu" else z * torch.sigmoid(z) if act == "silu" else z
        return (y * c.double()).sum()

    _, mean, rstd = forward(x, 2, w, b, 1e-3, activation=act)
    got = backward(c, x, mean, rstd, w, b, activation=act)
    args = [t.double() for t in (x, w, b)]
    for k, grad in enumerate(got):
        for i in range(0, args[k].numel(), 5):
            step = torch.zeros_like(args[k]).flatten()
            step[i] = 1e-5
            step = step.view_as(args[k])
            up, down = list(args), list(args)
            up[k], down[k] = args[k] + step, args[k] - step
            want = (loss(*up) - loss(*down)) / 2e-5
            assert abs(float(grad.flatten()[i]) - float(want)) <= 2e-6


def test_refusals():
    x, dy, w, b = draw((2, 2, 10, 24), "f32", seed=19)
    y, mean, rstd = forward(x, 4, w, b)
    q, scales = liec.liec_activation_compress(x)
    for bad, words in ((lambda: forward(x, 5), "groups must divide"), (lambda: forward(x, 4, activation="gelu"), "activation must be"),
                       (lambda: forward(x.half(), 4), "float32 or bfloat16"), (lambda: forward(x[0, 0], 4), "samples"), (lambda: forward(x.cpu(), 4), "CUDA"),
                       (lambda: forward(x, 4, w.double()), "weight must be"), (lambda: forward(x, 4, w[:, :12]), "weight must be"),
                       (lambda: forward(x, 4, y=torch.empty(2, 2, 10, 25, device="cuda")), "shape and type"),
                       (lambda: forward(x, 4, q=q[:1]), "q must be"), (lambda: backward(dy, x, mean[:1], rstd, w), "mean must be"),
                       (lambda: backward(dy, (q, scales[..., :0]), mean, rstd, w), "scales must be"),
                       (lambda: backward(dy, x[:, :, :5], mean, rstd, w), "shape and type"),
                       (lambda: backward(dy, x, mean, rstd, w, dweight=torch.empty(24, device="cuda")), "number of axes|of their own"),
                       (lambda: backward(dy, x, mean, rstd, w, dweight=torch.empty(24, device="cuda"), dbias=torch.empty(24, device="cuda")), "of their own"),
                       (lambda: forward(x, 4, w, workspace=torch.empty(10000, 2, dtype=torch.uint8, device="cuda")[:, 0]), "workspace must be contiguous")):
        with pytest.raises(ValueError, match=words):
            bad()
    for bad, words in ((lambda: forward(x, 4, y=x), "overlaps an input"), (lambda: forward(x, 4, y=y[:, :1].expand_as(y)), "rows of y overlap"),
                       (lambda: backward(dy, x, mean, rstd, w, dx=dy), "overlaps an input"), (lambda: backward(dy, x, mean, rstd, w, dx=x), "overlaps an input"),
                       (lambda: backward(dy, x, mean, rstd, w, dweight=w, dbias=b), "overlaps an input"),
                       (lambda: forward(x, 4, eps=-1.0), "eps")):
        with pytest.raises(liec.LiecError, match=words):
            bad()

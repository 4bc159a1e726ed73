"""The operators on activations as they are used: one after another, side by side, replayed, and in tensors whose offsets
pass 32 bits."""
import pytest
import torch

from activation_helpers import DT, check_group_norm_backward, check_group_norm_forward, check_weight_grad, restored64
from paper_2402_11857_b200 import liec

pytestmark = pytest.mark.gpu
N, S, OUT = 2, 3, 40


def inputs(pixels, C, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return (r(N, S, pixels, C) + r(C)).bfloat16(), (0.1 * r(N, S, pixels, C)).bfloat16(), 1 + 0.3 * r(N, C), 0.3 * r(N, C), (0.1 * r(N, S * pixels, OUT)).bfloat16()


def layer(x, dy, w, b, dz, space=(None, None, None), **kw):
    """A normalised layer whose input is kept in 8 bits, and the gradient of a linear layer on the same input."""
    C = x.shape[-1]
    y, mean, rstd, q, scales = liec.liec_group_norm_forward(x, 8, w, b, activation="silu", compress=True, workspace=space[0], **kw)
    grads = liec.liec_group_norm_backward(dy, (q, scales), mean, rstd, w, b, activation="silu", workspace=space[1], **kw)
    dweight = liec.liec_weight_grad(dz, q.view(N, -1, q.shape[-1]), scales.view(N, -1, scales.shape[-1]), C, workspace=space[2], **kw)
    return y, mean, rstd, q, scales, *grads, dweight


def equal(a, b):
    return all(torch.equal(s, t) for s, t in zip(a, b))


@pytest.mark.parametrize("pixels,C", [(49, 72), (3000, 64)])
def test_one_after_another(pixels, C):
    x, dy, w, b, dz = inputs(pixels, C, seed=1)
    y, mean, rstd, q, scales, dx, dw, db, dweight = layer(x, dy, w, b, dz)
    kept = restored64(q, scales, C)
    check_group_norm_forward(x, w, b, 8, 1e-5, "silu", "bf16", y, mean, rstd)
    check_group_norm_backward(dy, kept, mean, rstd, w, b, "silu", "bf16", "f32", dx, dw, db)
    check_weight_grad(dz, kept.flatten(1, 2), "f32", dweight)


@pytest.mark.parametrize("pixels,C", [(49, 72), (3000, 64)])
def test_side_by_side(pixels, C):
    """Two streams at once, many times: nothing is shared between calls."""
    sets = [inputs(pixels, C, seed) for seed in (2, 3)]
    want = [layer(*s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got = [layer(*given, stream=s) for given, s in zip(sets, streams)]
        torch.cuda.synchronize()
        assert equal(got[0], want[0]) and equal(got[1], want[1])


@pytest.mark.parametrize("pixels,C", [(49, 72), (3000, 64)])
def test_graphs_that_share_workspaces(pixels, C):
    sets = [inputs(pixels, C, seed) for seed in (4, 5)]
    want = [layer(*s) for s in sets]
    space = [torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
    graphs, got = [], []
    for given in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(layer(*given, space=space))
        graphs.append(g)
    for k in (0, 1, 1, 0, 1, 0):
        graphs[k].replay()
    assert equal(got[0], want[0]) and equal(got[1], want[1])


FAR = 2 ** 31 + 8


@pytest.mark.parametrize("pixels", [40, 5000])
def test_images_far_apart(pixels):
    """Workers 2^31 + 8 elements apart, in what is read and in what is written."""
    shape = (3, 1, pixels, 64)
    x, dy, y = (torch.zeros(2 * FAR + pixels * 64, dtype=torch.bfloat16, device="cuda").as_strided(shape, (FAR, pixels * 64, 64, 1)) for _ in range(3))
    gen = torch.Generator(device="cuda").manual_seed(6)
    x.copy_(torch.randn(shape, generator=gen, device="cuda"))
    dy.copy_(torch.randn(shape, generator=gen, device="cuda"))
    want = liec.liec_group_norm_forward(x.contiguous(), 8, activation="relu", compress=True)
    got = liec.liec_group_norm_forward(x, 8, activation="relu", compress=True, y=y)
    assert equal(got, want)
    want = liec.liec_group_norm_backward(dy.contiguous(), want[3:], *want[1:3], activation="relu")
    y.zero_()
    assert equal(liec.liec_group_norm_backward(dy, got[3:], *got[1:3], activation="relu", dx=y), want)


def test_checkpoint_of_more_than_32_bits():
    """More than 2^32 bytes of q: the last image, and the last rows of a sum over all."""
    samples, pixels, C = 66000, 64, 1024
    x = torch.empty(1, samples, pixels, C, dtype=torch.bfloat16, device="cuda").normal_()
    y, mean, rstd, q, scales = liec.liec_group_norm_forward(x, 8, compress=True)
    assert q.numel() > 2 ** 32
    last = slice(samples - 2, samples)
    one = torch.ones(1, C, device="cuda")
    check_group_norm_forward(x[:, last], one, 0 * one, 8, 1e-5, "none", "bf16", y[:, last], mean[:, last], rstd[:, last])
    del y
    dy = torch.zeros(1, samples, pixels, C, dtype=torch.bfloat16, device="cuda")
    dy[:, last] = x[:, :2]
    del x
    kept = restored64(q[:, last].contiguous(), scales[:, last].contiguous(), C)
    dx, dw, db = liec.liec_group_norm_backward(dy, (q, scales), mean, rstd)
    check_group_norm_backward(dy[:, last], kept, mean[:, last], rstd[:, last], one, 0 * one, "none", "bf16", "f32", dx[:, last], dw, db)   # (the other images give zeros)
    assert not dx[:, :-2].any()
    rows = dy[..., :24].flatten(1, 2)
    got = liec.liec_weight_grad(rows, q.flatten(1, 2), scales.flatten(1, 2), C)
    check_weight_grad(rows[:, -2 * pixels:], kept.flatten(1, 2), "f32", got)


def test_weight_gradients_far_apart():
    gen = torch.Generator(device="cuda").manual_seed(7)
    dy = torch.zeros(2 * FAR + 200 * 48, dtype=torch.bfloat16, device="cuda").as_strided((3, 200, 48), (FAR, 48, 1))
    dy.copy_(torch.randn(3, 200, 48, generator=gen, device="cuda"))
    q, scales = liec.liec_activation_compress(torch.randn(3, 200, 64, generator=gen, device="cuda"))
    want = liec.liec_weight_grad(dy.contiguous(), q, scales, 64)
    for dtype in DT.values():
        dweight = torch.zeros(2 * FAR + 48 * 64, dtype=dtype, device="cuda").as_strided((3, 48, 64), (FAR, 64, 1))
        liec.liec_weight_grad(dy, q, scales, 64, dweight=dweight)
        assert torch.equal(dweight, want.to(dtype))
        del dweight

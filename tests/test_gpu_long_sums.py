"""Sums keep their digits: where the first pixel of an image, or any other, is far from all others, where chains of
additions would be long, and where what the tensor cores cut would add up."""
import ctypes as C

import pytest
import torch

from activation_helpers import DT, U, U_BF, check_weight_grad, restored64
from paper_2402_11857_b200 import liec

pytestmark = pytest.mark.gpu
forward, backward = liec.liec_group_norm_forward, liec.liec_group_norm_backward


def statistics64(x, groups, eps):
    g = x.double().unflatten(-1, (groups, -1))
    m = g.mean((2, 4))
    v = (g - m[:, :, None, :, None]).square().mean((2, 4))
    return m, v, 1 / torch.sqrt(v + eps)


# Relative error of a variance.  A thread adds the squares of at most 64 entries about its first one, of those after the fourth about the
# mean of four, of those after the sixteenth about the mean of sixteen (held images: at most 56 entries, after the 14th and the 28th).
# n entries about the mean of the N before them: N (mean of the n - mean of the N)^2 n / (N + n) is among the squares of all about their
# common mean, so theirs come to at most n / N times those more: 3 times (held: 13 times at first, then once).  The roundings of
# the additions, 3 for an entry's square and 8 per move are so at most 4 (64 + 3 + 16) u = 332 u (held: 14 (14 + 11) + 2 (14 + 11) +
# 2 (28 + 11) = 478 u).  Up to 64 threads meet: 64 u more, and a held image's channels 40 u.  rstd has half of that, 291 u, and 4 u of its own.
RSTD = 295 * U


def check_statistics(x, groups, eps, mean, rstd):
    """The mean: each channel's is off by what 64 + 64 additions of values at most `far` from a thread's first entry lose, and one
    rounding of its own."""
    m, v, r = statistics64(x, groups, eps)
    worst = float(((rstd.double() - r).abs() / r).max())
    assert worst <= RSTD, f"rstd: {worst / U:.0f} u"
    g = x.double().unflatten(-1, (groups, -1))
    far = (g - m[:, :, None, :, None]).abs().amax((2, 4))
    assert ((mean.double() - m).abs() <= 2 * U * m.abs() + 128 * U * far).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mean", [0.0, 30.0, 300.0])
@pytest.mark.parametrize("border", [1, 57])
@pytest.mark.parametrize("N,S,pixels,ch,groups", [(2, 3, 49, 64, 8), (1, 2, 784, 64, 8), (2, 2, 1024, 48, 6), (2, 2, 1024, 45, 5), (1, 4, 4096, 32, 4), (1, 3, 12544, 40, 8),
                                                  (1, 2, 65536, 32, 4), (1, 2, 20001, 63, 9), (40, 16, 3136, 64, 32)])
def test_a_border_of_zeros_before_a_far_mean(N, S, pixels, ch, groups, border, mean, dtype):
    gen = torch.Generator(device="cuda").manual_seed(pixels + ch)
    x = (torch.randn(N, S, pixels, ch, generator=gen, device="cuda") + mean).to(DT[dtype])
    x[:, :, :min(border, pixels // 4)] = 0
    _, m, r = forward(x, groups)
    check_statistics(x, groups, 1e-5, m, r)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("where", [0, 1, 40, -1])
@pytest.mark.parametrize("pixels", [64, 3000, 30000])
def test_one_pixel_far_from_all_others(pixels, where, dtype):
    gen = torch.Generator(device="cuda").manual_seed(pixels)
    x = (torch.randn(2, 2, pixels, 64, generator=gen, device="cuda")).to(DT[dtype])
    x[:, :, where] = 1e4
    _, m, r = forward(x, 8)
    check_statistics(x, 8, 1e-5, m, r)


def test_equal_squares_in_long_images():
    """Images of so many pixels and so many of them that a thread has thousands; every square is the same number, so the roundings of
    a chain all go the same way."""
    pixels, ch, images = 65536, 128, 600
    gen = torch.Generator(device="cuda").manual_seed(1)
    for a in (1.0003, 1.137, 0.771):
        sign = torch.randint(0, 2, (1, 1, pixels, ch), generator=gen, device="cuda") * 2 - 1
        x = (sign * a).float()
        x[:, :, 0] = 0
        _, m, r = forward(x.expand(1, images, pixels, ch), 32)
        assert torch.equal(r, r[:, :1].expand_as(r))
        check_statistics(x, 32, 1e-5, m[:, :1], r[:, :1])


@pytest.mark.parametrize("source", ["x", "checkpoint"])
def test_gradients_of_equal_terms_in_long_images(source):
    """dy is one number everywhere, in images as above.  (dx, which would need memory, is not asked for.)  Chains of at most 64
    additions, 64 where threads meet, the rest in binary64; 4 roundings of a term, one of the result: 134 u."""
    pixels, ch, images, groups = 65536, 128, 600, 32
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(1, 1, pixels, ch, generator=gen, device="cuda")
    x = x.abs() if source == "x" else torch.rand(1, 1, pixels, ch, generator=gen, device="cuda").bfloat16().float()
    mean, rstd = torch.zeros(1, images, groups, device="cuda"), torch.full((1, images, groups), 0.7, device="cuda")
    q, scales = liec.liec_activation_compress(x.expand(1, images, pixels, ch)) if source == "checkpoint" else (None, None)
    read = restored64(q[:, :1], scales[:, :1], ch) if source == "checkpoint" else x.double()
    lib = liec.load_library()
    for c in (1.0003, 1.137, 0.771):
        dy = torch.full((ch,), c, device="cuda")
        dw, db = torch.empty(ch, device="cuda"), torch.empty(ch, device="cuda")
        d = liec.liec_group_norm_desc()
        d.workers, d.samples, d.pixels, d.channels, d.groups = 1, images, pixels, ch, groups
        d.dtype, d.grad_dtype, d.activation = liec.F32, liec.F32, 0
        d.x_pixel_stride = ch                                       # samples repeat
        need = lib.liec_group_norm_workspace_bytes(C.byref(d), 1)
        space = torch.empty(need, dtype=torch.uint8, device="cuda")
        st = lib.liec_group_norm_backward(C.byref(d), dy.data_ptr(), x.data_ptr() if q is None else None, None if q is None else q.data_ptr(),
                                          None if q is None else scales.data_ptr(), mean.data_ptr(), rstd.data_ptr(), None, None, None,
                                          dw.data_ptr(), db.data_ptr(), space.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
        assert st == 0
        c = float(dy[0])
        want = images * c * float(rstd[0, 0, 0]) * read[0, 0].sum(0)
        assert float(((dw.double() - want).abs() / want).max()) <= 134 * U, "dweight"
        assert float((db.double() / (images * pixels * c) - 1).abs().max()) <= 134 * U, "dbias"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,S,pixels,ch,groups,act", [(2, 3, 49, 64, 8, "none"), (1, 2, 3136, 64, 32, "silu"), (1, 1, 9001, 40, 8, "relu"), (1, 1, 65536, 32, 4, "none"),
                                                      (30, 40, 3136, 48, 6, "silu")])
def test_gradients_keep_their_digits(N, S, pixels, ch, groups, act, dtype):
    """Ordinary data.  Each sum: 64 + 64 + 8 roundings of at most u of the sum of the magnitudes, the short exponential of bfloat16 (2^-22 (4 + 2 |z|)
    of the slope, |z| below 8: 2^-17.6), a slope's own 40 u at |z| below 8."""
    gen = torch.Generator(device="cuda").manual_seed(ch)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, dy = (r(N, S, pixels, ch) + r(ch)).to(DT[dtype]), r(N, S, pixels, ch).to(DT[dtype])
    w, b = 1 + 0.1 * r(N, ch), 0.1 * r(N, ch)
    _, mean, rstd = forward(x, groups, w, b, activation=act)
    check_statistics(x[-1:], groups, 1e-5, mean[-1:], rstd[-1:])
    _, dw, db = backward(dy, x, mean, rstd, w, b, activation=act)
    width = ch // groups
    xh = (x[-1].double() - mean[-1].double().repeat_interleave(width, -1)[:, None]) * rstd[-1].double().repeat_interleave(width, -1)[:, None]
    z = xh * w[-1].double() + b[-1].double()
    s = torch.sigmoid(z)
    slope = (z > 0).double() if act == "relu" else s * (1 + z * (1 - s)) if act == "silu" else torch.ones_like(z)
    each = (136 + (40 if act == "silu" else 0)) * U + (2.0 ** -17.6 if act == "silu" and dtype == "bf16" else 0)
    for got, term in ((dw, dy[-1].double() * slope * xh), (db, dy[-1].double() * slope)):
        off = (got[-1].double() - term.sum((0, 1))).abs() / term.abs().sum((0, 1))
        assert float(off.max()) <= each, f"{float(off.max()) / U:.0f} u"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1 << 16, 1 << 20])
def test_bfloat16_weight_gradients_of_many_tokens(rows, dtype):
    """Positive terms, a tile for every pair of SMs, so that no plan cuts them.  At most 1024 additions (of 16 products each) to a sum in tensor
    memory, each cutting less than 2 u of it: 2048 u = 2^-13; these sums are added with rounding, at most 64 of them.  Then half a
    bfloat16 step.  On the average over the 18,944 outputs what is cut stays: against the outputs' own roundings, an output is a step of
    2^-8 lower where a border between steps lies within what was cut from it.  The outputs of 2^16 tokens are spread by 107 around 2^16, a step
    below which is 256, so that the share of them between two places is at most 0.4 / 107 of the distance: at most 0.4 / 107 x 256 = 0.96 of 2^-13 on the
    average, and six standard deviations of that count (at most 290) are 2e-5.  (The outputs' own roundings have an average that is not zero, as
    nearly all of them lie less than two steps from 2^16: 3.9e-4.)"""
    gen = torch.Generator(device="cuda").manual_seed(13)
    dy = (torch.rand(74, rows, 8, generator=gen, device="cuda") + 0.5).to(DT[dtype])
    q, scales = liec.liec_activation_compress((torch.rand(74, rows, 32, generator=gen, device="cuda") + 0.5).bfloat16())
    got = liec.liec_weight_grad(dy, q, scales, 32, dweight=torch.empty(74, 8, 32, dtype=torch.bfloat16, device="cuda")).double()
    want = torch.stack([dy[n].double().t() @ restored64(q[n], scales[n], 32) for n in range(74)])
    off = got / want - 1
    assert float(off.abs().max()) <= U_BF + 2.0 ** -13 + 64 * U
    assert abs(float((off - (want.to(torch.bfloat16).double() / want - 1)).mean())) <= 2.0 ** -13 + 64 * U + 2e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,rows,h,out", [(1, 16385, 40, 30), (2, 40000, 300, 600), (75, 16500, 33, 520), (160, 17000, 20, 8)])
def test_bfloat16_weight_gradients_through_the_workspace(N, rows, h, out, dtype):
    """Tiles of one run and of several, full ones and those with fewer outputs: what lies beside the gradient is left alone, equal calls give
    equal bits."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    dy = torch.randn(N, rows, out, generator=gen, device="cuda").to(DT[dtype])
    q, scales = liec.liec_activation_compress(torch.randn(N, rows, h, generator=gen, device="cuda").bfloat16())
    grads = torch.full((N, out * h + 9), 5.0, dtype=torch.bfloat16, device="cuda")
    got = liec.liec_weight_grad(dy, q, scales, h, dweight=grads[:, 4:4 + out * h].unflatten(1, (out, h)))
    for n in (0, N - 1):
        check_weight_grad(dy[n:n + 1], restored64(q[n:n + 1], scales[n:n + 1], h), "bf16", got[n:n + 1])
    assert (grads[:, :4] == 5).all() and (grads[:, -5:] == 5).all()
    again = liec.liec_weight_grad(dy, q, scales, h, dweight=torch.empty(N, out, h, dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(again, got)


@pytest.mark.parametrize("pixels,ch,groups", [(64, 64, 8), (200, 96, 3), (49, 90, 5), (5000, 64, 8)])
def test_channels_far_apart_in_a_group(pixels, ch, groups):
    """Two channels of each group at 1000 and -1000: their sum is exact in binary64, so a group's mean is off by what its channels' own sums lose, 64 + 64 + 8
    roundings of what lies about a channel's mean, and by the roundings of its own."""
    gen = torch.Generator(device="cuda").manual_seed(ch)
    x = torch.randn(2, 4, pixels, ch, generator=gen, device="cuda")
    width = ch // groups
    x[..., 0::width] += 1000
    x[..., 1::width] -= 1000
    _, mean, rstd = forward(x, groups)
    m, _, r = statistics64(x, groups, 1e-5)
    about = (x.double() - x.double().mean(2, keepdim=True)).abs().mean(2).unflatten(-1, (groups, width)).mean(-1)
    assert ((mean.double() - m).abs() <= 2 * U * m.abs() + 136 * U * about).all(), float(((mean.double() - m).abs() / about).max() / U)
    assert ((rstd.double() - r).abs() <= RSTD * r).all()

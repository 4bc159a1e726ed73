"""Sums keep their digits: where the first pixel of an image, or any other, is far from all others."""

import pytest
import torch

from activation_helpers import DT, U
from paper_2402_11857_b200 import liec

pytestmark = pytest.mark.gpu
forward = liec.liec_group_norm_forward


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

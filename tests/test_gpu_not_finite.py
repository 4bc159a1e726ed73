"""What group normalisation does with an infinity or NaN in x, for every activation: the group is NaN in y, dx and dweight; dbias is the sum of
dz alone, which sees x through SiLU's slope only."""
import pytest
import torch

from activation_helpers import DT, restored64
from paper_2402_11857_b200 import liec

pytestmark = pytest.mark.gpu
forward, backward = liec.liec_group_norm_forward, liec.liec_group_norm_backward


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("pixels", [30, 7000])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("checkpoint", [False, True])
def test_what_the_group_leaves(checkpoint, value, pixels, act, dtype):
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn(2, 3, pixels, 64, generator=gen, device="cuda").to(DT[dtype]) for _ in range(2))
    x[1, 2, pixels // 2, 17] = value                                # group 2 of 8, channels 16 to 23
    y, mean, rstd, q, scales = forward(x, 8, activation=act, compress=True)
    dx, dw, db = backward(dy, (q, scales) if checkpoint else x, mean, rstd, activation=act)
    assert y[1, 2, :, 16:24].isnan().all() and dx[1, 2, :, 16:24].isnan().all() and dw[1, 16:24].isnan().all()
    assert not mean[1, 2, 2].isfinite() and int(mean.isfinite().logical_not().sum()) == 1
    if act == "silu":
        assert db[1, 16:24].isnan().all()
    elif act == "relu":                                             # a z that is NaN is not above zero
        others = torch.ones(2, 3, dtype=torch.bool, device="cuda")
        others[1, 2] = False
        read = restored64(q, scales, 64).to(x.dtype) if checkpoint else x
        clean = backward(dy[others][None], read[others][None], mean[others][None].contiguous(), rstd[others][None].contiguous(), activation=act)[2]
        both = db.sum(0)[16:24].double()
        assert ((both - clean[0, 16:24].double()).abs() <= 1e-4 * dy[others].double().abs().sum((0, 1))[16:24]).all()
    else:
        assert ((db.double() - dy.double().sum((1, 2))).abs() <= 1e-5 * dy.double().abs().sum((1, 2))).all()
    # what a checkpoint's block of 32 channels loses besides is its own pixel's
    bad = torch.zeros_like(dx, dtype=torch.bool)
    bad[1, 2, :, 16:24] = True
    if checkpoint:
        bad[1, 2, :, 0:32] = True
    assert dx[~bad].isfinite().all() and dw[0].isfinite().all() and dw[1, 32:].isfinite().all()
    assert checkpoint or (dw[1, :16].isfinite().all() and dw[1, 24:].isfinite().all())

"""Group normalisation where one of weight and bias is shared by the workers and the other is their own."""
import pytest
import torch

from activation_helpers import check_group_norm_backward, check_group_norm_forward
from paper_2402_11857_b200 import liec

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shared", ["weight", "bias"])
@pytest.mark.parametrize("pixels", [40, 6000])
def test_one_vector_shared(pixels, shared):
    gen = torch.Generator(device="cuda").manual_seed(pixels)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, dy = r(3, 2, pixels, 48), r(3, 2, pixels, 48)
    own = {"weight": 1 + 0.3 * r(3, 48), "bias": 0.3 * r(3, 48)}
    full = own | {shared: own[shared][:1].expand(3, 48)}
    given = own | {shared: own[shared][0]}
    y, mean, rstd = liec.liec_group_norm_forward(x, 6, given["weight"], given["bias"], activation="silu")
    check_group_norm_forward(x, full["weight"], full["bias"], 6, 1e-5, "silu", "f32", y, mean, rstd)
    dx, dw, db = liec.liec_group_norm_backward(dy, x, mean, rstd, given["weight"], given["bias"], activation="silu")
    assert dw.shape == db.shape == (3, 48)
    check_group_norm_backward(dy, x, mean, rstd, full["weight"], full["bias"], "silu", "f32", "f32", dx, dw, db)
    dx2, dw2, db2 = liec.liec_group_norm_backward(dy, x, mean, rstd, given["weight"], given["bias"], activation="silu", dweight=torch.zeros(3, 48, device="cuda"))
    assert torch.equal(dx2, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)

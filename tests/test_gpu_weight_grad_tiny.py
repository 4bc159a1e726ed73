"""Weight gradients of a binary32 dy at the lower end of its range: exact products while all of its bits lie at 2^-133 or above, the last bit of a
subnormal bfloat16 number; what lies below is cut."""
import pytest
import torch

from paper_2402_11857_b200 import liec

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exponent", [-90, -109, -110, -111, -118, -126, -130, -140])
def test_what_is_cut(exponent):
    gen = torch.Generator(device="cuda").manual_seed(-exponent)
    q, scales = liec.liec_activation_compress(torch.full((1, 1, 32), 2.0 ** 60, device="cuda"))
    bits = torch.randint(0, 1 << 22, (64,), generator=gen, device="cuda").double() * 2 + 1
    dy = ((1 + bits / 2 ** 23) * 2.0 ** exponent).float()
    want = dy.double() * 2.0 ** 60
    got = liec.liec_weight_grad(dy[None, None], q, scales, 32)[0, :, 7].double()
    if exponent >= -110:
        assert torch.equal(got, want)
    assert ((got - want).abs() < 2.0 ** (60 - 133)).all() and (got <= want).all()

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

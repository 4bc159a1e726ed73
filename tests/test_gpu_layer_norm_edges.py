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

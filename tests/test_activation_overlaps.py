"""Calls of group normalisation that are refused before any CUDA call: outputs of the backward pass over the statistics that it reads, and more
images than a launch holds."""
import ctypes as C

import pytest

from paper_2402_11857_b200 import liec
from test_activation_arguments import AT, group_norm
from test_operator_arguments import lib  # noqa: F401  (fixture)

STATISTICS = 4 * 2 * 3 * 4   # bytes of mean and of rstd


@pytest.mark.parametrize("from_checkpoint", [False, True])
@pytest.mark.parametrize("name,at", [(n, at) for n in ("dx", "dweight", "dbias") for at in (3 * AT, 3 * AT + STATISTICS - 4, 4 * AT, 4 * AT + STATISTICS - 4)])
def test_outputs_over_the_statistics(lib, name, at, from_checkpoint):
    x, q, scales = (None, 11 * AT, 12 * AT) if from_checkpoint else (2 * AT, None, None)
    places = {"dx": 7 * AT, "dweight": 8 * AT, "dbias": 9 * AT} | {name: at}
    st = lib.liec_group_norm_backward(C.byref(group_norm()), AT, x, q, scales, 3 * AT, 4 * AT, 5 * AT, 6 * AT, places["dx"], places["dweight"], places["dbias"],
                                      10 * AT, 1 << 24, None)
    assert st == 1 and b"an output overlaps an input" in lib.liec_last_error(None)


def test_shared_gradients_over_the_statistics(lib):
    d = group_norm(shared_grads=1, weight_stride=0, bias_stride=0)
    for dweight, dbias in ((3 * AT + 8, 9 * AT), (8 * AT, 4 * AT - 92)):
        assert lib.liec_group_norm_backward(C.byref(d), AT, 2 * AT, None, None, 3 * AT, 4 * AT, None, None, None, dweight, dbias, 10 * AT, 1 << 24, None) == 1
        assert b"an output overlaps an input" in lib.liec_last_error(None)


def test_without_images_there_are_no_statistics(lib):
    assert lib.liec_group_norm_backward(C.byref(group_norm(pixels=0)), None, None, None, None, 3 * AT, 4 * AT, None, None, 3 * AT, None, None, None, 0, None) == 0


def test_images_that_a_launch_cannot_hold(lib):
    """2^31 blocks are one too many: refused by name, before the launch is."""
    at = [AT << 12 | k << 40 for k in range(1, 8)]
    d = group_norm(workers=2, samples=1 << 30, channels=1, groups=1, pixels=1, **{f"{n}_{axis}_stride": 1 << 30 if axis == "worker" else 1 for n in ("x", "y", "dx")
                                                                                 for axis in ("pixel", "sample", "worker")})
    assert lib.liec_group_norm_workspace_bytes(C.byref(d), 0) == 0
    assert lib.liec_group_norm_forward(C.byref(d), at[0], None, None, at[1], at[2], at[3], None, None, at[4], 1 << 40, None) == 2
    assert b"2^31 images" in lib.liec_last_error(None)
    assert lib.liec_group_norm_backward(C.byref(d), at[0], at[1], None, None, at[2], at[3], None, None, None, at[4], at[5], at[6], 1 << 40, None) == 2
    d = group_norm(workers=1, samples=(1 << 31) - 1, channels=1, groups=1, pixels=0)
    assert lib.liec_group_norm_forward(C.byref(d), at[0], None, None, at[1], at[2], at[3], None, None, at[4], 1 << 40, None) == 0

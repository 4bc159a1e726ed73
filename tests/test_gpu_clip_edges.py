"""Gradient norms and clipping at the edges of what a call may be given: the most tiles a row can have, waits
that run out, tables and buffers that do not fit together."""
import gc

import numpy as np
import pytest
import torch

from gpu_helpers import DEV
from paper_2402_11857_b200 import liec

pytestmark = pytest.mark.gpu

SIGN = liec.COMP_SCALED_SIGN
TILE, PASS = 8192, 4096      # elements per tile; tile sums that a row's join takes at a time
TDT = {liec.F32: torch.float32, liec.BF16: torch.bfloat16}


def small_integers(N, d, dtype, seed):
    """Rows of integers from -3 to 3, and their norms: sums of squares below 2^53 are exact in any order."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    G, norms = torch.empty(N, d, dtype=dtype, device=DEV), []
    for i in range(N):
        total = 0
        for a in range(0, d, 1 << 28):
            part = torch.randint(-3, 4, (min(d, a + (1 << 28)) - a,), generator=gen, device=DEV, dtype=torch.int8)
            G[i, a:a + len(part)] = part.to(dtype)
            total += int((part * part).sum(dtype=torch.int64))
        norms.append(np.float32(np.sqrt(np.float64(total))))
    return G, np.asarray(norms)


@pytest.mark.parametrize("gdt", [liec.F32, liec.BF16])
@pytest.mark.parametrize("passes", [3, 5])
def test_rows_of_several_passes(passes, gdt):
    """Counts of passes that are no power of two, rows that join one after another."""
    N, d = 3, (passes - 1) * PASS * TILE + 3 * TILE + 5
    off = [0, 1, TILE + 1, d]
    G, norms = small_integers(N, d, TDT[gdt], passes)
    ctx = liec.Context(torch.zeros(N, d, device=DEV), torch.zeros(d, device=DEV), off, SIGN, SIGN, grad_dtype=gdt)
    got = ctx.liec_clip_grads(G, float("inf"))
    assert np.array_equal(got.cpu().numpy(), norms)
    out, limit = torch.empty_like(G), float(np.sort(norms)[1])
    ctx.liec_clip_grads(G, limit, out=out)
    for i in range(N):
        factor = np.float32(np.float64(np.float32(limit)) / np.float64(norms[i])) if norms[i] > limit else np.float32(1)
        # (the factor is divided by the norm before its rounding to binary32: one step of difference at most)
        near = [np.nextafter(factor, np.float32(0)), factor, np.nextafter(factor, np.float32(2))]
        assert any(torch.equal(out[i], (G[i].float() * float(f)).to(G.dtype)) for f in near)
    assert ctx.liec_device_status() == 0


def test_norm_of_the_most_tiles():
    """dim just below 2^32 in 60,001 segments, 60,000 of them of one element: 143 passes, more than a power of two
    below the kernel's array."""
    gc.collect()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GiB of free device memory")
    d = (1 << 32) - TILE
    off = list(range(60_001)) + [d]
    tiles = 60_000 + (d - 60_000 + TILE - 1) // TILE
    assert 128 < (tiles + PASS - 1) // PASS <= 145
    G, norms = small_integers(1, d, torch.bfloat16, 7)
    ctx = liec.Context(torch.zeros(1, d, device=DEV), torch.zeros(d, device=DEV), off, SIGN, SIGN, grad_dtype=liec.BF16)
    assert np.array_equal(ctx.liec_clip_grads(G, float("inf")).cpu().numpy(), norms)
    assert ctx.liec_device_status() == 0
    del ctx, G
    gc.collect()
    torch.cuda.empty_cache()

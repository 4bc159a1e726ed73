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


@pytest.mark.parametrize("tiles", [2, 40, 60])
def test_table_that_is_not_there_yet_or_of_another_type(tiles):
    """A captured liec_set_tensors has not written the table before its first replay, and a replay brings its own table
    back: a gather that expects another type reads no tensor, says so, and the next right one is right."""
    N, d = 2, tiles * TILE + 24
    off = [0, 1000, d]
    sets = {dt: [[torch.randint(-3, 4, (b - a,), device=DEV).to(dt) for a, b in zip(off, off[1:])] for _ in range(N)]
            for dt in (torch.float32, torch.bfloat16)}
    rows = {dt: torch.stack([torch.cat([t.float() for t in ts]) for ts in s]) for dt, s in sets.items()}
    ctx = liec.Context(torch.zeros(N, d, device=DEV), torch.zeros(d, device=DEV), off, SIGN, SIGN)
    out = torch.full((N, d), 7.0, device=DEV)

    def refused():
        out.fill_(7.0)
        norms = ctx.liec_gather_grads(out)
        assert ctx.liec_device_status() == 64 and (out == 0).all() and (norms == 0).all()
        ctx.liec_clear_status()

    def right(dt):
        out.fill_(7.0)
        norms = ctx.liec_gather_grads(out)
        assert torch.equal(out, rows[dt])
        assert torch.equal(norms, rows[dt].double().square().sum(1).sqrt().float())
        assert ctx.liec_device_status() == 0

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.liec_set_tensors(sets[torch.bfloat16])
    refused()                                   # not replayed yet
    graph.replay()
    right(torch.bfloat16)
    ctx.liec_set_tensors(sets[torch.float32])
    right(torch.float32)
    graph.replay()                              # the bfloat16 table is back, the host expects binary32
    refused()
    ctx.liec_set_tensors(sets[torch.float32])
    right(torch.float32)


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tiles", [1, 50])
def test_tensors_within_the_rows(tiles, src):
    """Tensors that share memory with the rows they are gathered into are refused; beside them they are not."""
    N, off = 2, [0, 24, tiles * TILE]
    d = off[-1]
    size = torch.empty(0, dtype=src).element_size()
    memory = torch.zeros(4 * N * d + 64, device=DEV)
    rows = memory[:N * d].view(N, d)
    beyond = memory.view(src)[N * d * 4 // size:]           # begins where the rows end
    ctx = liec.Context(torch.zeros(N, d, device=DEV), torch.zeros(d, device=DEV), off, SIGN, SIGN)

    def tensors(first):
        rest = [torch.ones(b - a, dtype=src, device=DEV) for _ in range(N) for a, b in zip(off, off[1:])][1:]
        return [[first] + rest[:1], rest[1:]]

    inside = memory.view(src)
    for first in (inside[:24], inside[(N * d - 4) * 4 // size:][:24], inside[d * 4 // size - 5:][:24]):
        ctx.liec_set_tensors(tensors(first))
        with pytest.raises(liec.LiecError, match="overlaps") as err:
            ctx.liec_gather_grads(rows)
        assert err.value.status == 1
    assert (memory == 0).all()
    ctx.liec_set_tensors(tensors(beyond[:24]))
    norms = ctx.liec_gather_grads(rows)
    assert torch.equal(norms.cpu(), torch.tensor([(d - 24.0) ** 0.5, d ** 0.5]))
    assert (rows[0, :24] == 0).all() and (rows[0, 24:] == 1).all() and (rows[1] == 1).all() and (memory[N * d:] == 0).all()
    ctx.liec_set_tensors([[None, None], [None, None]])      # no tensors at all
    assert (ctx.liec_gather_grads(rows) == 0).all() and (rows == 0).all()
    assert ctx.liec_device_status() == 0


@pytest.mark.parametrize("gdt", [liec.F32, liec.BF16])
@pytest.mark.parametrize("N,tiles", [(2, 40), (1, 9000), (3, 1500)])
@pytest.mark.parametrize("withhold", [1, 2, 3])
def test_norm_wait_runs_out(withhold, N, tiles, gdt):
    """A tile's sum or a row's factor that is never handed over: whoever waits for it (a row's join, the scaling, the
    producer once its ring is full) gives up at its limit, bit 32 is set, no row is written, and the next call is right.
    The long rows have three passes of tile sums to join, and more tiles than the rings of all SMs hold."""
    d = tiles * TILE - 3
    off = [0, TILE + 1, d]
    G, norms = small_integers(N, d, TDT[gdt], tiles)
    ctx = liec.Context(torch.zeros(N, d, device=DEV), torch.zeros(d, device=DEV), off, SIGN, SIGN, grad_dtype=gdt)
    out, before = torch.full_like(G, 7.0), G.clone()
    limit = 0.5 * float(norms.min())
    ctx.liec_set_norm_wait(poll_limit=500, withhold=withhold)
    ctx.liec_clip_grads(G, limit, out=out)
    assert ctx.liec_device_status() == 32
    assert (out == 7).all() and torch.equal(G, before)
    ctx.liec_clear_status()
    ctx.liec_clip_grads(G, limit)                                 # in place
    assert ctx.liec_device_status() == 32 and torch.equal(G, before)
    ctx.liec_clear_status()
    got = ctx.liec_clip_grads(G, float("inf"))                    # norms alone: nobody waits for a factor
    if withhold == 2:
        assert ctx.liec_device_status() == 0 and np.array_equal(got.cpu().numpy(), norms)
    else:
        assert ctx.liec_device_status() == 32
    ctx.liec_set_norm_wait()
    ctx.liec_clear_status()
    assert np.array_equal(ctx.liec_clip_grads(G, limit, out=out).cpu().numpy(), norms)
    factor = (np.float64(np.float32(limit)) / norms.astype(np.float64))
    error = (out.double() - G.double() * torch.from_numpy(factor).to(DEV)[:, None]).abs()
    assert (error <= G.double().abs() * (2.0 ** -8 if gdt == liec.BF16 else 2.0 ** -22) * float(factor.max())).all()
    assert ctx.liec_device_status() == 0
    with pytest.raises(liec.LiecError) as err:
        ctx.liec_set_norm_wait(withhold=4)
    assert err.value.status == 1

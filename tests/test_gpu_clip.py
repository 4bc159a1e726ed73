"""Gradient norms and clipping on the GPU against a plain evaluation: bit for bit where the order of
the sums is fixed (tile trees, then the tree over the row's tiles), and against ordinary binary64 sums."""
import numpy as np
import pytest
import torch

import oracle
from gpu_helpers import DEV, f32, widen
from liec_synth import flat_layout, make_gradients, ragged_layout, resnet18_layout, scaled_layout
from liec_synth.layouts import Layout
from paper_2402_11857_b200 import liec

pytestmark = pytest.mark.gpu

SIGN = liec.COMP_SCALED_SIGN
TILE = 8192
TDT = {liec.F32: torch.float32, liec.BF16: torch.bfloat16}


def balanced(sums):
    """Balanced binary tree over a list zero-padded to a power of two."""
    s = np.asarray(sums, np.float64)
    n = 1
    while n < len(s):
        n *= 2
    s = np.concatenate([s, np.zeros(n - len(s))])
    while len(s) > 1:
        s = s[0::2] + s[1::2]
    return float(s[0])


def reference(rows, off, max_norm, zero_nonfinite=False):
    """(clipped rows in binary32 before the rounding to the rows' type, norms) of binary32 rows, numpy."""
    out, norms = np.empty_like(rows), []
    max_norm = float(np.float32(max_norm))
    with np.errstate(all="ignore"):
        for i, g in enumerate(rows):
            sums = []
            for t in range(len(off) - 1):
                seg = g[off[t]:off[t + 1]]
                sums += [oracle.tree_sumsq(seg[b:b + TILE]) for b in range(0, len(seg), TILE)]
            norm = np.sqrt(np.float64(balanced(sums)))
            factor = np.float32(max_norm / norm) if norm > max_norm else np.float32(1.0)
            out[i] = np.zeros_like(g) if zero_nonfinite and not np.isfinite(norm) else g * factor
            norms.append(np.float32(norm))
    return out, np.asarray(norms, np.float32)


def bits(t):
    t = t.detach().cpu()
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).numpy()


def same(a, b):
    """Equal bits, NaNs counted as equal to one another."""
    a, b = a.detach().cpu(), b.detach().cpu()
    assert a.dtype == b.dtype and a.shape == b.shape
    nan = torch.isnan(a) & torch.isnan(b)
    diff = (bits(a) != bits(b)) & ~nan.numpy()
    return int(diff.sum()) == 0


def context(N, off, gdt):
    d = int(off[-1])
    return liec.Context(torch.zeros(N, d, device=DEV), torch.zeros(d, device=DEV), off, SIGN, SIGN, grad_dtype=gdt)


def rounded(rows32, gdt):
    return torch.from_numpy(rows32).to(TDT[gdt])


LAYOUTS = {
    "one": flat_layout(1), "seven": flat_layout(7), "tile": flat_layout(TILE), "tile+1": flat_layout(TILE + 1),
    "flat": flat_layout(65536), "ragged": ragged_layout(), "resnet/40": scaled_layout(resnet18_layout(), 40),
    "many": Layout("many", tuple(1 + (7 * q) % 53 for q in range(2000))),
    "long": flat_layout(2050 * TILE + 3),
}


@pytest.mark.parametrize("gdt", [liec.F32, liec.BF16])
@pytest.mark.parametrize("name,N", [("one", 3), ("seven", 2), ("tile", 1), ("tile+1", 4), ("flat", 4), ("ragged", 5),
                                    ("resnet/40", 33), ("many", 2), ("long", 2)])
def test_clip_rows(name, N, gdt):
    lay = LAYOUTS[name]
    off = lay.seg_offsets
    G = make_gradients("bf16_outliers" if gdt == liec.BF16 else "normal", 0.02, N, lay.dim, 0, base_seed=11)
    G = (G.float() * torch.linspace(0.25, 2.0, N)[:, None]).to(TDT[gdt])
    rows = widen(G)
    max_norm = float(np.median(np.linalg.norm(rows.astype(np.float64), axis=1)))
    want, norms = reference(rows, off, max_norm)
    ctx = context(N, off, gdt)
    Gd, out = G.to(DEV), torch.full((N, lay.dim), 7.0, dtype=TDT[gdt], device=DEV)
    got = ctx.liec_clip_grads(Gd, max_norm, out=out)
    assert same(got, torch.from_numpy(norms))
    assert same(out, rounded(want, gdt)) and same(Gd, G)
    # plain binary64 sums: the tree differs from them by at most d roundings of 2^-53, the norm by 2^-24
    plain = np.sqrt((rows.astype(np.float64) ** 2).sum(1))
    assert np.all(np.abs(f32(got) - plain) <= plain * (2.0 ** -24 + lay.dim * 2.0 ** -53))
    # in place, into a caller's norms, twice over the first result (no kept state)
    mine = torch.empty(N, device=DEV)
    assert ctx.liec_clip_grads(Gd, max_norm, norms=mine) is mine
    assert same(Gd, rounded(want, gdt)) and same(mine, torch.from_numpy(norms))
    # no clipping: the norms and a copy
    out.fill_(-1)
    Gd.copy_(G)
    got = ctx.liec_clip_grads(Gd, float("inf"), out=out)
    assert same(got, torch.from_numpy(norms)) and same(out, G)
    assert ctx.liec_device_status() == 0


@pytest.mark.parametrize("src", [liec.F32, liec.BF16])
@pytest.mark.parametrize("gdt", [liec.F32, liec.BF16])
@pytest.mark.parametrize("name,N", [("one", 1), ("ragged", 3), ("tile+1", 2), ("resnet/40", 8), ("many", 3), ("long", 1)])
def test_gather(name, N, gdt, src):
    """Tensors at odd addresses, some of them missing, of either type into rows of either type."""
    lay = LAYOUTS[name]
    off = lay.seg_offsets
    G = make_gradients("normal", 0.02, N, lay.dim, 1, base_seed=12).to(TDT[src])
    tensors, keep = [], []
    for i in range(N):
        ts = []
        for t in range(lay.num_segments):
            if (i + 3 * t) % 7 == 6:
                G[i, off[t]:off[t + 1]] = 0
                ts.append(None)
                continue
            n, shift = int(off[t + 1] - off[t]), (i + t) % 5
            buf = torch.empty(n + shift, dtype=TDT[src], device=DEV)
            keep.append(buf)
            buf[shift:] = G[i, off[t]:off[t + 1]]
            ts.append(buf[shift:])
        tensors.append(ts)
    rows = widen(G)
    max_norm = 0.7 * float(np.median(np.linalg.norm(rows.astype(np.float64), axis=1))) or 1.0
    want, norms = reference(rows, off, max_norm)
    ctx = context(N, off, gdt)
    ctx.liec_set_tensors(tensors)
    out = torch.full((N, lay.dim), 7.0, dtype=TDT[gdt], device=DEV)
    got = ctx.liec_gather_grads(out, max_norm)
    assert same(got, torch.from_numpy(norms)) and same(out, rounded(want, gdt))
    # new contents behind the same table, then no clipping
    for buf in keep:
        buf.mul_(-2.0)
    want, norms = reference(widen((G.float() * -2.0).to(TDT[src])), off, np.inf)
    got = ctx.liec_gather_grads(out)
    assert same(got, torch.from_numpy(norms)) and same(out + 0, rounded(want, gdt) + 0)


@pytest.mark.parametrize("zero_nonfinite", [False, True])
@pytest.mark.parametrize("gdt", [liec.F32, liec.BF16])
def test_extreme_values(gdt, zero_nonfinite):
    """Values whose squares leave binary32 at either end, zeros, infinities, NaN, each in a row of its own."""
    lay = ragged_layout()
    off, d = lay.seg_offsets, lay.dim
    G = make_gradients("normal", 1.0, 8, d, 0, base_seed=13)
    G[1] = 3.0e38
    G[2] = G[2] * 1e-30
    G[3] = 1e-42 if gdt == liec.F32 else 9.2e-41
    G[4] = 0.0
    G[4, ::2] = -0.0
    G[5, d - 1] = float("inf")
    G[6, 8192] = float("nan")
    G[7, 3] = float("-inf")
    G[7, 5] = float("nan")
    G = G.to(TDT[gdt])
    want, norms = reference(widen(G), off, 1.5, zero_nonfinite)
    ctx = context(8, off, gdt)
    Gd, out = G.to(DEV), torch.empty(8, d, dtype=TDT[gdt], device=DEV)
    for _ in range(2):
        got = ctx.liec_clip_grads(Gd, 1.5, out=out, zero_nonfinite=zero_nonfinite)
        assert same(got, torch.from_numpy(norms)) and same(out, rounded(want, gdt))
    got = ctx.liec_clip_grads(Gd, 1.5, zero_nonfinite=zero_nonfinite)
    assert same(got, torch.from_numpy(norms)) and same(Gd, rounded(want, gdt))


@pytest.mark.parametrize("gdt", [liec.F32, liec.BF16])
@pytest.mark.parametrize("N,tiles", [(300, 3), (150, 7), (150, 8), (40, 20), (300, 12), (40, 33), (2, 700), (1, 4100)])
def test_many_rows_and_norms_only(N, tiles, gdt):
    """Rows of a few tiles to a few thousand, few and many of them: clipped, and in place with nothing to clip,
    where only the norms are wanted and the rows stay as they are."""
    off = [0, 5 * TILE // 2, tiles * TILE - 9] if tiles > 2 else [0, tiles * TILE]
    d = off[-1]
    gen = torch.Generator(device=DEV).manual_seed(tiles)
    G = (torch.randn(N, d, generator=gen, device=DEV) * torch.linspace(0.5, 1.5, N, device=DEV)[:, None]).to(TDT[gdt])
    rows = widen(G.cpu())
    max_norm = float(np.median(np.linalg.norm(rows.astype(np.float64), axis=1)))
    want, norms = reference(rows, off, max_norm)
    ctx = context(N, off, gdt)
    Gd = G.clone()
    assert same(ctx.liec_clip_grads(Gd, float("inf")), torch.from_numpy(norms)) and torch.equal(Gd, G)
    out = torch.full((N, d), 7.0, dtype=TDT[gdt], device=DEV)
    assert same(ctx.liec_clip_grads(Gd, max_norm, out=out), torch.from_numpy(norms))
    assert same(out, rounded(want, gdt)) and torch.equal(Gd, G)
    assert same(ctx.liec_clip_grads(Gd, max_norm), torch.from_numpy(norms)) and same(Gd, out)
    assert ctx.liec_device_status() == 0


@pytest.mark.parametrize("gdt", [liec.F32, liec.BF16])
def test_copy_wait_runs_out(gdt):
    """A bulk copy whose barrier never completes: the wait ends by its limit, bit 8 is set, no row is written,
    and the next call with the limit restored is right."""
    off, N = [0, 40 * TILE], 2
    G = make_gradients("normal", 0.1, N, off[-1], 0, base_seed=15).to(TDT[gdt])
    want, norms = reference(widen(G), off, 1.0)
    ctx = context(N, off, gdt)
    Gd, out = G.to(DEV), torch.full((N, off[-1]), 7.0, dtype=TDT[gdt], device=DEV)
    ctx.liec_set_copy_wait(poll_limit=1000, expect_extra_bytes=16)
    ctx.liec_clip_grads(Gd, 1.0, out=out)
    torch.cuda.synchronize()
    assert ctx.liec_device_status() & 8
    assert (out == 7).all() and same(Gd, G)
    ctx.liec_set_copy_wait()
    ctx.liec_clear_status()
    assert same(ctx.liec_clip_grads(Gd, 1.0, out=out), torch.from_numpy(norms)) and same(out, rounded(want, gdt))
    assert ctx.liec_device_status() == 0


def test_norm_at_the_limit_is_left_alone():
    """norm == max_norm is not clipped; one step of binary32 above it is."""
    off = [0, 4]
    ctx = context(2, off, liec.F32)
    G = torch.tensor([[3.0, 0.0, 4.0, 0.0], [3.0, 0.0, 4.0, 0.0]], device=DEV)
    G[1, 2] = float(np.nextafter(np.float32(4.0), np.float32(5.0)))
    out = torch.empty_like(G)
    ctx.liec_clip_grads(G, 5.0, out=out)
    assert torch.equal(out[0], G[0]) and not torch.equal(out[1], G[1])


def test_clipped_step_side_stream_and_graph():
    """Gather, clip and the compressed step on a stream of their own, plain and replayed from a graph, against
    the oracle's step on the clipped rows."""
    lay = ragged_layout()
    off, N = lay.seg_offsets, 3
    ctx = context(N, off, liec.F32)
    G = make_gradients("normal", 0.5, N, lay.dim, 0, base_seed=14)
    tensors = [[G[i, off[t]:off[t + 1]].to(DEV).clone() for t in range(lay.num_segments)] for i in range(N)]
    rows = torch.empty(N, lay.dim, device=DEV)
    norms = torch.empty(N, device=DEV)
    torch.cuda.synchronize()
    Xh, eh = np.zeros((N, lay.dim), np.float32), np.zeros(lay.dim, np.float32)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx.liec_set_tensors(tensors)
        ctx.liec_gather_grads(rows, 3.0, norms=norms)
        ctx.liec_step(rows, 0.1)
    s.synchronize()
    want, wn = reference(G.numpy(), off, 3.0)
    oracle.step(Xh, eh, want, 0.1, off, SIGN, SIGN)
    assert same(norms, torch.from_numpy(wn)) and same(rows, torch.from_numpy(want))
    assert same(ctx.params, torch.from_numpy(Xh)) and same(ctx.error, torch.from_numpy(eh))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.liec_set_tensors(tensors)
        ctx.liec_gather_grads(rows, 3.0, norms=norms)
        ctx.liec_step(rows, 0.1)
    for step in range(1, 4):
        G = make_gradients("normal", 0.5, N, lay.dim, step, base_seed=14)
        for i in range(N):
            for t in range(lay.num_segments):
                tensors[i][t].copy_(G[i, off[t]:off[t + 1]])
        graph.replay()
        torch.cuda.synchronize()
        want, wn = reference(G.numpy(), off, 3.0)
        oracle.step(Xh, eh, want, 0.1, off, SIGN, SIGN)
        assert same(norms, torch.from_numpy(wn)) and same(rows, torch.from_numpy(want))
        assert same(ctx.params, torch.from_numpy(Xh)) and same(ctx.error, torch.from_numpy(eh))
    assert ctx.liec_device_status() == 0


def test_refusals():
    lay = ragged_layout()
    off, d = lay.seg_offsets, lay.dim
    ctx = context(2, off, liec.F32)
    G = torch.zeros(2, d, device=DEV)

    def status(call):
        with pytest.raises(liec.LiecError) as err:
            call()
        return err.value.status

    for bad in (0.0, -1.0, float("nan")):
        assert status(lambda: ctx.liec_clip_grads(G, bad)) == 1
    assert status(lambda: ctx.liec_gather_grads(G, 1.0)) == 4            # no tensors given yet
    both = torch.zeros(3 * d + 8, device=DEV)
    a, b = both[:2 * d].view(2, d), both[d // 4 * 4:][:2 * d].view(2, d)
    assert status(lambda: ctx.liec_clip_grads(a, 1.0, out=b)) == 1       # overlapping, not the same
    assert status(lambda: ctx.liec_clip_grads(both[1:2 * d + 1].view(2, d), 1.0)) == 1   # not 16-byte aligned
    for wrong in (G.to(torch.bfloat16), G[:1], G.cpu()):
        with pytest.raises(ValueError):
            ctx.liec_clip_grads(wrong, 1.0)
    with pytest.raises(ValueError):
        ctx.liec_clip_grads(G, 1.0, norms=torch.zeros(3, device=DEV))
    ts = [[torch.zeros(n, device=DEV) for n in lay.sizes] for _ in range(2)]
    for spoil in (lambda: ts[:1], lambda: [ts[0], ts[1][:-1]], lambda: [ts[0], ts[1][:-1] + [torch.zeros(3, device=DEV)]],
                  lambda: [ts[0], ts[1][:-1] + [ts[1][-1].bfloat16()]], lambda: [ts[0], ts[1][:-1] + [ts[1][-1].cpu()]],
                  lambda: [[t.half() for t in row] for row in ts]):
        with pytest.raises(ValueError):
            ctx.liec_set_tensors(spoil())
    assert status(lambda: ctx.liec_gather_grads(G, 1.0)) == 4            # a refused table is no table
    ctx.liec_set_tensors(ts)
    ctx.liec_uplink_compress(G)
    assert status(lambda: ctx.liec_clip_grads(G, 1.0)) == 4              # between the stages
    assert status(lambda: ctx.liec_gather_grads(G, 1.0)) == 4
    ctx.liec_abort_step()
    ctx.liec_gather_grads(G, 1.0)
    lib = liec.load_library()
    assert lib.liec_set_tensors(ctx._ctx, None, liec.F32, None) == 1
    ptrs = np.full(2 * lay.num_segments, 258, np.uint64)
    assert lib.liec_set_tensors(ctx._ctx, ptrs.ctypes.data, liec.F32, None) == 1     # 258 is not a multiple of 4
    assert lib.liec_set_tensors(ctx._ctx, ptrs.ctypes.data, 7, None) == 1
    assert lib.liec_clip_grads(ctx._ctx, None, G.data_ptr(), 1.0, 0, None, None) == 1
    assert lib.liec_clip_grads(ctx._ctx, G.data_ptr(), None, 1.0, 0, None, None) == 1
    torch.cuda.synchronize()
    assert ctx.liec_device_status() == 0

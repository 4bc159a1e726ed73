// How the weight gradient's work is dealt out: plain arithmetic, for the host and the kernels.
#pragma once
#include <algorithm>
#include <cstdint>

#ifdef __CUDACC__
#define WG_BOTH __host__ __device__
#else
#define WG_BOTH
#endif

namespace liec {

constexpr int WG_TOKENS = 32;      // of a stage
constexpr int WG_CHANNELS = 128;   // of a CTA
constexpr int WG_SLAB = 256;       // outputs of one product of a pair of CTAs, 128 from each
constexpr int WG_PAIRS = 74;       // of SMs
// Stages that one sum in tensor memory takes.  The products' additions there cut what does not fit: always towards zero, which over
// 8192 tokens comes to 6e-6 of a gradient (measured), ten times what rounded additions lose, and grows with the tokens.  So a binary32
// gradient is summed there 1792 tokens at a time at most, and these sums are added with rounding: 8e-7.  Each such sum takes 10 us, 5 of
// them an SM's way out for its 256 KB: 8 x 8192 x 768 x 2304 took 242 us with them on one card (186 in one sum, 203 with 4096 tokens
// and 2.5e-6, 233 with 2048 and 1.2e-6).  A bfloat16 gradient keeps 2^-9 anyway: 16,384 tokens at a time, which cut at most 2^-13 and 2e-5 on the
// average, a hundredth of that.
constexpr int WG_SUM_STAGES = 56, WG_SUM_STAGES_BF16 = 512;
constexpr int wg_slabs(int dtype) { return dtype == 0 ? 1 : 2; }   // of a tile

// The work: all workers' tiles, full ones first, then those with the last, fewer slabs.  As many full tiles as fill the
// pairs evenly are taken whole; the rest is cut into runs of tokens, whose sums go through the workspace and are joined by
// another kernel.  Pair k takes items k, k + pairs, ...: neighbours in the list, which read the same operands (channels
// vary fastest), run side by side and meet in the L2 cache.  (Equal shares of one long line of work instead, cut wherever
// they end: neighbours then read different tokens, and 8 x 8192 x 768 x 2304 took 270 us before its join, all operands from HBM.)
struct WgItem {
    int64_t slot;                // where the sums go in the workspace, in floats; -1: to dW
    int32_t worker, c_tile, o_tile, slabs, stage, stages;   // first stage and number
};
struct WgPlan {
    int64_t full, whole, last, items;              // tiles: full ones, those taken whole, with the last slabs
    int32_t stages, runs, run, last_runs, last_run;   // stages of a tile; runs of a cut tile and their stages, full and last
    int32_t c_tiles, o_full, slabs, last_slabs, pairs;
    int32_t joined;                                // all tiles go through the workspace, those in one run too, and none is taken whole
    WG_BOTH bool cut_joins() const { return runs > 1 || joined != 0; }
    WG_BOTH bool last_joins() const { return last_runs > 1 || joined != 0; }
    WG_BOTH int64_t slot_size(bool is_last) const { return (int64_t)(is_last ? last_slabs : slabs) * WG_SLAB * 2 * WG_CHANNELS; }
    WG_BOTH int64_t slots() const {
        return (cut_joins() ? (full - whole) * runs * slot_size(false) : 0) + (last_joins() ? last * last_runs * slot_size(true) : 0);
    }
    WG_BOTH WgItem tile_of(int64_t tile) const {
        WgItem t{};
        t.slot = -1;
        if (tile < full) {
            const int64_t each = (int64_t)c_tiles * o_full;
            t.worker = (int32_t)(tile / each);
            const int32_t rest = (int32_t)(tile - t.worker * each);
            t.o_tile = rest / c_tiles;
            t.c_tile = rest - t.o_tile * c_tiles;
            t.slabs = slabs;
        } else {
            t.worker = (int32_t)((tile - full) / c_tiles);
            t.c_tile = (int32_t)(tile - full - (int64_t)t.worker * c_tiles);
            t.o_tile = o_full;
            t.slabs = last_slabs;
        }
        t.stages = stages;
        return t;
    }
    WG_BOTH WgItem item(int64_t i) const {
        if (i < whole) return tile_of(i);
        i -= whole;
        const int64_t cut = full - whole;
        const bool is_last = i >= cut * runs;
        if (is_last) i -= cut * runs;
        const int64_t tiles = is_last ? last : cut, run_index = i / tiles;
        const int32_t n = is_last ? last_runs : runs, length = is_last ? last_run : run;
        WgItem t = tile_of((is_last ? full : whole) + i - run_index * tiles);
        if (is_last ? last_joins() : cut_joins()) {
            t.slot = i * slot_size(is_last) + (is_last && cut_joins() ? cut * runs * slot_size(false) : 0);
            t.stage = (int32_t)run_index * length;
            t.stages = length < stages - t.stage ? length : stages - t.stage;
        }
        return t;
    }
};

// How many runs a cut tile has: the least time of the pair that has most to do, by what was measured (us): an item's start
// takes 2, a stage 0.36, with one slab 0.26 (0.7 with three parts of dy), a slab's end 2 (an SM's way out for its sums); a run
// of a cut tile 0.07 per slab (read and added), the joining launch 5.  Full tiles and those with fewer slabs have runs that take
// as long.  bf16_grad: a bfloat16 gradient cannot hold the sums so far of one that takes several, so these go through the workspace.
inline WgPlan wg_plan(int workers, int64_t rows, int in, int out, int dtype, bool bf16_grad = false) {
    WgPlan p{};
    const int slabs_all = (out + WG_SLAB - 1) / WG_SLAB;
    p.slabs = wg_slabs(dtype);
    p.c_tiles = (in + 2 * WG_CHANNELS - 1) / (2 * WG_CHANNELS);
    p.o_full = slabs_all / p.slabs;
    p.last_slabs = slabs_all % p.slabs;
    p.stages = (int32_t)((rows + WG_TOKENS - 1) / WG_TOKENS);
    p.full = (int64_t)workers * p.c_tiles * p.o_full;
    p.last = p.last_slabs ? (int64_t)workers * p.c_tiles : 0;
    p.joined = bf16_grad && p.stages > WG_SUM_STAGES_BF16;
    p.whole = p.joined ? 0 : p.full / WG_PAIRS * WG_PAIRS;
    const auto stage = [dtype](int slabs) { return dtype == 0 ? 0.7 * slabs : 0.16 + 0.1 * slabs; };
    const int64_t cut = p.full - p.whole;
    double best = 0.0;
    for (int n = 1; n <= WG_PAIRS && n <= p.stages; ++n) {
        const int run = (p.stages + n - 1) / n, runs = cut ? (p.stages + run - 1) / run : 1;
        const int last_n = cut ? std::max(1, (int)(n * stage(p.last_slabs) / stage(p.slabs) + 0.5)) : n;
        const int last_run = (p.stages + last_n - 1) / last_n, last_runs = p.last ? (p.stages + last_run - 1) / last_run : 1;
        const int64_t items = cut * runs + p.last * last_runs;
        if (items > 16 * WG_PAIRS && n > 1) break;
        double cost = 0.0;
        for (int64_t i = 0; i < items && i < 16 * WG_PAIRS; i += WG_PAIRS) cost += 2.0 + (i < cut * runs ? p.slabs * 2.0 + stage(p.slabs) * run : p.last_slabs * 2.0 + stage(p.last_slabs) * last_run);
        if (p.joined || runs > 1 || last_runs > 1) cost += 5.0 + 0.07 * (double)((p.joined || runs > 1 ? cut * runs * p.slabs : 0) + (p.joined || last_runs > 1 ? p.last * last_runs * p.last_slabs : 0));
        if (n > 1 && cost >= best) continue;
        best = cost;
        p.runs = runs; p.run = run; p.last_runs = last_runs; p.last_run = last_run;
        p.items = p.whole + items;
    }
    p.pairs = (int32_t)std::min<int64_t>(WG_PAIRS, p.items);
    return p;
}

}  // namespace liec

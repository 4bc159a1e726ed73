// Norm of every worker's gradient over all its tensors, and clipping.  For worker i with entries g_j:
//   norm_i = sqrt(sum_j g_j^2),  c_i = max_norm / norm_i if norm_i > max_norm, else 1,  out_j = round(c_i g_j)
// The squares are exact in binary64; a tile's sum is the balanced tree over its 8192 entries, and the
// row's sum the balanced tree over the row's tile sums in tile order, zero-padded to a power of two, so
// that the norm does not depend on how the tiles are spread over CTAs.  The gradients come as rows
// [N][d] or as N*T separate tensors (a table of pointers); a missing tensor counts as zeros.
//
// No entry can be written before the whole row has been read, so HBM's part is one read and one write only
// if the row is still on the chip when it is scaled.  Short rows: one cluster per row (clip_cluster_kernel).
// Others: one kernel that sums everything, then scales everything (clip_stream_kernel); it moves its two reads and
// one write at HBM's rate (GPT-2-small list, eight workers in bfloat16: 914 us = 6.5 TB/s).  Scaling row by row,
// behind the row's sum, was built and measured too: L2 keeps only the last 60 to 70 MB, and the wait
// for each row's norm costs more than that saves (1046 us; ResNet-18 list 189 against 178 us).
// Between the two, rows of some hundred tiles are bound by neither HBM nor the launch: every tile is fetched a second time
// although all of them would fit the rings together, and the start, the tickets of few tiles and the join of
// each row are not hidden (8 rows of 64 tiles in binary32 17 us, of 512 tiles 73 us; bytes at HBM's rate 5 and 41).
#include <cooperative_groups.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "balanced_join.h"
#include "device_common.cuh"
#include "granule.cuh"
#include "kernels.h"

namespace liec {

// ---- VEC consecutive elements as they lie in memory (aligned to min(16, VEC * size) bytes), and in binary32 ----
template <typename ST, int VEC>
struct Raw {
    static constexpr int WORDS = VEC * (int)sizeof(ST) / 4;
    uint32_t w[WORDS];
    template <bool LAST>   // LAST: not needed again
    __device__ __forceinline__ void load(const ST *ptr) {
        if constexpr (WORDS == 2) {
            const uint2 *from = reinterpret_cast<const uint2 *>(ptr);
            const uint2 q = LAST ? __ldcs(from) : *from;
            w[0] = q.x; w[1] = q.y;
        } else {
#pragma unroll
            for (int k = 0; k < WORDS; k += 4) {
                const uint4 *from = reinterpret_cast<const uint4 *>(reinterpret_cast<const uint32_t *>(ptr) + k);
                const uint4 q = LAST ? __ldcs(from) : *from;
                w[k] = q.x; w[k + 1] = q.y; w[k + 2] = q.z; w[k + 3] = q.w;
            }
        }
    }
    // element by element; those at or beyond `left` are +0
    __device__ __forceinline__ void load_guarded(const ST *ptr, int left) {
        if constexpr (sizeof(ST) == 4) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) w[k] = k < left ? reinterpret_cast<const uint32_t *>(ptr)[k] : 0u;
        } else {
#pragma unroll
            for (int k = 0; k < VEC; k += 2) {
                const unsigned short *h = reinterpret_cast<const unsigned short *>(ptr);
                w[k / 2] = (k < left ? (uint32_t)h[k] : 0u) | (k + 1 < left ? (uint32_t)h[k + 1] << 16 : 0u);
            }
        }
    }
    // from any place that is not on 16 bytes: out of the granules that hold them, all of which are read
    __device__ __forceinline__ void load_cut(const ST *ptr) {
        const uint32_t shift = (uint32_t)reinterpret_cast<uintptr_t>(ptr) & 15u;
        if constexpr (WORDS == 2) {
            const uint32_t *q = reinterpret_cast<const uint32_t *>(reinterpret_cast<const char *>(ptr) - (shift & 2u));
            const uint32_t w0 = q[0], w1 = q[1], w2 = (shift & 2u) ? q[2] : 0u, half = (shift & 2u) * 8u;
            w[0] = __funnelshift_r(w0, w1, half);
            w[1] = __funnelshift_r(w1, w2, half);
        } else {
            const uint4 *g = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(ptr) - shift);
            uint4 a = g[0];
#pragma unroll
            for (int k = 0; k < WORDS; k += 4) {
                const uint4 b = g[k / 4 + 1], q = cut_granules<(int)sizeof(ST)>(a, b, shift);
                w[k] = q.x; w[k + 1] = q.y; w[k + 2] = q.z; w[k + 3] = q.w;
                a = b;
            }
        }
    }
    __device__ __forceinline__ float get(int k) const {
        if constexpr (sizeof(ST) == 4) return __uint_as_float(w[k]);
        else return __uint_as_float((k & 1) ? (w[k / 2] & 0xffff0000u) : (w[k / 2] << 16));
    }
    __device__ __forceinline__ void set(int k, float v) {   // (v is a value of ST; elements are set in order)
        if constexpr (sizeof(ST) == 4) w[k] = __float_as_uint(v);
        else w[k / 2] = (k & 1) ? (w[k / 2] & 0xffffu) | __float_as_uint(v) : __float_as_uint(v) >> 16;
    }
};
__device__ __forceinline__ void store_vec(float *ptr, const float (&v)[4]) { __stcs(reinterpret_cast<float4 *>(ptr), make_float4(v[0], v[1], v[2], v[3])); }
__device__ __forceinline__ void store_vec(__nv_bfloat16 *ptr, const float (&v)[8]) {
    auto two = [](float lo, float hi) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    };
    __stcs(reinterpret_cast<uint4 *>(ptr), make_uint4(two(v[0], v[1]), two(v[2], v[3]), two(v[4], v[5]), two(v[6], v[7])));
}
__device__ __forceinline__ void store1(float *ptr, float v) { *ptr = v; }
__device__ __forceinline__ void store1(__nv_bfloat16 *ptr, float v) { *ptr = __float2bfloat16_rn(v); }

// Balanced tree over the squares of VEC (4 or 8) consecutive elements.  A square is exact in binary64, so
// the fused form rounds a pair's sum once, as the tree asks.
__device__ __forceinline__ double pair_sq(float a, float b) {
    const double x = (double)a, y = (double)b;
    return __fma_rn(y, y, __dmul_rn(x, x));
}
template <typename R>
__device__ __forceinline__ double leaf_sq4(const R &r, int k) { return __dadd_rn(pair_sq(r.get(k), r.get(k + 1)), pair_sq(r.get(k + 2), r.get(k + 3))); }
__device__ __forceinline__ double leaf_sq(const Raw<float, 4> &r) { return leaf_sq4(r, 0); }
__device__ __forceinline__ double leaf_sq(const Raw<__nv_bfloat16, 8> &r) { return __dadd_rn(leaf_sq4(r, 0), leaf_sq4(r, 4)); }

// Sums of squares of 1024 consecutive elements of a tile per warp (thread t of 256; the balanced tree over the
// warp's elements, in every lane): rows of 32 chunks of 16 bytes.
template <typename ST>
__device__ __forceinline__ double warp_sumsq(const ST *src, int len, int t) {
    constexpr int VEC = 16 / (int)sizeof(ST), ROWS = 32 / VEC;
    const int warp = t >> 5, lane = t & 31;
    Raw<ST, VEC> raw[ROWS];
    const int first = warp * 1024 + lane * VEC;
    const bool aligned = (reinterpret_cast<uintptr_t>(src) & 15u) == 0;
    if (aligned && len == TILE) {
#pragma unroll
        for (int j = 0; j < ROWS; ++j) raw[j].template load<false>(src + first + j * 32 * VEC);
    } else {
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            const int pos = first + j * 32 * VEC;
            if (aligned && pos + VEC <= len) raw[j].template load<false>(src + pos);
            else raw[j].load_guarded(src + pos, len - pos);
        }
    }
    double leaf[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) leaf[j] = leaf_sq(raw[j]);
    return warp_tree_reduce<ROWS>(leaf, lane);
}

// One tile of the output: round(c * source), or zeros where src is NULL.  Chunks of 16 bytes of the
// destination, wherever in them the tile starts; the few elements before and after one by one.
template <typename ST, typename DT>
__device__ __forceinline__ void scale_tile(const ST *src, DT *dst, int len, float c, int t /*of 256*/) {
    constexpr int VEC = 16 / (int)sizeof(DT), SRC_ALIGN = VEC * (int)sizeof(ST) < 16 ? VEC * (int)sizeof(ST) : 16;
    const int head = min(len, (int)(((16u - (unsigned)(reinterpret_cast<uintptr_t>(dst) & 15u)) & 15u) / sizeof(DT)));
    const int chunks = (len - head) / VEC;
    const int tail = head + chunks * VEC;
    if (t < head) store1(dst + t, src ? __fmul_rn(load1(src + t), c) : 0.0f);
    if (tail + t < len) store1(dst + tail + t, src ? __fmul_rn(load1(src + tail + t), c) : 0.0f);
    if (!src) {
        float v[VEC];
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[q] = 0.0f;
        for (int k = t; k < chunks; k += THREADS) store_vec(dst + head + k * VEC, v);
        return;
    }
    constexpr int DEEP = TILE / VEC / THREADS;   // chunks of a full tile per thread, all in flight
    const bool aligned = (reinterpret_cast<uintptr_t>(src + head) & (SRC_ALIGN - 1)) == 0;
    Raw<ST, VEC> raw[DEEP];
#pragma unroll
    for (int j = 0; j < DEEP; ++j) {
        const int k = t + j * THREADS;
        if (k < chunks) {
            if (aligned) raw[j].template load<true>(src + head + k * VEC);
            else raw[j].load_guarded(src + head + k * VEC, VEC);
        }
    }
#pragma unroll
    for (int j = 0; j < DEEP; ++j) {
        const int k = t + j * THREADS;
        if (k < chunks) {
            float v[VEC];
#pragma unroll
            for (int q = 0; q < VEC; ++q) v[q] = __fmul_rn(raw[j].get(q), c);
            store_vec(dst + head + k * VEC, v);
        }
    }
}

struct RowFactor {
    float factor;
    bool clear;   // the row is written as zeros
};

__device__ __forceinline__ RowFactor row_factor(const ClipArgs &a, double sumsq, float &norm32) {
    const double norm = sqrt(sumsq);
    norm32 = (float)norm;
    RowFactor f;
    f.factor = norm > (double)a.max_norm ? (float)((double)a.max_norm / norm) : 1.0f;
    f.clear = a.zero_nonfinite && !isfinite(norm);
    return f;
}

// Whether the table holds tensors of the kernel's source type.  If not (see TABLE_F32), no tensor is read: all count
// as missing, and the status word says so.
constexpr unsigned STATUS_TENSOR_TABLE = 64;
template <typename ST>
__device__ __forceinline__ bool table_fits(const Params &p, const ClipArgs &a) {
    const void *const *behind = a.table + (int64_t)p.N * p.T;
    return __ldg(reinterpret_cast<const unsigned long long *>(behind)) == (sizeof(ST) == 4 ? TABLE_F32 : TABLE_BF16);
}

// ---- rows of at most CLUSTER_TILES tiles: one cluster per row -------------------------------------
//
// 256 threads take a tile, up to four tiles a CTA, up to eight CTAs the cluster.  Every tile sum goes to all of
// the cluster through distributed shared memory; the cluster meets once; every warp forms the row's factor
// from the sums; the tiles are scaled (out of L1 or L2).  One launch, nothing to prepare: what such a row
// costs is latency: four rows of 8 tiles 4.9 us, of 32 tiles 8.8 us (binary32).
constexpr int CLUSTER_TILES = 32, CLUSTER_SIZE = 8;

template <typename ST, typename DT>
__global__ void __launch_bounds__(CLUSTER_TILES / CLUSTER_SIZE * THREADS) clip_cluster_kernel(const __grid_constant__ Params p, const __grid_constant__ ClipArgs a) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    __shared__ double warp_sums[CLUSTER_TILES / CLUSTER_SIZE][8];
    __shared__ double sums[CLUSTER_TILES];
    const int size = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int row = blockIdx.x / size, g = threadIdx.x / THREADS, t = threadIdx.x % THREADS, lane = t & 31;
    if (threadIdx.x < CLUSTER_TILES) sums[threadIdx.x] = 0.0;
    cluster.barrier_arrive();   // (no CTA writes into another's array before it is there and zeroed)
    const int tile = rank + g * size;
    const bool mine = tile < p.TT;
    const ST *src = nullptr;
    int64_t at = 0;
    int len = 0;
    if (mine) {
        at = __ldg(p.tile_at + tile);
        len = __ldg(p.tile_len + tile);
        if (a.table) {
            const int seg = __ldg(p.tile_seg + tile);
            const ST *tensor = reinterpret_cast<const ST *>(__ldg(reinterpret_cast<const unsigned long long *>(a.table) + (int64_t)row * p.T + seg));
            const int64_t tensor_at = __ldg(p.seg_off + seg);
            const bool fits = table_fits<ST>(p, a);
            if (tensor && fits) src = tensor + (at - tensor_at);
            if (!fits && tile == 0 && t == 0) atomicOr(p.status, STATUS_TENSOR_TABLE);
        } else {
            src = reinterpret_cast<const ST *>(a.rows) + (int64_t)row * p.d + at;
        }
        const double w = warp_sumsq<ST>(src, src ? len : 0, t);
        if (lane == 0) warp_sums[g][t >> 5] = w;
    }
    __syncthreads();
    cluster.barrier_wait();
    if (mine && t < size) {   // thread t: to CTA t
        const double *b = warp_sums[g];
        *cluster.map_shared_rank(&sums[tile], t) = __dadd_rn(__dadd_rn(__dadd_rn(b[0], b[1]), __dadd_rn(b[2], b[3])),
                                                             __dadd_rn(__dadd_rn(b[4], b[5]), __dadd_rn(b[6], b[7])));
    }
    cluster.sync();
    if (!mine) return;
    double s = sums[lane];
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) s = __dadd_rn(s, shfl_xor_f64(s, m));
    float norm;
    const RowFactor f = row_factor(a, s, norm);
    if (tile == 0 && t == 0 && a.norms) a.norms[row] = norm;
    if (a.in_place && f.factor == 1.0f && !f.clear) return;   // the row stays as it is
    scale_tile<ST, DT>(f.clear ? nullptr : src, reinterpret_cast<DT *>(a.out) + (int64_t)row * p.d + at, len, f.factor, t);
}

// ---- longer rows -----------------------------------------------------------------------------------
//
// One CTA per SM.  A producer warp takes tiles from two counters in global memory, fetches them by bulk copies
// into a ring of buffers and describes them to the consumer groups in op slots; six groups of 128 threads
// take the ops in turn.  First the sums of squares of all rows' tiles (OP_SUM), a row being joined (OP_JOIN)
// by the CTA that took its last tile; then the scaling (OP_SCALE), backwards, so that what was read last
// comes out of L2, but with the last row after the one before it, whose norm is known by then.  Tiles are
// dealt out by tickets because SMs read at different speeds (dealt evenly, the last one was a third late).
// Tile sums and row factors cross the GPU as single 64-bit words that hold UNSET before: whoever needs one
// reads until it is there, and no fence (which would wait for all of an SM's stores) is needed.  An op
// waits only for ops with earlier tickets, which never wait for it, so the CTAs need not all be resident.
constexpr int GROUPS = 6, GROUP = 128, OP_SLOTS = 32;   // (one slot per producer lane)
constexpr int STREAM_THREADS = GROUPS * GROUP + 32;
constexpr int PASS_TILES = 8 * GROUP * 4;   // tile sums that row_tree takes in one pass
constexpr int ROW_PASSES = 160;
static_assert((int64_t)ROW_PASSES * PASS_TILES >= (int64_t(1) << 32) / TILE + 65535, "passes for the most tiles: dim below 2^32, at most 65535 segments");
constexpr unsigned STATUS_NORM_TIMEOUT = 32;   // bit of the status word: a row's norm did not arrive within the wait limit
// (norm_wait_limit: polls of 40 ns and a load for sums and factors, of 200 ns by the producer for ops to be worked off)

template <typename ST>
struct StreamShape {
    static constexpr int STRIDE = TILE * (int)sizeof(ST) + 16;         // a tile lies at its address modulo 16
    static constexpr int RING = 200 * 1024 / STRIDE;                   // 6 or 12 tiles
    static constexpr int SMEM = RING * STRIDE;
    static constexpr int BATCH = sizeof(ST) == 4 ? 4 : 8;              // most tiles per ticket
};

enum { OP_SUM = 0, OP_JOIN = 1, OP_SCALE = 2, OP_END = 3 };
struct Op {
    const void *src;   // the tile's first element, or NULL
    int64_t at;        // the same within the rows
    int kind, row, tile, len, buffer;
    int open;          // whether the granules at the tile's ends may be read whole: 1 the first, 2 the last
};

// Before the kernel all counters, sums and factors are filled with bytes 0xC0: a negative number as a sum of
// squares, and no factor.
constexpr unsigned long long UNSET64 = 0xC0C0C0C0C0C0C0C0ull;
// a row's answer: its factor, and bit 32 where the row is written as zeros
__device__ __forceinline__ unsigned long long pack_factor(RowFactor f) { return __float_as_uint(f.factor) | (f.clear ? 1ull << 32 : 0ull); }
__device__ __forceinline__ RowFactor unpack_factor(unsigned long long w) { return RowFactor{__uint_as_float((uint32_t)w), (w >> 32) != 0}; }
__device__ __forceinline__ unsigned long long peek(const void *p) {
    unsigned long long v;
    asm volatile("ld.relaxed.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void post(void *p, unsigned long long v) { asm volatile("st.relaxed.gpu.global.u64 [%0], %1;" ::"l"(p), "l"(v) : "memory"); }

// As group_sync, and whether the flag is set in any of the group's threads.
__device__ __forceinline__ bool group_any(int g, bool flag) {
    int any;
    __syncwarp();   // (see group_sync)
    asm volatile("{ .reg .pred p, q; setp.ne.s32 p, %2, 0; bar.red.or.pred q, %1, %3, p; selp.s32 %0, 1, 0, q; }"
                 : "=r"(any) : "r"(g + 1), "r"((int)flag), "n"(GROUP) : "memory");
    return any != 0;
}
// The group's barrier.  A warp whose first lane comes out of a branch of its own has to be brought together
// first: it would stay split behind the barrier, and every shuffle of the sums would wait for both halves
// (measured: ten times slower).
__device__ __forceinline__ void group_sync(int g) {
    __syncwarp();
    asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "n"(GROUP) : "memory");
}

__device__ __forceinline__ void mbar_init(unsigned long long *bar) { asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(bar))); }
__device__ __forceinline__ void mbar_arrive(unsigned long long *bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory"); }

__device__ __forceinline__ bool mbar_test(unsigned long long *bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{ .reg .pred q; mbarrier.test_wait.parity.shared::cta.b64 q, [%1], %2; selp.u32 %0, 1, 0, q; }"
                 : "=r"(done) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return done != 0;
}

// A bulk copy into a buffer that ordinary stores never touch: what was read from it before is ordered by the
// barrier that the producer waited for.  (The proxy fence that bulk_copy_g2s begins with waits for all that
// the thread has under way, among it the next ticket.)
__device__ __forceinline__ void fetch_bulk(void *dst_smem, const void *src, uint32_t bytes, uint32_t expect, unsigned long long *bar) {
    const uint32_t b = smem_u32(bar);
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(b), "r"(expect) : "memory");
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst_smem)), "l"(src), "r"(bytes), "r"(b) : "memory");
}

// The part of a tile that a bulk copy can bring: elements [beg, end), out of 16-byte granules [lo, hi) counted in
// bytes from the one in which the tile starts.  A granule at an end is among them only where the array goes on
// beyond the tile (`open`); the neighbour's elements in it, which another group may just be writing, are not used.
template <typename ST>
struct Staged {
    int beg, end, shift, lo, hi;   // shift: the tile's first byte in its buffer
    __device__ __forceinline__ Staged(const ST *src, int len, int open) {
        shift = (int)(reinterpret_cast<uintptr_t>(src) & 15u);
        const int bytes = shift + len * (int)sizeof(ST);
        lo = (open & 1) ? 0 : (shift + 15) & ~15;
        hi = (open & 2) ? (bytes + 15) & ~15 : bytes & ~15;
        if (!src || hi <= lo) lo = hi = shift;   // nothing
        beg = max(lo - shift, 0) / (int)sizeof(ST);
        end = min((hi - shift) / (int)sizeof(ST), len);
    }
};

// VEC elements from `pos` on: out of the buffer where they were staged, else from the source; +0 beyond len.
template <typename ST, int VEC>
__device__ __forceinline__ void read_tile(Raw<ST, VEC> &raw, const ST *src, const ST *buf, const Staged<ST> &in, int pos, int len) {
    constexpr int ALIGN = VEC * (int)sizeof(ST) < 16 ? VEC * (int)sizeof(ST) : 16;
    if (pos >= in.beg && pos + VEC <= in.end) {
        if ((smem_u32(buf + pos) & (ALIGN - 1)) == 0) raw.template load<false>(buf + pos);
        else raw.load_cut(buf + pos);   // (what is staged begins and ends with whole granules)
        return;
    }
    for (int k = 0; k < VEC; ++k) {   // at the ends of the tile
        const int e = pos + k;
        const float v = e >= len || !src ? 0.0f : e >= in.beg && e < in.end ? load1(buf + e) : load1(src + e);
        raw.set(k, v);
    }
}

// Balanced tree over the sums of the group's four warps (result in every thread).
__device__ __forceinline__ double group_tree(double warp_sum, double *warp_sums, int g) {
    const int warp = (threadIdx.x / 32) % (GROUP / 32), lane = threadIdx.x & 31;
    if (lane == 0) warp_sums[warp] = warp_sum;
    group_sync(g);
    const double *b = warp_sums;
    return __dadd_rn(__dadd_rn(b[0], b[1]), __dadd_rn(b[2], b[3]));
}

// Balanced tree over a row's tile sums as they come in (a group; result in its thread 0).  A warp takes 1024
// consecutive sums as 16 rows of 64, two per lane; `missing` is set when they did not all come within `limit` polls
// (of the row, not of a pass), or the CTA stops.
__device__ __noinline__ double row_tree(const double *src, int tiles, double *warp_sums /*[4]*/, double *pass_sums /*[ROW_PASSES]*/,
                                           int g, const volatile int *stop, unsigned limit, bool &missing) {
    const int t = threadIdx.x % GROUP, warp = t / 32, lane = t & 31;
    const int passes = (tiles + PASS_TILES - 1) / PASS_TILES;
    missing = false;
    unsigned tries = 0;
    for (int q = 0; q < passes; ++q) {
        double part[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int first = q * PASS_TILES + warp * 1024 + half * 512 + lane * 2;
            unsigned long long v[8][2];
            for (;; ++tries) {   // all sixteen again until they are there
                bool unset = false;
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int k = 0; k < 2; ++k) v[j][k] = first + j * 64 + k < tiles ? peek(src + first + j * 64 + k) : 0ull;
#pragma unroll
                for (int j = 0; j < 8; ++j) unset |= v[j][0] == UNSET64 || v[j][1] == UNSET64;
                if (!__any_sync(0xffffffffu, unset)) break;
                if (__any_sync(0xffffffffu, tries >= limit || *stop)) { missing = true; break; }
                __nanosleep(40);
            }
            double leaf[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) leaf[j] = __dadd_rn(__longlong_as_double((long long)v[j][0]), __longlong_as_double((long long)v[j][1]));
            part[half] = warp_tree_reduce<8>(leaf, lane);
        }
        const double s = group_tree(__dadd_rn(part[0], part[1]), warp_sums, g);
        if (t == 0) pass_sums[q] = s;
        missing = group_any(g, missing);
        if (missing) break;
    }
    return t == 0 ? balanced_join(pass_sums, passes) : 0.0;
}

// The two ops on tiles that are not whole or not aligned.  (These and row_tree are functions of their own:
// inlined, the consumers' code no longer fits the instruction cache and every op waits for instructions.)
template <typename ST>
__device__ __noinline__ double sum_ragged(const ST *src, const ST *buf, int len, int open, int first /*this lane's place among 1024 elements*/) {
    constexpr int VEC = 16 / (int)sizeof(ST), ROWS = 32 / VEC;
    const Staged<ST> in(src, len, open);
    double leaf[ROWS];
    const int base = first - (int)(threadIdx.x & 31) * VEC;
    if (base >= in.beg && base + 1024 <= in.end && in.shift != 0) {   // all of the warp's elements, off the granules
        Raw<ST, VEC> raw[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j) raw[j].load_cut(buf + first + j * 32 * VEC);
#pragma unroll
        for (int j = 0; j < ROWS; ++j) leaf[j] = leaf_sq(raw[j]);
    } else {
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            Raw<ST, VEC> raw;
            read_tile<ST, VEC>(raw, src, buf, in, first + j * 32 * VEC, len);
            leaf[j] = leaf_sq(raw);
        }
    }
    return warp_tree_reduce<ROWS>(leaf, threadIdx.x & 31);
}

template <typename ST, typename DT>
__device__ __noinline__ void scale_ragged(const ST *src, const ST *buf, int len, int open, DT *dst, RowFactor rf) {
    constexpr int VEC = 16 / (int)sizeof(DT);
    const Staged<ST> in(src, len, open);
    const ST *from = rf.clear ? nullptr : src;
    const int t = threadIdx.x % GROUP;
    const int lead = min(len, (int)(((16u - (unsigned)(reinterpret_cast<uintptr_t>(dst) & 15u)) & 15u) / sizeof(DT)));
    const int chunks = (len - lead) / VEC, rest = lead + chunks * VEC;
    auto one = [&](int e) { store1(dst + e, from ? __fmul_rn(e >= in.beg && e < in.end ? load1(buf + e) : load1(src + e), rf.factor) : 0.0f); };
    if (t < lead) one(t);
    if (rest + t < len) one(rest + t);
#pragma unroll 2
    for (int k = t; k < chunks; k += GROUP) {
        Raw<ST, VEC> raw;
        read_tile<ST, VEC>(raw, from, buf, in, lead + k * VEC, len);
        float v[VEC];
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[q] = rf.clear ? 0.0f : __fmul_rn(raw.get(q), rf.factor);
        store_vec(dst + lead + k * VEC, v);
    }
}

template <typename ST, typename DT>
__global__ void __launch_bounds__(STREAM_THREADS, 1) clip_stream_kernel(const __grid_constant__ Params p, const __grid_constant__ ClipArgs a) {
    using Shape = StreamShape<ST>;
    extern __shared__ __align__(128) char ring[];
    __shared__ __align__(8) unsigned long long full[OP_SLOTS], done[OP_SLOTS];
    __shared__ Op ops[OP_SLOTS];
    __shared__ double warp_sums[GROUPS][GROUP / 32];
    __shared__ double pass_sums[GROUPS][ROW_PASSES];
    __shared__ RowFactor factors[GROUPS];
    __shared__ int no_norm[GROUPS];
    __shared__ uint32_t stream_op[64];   // producer: the op that took a place in the order of buffers
    __shared__ __align__(8) unsigned long long idle;   // never completes
    __shared__ volatile int stop;                       // a wait ran out: everyone leaves
    if (threadIdx.x == 0) {
        for (int s = 0; s < OP_SLOTS; ++s) { mbar_init(&full[s]); mbar_init(&done[s]); }
        mbar_init(&idle);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        stop = 0;
    }
    __syncthreads();
    const int warp_id = threadIdx.x >> 5;
    if (warp_id == GROUPS * (GROUP / 32)) {
        // ---- producer warp: a batch of ops at a time, one per lane ----
        // An op waits until its slot is free (the op 32 earlier is worked off) and its buffer is (buffers are used
        // in turn: the op that used it last is worked off).
        const int lane = threadIdx.x & 31;
        uint32_t next_op = 0, next_stream = 0;
        auto stopping = [&] { return (bool)__any_sync(0xffffffffu, stop); };   // (one answer for the warp)
        // what a lane has to know of its tile: loaded one batch ahead and not touched before it is used, so that
        // the warp, which executes in order, does not wait for the tables
        struct Look {
            const ST *tensor;         // gather: the tile's tensor ...
            long long at, tensor_at, tensor_end;  // (the tile's and) its first element within the row, and its end
            int row, tile, len;
        };
        auto look = [&](bool valid, int row, int tile) {
            Look l{nullptr, 0, 0, 0, row, tile, 0};
            if (valid) {
                l.at = __ldg(reinterpret_cast<const long long *>(p.tile_at) + tile);
                l.len = __ldg(p.tile_len + tile);
                if (a.table) {
                    const int seg = __ldg(p.tile_seg + tile);
                    l.tensor = reinterpret_cast<const ST *>(__ldg(reinterpret_cast<const unsigned long long *>(a.table) + (int64_t)row * p.T + seg));
                    l.tensor_at = __ldg(reinterpret_cast<const long long *>(p.seg_off) + seg);
                    l.tensor_end = __ldg(reinterpret_cast<const long long *>(p.seg_off) + seg + 1);
                }
            }
            return l;
        };
        const bool fits = !a.table || table_fits<ST>(p, a);
        if (!fits && lane == 0) atomicOr(p.status, STATUS_TENSOR_TABLE);
        auto source = [&](const Look &l) -> const ST * {
            if (a.table) return l.tensor && fits ? l.tensor + (l.at - l.tensor_at) : nullptr;
            return reinterpret_cast<const ST *>(a.rows) + (int64_t)l.row * p.d + l.at;
        };
        // (the rows as a whole begin on 16 bytes; a tile that does not begin its tensor has 8192 elements before it)
        auto open_ends = [&](const Look &l, const ST *src) {
            const int more = (int)(-(intptr_t)(src + l.len) & 15) / (int)sizeof(ST);   // elements after the tile in its last granule
            if (a.table) return (l.at > l.tensor_at ? 1 : 0) | (l.at + l.len + more <= l.tensor_end ? 2 : 0);
            return 1 | ((int64_t)l.row * p.d + l.at + l.len + more <= (int64_t)p.N * p.d ? 2 : 0);
        };
        auto issue = [&](int kind, int count, const Look &l) {
            bool pending = lane < count;
            const uint32_t first_op = next_op, op = first_op + lane, m = next_stream + lane;
            const int slot = op % OP_SLOTS;
            const bool streams = kind == OP_SUM || kind == OP_SCALE;
            const ST *src = source(l);
            const Op o{src, l.at, kind, l.row, l.tile, l.len, (int)(m % Shape::RING), open_ends(l, src)};
            uint32_t before = op;   // the op that the buffer waits for (op itself: none)
            if (pending && streams) stream_op[m % 64] = op;
            __syncwarp();
            if (pending && streams && m >= (uint32_t)Shape::RING) before = stream_op[(m - Shape::RING) % 64];
            // (ops more than a full turn of the slots before this batch are worked off: their slots were used again)
            bool wait_slot = op >= OP_SLOTS, wait_buffer = before != op && (int)(first_op - before) <= OP_SLOTS;
            unsigned polls = 0;
            while (__any_sync(0xffffffffu, pending)) {
                if (pending && wait_slot) wait_slot = !mbar_test(&done[slot], ((op - OP_SLOTS) / OP_SLOTS) & 1u);
                if (pending && wait_buffer) wait_buffer = !mbar_test(&done[before % OP_SLOTS], (before / OP_SLOTS) & 1u);
                if (pending && !wait_slot && !wait_buffer) {
                    pending = false;
                    ops[slot] = o;
                    const Staged<ST> in(src, o.len, o.open);
                    const uint32_t bytes = streams ? (uint32_t)(in.hi - in.lo) : 0u;   // (the other ops have no buffer)
                    if (bytes) {
                        char *dst = ring + (size_t)o.buffer * Shape::STRIDE + in.lo;
                        fetch_bulk(dst, reinterpret_cast<const char *>(src) - in.shift + in.lo, bytes, bytes + p.copy_expect_extra, &full[slot]);
                    } else {
                        mbar_arrive(&full[slot]);
                    }
                }
                if (++polls > p.norm_wait_limit) { atomicOr(p.status, STATUS_NORM_TIMEOUT); stop = 1; }
                if (stopping()) return;
                // (polling without a pause made the consumers' shuffles ten times slower: both use the shared memory pipe)
                if (__any_sync(0xffffffffu, pending)) __nanosleep(200);
            }
            next_op += count;
            if (streams) next_stream += count;
        };
        // the next ticket of a counter, in lane 0: the first of BATCH tiles (asked for one batch ahead, too)
        const long long K = (long long)p.N * p.TT;
        auto take = [&](unsigned long long *counter) {
            unsigned long long t = 0;
            // (written out: the compiler gathers a warp's atomicAdd into one and waits for its result at once)
            if (lane == 0) asm volatile("atom.relaxed.gpu.global.add.u64 %0, [%1], %2;" : "=l"(t) : "l"(counter), "l"((unsigned long long)a.batch) : "memory");
            return t;
        };
        auto all = [&](unsigned long long t) { return min((long long)(__shfl_sync(0xffffffffu, t, 0) - UNSET64), K); };
        auto row_of = [&](long long k) { return K <= 0xffffffffll ? (int)((unsigned)k / (unsigned)p.TT) : (int)(k / p.TT); };
        auto size = [&](long long k) { return (int)min((long long)a.batch, K - k); };
        const Look none = look(false, 0, 0);
        {
            auto place = [&](long long k) {
                const int row = row_of(k + lane);
                return look(lane < size(k), row, (int)(k + lane - (long long)row * p.TT));
            };
            long long k = all(take(a.sum_ticket));
            unsigned long long ticket = take(a.sum_ticket);
            Look now = place(k);
            while (k < K && !stopping()) {
                const long long k1 = all(ticket);
                const Look next = place(k1);
                ticket = take(a.sum_ticket);
                issue(OP_SUM, size(k), now);
                unsigned ends = __ballot_sync(0xffffffffu, lane < size(k) && now.tile == p.TT - 1);
                for (; ends && !stopping(); ends &= ends - 1) {
                    Look j = none;
                    j.row = __shfl_sync(0xffffffffu, now.row, __ffs(ends) - 1);
                    issue(OP_JOIN, 1, j);
                }
                k = k1;
                now = next;
            }
        }
        if (!a.norms_only) {
            auto place = [&](long long k) {
                const int r = row_of(k + lane);
                int row = p.N - 1 - r;
                if (p.N > 1 && row >= p.N - 2) row = 2 * p.N - 3 - row;   // (the last two rows change places)
                return look(lane < size(k), row, p.TT - 1 - (int)(k + lane - (long long)r * p.TT));
            };
            long long k = all(take(a.scale_ticket));
            unsigned long long ticket = take(a.scale_ticket);
            Look now = place(k);
            int known = -1;        // in place: the row that `still` is about
            bool still = false;    // it stays as it is
            while (k < K && !stopping()) {
                const long long k1 = all(ticket);
                const Look next = place(k1);
                ticket = take(a.scale_ticket);
                bool skip = false;
                if (a.in_place) {   // (rows that stay as they are are not read again)
                    const int first = __shfl_sync(0xffffffffu, now.row, 0), last = __shfl_sync(0xffffffffu, now.row, size(k) - 1);
                    if (first == last) {
                        if (first != known) {
                            const unsigned long long w = __shfl_sync(0xffffffffu, lane == 0 ? peek(a.answer + first) : 0ull, 0);
                            still = w != UNSET64 && unpack_factor(w).factor == 1.0f && !unpack_factor(w).clear;
                            known = w != UNSET64 ? first : -1;
                        }
                        skip = still;
                    }
                }
                if (!skip) issue(OP_SCALE, size(k), now);
                k = k1;
                now = next;
            }
        }
        if (!stopping()) issue(OP_END, GROUPS, none);
    } else {
        // ---- consumers ----
        const int g = threadIdx.x / GROUP, t = threadIdx.x % GROUP, warp = t / 32, lane = threadIdx.x & 31;
        RowFactor rf{1.0f, false};
        int rf_row = -1;   // the row that rf belongs to
        for (uint32_t op = g;; op += GROUPS) {
            const int slot = op % OP_SLOTS;
            if (t == 0) {   // (one thread polls, the others sleep at the barrier: spinning warps starve the producer)
                unsigned polls = 0;
                while (!stop && !mbar_test(&full[slot], (op / OP_SLOTS) & 1u)) {
                    if (++polls > p.copy_wait_limit) { atomicOr(p.status, STATUS_COPY_TIMEOUT); stop = 1; }
                    __nanosleep(100);
                }
            }
            if (group_any(g, stop)) break;   // (one answer for the whole group)
            const Op o = ops[slot];
            if (o.kind == OP_END) break;
            const ST *src = reinterpret_cast<const ST *>(o.src);
            const Staged<ST> in(src, o.len, o.open);
            const ST *buf = reinterpret_cast<const ST *>(ring + (size_t)o.buffer * Shape::STRIDE + in.shift);
            if (o.kind == OP_SUM) {
                constexpr int VEC = 16 / (int)sizeof(ST), ROWS = 32 / VEC, PER_WARP = TILE / (GROUP / 32);
                const bool plain = o.len == TILE && in.end == TILE && in.shift == 0;   // (then beg = 0 as well)
                static_assert(PER_WARP == 2048, "two subtrees of 1024 elements per warp");
                double sum = 0.0;
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    const int first = warp * PER_WARP + half * 1024 + lane * VEC;
                    double part;
                    if (plain) {
                        Raw<ST, VEC> raw[ROWS];
#pragma unroll
                        for (int j = 0; j < ROWS; ++j) raw[j].template load<false>(buf + first + j * 32 * VEC);
                        double leaf[ROWS];
#pragma unroll
                        for (int j = 0; j < ROWS; ++j) leaf[j] = leaf_sq(raw[j]);
                        part = warp_tree_reduce<ROWS>(leaf, lane);
                    } else {
                        part = sum_ragged(src, buf, o.len, o.open, first);
                    }
                    sum = half == 0 ? part : __dadd_rn(sum, part);
                }
                const double s = group_tree(sum, warp_sums[g], g);
                if (t == 0) {
                    mbar_arrive(&done[slot]);
                    if (!(p.norm_withhold & WITHHOLD_SUM) || o.tile != 0)
                        post(a.partials + (int64_t)o.row * p.TT + o.tile, (unsigned long long)__double_as_longlong(s));
                }
            } else if (o.kind == OP_JOIN) {
                bool missing;
                const double sum = row_tree(a.partials + (int64_t)o.row * p.TT, p.TT, warp_sums[g], pass_sums[g], g, &stop, p.norm_wait_limit, missing);
                if (t == 0) {
                    mbar_arrive(&done[slot]);
                    if (missing) {
                        if (!stop) atomicOr(p.status, STATUS_NORM_TIMEOUT);
                        stop = 1;
                    } else {
                        float norm;
                        const unsigned long long factor = pack_factor(row_factor(a, sum, norm));
                        if (!(p.norm_withhold & WITHHOLD_FACTOR)) post(a.answer + o.row, factor);
                        if (a.norms) a.norms[o.row] = norm;
                    }
                }
            } else {
                if (rf_row != o.row) {   // the group's first op of this row
                    if (t == 0) {
                        unsigned tries = 0;
                        unsigned long long word = peek(a.answer + o.row);
                        while (!stop && word == UNSET64) {
                            __nanosleep(40);
                            // (a CTA that gave up ends the others' waits as well)
                            if (++tries > p.norm_wait_limit || ((tries & 63u) == 0 && peek(a.gave_up) != UNSET64)) {
                                atomicOr(p.status, STATUS_NORM_TIMEOUT);
                                stop = 1;
                            }
                            word = peek(a.answer + o.row);
                        }
                        factors[g] = unpack_factor(word);
                        no_norm[g] = stop;
                    }
                    group_sync(g);
                    if (no_norm[g]) break;
                    rf = factors[g];
                    rf_row = o.row;
                }
                if (!(a.in_place && rf.factor == 1.0f && !rf.clear)) {
                    DT *dst = reinterpret_cast<DT *>(a.out) + (int64_t)o.row * p.d + o.at;
                    constexpr int VEC = 16 / (int)sizeof(DT), DEEP = TILE / VEC / GROUP, TURN = 4;
                    if (o.len == TILE && in.end == TILE && in.shift == 0 && (reinterpret_cast<uintptr_t>(dst) & 15u) == 0 && !rf.clear) {
#pragma unroll 1
                        for (int j0 = 0; j0 < DEEP; j0 += TURN) {
                            Raw<ST, VEC> raw[TURN];
#pragma unroll
                            for (int j = 0; j < TURN; ++j) raw[j].template load<false>(buf + (t + (j0 + j) * GROUP) * VEC);
#pragma unroll
                            for (int j = 0; j < TURN; ++j) {
                                float v[VEC];
#pragma unroll
                                for (int q = 0; q < VEC; ++q) v[q] = __fmul_rn(raw[j].get(q), rf.factor);
                                store_vec(dst + (t + (j0 + j) * GROUP) * VEC, v);
                            }
                        }
                    } else {
                        scale_ragged<ST, DT>(src, buf, o.len, o.open, dst, rf);
                    }
                }
                group_sync(g);
                if (t == 0) mbar_arrive(&done[slot]);
            }
        }
    }
    __syncthreads();
    if (stop && threadIdx.x == 0) {
        post(a.gave_up, 1ull);
        mbar_drain(&idle, 0u);   // a millisecond, so that copies still under way land before the shared memory goes
    }
}

// The pointer table travels as kernel arguments: the call is ordered on the stream, can be captured,
// and leaves no host buffer behind that a later call could overwrite too early.
template <int CAP>
struct PointerBlock { const void *ptr[CAP]; };

template <int CAP>
__global__ void upload_pointers_kernel(const __grid_constant__ PointerBlock<CAP> block, const void **table, int count, unsigned long long *word, unsigned long long tag) {
    for (int q = threadIdx.x; q < count; q += blockDim.x) table[q] = block.ptr[q];
    if (threadIdx.x == 0) *word = tag;
}

template <int CAP>
static cudaError_t upload_block(const void *const *tensors, const void **table, int count, unsigned long long *word, unsigned long long tag, cudaStream_t st) {
    PointerBlock<CAP> block;
    for (int q = 0; q < count; ++q) block.ptr[q] = tensors[q];
    upload_pointers_kernel<CAP><<<1, THREADS, 0, st>>>(block, table, count, word, tag);
    return cudaGetLastError();
}

// Arguments of up to 4 KB are the cheap kind; longer tables go in blocks of 31 KB, near the 32,764-byte limit.
cudaError_t launch_upload_pointers(const void *const *tensors, int dtype, const void **table, int64_t count, cudaStream_t st, int64_t *launches) {
    constexpr int SMALL = 480, LARGE = 3968;
    unsigned long long *word = reinterpret_cast<unsigned long long *>(table + count);
    for (int64_t at = 0; at < count;) {
        const int64_t left = count - at;
        const int here = (int)(left < LARGE ? left : LARGE);
        const unsigned long long tag = at + here < count ? 0ull : dtype == DT_F32 ? TABLE_F32 : TABLE_BF16;   // (a table that is only half written is none)
        const cudaError_t e = here <= SMALL ? upload_block<SMALL>(tensors + at, table + at, here, word, tag, st)
                                            : upload_block<LARGE>(tensors + at, table + at, here, word, tag, st);
        if (e != cudaSuccess) return e;
        ++*launches;
        at += here;
    }
    return cudaSuccess;
}

template <typename ST, typename DT>
static cudaError_t launch_clip_t(const Params &p, ClipArgs a, cudaStream_t st, int64_t *launches) {
    // One cluster per row while a tile has a CTA of its own (TT <= 8: 2000 rows of 8 tiles 202 us, 245 us by the
    // streaming kernel), or while all clusters run at once (32 rows of 16 tiles 8.6 against 16.6 us); CTAs of two to
    // four tiles that come in several waves lose (256 rows of 32 tiles 159 against 130 us; equal near 1024 tiles).
    if (p.TT <= CLUSTER_SIZE || (p.TT <= CLUSTER_TILES && (int64_t)p.N * p.TT <= 1024)) {
        int size = 1;
        while (size < CLUSTER_SIZE && size < p.TT) size <<= 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(p.N * size));
        cfg.blockDim = dim3((p.TT + size - 1) / size * THREADS);
        cfg.stream = st;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = size;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        const cudaError_t e = cudaLaunchKernelEx(&cfg, clip_cluster_kernel<ST, DT>, p, a);
        if (e != cudaSuccess) return e;
        ++*launches;
        return cudaGetLastError();
    }
    a.norms_only = a.in_place && std::isinf(a.max_norm) && !a.zero_nonfinite;
    // (a batch per ticket keeps the producer ahead of HBM; short work is dealt out finer: at least six tickets per CTA)
    a.batch = (int)std::max<int64_t>(1, std::min<int64_t>(StreamShape<ST>::BATCH, (int64_t)p.N * p.TT / (6 * (p.num_sms > 0 ? p.num_sms : 148))));
    const cudaError_t e = cudaMemsetAsync(a.partials, 0xC0, CLIP_STREAM_BYTES(p.N, p.TT), st);   // (all four arrays: UNSET)
    if (e != cudaSuccess) return e;
    clip_stream_kernel<ST, DT><<<p.num_sms > 0 ? p.num_sms : 148, STREAM_THREADS, StreamShape<ST>::SMEM, st>>>(p, a);
    ++*launches;
    return cudaGetLastError();
}

cudaError_t configure_clip_kernels() {
    cudaError_t e = cudaFuncSetAttribute(clip_stream_kernel<float, float>, cudaFuncAttributeMaxDynamicSharedMemorySize, StreamShape<float>::SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(clip_stream_kernel<float, __nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, StreamShape<float>::SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(clip_stream_kernel<__nv_bfloat16, float>, cudaFuncAttributeMaxDynamicSharedMemorySize, StreamShape<__nv_bfloat16>::SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(clip_stream_kernel<__nv_bfloat16, __nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, StreamShape<__nv_bfloat16>::SMEM);
    return e;
}

cudaError_t launch_clip(const Params &p, const ClipArgs &a, cudaStream_t st, int64_t *launches) {
    if (a.src_dtype == DT_F32)
        return p.gdt == DT_F32 ? launch_clip_t<float, float>(p, a, st, launches) : launch_clip_t<float, __nv_bfloat16>(p, a, st, launches);
    return p.gdt == DT_F32 ? launch_clip_t<__nv_bfloat16, float>(p, a, st, launches)
                           : launch_clip_t<__nv_bfloat16, __nv_bfloat16>(p, a, st, launches);
}

}  // namespace liec

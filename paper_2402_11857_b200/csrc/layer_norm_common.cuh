// Layer normalisation kernels: how a row is spread over threads, how rows reach them, packed binary32
// arithmetic.
//
// TPR threads share a row (a "slot" of a CTA).  A chunk is 16 bytes of elements (VEC = 4 of binary32, 8 of
// bfloat16); thread t of the slot owns the chunks v TPR + t, v < NV, of its row, whatever the row's
// alignment, so that the order of a row's sums depends on h and the element type alone, that of the column sums of the
// backward pass on the numbers of rows and workers as well, and no bit of a result on strides or alignment.  Rows
// pass through a ring in shared memory, STAGES rows deep per slot; what lies beyond column h there is
// zero.  The bytes in flight so cost no registers, which the backward pass needs for its column sums.
// WHOLE says how a row is fetched:
//   true   every row starts on 16 bytes and h is a multiple of VEC: a thread fetches its own chunks with
//          16-byte cp.async and is the only one to read them, so no barrier guards the ring
//   false  rows of any width and place: the ring holds the 16-byte granules of memory that the row touches, as
//          they lie (cp.async of whole granules, of a part at the end; the elements of a first granule that the
//          row does not fill one by one), and a thread cuts its chunk out of two of them; results go back through
//          the ring and leave as granules too.  A barrier of the slot per row.  (32 x 4095 rows of 767 bfloat16:
//          forward 109 us, backward 191 us; 114 and 846 us with 2-byte loads through registers.  768 columns,
//          which the first form takes: 71 and 105 us.)
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

#include "granule.cuh"
#include "layer_norm.h"

namespace liec {

__device__ __forceinline__ void ln_store(float *p, float v) { *p = v; }
__device__ __forceinline__ void ln_store(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// ---- two binary32 values in a register pair, one instruction for both (each rounded as the scalar one) ----
struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 f2(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ F2 f2(float x) { return f2(x, x); }
__device__ __forceinline__ float lo(F2 a) { return __uint_as_float((uint32_t)a.v); }
__device__ __forceinline__ float hi(F2 a) { return __uint_as_float((uint32_t)(a.v >> 32)); }
__device__ __forceinline__ F2 add(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 mul(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
// A product that is rounded before anything is added to it: a packed mul and the packed add behind it come out as
// one fused operation although both name their rounding (seen as a residue where q - q had to be zero).
__device__ __forceinline__ F2 rounded_mul(F2 a, F2 b) { return f2(__fmul_rn(lo(a), lo(b)), __fmul_rn(hi(a), hi(b))); }

// ---- a chunk as pairs ----
template <typename T> struct LnChunk;
template <> struct LnChunk<float> {
    static constexpr int VEC = 4;
    static __device__ __forceinline__ void read(uint4 q, F2 (&out)[2]) {
        out[0] = f2(__uint_as_float(q.x), __uint_as_float(q.y));
        out[1] = f2(__uint_as_float(q.z), __uint_as_float(q.w));
    }
    static __device__ __forceinline__ void write(void *p, const F2 (&in)[2]) {
        *reinterpret_cast<float4 *>(p) = make_float4(lo(in[0]), hi(in[0]), lo(in[1]), hi(in[1]));
    }
};
template <> struct LnChunk<__nv_bfloat16> {
    static constexpr int VEC = 8;
    static __device__ __forceinline__ F2 pair(uint32_t w) { return f2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
    static __device__ __forceinline__ uint32_t word(F2 a) {
        uint32_t w;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi(a)), "f"(lo(a)));
        return w;
    }
    static __device__ __forceinline__ void read(uint4 q, F2 (&out)[4]) {
        out[0] = pair(q.x); out[1] = pair(q.y); out[2] = pair(q.z); out[3] = pair(q.w);
    }
    static __device__ __forceinline__ void write(void *p, const F2 (&in)[4]) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(word(in[0]), word(in[1]), word(in[2]), word(in[3]));
    }
};

__device__ __forceinline__ void copy_async(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// the first `bytes` (0 to 16) of 16, zeros behind them; nothing beyond them is read
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }

// All threads of a slot.  Slots of less than a warp meet as a warp (their turns are the same).
template <int TPR>
__device__ __forceinline__ void slot_sync(int slot) {
    if constexpr (TPR <= 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(slot + 1), "n"(TPR) : "memory");
}

// Two sums (R = 1) or twice two (R = 2 rows at once) over a slot, in every thread.  The first steps hand
// different values to different lanes, so that all of them together cost one shuffle per further step;
// warps meet in `box` (two buffers in turn: whoever writes one has passed the barrier that follows
// everyone's reading of it).
template <int TPR, int WARPS, int R>
__device__ __forceinline__ void slot_sums(float (&a)[R], float (&b)[R], int t, int slot, float (*box)[WARPS][2 * R]) {
    constexpr int LANES = TPR < 32 ? TPR : 32, HALF = LANES / 2, QUARTER = LANES / 4;
    constexpr unsigned ALL = 0xffffffffu;
    const bool upper = (t & HALF) != 0, odd = (t & QUARTER) != 0;
    float v;
    if constexpr (R == 1) {
        v = (upper ? b[0] : a[0]) + __shfl_xor_sync(ALL, upper ? a[0] : b[0], HALF);
        v += __shfl_xor_sync(ALL, v, QUARTER);
    } else {
        const float p = (upper ? a[1] : a[0]) + __shfl_xor_sync(ALL, upper ? a[0] : a[1], HALF);
        const float q = (upper ? b[1] : b[0]) + __shfl_xor_sync(ALL, upper ? b[0] : b[1], HALF);
        v = (odd ? q : p) + __shfl_xor_sync(ALL, odd ? p : q, QUARTER);
    }
#pragma unroll
    for (int m = QUARTER / 2; m >= 1; m >>= 1) v += __shfl_xor_sync(ALL, v, m);
    if constexpr (WARPS == 1) {
        if constexpr (R == 1) {
            const float other = __shfl_xor_sync(ALL, v, HALF);
            a[0] = upper ? other : v;
            b[0] = upper ? v : other;
        } else {
            const float other = __shfl_xor_sync(ALL, v, QUARTER);
            const float p = odd ? other : v, q = odd ? v : other;
            const float p2 = __shfl_xor_sync(ALL, p, HALF), q2 = __shfl_xor_sync(ALL, q, HALF);
            a[0] = upper ? p2 : p;
            a[1] = upper ? p : p2;
            b[0] = upper ? q2 : q;
            b[1] = upper ? q : q2;
        }
    } else {
        // order in the box: R = 1: a, b; R = 2: a0, b0, a1, b1
        if (R == 1 ? (t & 15) == 0 : (t & 7) == 0) box[slot][t >> 5][R == 1 ? (t & 31) >> 4 : (t & 31) >> 3] = v;
        slot_sync<TPR>(slot);
#pragma unroll
        for (int r = 0; r < R; ++r) a[r] = b[r] = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; w += 2 / R) {
            const float4 q = *reinterpret_cast<const float4 *>(box[slot][w]);
            a[0] += q.x;
            b[0] += q.y;
            a[R - 1] += q.z;
            b[R - 1] += q.w;
        }
    }
}

// ---- rows wider than a CTA: a cluster holds one, each CTA a range of its columns ----
__device__ __forceinline__ int cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return (int)r; }
__device__ __forceinline__ int cluster_size() { uint32_t r; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return (int)r; }
__device__ __forceinline__ void cluster_sync() {   // every thread of every CTA, warps whole
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The CTAs' sums (equal in all threads of a CTA) meet: each hands its own to every other, and all add them up in
// the same order.  `meet` as the box of slot_sums: two in turn.
template <int R>
__device__ __forceinline__ void cluster_sums(float (&a)[R], float (&b)[R], int rank, int size, float2 (*meet)[8]) {
    if ((int)threadIdx.x < size) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            uint32_t to;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(&meet[j][rank])), "r"(threadIdx.x));
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(a[j]), "f"(b[j]) : "memory");
        }
    }
    __syncwarp();
    cluster_sync();
#pragma unroll
    for (int j = 0; j < R; ++j) {
        a[j] = b[j] = 0.0f;
        for (int q = 0; q < size; ++q) {
            const float2 v = meet[j][q];
            a[j] += v.x;
            b[j] += v.y;
        }
    }
}

template <typename T, bool WHOLE, int NV, int TPR, int SLOTS, int MINB, int R, int ARRAYS>
struct LnShape {
    static constexpr int VEC = LnChunk<T>::VEC, E = VEC * NV, THREADS = TPR * SLOTS, COLS = TPR * E;
    // (a row that starts inside a granule touches one more; a result lies 16 bytes into its place, see ln_store_row)
    static constexpr int ROW_BYTES = COLS * (int)sizeof(T) + (WHOLE ? 0 : 32);
    static constexpr int STAGE_BYTES = ARRAYS * SLOTS * R * ROW_BYTES;   // a stage holds the R rows of a turn, for every slot
    // About 40 KB per SM have to be in flight to cover HBM's latency at its bandwidth: 2 to 6 stages
    // give that for every shape within the 200 KB that the MINB CTAs of an SM share.
    // The backward pass either keeps what the rows gave in registers while their sums meet, or reads the rows once
    // more: bfloat16 would have to be widened twice (4 x 4096 rows of 4096: 80 us kept, 89 us read again; binary32,
    // 4 x 8192 rows of 2048: 141 and 139 us, 16 x 8192 of 511: 156 and 145 us).  Results then need a place of their own.
    static constexpr bool KEEP = ARRAYS == 1 || sizeof(T) == 2;
    static constexpr int RESULT_BYTES = WHOLE || KEEP ? 0 : SLOTS * R * ROW_BYTES;
    static constexpr int FIT = (200 * 1024 / MINB - RESULT_BYTES) / STAGE_BYTES;
    static constexpr int STAGES = FIT < 2 ? 2 : FIT > 6 ? 6 : FIT;
    static constexpr int RING_BYTES = STAGES * STAGE_BYTES;
    static constexpr int WARPS = TPR < 32 ? 1 : TPR / 32;      // warps per slot
};

// An element of a row's first granule on its way to the ring (to = 0: none).
struct LnHead { uint32_t to, value; };

// The rows of one array on their way to one place in the stages.
template <typename T, typename S, bool WHOLE, int NV, int TPR>
struct LnPipe {
    char *ring;             // this slot's row of stage 0
    uint32_t ring_u32;
    uint32_t now;           // !WHOLE: low bits of the address of this turn's row
    __device__ __forceinline__ void place(char *smem, int row_of_stage) {
        ring = smem + row_of_stage * S::ROW_BYTES;
        ring_u32 = (uint32_t)__cvta_generic_to_shared(ring);
    }
    // start fetching a row into a stage; head: what land() still has to put there
    __device__ __forceinline__ void fetch(const T *row, int t, int cols, int stage, LnHead &head) {
        const uint32_t to = ring_u32 + stage * S::STAGE_BYTES;
        const int bytes = cols * (int)sizeof(T);
        if constexpr (WHOLE) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int at = (v * TPR + t) * 16;
                if (at < bytes) copy_async(to + at, reinterpret_cast<const char *>(row) + at);
            }
        } else {
            const int shift = (int)(reinterpret_cast<uintptr_t>(row) & 15u), end = shift + bytes;
            const char *from = reinterpret_cast<const char *>(row) - shift;
            if (shift == 0 || t > 0) {
                if (t * 16 + 16 <= end) copy_async(to + t * 16, from + t * 16);
            }
#pragma unroll
            for (int v = 1; v <= NV; ++v) {
                const int at = (v * TPR + t) * 16;
                if (at + 16 <= end) copy_async(to + at, from + at);
            }
            // the last granule's first bytes, and zeros behind them and in the granule that a chunk may reach into
            const int tail = (end & ~15) + t * 16;
            if (t < 2 && tail <= bytes + 14) {
                if (tail > 0 || shift == 0) copy_async(to + tail, tail < end ? from + tail : from, max(end - tail, 0) & 15);
            }
            const int at = t * (int)sizeof(T);
            head.to = 0u;
            if (shift != 0 && at >= shift && at < 16) {   // (zeros behind a row that ends in its first granule)
                head.to = to + at;
                head.value = 0u;
                if (at < end) {
                    if constexpr (sizeof(T) == 4) head.value = __ldg(reinterpret_cast<const unsigned *>(from + at));
                    else head.value = __ldg(reinterpret_cast<const unsigned short *>(from + at));
                }
            }
        }
    }
    static __device__ __forceinline__ void land(const LnHead &head) {
        if constexpr (!WHOLE) {
            if (head.to != 0u) {
                if constexpr (sizeof(T) == 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(head.to), "r"(head.value) : "memory");
                else asm volatile("st.shared.b16 [%0], %1;" ::"r"(head.to), "h"((unsigned short)head.value) : "memory");
            }
        }
    }
    __device__ __forceinline__ void read(int v, int t, int stage, F2 (&out)[S::VEC / 2]) const {
        const uint4 *g = reinterpret_cast<const uint4 *>(ring + stage * S::STAGE_BYTES + (v * TPR + t) * 16);
        if constexpr (WHOLE) LnChunk<T>::read(g[0], out);
        else LnChunk<T>::read(cut_granules<(int)sizeof(T)>(g[0], g[1], now & 15u), out);
    }
    // where a result's chunk waits for ln_store_row
    __device__ __forceinline__ char *result(int v, int t, int stage) const { return ring + stage * S::STAGE_BYTES + 16 + (v * TPR + t) * 16; }
};

// Zeros behind the last granule that a fetch writes, in every place for a row.
template <typename S, bool WHOLE>
__device__ __forceinline__ void ln_clear_tails(char *ring, int bytes) {
    const int first = WHOLE ? bytes / 16 : (bytes + 14) / 16 + 1, left = S::ROW_BYTES / 16 - first;
    for (int q = threadIdx.x; q < S::RING_BYTES / S::ROW_BYTES * left; q += S::THREADS)
        *reinterpret_cast<uint4 *>(ring + q / left * S::ROW_BYTES + (first + q % left) * 16) = make_uint4(0u, 0u, 0u, 0u);
}

// A finished row leaves the ring's stage, where its first element lies at byte 16, in granules of memory; the
// elements of a first and a last granule that it does not fill go one by one.
template <typename T, int NV, int TPR>
__device__ __forceinline__ void ln_store_row(T *row, const char *stage, int t, int cols) {
    const int shift = (int)(reinterpret_cast<uintptr_t>(row) & 15u), end = shift + cols * (int)sizeof(T);
    char *to = reinterpret_cast<char *>(row) - shift;
    const char *from = stage + 16 - shift;
    const char *g = stage + (shift == 0 ? 16 : 0);
    const uint32_t turn = (uint32_t)(16 - shift) & 15u;
#pragma unroll
    for (int v = 0; v <= NV; ++v) {
        const int at = (v * TPR + t) * 16;
        if (at + 16 <= end && (v > 0 || at >= shift)) {
            const uint4 *q = reinterpret_cast<const uint4 *>(g + at);
            *reinterpret_cast<uint4 *>(to + at) = cut_granules<(int)sizeof(T)>(q[0], q[1], turn);
        }
    }
    if (t < LnChunk<T>::VEC) {
        const int first = t * (int)sizeof(T), last = (end & ~15) + first;
        if (shift != 0 && first >= shift && first < end) *reinterpret_cast<T *>(to + first) = *reinterpret_cast<const T *>(from + first);
        if ((last >= 16 || shift == 0) && last < end) *reinterpret_cast<T *>(to + last) = *reinterpret_cast<const T *>(from + last);
    }
}

// The first `left` elements of a chunk, zeros behind them.
template <int P>
__device__ __forceinline__ void ln_keep(F2 (&x)[P], int left) {
#pragma unroll
    for (int k = 0; k < P; ++k) x[k] = f2(2 * k < left ? lo(x[k]) : 0.0f, 2 * k + 1 < left ? hi(x[k]) : 0.0f);
}

// A chunk's weights or biases: from column c of the worker's vector, `fill` where there is none.
template <int P>
__device__ __forceinline__ void ln_parameters(const float *base, int64_t offset, int c, int h, float fill, F2 (&out)[P]) {
    const float *p = base + offset + c;
    if (base && c + 2 * P <= h && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
#pragma unroll
        for (int k = 0; k < P; k += 2) {
            const float4 q = __ldg(reinterpret_cast<const float4 *>(p) + k / 2);
            out[k] = f2(q.x, q.y);
            out[k + 1] = f2(q.z, q.w);
        }
    } else {
#pragma unroll
        for (int k = 0; k < P; ++k)
            out[k] = f2(base && c + 2 * k < h ? __ldg(p + 2 * k) : fill, base && c + 2 * k + 1 < h ? __ldg(p + 2 * k + 1) : fill);
    }
}

// ---- shapes ----------------------------------------------------------------------------------------

constexpr int LN_SMS = 148;            // a B200's; on another count the grid is only less even
constexpr int LN_CTA_COLS = 8192;      // widest row that the 512 threads of a CTA hold
constexpr int LN_SUM_ROWS = 1024;      // rows that one binary32 column accumulator may take

// Rows to CTAs, in whole turns of turn_rows.  SMs do not move data equally fast, so with `uneven` a resident
// set of CTAs takes 85 % of the rows in equal shares and the rest comes in small shares, two per resident
// CTA, that go to whichever place is free first; without, every resident CTA takes an equal share (for
// kernels whose shares have a price of their own).  No share is longer than max_turns.
inline LnShare ln_share(int64_t total, int turn_rows, int resident, int64_t max_turns, bool uneven) {
    auto whole = [&](int64_t rows) { return (rows + turn_rows - 1) / turn_rows * turn_rows; };
    LnShare s{0, 0, 0, 0};
    const int64_t even = (total + resident - 1) / resident;
    s.small_rows = std::min(whole(even), max_turns * turn_rows);
    if (uneven && even >= 8 * turn_rows && even <= max_turns * turn_rows) {
        s.large = resident;
        s.large_rows = even * 85 / 100 / turn_rows * turn_rows;
        s.small_rows = whole((total - s.large * s.large_rows + 2 * resident - 1) / (2 * resident));
    }
    s.ctas = s.large + (total - s.large * s.large_rows + s.small_rows - 1) / s.small_rows;
    return s;
}

// Places for CTAs of minb per SM, or for clusters: not every SM finds a place in a cluster (a cluster lies within
// one group of SMs), so these get shares of a quarter of the rows that one place would take.
inline int ln_resident(int minb, int parts) { return parts == 1 ? LN_SMS * minb : (parts == 2 ? 1 : 4) * LN_SMS / parts; }

// Threads per row, elements per thread, slots per CTA and CTAs per SM for h columns:
// f.template operator()<TPR, E, SLOTS, MINB>().  Up to 1024 columns a warp or less takes a row: its sums meet
// by shuffles alone, without a barrier between warps, and 24 or 32 elements per thread are still faster than two
// warps per row; beyond, 16 elements per thread, the most with which two rows (forward) or a row and its column
// sums (backward) fit the registers of two CTAs of 256 threads.
template <typename F>
auto ln_forward_shape(int h, F &&f) {
    if (h <= 64) return f.template operator()<8, 8, 32, 3>();
    if (h <= 128) return f.template operator()<16, 8, 16, 3>();
    if (h <= 256) return f.template operator()<32, 8, 8, 3>();
    if (h <= 512) return f.template operator()<32, 16, 8, 2>();
    if (h <= 768) return f.template operator()<32, 24, 4, 4>();
    if (h <= 1024) return f.template operator()<32, 32, 4, 3>();
    if (h <= 2048) return f.template operator()<128, 16, 2, 2>();
    if (h <= 4096) return f.template operator()<256, 16, 1, 2>();
    return f.template operator()<512, 16, 1, 1>();
}

template <typename F>
auto ln_backward_shape(int h, F &&f) {
    if (h <= 64) return f.template operator()<8, 8, 32, 3>();
    if (h <= 128) return f.template operator()<16, 8, 16, 3>();
    if (h <= 256) return f.template operator()<32, 8, 8, 3>();
    if (h <= 512) return f.template operator()<32, 16, 8, 2>();
    if (h <= 768) return f.template operator()<32, 24, 4, 3>();
    if (h <= 1024) return f.template operator()<32, 32, 4, 2>();
    if (h <= 2048) return f.template operator()<128, 16, 2, 2>();
    if (h <= 4096) return f.template operator()<256, 16, 1, 2>();
    return f.template operator()<512, 16, 1, 1>();
}

template <typename F>
auto ln_wide_shape(F &&f) { return f.template operator()<512, 16, 1, 1>(); }   // per CTA of a row's cluster

// CTAs per row, and columns of each (a multiple of 8, so that what starts on 16 bytes does so in every CTA).
inline int ln_parts(int h) { return (h + LN_CTA_COLS - 1) / LN_CTA_COLS; }
inline int ln_part_cols(int h) { return ((h + ln_parts(h) - 1) / ln_parts(h) + 7) / 8 * 8; }

template <typename A>
cudaError_t ln_launch(void (*kernel)(A), const A &a, int64_t ctas, int parts, int threads, int smem, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(ctas * parts));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)parts;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

// Dynamic shared memory beyond 48 KB (static included) needs the kernel's consent, once per device.
template <typename K>
cudaError_t ln_allow_smem(K kernel, int bytes, std::atomic<uint64_t> &done) {
    if (bytes <= 40 * 1024) return cudaSuccess;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0ull;
    if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
    else cudaGetLastError();   // (reported here; the next launch starts clean)
    return e;
}

// All rows of an array start and end on 16 bytes.
inline bool ln_whole(const void *p, int64_t row, int64_t group, int64_t rows, int groups, int cols, int esz) {
    uint64_t bits = reinterpret_cast<uintptr_t>(p) | (uint64_t)cols * esz;
    if (rows > 1) bits |= (uint64_t)row * esz;
    if (groups > 1) bits |= (uint64_t)group * esz;
    return (bits & 15u) == 0;
}

}  // namespace liec

// Layer normalisation kernels: how a row is spread over threads, how rows reach them, packed binary32
// arithmetic.
//
// TPR threads share a row (a "slot" of a CTA).  A chunk is 16 bytes of elements (VEC = 4 of binary32, 8 of
// bfloat16); thread t of the slot owns the chunks v TPR + t, v < NV, of its row, whatever the row's
// alignment, so that the order of every sum, hence every bit of the result, depends on h alone.  Rows
// pass through a ring in shared memory, STAGES rows deep per slot, where they lie in column order from a
// 16-byte boundary; what lies beyond column h in the ring is zero.  The bytes in flight so cost no
// registers, which the backward pass needs for its column sums.  PIECE says how a row is fetched:
//   16  every row starts on 16 bytes and h is a multiple of VEC: a thread fetches its own chunks with
//       cp.async and is the only one to read them, so no barrier guards the ring
//    4  rows start on 4 bytes: 4-byte cp.async, neighbouring threads fetch neighbouring words; a barrier
//       of the slot per row
//    2  bfloat16 rows of odd width or at odd places: 2-byte loads through registers
// Results of the PIECE < 16 forms go back through the ring as well, so that neighbouring threads store
// neighbouring words.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

#include "layer_norm.h"

namespace liec {

__device__ __forceinline__ float ln_load(const float *p) { return __ldg(p); }
__device__ __forceinline__ float ln_load(const __nv_bfloat16 *p) {
    return __uint_as_float((uint32_t)__ldg(reinterpret_cast<const unsigned short *>(p)) << 16);
}
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

// ---- a chunk as pairs ----
template <typename T> struct LnChunk;
template <> struct LnChunk<float> {
    static constexpr int VEC = 4;
    static __device__ __forceinline__ void read(const void *p, F2 (&out)[2]) {
        const float4 q = *reinterpret_cast<const float4 *>(p);
        out[0] = f2(q.x, q.y);
        out[1] = f2(q.z, q.w);
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
    static __device__ __forceinline__ void read(const void *p, F2 (&out)[4]) {
        const uint4 q = *reinterpret_cast<const uint4 *>(p);
        out[0] = pair(q.x); out[1] = pair(q.y); out[2] = pair(q.z); out[3] = pair(q.w);
    }
    static __device__ __forceinline__ void write(void *p, const F2 (&in)[4]) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(word(in[0]), word(in[1]), word(in[2]), word(in[3]));
    }
};

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
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

template <typename T, int PIECE, int NV, int TPR, int SLOTS, int MINB, int R, int ARRAYS>
struct LnShape {
    static constexpr int VEC = LnChunk<T>::VEC, E = VEC * NV, THREADS = TPR * SLOTS, COLS = TPR * E;
    static constexpr int ROW_BYTES = COLS * (int)sizeof(T);
    static constexpr int STAGE_BYTES = ARRAYS * SLOTS * R * ROW_BYTES;   // a stage holds the R rows of a turn, for every slot
    // About 40 KB per SM have to be in flight to cover HBM's latency at its bandwidth: 2 to 6 stages
    // give that for every shape within the 200 KB that the MINB CTAs of an SM share.
    static constexpr int FIT = 200 * 1024 / MINB / STAGE_BYTES;
    static constexpr int STAGES = PIECE == 2 ? 2 : FIT < 2 ? 2 : FIT > 6 ? 6 : FIT;
    static constexpr int RING_BYTES = STAGES * STAGE_BYTES;
    static constexpr int WARPS = TPR < 32 ? 1 : TPR / 32;      // warps per slot
    static constexpr int PIECES = PIECE == 16 ? NV : E * (int)sizeof(T) / PIECE;   // fetches per thread and row
};

// The rows of one array on their way to one place in the stages.
template <typename T, typename S, int PIECE, int NV, int TPR>
struct LnPipe {
    char *ring;                                            // this slot's row of stage 0
    uint32_t ring_u32;
    unsigned short ahead[PIECE == 2 ? S::PIECES : 1];      // PIECE 2: the row after the next, in registers
    __device__ __forceinline__ void place(char *smem, int row_of_stage) {
        ring = smem + row_of_stage * S::ROW_BYTES;
        ring_u32 = (uint32_t)__cvta_generic_to_shared(ring);
    }
    // start fetching a row into a stage
    __device__ __forceinline__ void fetch(const T *row, int t, int cols, int stage) {
        const uint32_t to = ring_u32 + stage * S::STAGE_BYTES;
        const char *from = reinterpret_cast<const char *>(row);
        const int bytes = cols * (int)sizeof(T);
        if constexpr (PIECE >= 4) {
#pragma unroll
            for (int j = 0; j < S::PIECES; ++j) {
                const int at = (j * TPR + t) * PIECE;
                if (at < bytes) copy_async<PIECE>(to + at, from + at);
            }
        } else {
#pragma unroll
            for (int j = 0; j < S::PIECES; ++j) {
                const int at = (j * TPR + t) * PIECE;
                if (at < bytes) ahead[j] = __ldg(reinterpret_cast<const unsigned short *>(from + at));
            }
        }
    }
    // PIECE 2: what fetch brought into the registers goes to a stage
    __device__ __forceinline__ void land(int t, int cols, int stage) {
#pragma unroll
        for (int j = 0; j < S::PIECES; ++j) {
            const int at = (j * TPR + t) * PIECE;
            if (at < cols * (int)sizeof(T)) *reinterpret_cast<unsigned short *>(ring + stage * S::STAGE_BYTES + at) = ahead[j];
        }
    }
    __device__ __forceinline__ char *chunk(int v, int t, int stage) const { return ring + stage * S::STAGE_BYTES + (v * TPR + t) * 16; }
};

// A finished row leaves the ring's stage in pieces that neighbouring threads store side by side.
template <typename T, typename S, int PIECE, int TPR>
__device__ __forceinline__ void ln_store_row(T *row, const char *stage, int t, int cols) {
    char *to = reinterpret_cast<char *>(row);
#pragma unroll
    for (int j = 0; j < S::PIECES; ++j) {
        const int at = (j * TPR + t) * PIECE;
        if (at < cols * (int)sizeof(T)) {
            if constexpr (PIECE == 4) *reinterpret_cast<uint32_t *>(to + at) = *reinterpret_cast<const uint32_t *>(stage + at);
            else *reinterpret_cast<unsigned short *>(to + at) = *reinterpret_cast<const unsigned short *>(stage + at);
        }
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
constexpr int LN_REGISTER_COLS = 8192; // widest row that 512 threads hold
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

// Threads per row, elements per thread, slots per CTA and CTAs per SM for h columns:
// f.template operator()<TPR, E, SLOTS, MINB>().
template <typename F>
auto ln_forward_shape(int h, F &&f) {
    if (h <= 64) return f.template operator()<8, 8, 32, 4>();
    if (h <= 128) return f.template operator()<16, 8, 16, 4>();
    if (h <= 256) return f.template operator()<32, 8, 8, 4>();
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

// The largest piece (16, 4 or 2 bytes) at which all rows of an array start and end.
inline int ln_piece(const void *p, int64_t row, int64_t group, int64_t rows, int groups, int cols, int esz) {
    uint64_t bits = reinterpret_cast<uintptr_t>(p) | (uint64_t)cols * esz;
    if (rows > 1) bits |= (uint64_t)row * esz;
    if (groups > 1) bits |= (uint64_t)group * esz;
    return (bits & 15u) == 0 ? 16 : (bits & 3u) == 0 ? 4 : 2;
}

// generic kernels for rows beyond LN_REGISTER_COLS
cudaError_t launch_layer_norm_forward_wide(const LnForward &a, int dtype, cudaStream_t st);
cudaError_t launch_layer_norm_backward_wide(LnBackward &a, int dtype, cudaStream_t st);
int64_t ln_wide_runs(int64_t rows);

}  // namespace liec

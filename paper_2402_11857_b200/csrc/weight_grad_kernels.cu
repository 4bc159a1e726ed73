// Weight gradient of a linear layer from the 8-bit checkpoint of its input: dW[o][c] = sum over tokens t of
// dy[t][o] x^[t][c], for N workers, on the tensor cores.
//
// x^ = q 2^e is a bfloat16 number, so the products are those of the definition; a binary32 dy is cut into three bfloat16
// parts whose sum it is, and multiplied three times.  A pair of CTAs takes a tile of 256 channels c (the rows of the
// accumulator, 128 in each CTA) by 512 outputs o (256 for binary32), and one run of tokens.  Operands lie in shared memory
// as in global memory, a token as a row of 128-byte pieces: one thread of each CTA has the tensor memory accelerator bring
// q and dy, sixteen warps widen q (four groups of four, a stage each in turn, so that one's latency hides behind the
// others), one thread of the pair issues the products.  Each CTA so widens 128 channels and reads half of the outputs: a
// tile of the same size in one CTA would need half again the shared memory traffic of a product.  Lanes of the accumulator
// are channels, so a warp writes 32 neighbours of a row of dW.
#include <cuda.h>

#include <algorithm>

#include "activation.cuh"
#include "tensor_core.cuh"

namespace liec {

constexpr int WG_TOKENS = 32;                  // of a stage
constexpr int WG_CHANNELS = 128;               // of a CTA
constexpr int WG_BLOCK_BYTES = WG_TOKENS * 128;
constexpr int WG_A_BYTES = 2 * WG_BLOCK_BYTES, WG_RAW_BYTES = WG_TOKENS * WG_CHANNELS;
constexpr int WG_GROUPS = 4, WG_GROUP = 128;   // groups of widening threads
constexpr int WG_WIDENERS = WG_GROUPS * WG_GROUP, WG_THREADS = WG_WIDENERS + 64;
constexpr int WG_SLAB = 256;                   // outputs of one product of the pair, 128 from each CTA
constexpr uint32_t WG_POLLS = 1u << 20;

// PARTS: bfloat16 parts of dy.  SLABS: products side by side.
template <int PARTS_>
struct WgShape {
    static constexpr int PARTS = PARTS_, SLABS = PARTS == 1 ? 2 : 1, OUTPUTS = SLABS * WG_SLAB, COLUMNS = OUTPUTS;
    static constexpr int B_BYTES = 2 * WG_BLOCK_BYTES;                       // of a slab's part
    static constexpr int STAGE_BYTES = WG_A_BYTES + SLABS * PARTS * B_BYTES + WG_RAW_BYTES;
    static constexpr int STAGES = PARTS == 1 ? 7 : 6;                        // what fits
    static constexpr int SMEM_BYTES = 1024 + STAGES * STAGE_BYTES;
};
inline int wg_parts(int dtype) { return dtype == 0 ? 3 : 1; }
inline int wg_outputs(int dtype) { return dtype == 0 ? WgShape<3>::OUTPUTS : WgShape<1>::OUTPUTS; }

struct WgPlan {
    int64_t tiles, run;          // per worker; tokens of a run (whole stages)
    int32_t c_tiles, o_tiles, runs;
};

// 16 bytes of q times their power, as 16 bfloat16 numbers.  Byte b with last seven bits l and sign bit s is l - 128 s:
// as bfloat16, 0x4300 | l is 128 + l and 0x4300 | (b & 0x80) is 128 + 128 s.
__device__ __forceinline__ void wg_widen(uint4 q, uint32_t byte, uint4 (&out)[2]) {
    const uint32_t words[4] = {q.x, q.y, q.z, q.w}, power2 = (byte << 7) * 0x10001u;
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t two = __byte_perm(words[i / 2], 0x43u, i % 2 ? 0x4342 : 0x4140);
        const uint32_t up = two & 0xff7fff7fu, down = two & 0xff80ff80u;
        uint32_t v;
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(v) : "r"(up), "r"(down));
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r[i]) : "r"(v), "r"(power2));
    }
    out[0] = make_uint4(r[0], r[1], r[2], r[3]);
    out[1] = make_uint4(r[4], r[5], r[6], r[7]);
}

// x = p[0] + p[1] + p[2], each the upper half of a binary32 number: 8 bits of the significand at a time.
__device__ __forceinline__ void wg_split(float x, uint32_t (&p)[3]) {
    const uint32_t bits = __float_as_uint(x);
    if ((bits & 0x7f800000u) == 0x7f800000u) {   // infinities and NaN as they are
        p[0] = (bits & 0x007fffffu) != 0u ? bits | 0x00400000u : bits;
        p[1] = p[2] = 0u;
        return;
    }
    p[0] = bits & 0xffff0000u;
    const float rest = x - __uint_as_float(p[0]);
    p[1] = __float_as_uint(rest) & 0xffff0000u;
    p[2] = __float_as_uint(rest - __uint_as_float(p[1]));
}

// dy as the tensor memory accelerator wants it: bfloat16 rows of a multiple of 8 columns without gaps, part after part.  A
// thread takes 8 columns of a row.
template <typename T>
__global__ void __launch_bounds__(256) wg_pack_kernel(const __grid_constant__ WgArgs a, int64_t row_chunks) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    const int64_t rows = a.workers * a.rows, i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / row_chunks;
    if (row >= rows) return;
    const int64_t w = row / a.rows;
    const int c = (int)(i - row * row_chunks) * 8;
    const T *from = static_cast<const T *>(a.dy) + w * a.dy_worker + (row - w * a.rows) * a.dy_row;
    uint4 *to = reinterpret_cast<uint4 *>(a.packed) + i;
    if constexpr (PARTS == 1) {
        *to = load_chunk(from, c, a.out);
    } else {
        const uint4 lo4 = load_chunk(from, c, a.out), hi4 = c + 4 < a.out ? load_chunk(from, c + 4, a.out) : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t x[8] = {lo4.x, lo4.y, lo4.z, lo4.w, hi4.x, hi4.y, hi4.z, hi4.w};
        uint32_t p[8][3];
#pragma unroll
        for (int e = 0; e < 8; ++e) wg_split(__uint_as_float(x[e]), p[e]);
#pragma unroll
        for (int k = 0; k < 3; ++k)
            to[k * rows * row_chunks] = make_uint4(__byte_perm(p[0][k], p[1][k], 0x7632), __byte_perm(p[2][k], p[3][k], 0x7632),
                                                   __byte_perm(p[4][k], p[5][k], 0x7632), __byte_perm(p[6][k], p[7][k], 0x7632));
    }
}

__device__ __forceinline__ void wg_store(float *p, float v) { *p = v; }
__device__ __forceinline__ void wg_store(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// 32 outputs of a channel, `step` elements apart.
template <typename T>
__device__ __forceinline__ void wg_store_column(T *to, int64_t step, int outputs, const float (&v)[32]) {
    if (outputs >= 32) {
#pragma unroll
        for (int e = 0; e < 32; ++e) wg_store(to + e * step, v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 32; ++e)
            if (e < outputs) wg_store(to + e * step, v[e]);
    }
}

template <int PARTS>
__global__ void __launch_bounds__(WG_THREADS, 1) wg_kernel(const __grid_constant__ WgArgs a, const __grid_constant__ WgPlan p,
                                                            const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap dy_map) {
    using S = WgShape<PARTS>;
    extern __shared__ char wg_smem[];
    __shared__ __align__(8) unsigned long long bars[3 * S::STAGES + 1];
    __shared__ uint32_t tmem_at;
    __shared__ int failed;
    const uint32_t bar = (uint32_t)__cvta_generic_to_shared(bars);
    const uint32_t base = ((uint32_t)__cvta_generic_to_shared(wg_smem) + 1023u) & ~1023u;
    auto loaded = [&](int s) { return bar + 8u * s; };                       // the copies of a stage, in this CTA
    auto full = [&](int s) { return bar + 8u * (S::STAGES + s); };           // both CTAs' operands (in the first CTA)
    auto empty = [&](int s) { return bar + 8u * (2 * S::STAGES + s); };      // the stage's products are done
    const uint32_t done = bar + 8u * 3 * S::STAGES;
    auto a_at = [&](int s) { return base + s * S::STAGE_BYTES; };
    auto b_at = [&](int s) { return a_at(s) + WG_A_BYTES; };
    auto raw_at = [&](int s) { return b_at(s) + S::SLABS * PARTS * S::B_BYTES; };
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = cluster_rank();

    int64_t b = blockIdx.x / 2;
    const int run = (int)(b % p.runs);
    b /= p.runs;
    const int worker = (int)(b / p.tiles), tile = (int)(b % p.tiles);
    const int o0 = tile / p.c_tiles * S::OUTPUTS, c0 = tile % p.c_tiles * 2 * WG_CHANNELS + rank * WG_CHANNELS;
    const int slabs = min(S::SLABS, (a.out - o0 + WG_SLAB - 1) / WG_SLAB);
    const int64_t first = run * p.run, tokens = min(p.run, a.rows - first);
    const int turns = (int)((tokens + WG_TOKENS - 1) / WG_TOKENS);

    if (warp == WG_WIDENERS / 32 + 1) {
        if (lane == 0) {
            for (int s = 0; s < S::STAGES; ++s) {
                barrier_init(loaded(s), 1);
                barrier_init(full(s), 2 * WG_GROUP / 32);
                barrier_init(empty(s), 1);
            }
            barrier_init(done, 1);
            failed = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            async_fence();
        }
        __syncwarp();
        tc_alloc_pair((uint32_t)__cvta_generic_to_shared(&tmem_at), S::COLUMNS);
    }
    tc_before_sync();
    __syncthreads();
    cluster_sync();
    tc_after_sync();
    const uint32_t tmem = tmem_at;

    if (warp == WG_WIDENERS / 32) {
        if (lane == 0) {   // copies
            asm volatile("griddepcontrol.wait;" ::: "memory");   // dy may come from the kernel before
            int i = 0;
            bool ok = true;
            for (; i < turns; ++i) {
                const int s = i % S::STAGES, t = (int)first + i * WG_TOKENS;
                if (i >= S::STAGES) ok = barrier_wait(empty(s), (i / S::STAGES - 1) & 1, WG_POLLS);
                if (!ok) break;
                barrier_expect(loaded(s), WG_RAW_BYTES + slabs * PARTS * S::B_BYTES);
                copy_box(raw_at(s), &q_map, c0, t, worker, loaded(s));
                for (int n = 0; n < slabs; ++n)
#pragma unroll
                    for (int part = 0; part < PARTS; ++part)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            copy_box(b_at(s) + (n * PARTS + part) * S::B_BYTES + h * WG_BLOCK_BYTES, &dy_map, o0 + n * WG_SLAB + rank * 128 + h * 64, t,
                                     part * a.workers + worker, loaded(s));
            }
            if (!ok) {   // nothing may be on its way into this CTA's memory when it ends
                failed = 1;
                for (int k = max(0, i - S::STAGES); k < i; ++k) barrier_wait(loaded(k % S::STAGES), (k / S::STAGES) & 1, WG_POLLS);
            }
        }
        __syncwarp();
    } else if (warp == WG_WIDENERS / 32 + 1) {
        if (lane == 0 && rank == 0) {   // products
            bool ok = true;
            for (int i = 0; i < turns; ++i) {
                const int s = i % S::STAGES;
                ok = barrier_wait(full(s), (i / S::STAGES) & 1, WG_POLLS);
                if (!ok) break;
                tc_after_sync();
#pragma unroll
                for (int k = 0; k < WG_TOKENS / 16; ++k) {
                    const uint64_t x = tc_descriptor(a_at(s) + k * 2048, WG_BLOCK_BYTES);
                    for (int n = 0; n < slabs; ++n)
#pragma unroll
                        for (int part = 0; part < PARTS; ++part)
                            tc_mma_pair(tmem + n * WG_SLAB, x, tc_descriptor(b_at(s) + (n * PARTS + part) * S::B_BYTES + k * 2048, WG_BLOCK_BYTES),
                                        tc_instruction(256, WG_SLAB), i > 0 || k > 0 || part > 0);
                }
                tc_commit_pair(empty(s));
            }
            if (!ok) {
                const uint32_t flag = (uint32_t)__cvta_generic_to_shared(&failed);
                for (int r = 0; r < 2; ++r) asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(in_cta(flag, r)), "r"(1) : "memory");
                asm volatile("fence.acq_rel.cluster;" ::: "memory");
            }
            tc_commit_pair(done);
        }
        __syncwarp();
    } else {
        // A thread's part of a stage: two chunks of q, 16 channels of one token each.  Eight threads that load or store
        // together meet all places of a 128-byte row, plain in one case and swizzled in the other.
        const int group = warp / 4, parity = lane >> 2 & 1, q_block = parity ^ (lane >> 3 & 1), q_piece = lane & 3;
        const int token = warp % 4 * 4 + (lane >> 4) * 2 + parity;           // and the one 16 further on
        const int64_t row_powers = (a.in + CK_BLOCK - 1) / CK_BLOCK;
        const int c = c0 + q_block * 64 + q_piece * 16, left = c < row_powers * CK_BLOCK ? (int)tokens : 0;
        const uint8_t *powers = a.scales + (worker * a.rows + first) * row_powers + c / CK_BLOCK;
        auto fetch = [&](int i, uint32_t (&power)[2]) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int t = i * WG_TOKENS + token + j * 16;
                power[j] = t < left ? __ldg(powers + t * row_powers) : 127u;
            }
        };
        auto turn = [&](int i, uint32_t (&power)[2]) {
            const int s = i % S::STAGES;
            if (!__all_sync(0xffffffffu, barrier_wait(loaded(s), (i / S::STAGES) & 1, WG_POLLS))) return false;
            const uint32_t to = a_at(s) + q_block * WG_BLOCK_BYTES, from = raw_at(s) + q_block * 64 + q_piece * 16 + token * 128;
            uint4 q[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q[j].x), "=r"(q[j].y), "=r"(q[j].z), "=r"(q[j].w) : "r"(from + j * 2048) : "memory");
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint4 x[2];
                wg_widen(q[j], power[j], x);
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + tc_swizzled(token, q_piece * 2 + h) + j * 2048),
                                 "r"(x[h].x), "r"(x[h].y), "r"(x[h].z), "r"(x[h].w) : "memory");
            }
            async_fence();
            __syncwarp();
            if (lane == 0) barrier_arrive_cluster(in_cta(full(s), 0));
            return true;
        };
        // the powers run two turns ahead
        bool ok = true;
        uint32_t even[2], odd[2];
        fetch(group, even);
        fetch(group + WG_GROUPS, odd);
        for (int i = group; i < turns && ok; i += 2 * WG_GROUPS) {
            ok = turn(i, even);
            fetch(i + 2 * WG_GROUPS, even);
            if (ok && i + WG_GROUPS < turns) {
                ok = turn(i + WG_GROUPS, odd);
                fetch(i + 3 * WG_GROUPS, odd);
            }
        }
        if (!ok) failed = 1;
        if (!barrier_wait(done, 0, WG_POLLS)) failed = 1;
        tc_after_sync();
        asm volatile("bar.sync 1, %0;" ::"n"(WG_WIDENERS) : "memory");   // everyone's verdict
        const bool good = *reinterpret_cast<volatile int *>(&failed) == 0;
        const int ch = c0 + (warp % 4) * 32 + lane;
        for (int col = group * 32; col < slabs * WG_SLAB && o0 + col < a.out; col += WG_GROUPS * 32) {
            float v[32];
            __syncwarp();
            tc_load(tmem + ((uint32_t)(warp % 4) << 21) + col, v);
            if (ch >= a.in) continue;
            if (!good) {   // an unfinished sum is never taken for one
#pragma unroll
                for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(0x7fffffffu);
            }
            const int o = o0 + col;
            if (p.runs > 1) wg_store_column(a.part + (((int64_t)run * a.workers + worker) * a.out + o) * a.in + ch, a.in, a.out - o, v);
            else if (a.grad_dtype == LIEC_F32) wg_store_column(static_cast<float *>(a.dweight) + worker * a.dw_worker + o * a.dw_row + ch, a.dw_row, a.out - o, v);
            else wg_store_column(static_cast<__nv_bfloat16 *>(a.dweight) + worker * a.dw_worker + o * a.dw_row + ch, a.dw_row, a.out - o, v);
        }
        tc_before_sync();
    }
    __syncthreads();
    cluster_sync();   // neither CTA ends while the other may still reach into it
    if (warp == WG_WIDENERS / 32 + 1) tc_free_pair(tmem, S::COLUMNS);
}

// The runs' sums, in their order, rounded once to the gradient's type; zeros without runs.
__global__ void __launch_bounds__(256) wg_join_kernel(const __grid_constant__ WgArgs a, int runs) {
    const int64_t n = (int64_t)a.workers * a.out * a.in, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float s = 0.0f;
    for (int r = 0; r < runs; ++r) s += __ldcs(a.part + r * n + i);
    const int64_t row = i / a.in, c = i - row * a.in, w = row / a.out, at = w * a.dw_worker + (row - w * a.out) * a.dw_row + c;
    if (a.grad_dtype == LIEC_F32) static_cast<float *>(a.dweight)[at] = s;
    else static_cast<__nv_bfloat16 *>(a.dweight)[at] = __float2bfloat16_rn(s);
}

// Runs of tokens: as many as make the GPU's 74 pairs of SMs busy, weighed against what joining them costs.  In units of a
// stage's products (512 cycles): a pair's start and end take about 12, writing and reading a run's sums of a tile 12.
static WgPlan wg_plan(const WgArgs &a, int dtype) {
    WgPlan p{};
    const int outputs = wg_outputs(dtype);
    p.c_tiles = (a.in + 2 * WG_CHANNELS - 1) / (2 * WG_CHANNELS);
    p.o_tiles = (a.out + outputs - 1) / outputs;
    p.tiles = (int64_t)p.c_tiles * p.o_tiles;
    const int64_t stages = (a.rows + WG_TOKENS - 1) / WG_TOKENS, places = p.tiles * a.workers;
    double best = 0.0;
    p.runs = 0;
    for (int runs = 1; runs <= 64 && runs <= std::max<int64_t>(stages, 1) && places * runs < int64_t(1) << 30; ++runs) {
        const int64_t length = (stages + runs - 1) / runs, used = std::max<int64_t>(1, (stages + length - 1) / std::max<int64_t>(length, 1));
        if (used != runs && runs > 1) continue;
        const double cost = (double)((places * runs + 73) / 74) * (double)(length + 12) + (runs > 1 ? 20.0 + 12.0 * (double)(places * runs) / 74.0 : 0.0);
        if (p.runs == 0 || cost < best) {
            best = cost;
            p.runs = runs;
            p.run = std::max<int64_t>(1, length) * WG_TOKENS;
        }
    }
    return p;
}

// dy goes to the products as it is where it is bfloat16 and its rows start on 16 bytes, one after another.
static bool wg_direct(const WgArgs &a, int dtype) {
    return dtype == 1 && ln_whole(a.dy, a.dy_row, a.dy_worker, a.rows, a.workers, 8, 2) && (a.rows == 1 || a.dy_row >= a.out) &&
           (a.workers == 1 || a.dy_worker >= a.out);
}
static size_t wg_part_bytes(const WgArgs &a, const WgPlan &p) {
    return p.runs > 1 ? (sizeof(float) * (size_t)p.runs * a.workers * a.out * a.in + 255) / 256 * 256 : 0;
}

size_t weight_grad_workspace(const WgArgs &a, int dtype) {
    if (a.rows == 0) return 0;
    const size_t packed = wg_direct(a, dtype) ? 0 : (size_t)wg_parts(dtype) * a.workers * a.rows * ((a.out + 7) / 8) * 16;
    return wg_part_bytes(a, wg_plan(a, dtype)) + packed;
}

// The function behind cuTensorMapEncodeTiled: asked of the runtime, so that the library links without the driver's.
typedef CUresult (*WgEncode)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                             CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static WgEncode wg_encode() {
    static std::atomic<void *> found{nullptr};
    void *f = found.load(std::memory_order_acquire);
    if (!f) {
        cudaDriverEntryPointQueryResult result;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &result) != cudaSuccess || result != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        found.store(f, std::memory_order_release);
    }
    return reinterpret_cast<WgEncode>(f);
}

// [workers][rows][cols], boxes of box_cols columns by a stage's tokens; what lies outside is read as zeros.
static bool wg_map(CUtensorMap *map, const void *base, bool bytes, int64_t cols, int64_t rows, int64_t workers, int64_t row, int64_t worker, int box_cols) {
    const WgEncode encode = wg_encode();
    if (!encode) return false;
    const int size = bytes ? 1 : 2;
    // (a single row or worker is never stepped over; the map wants a step all the same)
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)workers};
    const cuuint64_t row_step = rows > 1 ? (cuuint64_t)(row * size) : (cuuint64_t)((cols * size + 15) / 16 * 16);
    const cuuint64_t steps[2] = {row_step, workers > 1 ? (cuuint64_t)(worker * size) : row_step * (cuuint64_t)rows};
    const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)WG_TOKENS, 1}, one[3] = {1, 1, 1};
    return encode(map, bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, steps, box, one,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, bytes ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static cudaLaunchConfig_t wg_config(int64_t ctas, int threads, int smem, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    return cfg;
}

// after: the kernel before this one packs dy; this one starts while it ends and waits for it where it reads.
template <int PARTS>
static cudaError_t wg_launch(const WgArgs &a, const WgPlan &p, const CUtensorMap &q_map, const CUtensorMap &dy_map, bool after, cudaStream_t st) {
    static std::atomic<uint64_t> allowed{0};
    const auto kernel = wg_kernel<PARTS>;
    const cudaError_t e = ln_allow_smem(kernel, WgShape<PARTS>::SMEM_BYTES, allowed);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = wg_config(p.tiles * a.workers * p.runs * 2, WG_THREADS, WgShape<PARTS>::SMEM_BYTES, st);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = after ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, p, q_map, dy_map);
}

cudaError_t launch_weight_grad(WgArgs a, int dtype, cudaStream_t st) {
    int runs = 0;
    if (a.rows > 0) {
        const WgPlan p = wg_plan(a, dtype);
        const bool direct = wg_direct(a, dtype);
        const int64_t q_cols = ck_cols(a.in), dy_cols = (a.out + 7) / 8 * 8;
        a.packed = reinterpret_cast<char *>(a.part) + wg_part_bytes(a, p);
        CUtensorMap q_map, dy_map;
        if (!wg_map(&q_map, a.q, true, q_cols, a.rows, a.workers, q_cols, q_cols * a.rows, WG_CHANNELS) ||
            !(direct ? wg_map(&dy_map, a.dy, false, a.out, a.rows, a.workers, a.dy_row, a.dy_worker, 64)
                     : wg_map(&dy_map, a.packed, false, a.out, a.rows, (int64_t)wg_parts(dtype) * a.workers, dy_cols, dy_cols * a.rows, 64)))
            return cudaErrorNotSupported;
        if (!direct) {
            const int64_t chunks = a.workers * a.rows * (dy_cols / 8);
            const cudaLaunchConfig_t cfg = wg_config((chunks + 255) / 256, 256, 0, st);
            const cudaError_t e = cudaLaunchKernelEx(&cfg, dtype == 0 ? wg_pack_kernel<float> : wg_pack_kernel<__nv_bfloat16>, a, dy_cols / 8);
            if (e != cudaSuccess) return e;
        }
        const cudaError_t e = dtype == 0 ? wg_launch<3>(a, p, q_map, dy_map, !direct, st) : wg_launch<1>(a, p, q_map, dy_map, !direct, st);
        if (e != cudaSuccess || p.runs == 1) return e;
        runs = p.runs;
    }
    const int64_t n = (int64_t)a.workers * a.out * a.in;
    wg_join_kernel<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(a, runs);
    return cudaGetLastError();
}

}  // namespace liec

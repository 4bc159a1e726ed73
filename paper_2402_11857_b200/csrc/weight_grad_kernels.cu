// Weight gradient of a linear layer from the 8-bit checkpoint of its input: dW[o][c] = sum over tokens t of
// dy[t][o] x^[t][c], for N workers, on the tensor cores.
//
// x^ = q 2^e is a bfloat16 number, so the products are those of the definition; a binary32 dy is cut into three bfloat16
// parts whose sum it is, and multiplied three times.  A CTA takes 256 channels c (the rows of the accumulator, two halves of
// 128) by 256 outputs o (128 for binary32), and one run of tokens.  Eight warps bring both operands to shared memory, where
// each token is a row of 128-byte pieces as in memory; the bytes of q are widened on the way.  One thread issues the products.
// Lanes of the accumulator are channels, so a warp writes 32 neighbours of a row of dW.
#include <algorithm>

#include "activation.cuh"
#include "tensor_core.cuh"

namespace liec {

constexpr int WG_TOKENS = 32;                  // of a stage
constexpr int WG_CHANNELS = 256;               // of a tile
constexpr int WG_AHEAD = 3;                    // stages by which the copies run ahead
constexpr int WG_WORKERS = 256, WG_THREADS = WG_WORKERS + 32;
constexpr int WG_BLOCK_BYTES = WG_TOKENS * 128;
constexpr uint32_t WG_POLLS = 1u << 20;

template <typename T>
struct WgShape {
    static constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    static constexpr int OUTPUTS = sizeof(T) == 4 ? 128 : 256;
    static constexpr int A_BYTES = WG_CHANNELS / 64 * WG_BLOCK_BYTES, B_BYTES = OUTPUTS / 64 * WG_BLOCK_BYTES, STAGE_BYTES = A_BYTES + PARTS * B_BYTES;
    static constexpr int STAGES = sizeof(T) == 4 ? 4 : 5;   // what fits; copies that run ahead need two more than their lead
    static constexpr int RAW_BYTES = WG_TOKENS * WG_CHANNELS;
    static constexpr int SMEM_BYTES = 1024 + STAGES * STAGE_BYTES + (WG_AHEAD + 1) * RAW_BYTES;
    static constexpr int COLUMNS = 2 * OUTPUTS;
    static constexpr int DY_CHUNKS = WG_TOKENS * OUTPUTS / Bits<T>::VEC / WG_WORKERS;   // 16-byte chunks of dy per thread and stage
};

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

// ASYNC: rows of dy start on 16 bytes and are bfloat16; they go to shared memory without passing through registers.
template <typename T, bool ASYNC>
__global__ void __launch_bounds__(WG_THREADS, 1) wg_kernel(const __grid_constant__ WgArgs a, const __grid_constant__ WgPlan p) {
    using S = WgShape<T>;
    extern __shared__ char wg_smem[];
    __shared__ __align__(8) unsigned long long bars[2 * S::STAGES + 1];
    __shared__ uint32_t tmem_at;
    __shared__ int failed;
    const uint32_t bar = (uint32_t)__cvta_generic_to_shared(bars);
    const uint32_t base = ((uint32_t)__cvta_generic_to_shared(wg_smem) + 1023u) & ~1023u;
    auto full = [&](int s) { return bar + 8u * s; };
    auto empty = [&](int s) { return bar + 8u * (S::STAGES + s); };
    const uint32_t done = bar + 8u * 2 * S::STAGES;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    int64_t b = blockIdx.x;
    const int run = (int)(b % p.runs);
    b /= p.runs;
    const int worker = (int)(b / p.tiles), tile = (int)(b % p.tiles);
    const int o0 = tile / p.c_tiles * S::OUTPUTS, c0 = tile % p.c_tiles * WG_CHANNELS;
    const int64_t first = run * p.run, tokens = min(p.run, a.rows - first);
    const int turns = (int)((tokens + WG_TOKENS - 1) / WG_TOKENS);

    if (warp == WG_WORKERS / 32) {
        if (lane == 0) {
            for (int s = 0; s < S::STAGES; ++s) {
                barrier_init(full(s), WG_WORKERS / 32);
                barrier_init(empty(s), 1);
            }
            barrier_init(done, 1);
            failed = 0;
            async_fence();
        }
        __syncwarp();
        tc_alloc((uint32_t)__cvta_generic_to_shared(&tmem_at), S::COLUMNS);
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = tmem_at;

    if (warp == WG_WORKERS / 32) {
        if (lane == 0) {
            bool ok = true;
            for (int i = 0; i < turns && ok; ++i) {
                const int s = i % S::STAGES;
                ok = barrier_wait(full(s), (i / S::STAGES) & 1, WG_POLLS);
                if (!ok) break;
                tc_after_sync();
                const uint32_t at = base + s * S::STAGE_BYTES;
#pragma unroll
                for (int k = 0; k < WG_TOKENS / 16; ++k)
#pragma unroll
                    for (int part = 0; part < S::PARTS; ++part)
#pragma unroll
                        for (int half = 0; half < 2; ++half)
                            tc_mma(tmem + half * S::OUTPUTS, tc_descriptor(at + half * 2 * WG_BLOCK_BYTES + k * 2048, WG_BLOCK_BYTES),
                                   tc_descriptor(at + S::A_BYTES + part * S::B_BYTES + k * 2048, WG_BLOCK_BYTES), tc_instruction(128, S::OUTPUTS),
                                   i > 0 || k > 0 || part > 0);
                tc_commit(empty(s));
            }
            if (!ok) {
                failed = 1;
                __threadfence_block();
            }
            tc_commit(done);
        }
        __syncwarp();
    } else {
        // this thread's part of a stage: two chunks of q (16 channels of one token each; a warp takes two tokens, so that
        // the eight threads whose stores go together fill all places of the swizzle), and chunks of dy
        const int q_block = lane >> 3 & 3, q_piece = lane & 3;
        const int64_t q_cols = (a.in + CK_BLOCK - 1) / CK_BLOCK * CK_BLOCK, q_row0 = worker * a.rows + first;
        const int c = c0 + q_block * 64 + q_piece * 16;
        const bool c_live = c < q_cols;
        const T *dy = static_cast<const T *>(a.dy) + worker * a.dy_worker + first * a.dy_row;
        const uint32_t raw = base + S::STAGES * S::STAGE_BYTES + threadIdx.x * 16;
        uint32_t power[WG_AHEAD + 1][2];
        uint4 held[S::DY_CHUNKS];
        auto q_token = [&](int j) { return j * 16 + warp * 2 + (lane >> 2 & 1); };
        auto fetch = [&](int i, int slot) {   // turn i's copies
            const int64_t t0 = (int64_t)i * WG_TOKENS;
            if (i < turns) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int64_t t = t0 + q_token(j);
                    const bool live = c_live && t < tokens;
                    copy_async(raw + slot * S::RAW_BYTES + j * WG_WORKERS * 16, live ? a.q + (q_row0 + t) * q_cols + c : a.q, live ? 16 : 0);
                    power[slot][j] = live ? __ldg(a.scales + (q_row0 + t) * (q_cols / CK_BLOCK) + c / CK_BLOCK) : 127u;
                }
                if constexpr (ASYNC) {
                    const uint32_t to = base + (i % S::STAGES) * S::STAGE_BYTES + S::A_BYTES;
#pragma unroll
                    for (int j = 0; j < S::DY_CHUNKS; ++j) {
                        const int piece = threadIdx.x % 32, t = threadIdx.x / 32 + j * 8, o = o0 + piece * 8;
                        const int bytes = t0 + t < tokens ? min(16, max(0, (a.out - o) * 2)) : 0;
                        copy_async(to + piece / 8 * WG_BLOCK_BYTES + tc_swizzled(t, piece % 8), bytes > 0 ? dy + (t0 + t) * a.dy_row + o : dy, bytes);
                    }
                }
            }
            copy_commit();
        };
        auto hold = [&](int i) {   // turn i's chunks of dy into registers
            if constexpr (!ASYNC) {
                constexpr int ROW = S::OUTPUTS / Bits<T>::VEC;
#pragma unroll
                for (int j = 0; j < S::DY_CHUNKS; ++j) {
                    const int q = threadIdx.x + j * WG_WORKERS;
                    const int64_t t = (int64_t)i * WG_TOKENS + q / ROW;
                    held[j] = i < turns && t < tokens && o0 + q % ROW * Bits<T>::VEC < a.out ? load_chunk(dy + t * a.dy_row, o0 + q % ROW * Bits<T>::VEC, a.out)
                                                                                             : make_uint4(0u, 0u, 0u, 0u);
                }
            }
        };
        auto put = [&](int s) {   // and on to shared memory
            if constexpr (!ASYNC) {
                constexpr int ROW = S::OUTPUTS / Bits<T>::VEC;
                char *to = wg_smem + (base - (uint32_t)__cvta_generic_to_shared(wg_smem)) + s * S::STAGE_BYTES + S::A_BYTES;
#pragma unroll
                for (int j = 0; j < S::DY_CHUNKS; ++j) {
                    const int q = threadIdx.x + j * WG_WORKERS, t = q / ROW, o = q % ROW * Bits<T>::VEC;
                    char *at = to + o / 64 * WG_BLOCK_BYTES + tc_swizzled(t, o % 64 / 8) + o % 8 * 2;
                    if constexpr (S::PARTS == 1) {
                        *reinterpret_cast<uint4 *>(at) = held[j];
                    } else {
                        const uint32_t w[4] = {held[j].x, held[j].y, held[j].z, held[j].w};
                        uint32_t part[4][3];
#pragma unroll
                        for (int e = 0; e < 4; ++e) wg_split(__uint_as_float(w[e]), part[e]);
#pragma unroll
                        for (int k = 0; k < 3; ++k)
                            *reinterpret_cast<uint2 *>(at + k * S::B_BYTES) = make_uint2(__byte_perm(part[0][k], part[1][k], 0x7632), __byte_perm(part[2][k], part[3][k], 0x7632));
                    }
                }
            }
        };
        bool ok = true;
#pragma unroll
        for (int i = 0; i < WG_AHEAD; ++i) fetch(i, i);
        hold(0);
        for (int i0 = 0; i0 < turns && ok; i0 += WG_AHEAD + 1) {
#pragma unroll
            for (int j = 0; j < WG_AHEAD + 1; ++j) {
                const int i = i0 + j;
                if (i < turns && ok) {
                    // the place that is filled now is free: of the turn fetched ahead, or of this one
                    const int next = ASYNC ? i + WG_AHEAD : i;
                    if (next >= S::STAGES && next < turns) ok = barrier_wait(empty(next % S::STAGES), (next / S::STAGES - 1) & 1, WG_POLLS);
                    ok = __all_sync(0xffffffffu, ok);
                    if (ok) {
                        fetch(i + WG_AHEAD, (j + WG_AHEAD) % (WG_AHEAD + 1));
                        const int s = i % S::STAGES;
                        put(s);
                        hold(i + 1);
                        copy_wait<WG_AHEAD>();
                        const uint32_t to = base + s * S::STAGE_BYTES + q_block * WG_BLOCK_BYTES;
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            uint4 q, x[2];
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w)
                                         : "r"(raw + j * S::RAW_BYTES + k * WG_WORKERS * 16) : "memory");
                            wg_widen(q, power[j][k], x);
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + tc_swizzled(q_token(k), q_piece * 2 + h)),
                                             "r"(x[h].x), "r"(x[h].y), "r"(x[h].z), "r"(x[h].w) : "memory");
                        }
                        async_fence();
                        __syncwarp();
                        if (lane == 0) barrier_arrive(full(s));
                    }
                }
            }
        }
        copy_wait<0>();
        if (!ok) failed = 1;
        if (!barrier_wait(done, 0, WG_POLLS)) failed = 1;
        tc_after_sync();
        asm volatile("bar.sync 1, %0;" ::"n"(WG_WORKERS) : "memory");   // everyone's verdict
        const bool good = failed == 0;
        const int half = warp / 4, ch = c0 + half * 128 + (warp % 4) * 32 + lane;
        for (int col = 0; col < S::OUTPUTS && o0 + col < a.out; col += 32) {
            float v[32];
            __syncwarp();
            tc_load(tmem + ((uint32_t)(warp % 4) << 21) + half * S::OUTPUTS + col, v);
            if (ch < a.in) {
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const int o = o0 + col + e;
                    if (o >= a.out) break;
                    const float r = !good ? __uint_as_float(0x7fffffffu) : v[e];
                    if (p.runs > 1) a.part[(((int64_t)run * a.workers + worker) * a.out + o) * a.in + ch] = r;
                    else if (a.grad_dtype == LIEC_F32) static_cast<float *>(a.dweight)[worker * a.dw_worker + o * a.dw_row + ch] = r;
                    else static_cast<__nv_bfloat16 *>(a.dweight)[worker * a.dw_worker + o * a.dw_row + ch] = __float2bfloat16_rn(r);
                }
            }
        }
        tc_before_sync();
    }
    __syncthreads();
    if (warp == WG_WORKERS / 32) tc_free(tmem, S::COLUMNS);
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

// Runs of tokens: as many as make the GPU's places busy, weighed against what joining them costs.  In units of a stage's
// products (512 cycles): a CTA's start and end take about 12, writing and reading a run's sums of a tile 6.
static WgPlan wg_plan(const WgArgs &a, int dtype) {
    WgPlan p{};
    const int outputs = dtype == 0 ? WgShape<float>::OUTPUTS : WgShape<__nv_bfloat16>::OUTPUTS;
    p.c_tiles = (a.in + WG_CHANNELS - 1) / WG_CHANNELS;
    p.o_tiles = (a.out + outputs - 1) / outputs;
    p.tiles = (int64_t)p.c_tiles * p.o_tiles;
    const int64_t stages = (a.rows + WG_TOKENS - 1) / WG_TOKENS, places = p.tiles * a.workers;
    double best = 0.0;
    p.runs = 0;
    for (int runs = 1; runs <= 64 && runs <= std::max<int64_t>(stages, 1) && places * runs < int64_t(1) << 31; ++runs) {
        const int64_t length = (stages + runs - 1) / runs, used = std::max<int64_t>(1, (stages + length - 1) / std::max<int64_t>(length, 1));
        if (used != runs && runs > 1) continue;
        const double cost = (double)((places * runs + 147) / 148) * (double)(length + 12) + (runs > 1 ? 20.0 + 6.0 * (double)(places * runs) / 148.0 : 0.0);
        if (p.runs == 0 || cost < best) {
            best = cost;
            p.runs = runs;
            p.run = std::max<int64_t>(1, length) * WG_TOKENS;
        }
    }
    return p;
}

size_t weight_grad_workspace(const WgArgs &a, int dtype) {
    if (a.rows == 0) return 0;
    const WgPlan p = wg_plan(a, dtype);
    return p.runs > 1 ? sizeof(float) * (size_t)p.runs * a.workers * a.out * a.in : 0;
}

template <typename T, bool ASYNC>
static cudaError_t wg_launch(const WgArgs &a, const WgPlan &p, cudaStream_t st) {
    static std::atomic<uint64_t> allowed{0};
    const auto kernel = wg_kernel<T, ASYNC>;
    const cudaError_t e = ln_allow_smem(kernel, WgShape<T>::SMEM_BYTES, allowed);
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)(p.tiles * a.workers * p.runs), WG_THREADS, WgShape<T>::SMEM_BYTES, st>>>(a, p);
    return cudaGetLastError();
}

cudaError_t launch_weight_grad(WgArgs a, int dtype, cudaStream_t st) {
    int runs = 0;
    if (a.rows > 0) {
        const WgPlan p = wg_plan(a, dtype);
        const bool whole = dtype == 1 && ln_whole(a.dy, a.dy_row, a.dy_worker, a.rows, a.workers, 8, 2);
        const cudaError_t e = dtype == 0 ? wg_launch<float, false>(a, p, st) : whole ? wg_launch<__nv_bfloat16, true>(a, p, st) : wg_launch<__nv_bfloat16, false>(a, p, st);
        if (e != cudaSuccess || p.runs == 1) return e;
        runs = p.runs;
    }
    const int64_t n = (int64_t)a.workers * a.out * a.in;
    wg_join_kernel<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(a, runs);
    return cudaGetLastError();
}

}  // namespace liec

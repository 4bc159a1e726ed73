// Weight gradient of a linear layer from the 8-bit checkpoint of its input: dW[o][c] = sum over tokens t of
// dy[t][o] x^[t][c], for N workers, on the tensor cores.
//
// x^ = q 2^e is a bfloat16 number, so the products are those of the definition; a binary32 dy is cut into three bfloat16
// parts whose sum it is, and multiplied three times.  A pair of CTAs takes a tile of 256 channels c (the rows of the
// accumulator, 128 in each CTA) by 512 outputs o (256 for binary32), and as many tokens of it as its share of the work has.
// Operands lie in shared memory as in global memory, a token as a row of 128-byte pieces: one thread of each CTA has the
// tensor memory accelerator bring q and dy, sixteen warps widen q and cut a binary32 dy (four groups of four, a stage each in
// turn, so that one's latency hides behind the others), one thread of the pair issues the products.  Each CTA so widens 128
// channels and reads half of the outputs: a tile of the same size in one CTA would need half again the shared memory traffic
// of a product.  Lanes of the accumulator are channels, so a warp writes 32 neighbours of a row of dW.
//
// What bounds it: shared memory (bytes in, widened bytes out and in again, and the products' own reads share 128 bytes a cycle) and,
// where sums leave tensor memory, an SM's way out, 27 bytes a cycle.  In bursts at 1965 MHz, by the card: 16 x 3136 tokens of 512 x 2048
// into bfloat16 84 to 91 us, up to 1.25 PFLOP/s; 8 x 8192 of 768 x 2304 into binary32 235 to 250 us, 0.99; binary32 dy, 8 x 4096 of
// 1024 x 1024, 184 us, three times 0.37.  (In a loop of seconds the power cap holds the SMs at 1390 to 1590 MHz: 102 and 278 us.)
#include <cuda.h>

#include <algorithm>

#include "activation.cuh"
#include "tensor_core.cuh"
#include "weight_grad_plan.h"

namespace liec {

constexpr int WG_BLOCK_BYTES = WG_TOKENS * 128;
constexpr int WG_A_BYTES = 2 * WG_BLOCK_BYTES, WG_RAW_BYTES = WG_TOKENS * WG_CHANNELS;
constexpr int WG_GROUPS = 4, WG_GROUP = 128;   // groups of widening threads
constexpr int WG_WIDENERS = WG_GROUPS * WG_GROUP, WG_THREADS = WG_WIDENERS + 64;
constexpr uint32_t WG_POLLS = 1u << 20;

// PARTS: bfloat16 parts of dy; three of a binary32 dy, which comes as it is and is cut by those who widen q.  SLABS: products side by
// side.  A copied stage (bytes of q, dy) stays from the start of its copies to the end of its products (to the end of the cutting, where dy
// is cut), what the widening threads
// make of it (a group's place: channels, and parts of dy) from its widening on: as many of the first as fit beside one of
// the second per group.
template <int PARTS_>
struct WgShape {
    static constexpr int PARTS = PARTS_, SLABS = PARTS == 1 ? 2 : 1, OUTPUTS = SLABS * WG_SLAB;
    static constexpr int COLUMNS = 2 * WG_SLAB;   // two slabs; or one, and the products of the smaller parts of dy beside it
    static constexpr int B_BYTES = 2 * WG_BLOCK_BYTES;                       // of a slab's part
    static constexpr int DY_BYTES = PARTS == 1 ? B_BYTES : 2 * B_BYTES;      // of a slab's dy as it comes
    static constexpr int STAGE_BYTES = SLABS * DY_BYTES + WG_RAW_BYTES;
    static constexpr int PLACE_BYTES = WG_A_BYTES + (PARTS == 1 ? 0 : PARTS * B_BYTES);
    static constexpr int STAGES = PARTS == 1 ? 9 : 4;
    static constexpr int SMEM_BYTES = 1024 + STAGES * STAGE_BYTES + WG_GROUPS * PLACE_BYTES;
    static_assert(SMEM_BYTES <= 227 * 1024 - 512, "with the barriers");
    static_assert(STAGES >= WG_GROUPS, "the parities of the widening groups' waits");
};
static_assert(WgShape<1>::SLABS == wg_slabs(1) && WgShape<3>::SLABS == wg_slabs(0), "the plan's tiles");

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

// x = p[0] + p[1] + p[2], each the upper half of a binary32 number: 8 bits of the significand at a time (what lies below the last
// is zero; next to the end of the range it is not, and what of x lies below 2^-133 is cut).  An infinity or NaN would leave NaN as rest.
__device__ __forceinline__ void wg_split(float x, uint32_t (&p)[3]) {
    p[0] = __float_as_uint(x) & 0xffff0000u;
    const float rest = x - __uint_as_float(p[0]);
    p[1] = __float_as_uint(rest) & 0xffff0000u;
    p[2] = __float_as_uint(rest - __uint_as_float(p[1]));
}
__device__ __forceinline__ void wg_split_special(float x, uint32_t (&p)[3]) {   // infinities and NaN as they are
    const uint32_t bits = __float_as_uint(x);
    if ((bits & 0x7f800000u) != 0x7f800000u) return;
    p[0] = (bits & 0x007fffffu) != 0u ? bits | 0x00400000u : bits;
    p[1] = p[2] = 0u;
}

// dy as the tensor memory accelerator wants it: rows of a multiple of 16 bytes without gaps.  A thread takes 16 bytes.
template <typename T>
__global__ void __launch_bounds__(256) wg_pack_kernel(const __grid_constant__ WgArgs a, int64_t row_chunks) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / row_chunks;
    if (row >= a.workers * a.rows) return;
    const int64_t w = row / a.rows;
    const int c = (int)(i - row * row_chunks) * Bits<T>::VEC;
    reinterpret_cast<uint4 *>(a.packed)[i] = load_chunk(static_cast<const T *>(a.dy) + w * a.dy_worker + (row - w * a.rows) * a.dy_row, c, a.out);
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

// Adds 32 outputs to what this thread stored there; in its order, so equal calls give equal bits.
__device__ __forceinline__ void wg_add_column(float *to, int64_t step, int outputs, const float (&v)[32]) {
#pragma unroll
    for (int e = 0; e < 32; ++e)
        if (e < outputs) asm volatile("red.global.add.f32 [%0], %1;" ::"l"(to + e * step), "f"(v[e]) : "memory");
}

// Stages of each sum of an item.
__device__ __forceinline__ int wg_sum_stages(const WgArgs &a, int stages) {
    const int most = a.grad_dtype == LIEC_F32 ? WG_SUM_STAGES : WG_SUM_STAGES_BF16;
    if (stages <= most) return stages;
    const int sums = (stages + most - 1) / most;
    return (stages + sums - 1) / sums;
}

template <int PARTS>
__global__ void __launch_bounds__(WG_THREADS, 1) wg_kernel(const __grid_constant__ WgArgs a, const __grid_constant__ WgPlan p,
                                                            const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap dy_map) {
    using S = WgShape<PARTS>;
    extern __shared__ char wg_smem[];
    __shared__ __align__(8) unsigned long long bars[3 * S::STAGES + WG_GROUPS + 2];
    __shared__ uint32_t tmem_at;
    __shared__ int failed;
    const uint32_t bar = (uint32_t)__cvta_generic_to_shared(bars);
    const uint32_t base = ((uint32_t)__cvta_generic_to_shared(wg_smem) + 1023u) & ~1023u;
    auto loaded = [&](int s) { return bar + 8u * s; };                       // the copies of a stage, in this CTA
    auto empty = [&](int s) { return bar + 8u * (S::STAGES + s); };          // its products are done
    auto full = [&](int g) { return bar + 8u * (2 * S::STAGES + g); };       // a group's channels, in both CTAs (in the first CTA)
    const uint32_t done = full(WG_GROUPS), drained = done + 8u;              // a tile's products; its sums are read (in the first CTA)
    auto read = [&](int s) { return drained + 8u + 8u * s; };                // PARTS > 1: the widening threads are done with a stage, in this CTA
    auto b_at = [&](int s) { return base + s * S::STAGE_BYTES; };
    auto raw_at = [&](int s) { return b_at(s) + S::SLABS * S::DY_BYTES; };
    auto a_at = [&](int g) { return base + S::STAGES * S::STAGE_BYTES + g * S::PLACE_BYTES; };
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = cluster_rank();
    const int64_t pair = blockIdx.x / 2;
    auto first_channel = [&](const WgItem &g) { return g.c_tile * 2 * WG_CHANNELS + rank * WG_CHANNELS; };

    if (warp == WG_WIDENERS / 32 + 1) {
        if (lane == 0) {
            for (int s = 0; s < S::STAGES; ++s) {
                barrier_init(loaded(s), 1);
                barrier_init(empty(s), 1);
                barrier_init(read(s), WG_GROUP / 32);
            }
            for (int k = 0; k < WG_GROUPS; ++k) barrier_init(full(k), 2 * WG_GROUP / 32);
            barrier_init(done, 1);
            barrier_init(drained, 2 * WG_WIDENERS / 32);
            failed = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            async_fence();
        }
        __syncwarp();
        tc_alloc_pair((uint32_t)__cvta_generic_to_shared(&tmem_at), S::COLUMNS);
    }
    tc_before_sync();
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");

    if (warp == WG_WIDENERS / 32) {
        // copies: into this CTA's memory alone, so the first need not wait for the other CTA
        asm volatile("griddepcontrol.wait;" ::: "memory");   // dy may come from the kernel before
        int it = 0;
        bool ok = true;
        for (int64_t item = pair; ok && item < p.items; item += p.pairs) {
            const WgItem g = p.item(item);
            const int o0 = g.o_tile * S::OUTPUTS + rank * 128, c0 = first_channel(g), t0 = g.stage * WG_TOKENS;
            for (int i = 0; i < g.stages; ++i, ++it) {
                const int s = it % S::STAGES, t = t0 + i * WG_TOKENS;
                if (it >= S::STAGES) ok = barrier_wait_warp(PARTS == 1 ? empty(s) : read(s), (it / S::STAGES - 1) & 1, WG_POLLS);
                if (!ok) break;
                if (elected()) {
                    barrier_expect(loaded(s), WG_RAW_BYTES + g.slabs * S::DY_BYTES);
                    copy_box(raw_at(s), &q_map, c0, t, g.worker, loaded(s));
                    if constexpr (PARTS == 1) {
#pragma unroll
                        for (int n = 0; n < S::SLABS; ++n)
                            if (n < g.slabs)
#pragma unroll
                                for (int h = 0; h < 2; ++h)
                                    copy_box(b_at(s) + n * S::B_BYTES + h * WG_BLOCK_BYTES, &dy_map, o0 + n * WG_SLAB + h * 64, t, g.worker, loaded(s));
                    } else {
                        copy_box(b_at(s), &dy_map, o0, t, g.worker, loaded(s));
                    }
                }
                __syncwarp();
            }
        }
        // nothing may be on its way into this CTA's memory when it ends: the products' last arrivals, or copies
        // (PARTS > 1: a stage that has been read had its last products done, so a parity of `empty` tells its phase)
        for (int k = max(0, it - S::STAGES); ok && k < it; ++k) {
            if constexpr (PARTS > 1) ok = barrier_wait_warp(read(k % S::STAGES), (k / S::STAGES) & 1, WG_POLLS);
            ok = ok && barrier_wait_warp(empty(k % S::STAGES), (k / S::STAGES) & 1, WG_POLLS);
        }
        if (!ok) {
            failed = 1;
            for (int k = max(0, it - S::STAGES); k < it; ++k) barrier_wait_warp(loaded(k % S::STAGES), (k / S::STAGES) & 1, WG_POLLS);
        }
        __syncwarp();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // the other CTA has its barriers and tensor memory
    }
    tc_after_sync();
    const uint32_t tmem = tmem_at;

    if (warp == WG_WIDENERS / 32 + 1) {
        if (rank == 0) {   // products
            bool ok = true;
            int it = 0;
            int64_t n = 0;   // sums so far
            for (int64_t item = pair; ok && item < p.items; item += p.pairs) {
                const WgItem g = p.item(item);
                const int length = wg_sum_stages(a, g.stages);
                for (int i = 0, in_sum = 0; ok && i < g.stages; ++i, ++it) {
                    const int s = it % S::STAGES, k4 = it % WG_GROUPS;
                    if (in_sum == 0 && n > 0) ok = barrier_wait_warp(drained, (n - 1) & 1, WG_POLLS);
                    ok = ok && barrier_wait_warp(full(k4), (it / WG_GROUPS) & 1, WG_POLLS);
                    if (!ok) break;
                    tc_after_sync();
                    const uint64_t x = tc_descriptor(a_at(k4), WG_BLOCK_BYTES), y = tc_descriptor(PARTS == 1 ? b_at(s) : a_at(k4) + WG_A_BYTES, WG_BLOCK_BYTES);
                    const bool last = ++in_sum == length || i + 1 == g.stages;
                    if (elected()) {
#pragma unroll
                        for (int k = 0; k < WG_TOKENS / 16; ++k)
#pragma unroll
                            for (int n = 0; n < S::SLABS; ++n)
                                if (n < g.slabs)
#pragma unroll
                                    for (int part = 0; part < PARTS; ++part)   // (the address field counts 16 bytes)
                                        tc_mma_pair(tmem + (n + (part > 0)) * WG_SLAB, x + (k * 2048 >> 4), y + (((n * PARTS + part) * S::B_BYTES + k * 2048) >> 4),
                                                    tc_instruction(256, WG_SLAB), in_sum > 1 || k > 0 || part > 1);
                        tc_commit_pair(empty(s));
                        if (last) tc_commit_pair(done);
                    }
                    __syncwarp();
                    if (last) {
                        in_sum = 0;
                        ++n;
                    }
                }
                if (!ok && lane == 0) {
                    const uint32_t flag = (uint32_t)__cvta_generic_to_shared(&failed);
                    for (int r = 0; r < 2; ++r) asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(in_cta(flag, r)), "r"(1) : "memory");
                    asm volatile("fence.acq_rel.cluster;" ::: "memory");
                }
                __syncwarp();
            }
            if (!ok && elected()) tc_commit_pair(done);   // nobody is to wait for its limit
            __syncwarp();
        }
    } else if (warp < WG_WIDENERS / 32) {
        // A thread's part of a stage: two chunks of q, 16 channels of one token each.  Eight threads that load or store
        // together meet all places of a 128-byte row, plain in one case and swizzled in the other.
        const int group = warp / 4, parity = lane >> 2 & 1, q_block = parity ^ (lane >> 3 & 1), q_piece = lane & 3;
        const int token = warp % 4 * 4 + (lane >> 4) * 2 + parity;           // and the one 16 further on
        const int64_t row_powers = (a.in + CK_BLOCK - 1) / CK_BLOCK;
        bool ok = true;
        int it0 = 0;   // stages before this tile's
        int64_t n = 0;   // sums so far
        for (int64_t item = pair; item < p.items; item += p.pairs) {
            const WgItem g = p.item(item);
            const int length = wg_sum_stages(a, g.stages);
            for (int sum = 0, from = 0; sum < g.stages; sum += length, ++n) {
                // A group widens one stage of the next sum before it takes this one, so that its products wait for that alone.
                const int end = min(sum + length, g.stages), until = min(end + WG_GROUPS, g.stages);
                const int c0 = first_channel(g), c = c0 + q_block * 64 + q_piece * 16;
                const int64_t first = (int64_t)g.stage * WG_TOKENS;
                const int left = c < row_powers * CK_BLOCK ? (int)min(a.rows - first, (int64_t)g.stages * WG_TOKENS) : 0;
                const uint8_t *powers = a.scales + (g.worker * a.rows + first) * row_powers + c / CK_BLOCK;
                auto fetch = [&](int i, uint32_t (&power)[2]) {   // i: stage of this tile
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int t = i * WG_TOKENS + token + j * 16;
                        power[j] = t < left ? __ldg(powers + t * row_powers) : 127u;
                    }
                };
                auto turn = [&](int i, uint32_t (&power)[2]) {
                    const int s = (it0 + i) % S::STAGES;
                    // The group's place is free when the products of its last turn, WG_GROUPS stages ago, are done.  This wait comes
                    // first: a group does not see every phase of a stage's barriers, and a parity tells a phase from its
                    // neighbours only.  After it all stages up to the last turn's are done, so both barriers are in the phase
                    // that is waited for (STAGES >= WG_GROUPS; here the last turn's own wait vouches for 2 WG_GROUPS stages ago).
                    const int before = it0 + i - WG_GROUPS;
                    if (before >= 0 && !barrier_wait_warp(empty(before % S::STAGES), (before / S::STAGES) & 1, WG_POLLS)) return false;
                    if (!barrier_wait_warp(loaded(s), ((it0 + i) / S::STAGES) & 1, WG_POLLS)) return false;
                    const uint32_t to = a_at(group) + q_block * WG_BLOCK_BYTES, from = raw_at(s) + q_block * 64 + q_piece * 16 + token * 128;
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
                    if constexpr (PARTS > 1) {   // 8 outputs of a token at a time
#pragma unroll 2
                        for (int j = 0; j < 4; ++j) {
                            const int dy_token = warp % 4 * 8 + j * 2 + (lane >> 4), piece = lane & 15, swap = lane >> 2 & 1;   // (of eight lanes, four start with their second half: all places of a row)
                            float u[8], v[8];
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(u[4 * h]), "=f"(u[4 * h + 1]), "=f"(u[4 * h + 2]), "=f"(u[4 * h + 3])
                                             : "r"(b_at(s) + dy_token * 512 + piece * 32 + (h ^ swap) * 16) : "memory");
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = swap ? u[e ^ 4] : u[e];
                            uint32_t x[8][3], most = 0u;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                wg_split(v[e], x[e]);
                                most = max(most, __float_as_uint(v[e]) & 0x7fffffffu);
                            }
                            if (most >= 0x7f800000u)
#pragma unroll
                                for (int e = 0; e < 8; ++e) wg_split_special(v[e], x[e]);
#pragma unroll
                            for (int part = 0; part < 3; ++part)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a_at(group) + WG_A_BYTES + part * S::B_BYTES + (piece >> 3) * WG_BLOCK_BYTES +
                                                                                              tc_swizzled(dy_token, piece & 7)),
                                             "r"(__byte_perm(x[0][part], x[1][part], 0x7632)), "r"(__byte_perm(x[2][part], x[3][part], 0x7632)),
                                             "r"(__byte_perm(x[4][part], x[5][part], 0x7632)), "r"(__byte_perm(x[6][part], x[7][part], 0x7632)) : "memory");
                        }
                    }
                    async_fence();
                    __syncwarp();
                    if (lane == 0) {
                        barrier_arrive_cluster(in_cta(full(group), 0));
                        if constexpr (PARTS > 1) barrier_arrive_cluster(in_cta(read(s), rank));
                    }
                    return true;
                };
                // the powers run two turns ahead
                uint32_t even[2], odd[2];
                const int begin = from + (group - (it0 + from) % WG_GROUPS + WG_GROUPS) % WG_GROUPS;
                fetch(begin, even);
                fetch(begin + WG_GROUPS, odd);
                for (int i = begin; i < until && ok; i += 2 * WG_GROUPS) {
                    ok = turn(i, even);
                    fetch(i + 2 * WG_GROUPS, even);
                    if (ok && i + WG_GROUPS < until) {
                        ok = turn(i + WG_GROUPS, odd);
                        fetch(i + 3 * WG_GROUPS, odd);
                    }
                }
                if (ok) ok = barrier_wait(done, n & 1, WG_POLLS);
                if (!ok) failed = 1;
                tc_after_sync();
                asm volatile("bar.sync 1, %0;" ::"n"(WG_WIDENERS) : "memory");   // everyone's verdict
                if (*reinterpret_cast<volatile int *>(&failed)) ok = false;
                const int o0 = g.o_tile * S::OUTPUTS, mine = (warp % 4) * 32 + lane, ch = c0 + mine;
                float *part = a.part + g.slot + rank * WG_CHANNELS + mine;
                for (int col = group * 32; col < g.slabs * WG_SLAB && o0 + col < a.out; col += WG_GROUPS * 32) {
                    float v[32];
                    __syncwarp();
                    tc_load(tmem + ((uint32_t)(warp % 4) << 21) + col, v);
                    if constexpr (PARTS > 1) {
                        float rest[32];
                        tc_load(tmem + ((uint32_t)(warp % 4) << 21) + WG_SLAB + col, rest);
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] += rest[e];
                    }
                    if (!ok) {   // an unfinished sum is never taken for one (and stays NaN whatever is added)
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(0x7fffffffu);
                    }
                    const int o = o0 + col;
                    float *to = nullptr;
                    int64_t step = 2 * WG_CHANNELS;
                    int outputs = 32;
                    if (g.slot >= 0) {
                        to = part + col * step;
                    } else {
                        if (ch >= a.in) continue;
                        step = a.dw_row;
                        outputs = a.out - o;
                        if (a.grad_dtype == LIEC_F32) to = static_cast<float *>(a.dweight) + g.worker * a.dw_worker + o * step + ch;
                    }
                    if (!to) wg_store_column(static_cast<__nv_bfloat16 *>(a.dweight) + g.worker * a.dw_worker + o * step + ch, step, outputs, v);
                    else if (sum == 0) wg_store_column(to, step, outputs, v);
                    else wg_add_column(to, step, outputs, v);
                }
                tc_before_sync();
                __syncwarp();
                if (lane == 0 && (end < g.stages || item + p.pairs < p.items)) barrier_arrive_cluster(in_cta(drained, 0));   // the next sum's products wait for this
                from = until;
            }
            it0 += g.stages;
        }
    }
    tc_before_sync();
    __syncthreads();
    __syncwarp();
    if (failed) {   // arrivals that nobody waited for, and products: time to come to their end
        long long t0, t1;
        asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
        for (int spin = 0; spin < 1 << 22; ++spin) {
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t1));
            if (t1 - t0 > 1000000) break;
        }
    }
    cluster_sync();   // neither CTA ends while the other may still reach into it
    if (warp == WG_WIDENERS / 32 + 1) tc_free_pair(tmem, S::COLUMNS);
}

// A cut tile's runs, added in their order and rounded once to the gradient's type.  A block has 4 outputs of a cut tile, a thread 4
// channels of one: many threads with eight loads under way each (16 outputs per block, four loads: 13 us for six
// tiles in 11 and 5 runs, now 7).
constexpr int WG_JOIN_OUTPUTS = 4;
__global__ void __launch_bounds__(256) wg_join_kernel(const __grid_constant__ WgArgs a, const __grid_constant__ WgPlan p) {
    const uint32_t blocks = (uint32_t)p.slabs * WG_SLAB / WG_JOIN_OUTPUTS, tile = blockIdx.x / blocks, block = blockIdx.x - tile * blocks;
    const int64_t cut = p.cut_joins() ? p.full - p.whole : 0;
    const bool is_last = tile >= cut;
    const int64_t index = is_last ? tile - cut : tile, tiles = is_last ? p.last : cut, size = p.slot_size(is_last);
    const WgItem t = p.tile_of((is_last ? p.full : p.whole) + index);
    const int runs = is_last ? p.last_runs : p.runs, lane = threadIdx.x % 64, c = t.c_tile * 2 * WG_CHANNELS + lane * 4;
    const int row = (int)block * WG_JOIN_OUTPUTS + threadIdx.x / 64, o = t.o_tile * p.slabs * WG_SLAB + row;
    const float4 *from = reinterpret_cast<const float4 *>(a.part + index * size + (is_last ? cut * p.runs * p.slot_size(false) : 0) + row * 2 * WG_CHANNELS + lane * 4);
    const int64_t step = tiles * size / 4;
    asm volatile("griddepcontrol.wait;" ::: "memory");   // the sums are complete
    if (o >= a.out || row >= t.slabs * WG_SLAB || c >= a.in) return;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    int r = 0;
    auto add = [&](const float4 &v) { s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w; };
    for (; r + 8 <= runs; r += 8, from += 8 * step) {
        float4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __ldcs(from + k * step);
#pragma unroll
        for (int k = 0; k < 8; ++k) add(v[k]);
    }
#pragma unroll 4
    for (; r < runs; ++r, from += step) add(__ldcs(from));
    const float v[4] = {s.x, s.y, s.z, s.w};
    const int64_t to = t.worker * a.dw_worker + o * a.dw_row + c;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (c + e < a.in) {
            if (a.grad_dtype == LIEC_F32) static_cast<float *>(a.dweight)[to + e] = v[e];
            else static_cast<__nv_bfloat16 *>(a.dweight)[to + e] = __float2bfloat16_rn(v[e]);
        }
}

__global__ void __launch_bounds__(256) wg_zero_kernel(const __grid_constant__ WgArgs a) {   // no tokens
    const int64_t n = (int64_t)a.workers * a.out * a.in, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int64_t row = i / a.in, w = row / a.out, at = w * a.dw_worker + (row - w * a.out) * a.dw_row + i - row * a.in;
    if (a.grad_dtype == LIEC_F32) static_cast<float *>(a.dweight)[at] = 0.0f;
    else static_cast<__nv_bfloat16 *>(a.dweight)[at] = __float2bfloat16_rn(0.0f);
}

// dy goes to the kernel as it is where its rows start on 16 bytes, one after another.
static bool wg_direct(const WgArgs &a, int dtype) {
    return ln_whole(a.dy, a.dy_row, a.dy_worker, a.rows, a.workers, dtype == 0 ? 4 : 8, dtype == 0 ? 4 : 2) && (a.rows == 1 || a.dy_row >= a.out) &&
           (a.workers == 1 || a.dy_worker >= a.out);
}
static size_t wg_part_bytes(const WgPlan &p) { return sizeof(float) * (size_t)p.slots(); }

size_t weight_grad_workspace(const WgArgs &a, int dtype) {
    if (a.rows == 0) return 0;
    const int vec = dtype == 0 ? 4 : 8;
    const size_t packed = wg_direct(a, dtype) ? 0 : (size_t)a.workers * a.rows * ((a.out + vec - 1) / vec) * 16;
    return wg_part_bytes(wg_plan(a.workers, a.rows, a.in, a.out, dtype, a.grad_dtype == LIEC_BF16)) + packed;
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
static bool wg_map(CUtensorMap *map, const void *base, int size, int64_t cols, int64_t rows, int64_t workers, int64_t row, int64_t worker, int box_cols) {
    const WgEncode encode = wg_encode();
    if (!encode) return false;
    // (a single row or worker is never stepped over; the map wants a step all the same)
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)workers};
    const cuuint64_t row_step = rows > 1 ? (cuuint64_t)(row * size) : (cuuint64_t)((cols * size + 15) / 16 * 16);
    const cuuint64_t steps[2] = {row_step, workers > 1 ? (cuuint64_t)(worker * size) : row_step * (cuuint64_t)rows};
    const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)WG_TOKENS, 1}, one[3] = {1, 1, 1};
    return encode(map, size == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : size == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, const_cast<void *>(base), dims, steps, box, one,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, size == 2 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
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
    cudaLaunchConfig_t cfg = wg_config((int64_t)p.pairs * 2, WG_THREADS, WgShape<PARTS>::SMEM_BYTES, st);
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
    if (a.rows == 0) {
        wg_zero_kernel<<<(unsigned)(((int64_t)a.workers * a.out * a.in + 255) / 256), 256, 0, st>>>(a);
        return cudaGetLastError();
    }
    const WgPlan p = wg_plan(a.workers, a.rows, a.in, a.out, dtype, a.grad_dtype == LIEC_BF16);
    const bool direct = wg_direct(a, dtype);
    const int size = dtype == 0 ? 4 : 2, vec = 16 / size, box = dtype == 0 ? 128 : 64;
    const int64_t q_cols = ck_cols(a.in), dy_cols = (a.out + vec - 1) / vec * vec;
    a.packed = reinterpret_cast<char *>(a.part) + wg_part_bytes(p);
    CUtensorMap q_map, dy_map;
    if (!wg_map(&q_map, a.q, 1, q_cols, a.rows, a.workers, q_cols, q_cols * a.rows, WG_CHANNELS) ||
        !(direct ? wg_map(&dy_map, a.dy, size, a.out, a.rows, a.workers, a.dy_row, a.dy_worker, box)
                 : wg_map(&dy_map, a.packed, size, a.out, a.rows, a.workers, dy_cols, dy_cols * a.rows, box)))
        return cudaErrorNotSupported;
    cudaError_t e = cudaSuccess;
    if (!direct) {
        const int64_t chunks = a.workers * a.rows * (dy_cols / vec);
        const cudaLaunchConfig_t cfg = wg_config((chunks + 255) / 256, 256, 0, st);
        e = cudaLaunchKernelEx(&cfg, dtype == 0 ? wg_pack_kernel<float> : wg_pack_kernel<__nv_bfloat16>, a, dy_cols / vec);
        if (e != cudaSuccess) return e;
    }
    e = dtype == 0 ? wg_launch<3>(a, p, q_map, dy_map, !direct, st) : wg_launch<1>(a, p, q_map, dy_map, !direct, st);
    const int64_t joined = (p.cut_joins() ? p.full - p.whole : 0) + (p.last_joins() ? p.last : 0);
    if (e != cudaSuccess || joined == 0) return e;
    cudaLaunchConfig_t cfg = wg_config(joined * (p.slabs * WG_SLAB / WG_JOIN_OUTPUTS), 256, 0, st);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, wg_join_kernel, a, p);
}

}  // namespace liec

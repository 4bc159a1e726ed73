// Layer normalisation, forward pass.  Per row: m = mean(x), r = 1 / sqrt(mean((x - m)^2) + eps),
// y = (x - m) r w + b.  A row is read into registers once, its two sums meet (one exchange), y is written: every
// element crosses HBM once, and HBM bounds it.  Bfloat16: 32 x 4096 rows of 768 70.7 us (5.7 TB/s; a copy of the
// array takes 62.4 us), 4 x 4096 of 4096 44.8 us (copy 42.6), 16 x 4096 of 1024 51.5 us (copy 42.6: twelve warps
// per SM, which the 32 elements per thread leave room for); binary32, 4 x 8192 of 2048 88 us (copy 82.5).  Rows of
// odd width cost instructions on top (see the common header), calls below a few MB are latency: 4 x 32 rows of 256
// 3.5 us.  Two rows per turn, where the registers hold them, halve the exchanges; with E = 24 and 32 that spills
// (93 against 71 us at 768 columns).
#include "layer_norm_common.cuh"

namespace liec {

// A CTA takes its share of all groups * rows rows, group after group; every thread of the CTA makes the
// same number of turns, a turn being R consecutive rows for every slot.
template <typename T, bool WHOLE, bool WIDE, int NV, int TPR, int SLOTS, int MINB, int R>
__global__ void __launch_bounds__(TPR * SLOTS, MINB) ln_forward_kernel(const __grid_constant__ LnForward a) {
    using S = LnShape<T, WHOLE, NV, TPR, SLOTS, MINB, R, 1>;
    constexpr int VEC = S::VEC, P = VEC / 2;
    extern __shared__ __align__(16) char ln_ring[];
    __shared__ __align__(16) float box[2][SLOTS][S::WARPS][2 * R];
    const int slot = threadIdx.x / TPR, t = threadIdx.x % TPR;
    __shared__ float2 meet[2][R][8];
    // WIDE: this CTA's columns of the cluster's rows
    const int rank = WIDE ? cluster_rank() : 0, parts = WIDE ? cluster_size() : 1, c0 = WIDE ? rank * a.part_cols : 0;
    const int64_t cta = WIDE ? blockIdx.x / parts : blockIdx.x;
    const int h = WIDE ? min(a.part_cols, a.cols - c0) : a.cols;
    const float inv_h = 1.0f / (float)a.cols;
    LnPipe<T, S, WHOLE, NV, TPR> px[R];
#pragma unroll
    for (int j = 0; j < R; ++j) px[j].place(ln_ring, slot * R + j);
    ln_clear_tails<S, WHOLE>(ln_ring, h * (int)sizeof(T));
    if constexpr (WIDE) cluster_sync();   // (all have started: their shared memory may be written)
    else __syncthreads();
    int flip = 0;
    const int64_t total = (int64_t)a.groups * a.rows;
    const int64_t u_end = min(total, a.share.first(cta + 1));
    for (int64_t u = a.share.first(cta); u < u_end;) {
        const int group = (int)(u / a.rows);
        const int64_t r0 = u - (int64_t)group * a.rows;
        const int count = (int)(min(a.rows, r0 + (u_end - u)) - r0);    // rows of this group
        u += count;
        const int turns = (count + SLOTS * R - 1) / (SLOTS * R);
        const T *x_next = reinterpret_cast<const T *>(a.x) + group * a.x_group + (r0 + slot * R) * a.x_row + c0;   // the next row to fetch
        T *y = reinterpret_cast<T *>(a.y) + group * a.y_group + (r0 + slot * R) * a.y_row + c0;
        int64_t at = (int64_t)group * a.rows + r0 + slot * R;
        const int64_t x_step = (int64_t)SLOTS * R * a.x_row, y_step = (int64_t)SLOTS * R * a.y_row;
        auto row_of = [&](int turn, int j) { return (turn * SLOTS + slot) * R + j; };
        auto fetch = [&](int turn, int stage, LnHead (&head)[R]) {
#pragma unroll
            for (int j = 0; j < R; ++j) {
                head[j].to = 0u;
                if (row_of(turn, j) < count) px[j].fetch(x_next + j * a.x_row, t, h, stage, head[j]);
            }
            x_next += x_step;
            copy_commit();
        };
        auto land = [&](const LnHead (&head)[R]) {
#pragma unroll
            for (int j = 0; j < R; ++j) px[j].land(head[j]);
        };
#pragma unroll
        for (int j = 0; j < R; ++j) px[j].now = (uint32_t)reinterpret_cast<uintptr_t>(x_next + j * a.x_row);
        LnHead head[S::STAGES - 1][R];
#pragma unroll
        for (int s = 0; s < S::STAGES - 1; ++s) fetch(s, s, head[s]);
#pragma unroll
        for (int s = 0; s < S::STAGES - 2; ++s) land(head[s]);
        LnHead (&last)[R] = head[S::STAGES - 2];   // of the turn fetched last
        F2 w[NV][P], b[NV][P];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            ln_parameters<P>(a.weight, group * a.weight_stride + c0, (v * TPR + t) * VEC, h, 1.0f, w[v]);
            ln_parameters<P>(a.bias, group * a.bias_stride + c0, (v * TPR + t) * VEC, h, 0.0f, b[v]);
        }
        for (int i = 0, stage = 0; i < turns; ++i) {
            const int ahead = i + S::STAGES - 1;                               // turn to fetch now
            const int into = stage == 0 ? S::STAGES - 1 : stage - 1;
            if constexpr (WHOLE) {
                fetch(ahead, into, last);
                copy_wait<S::STAGES - 1>();
            } else {
                copy_wait<S::STAGES - 2>();
                land(last);
                slot_sync<TPR>(slot);      // the rows of turn i are complete, and all are done with turn i - 1
                fetch(ahead, into, last);
            }
            F2 x[R][NV][P];
            float mean[R], var[R];
#pragma unroll
            for (int j = 0; j < R; ++j) {
                F2 s2 = f2(0.0f), q2 = f2(0.0f);
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    px[j].read(v, t, stage, x[j][v]);   // (zeros beyond column h)
#pragma unroll
                    for (int k = 0; k < P; ++k) {
                        s2 = add(s2, x[j][v][k]);
                        q2 = fma(x[j][v][k], x[j][v][k], q2);
                    }
                }
                mean[j] = lo(s2) + hi(s2);
                var[j] = lo(q2) + hi(q2);
            }
            slot_sums<TPR, S::WARPS, R>(mean, var, t, slot, box[flip]);
            if constexpr (WIDE) cluster_sums<R>(mean, var, rank, parts, meet[flip]);
            flip ^= 1;
            if constexpr (!WHOLE && S::WARPS == 1) __syncwarp();   // all have read the rows, whose place the results take
            // var = mean(x^2) - mean^2 keeps its digits while mean^2 is at most a quarter of it (the difference
            // then carries at most 1.25 times the relative error of the sums) and nothing overflowed; other
            // rows sum the squares around their mean
            bool far[R], any_far = false;
#pragma unroll
            for (int j = 0; j < R; ++j) {
                mean[j] *= inv_h;
                var[j] = __fmaf_rn(-mean[j], mean[j], var[j] * inv_h);
                far[j] = !(mean[j] * mean[j] <= 0.25f * var[j] && var[j] < 1e37f);
                any_far |= far[j];
                const F2 minus = f2(-mean[j]);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int k = 0; k < P; ++k) x[j][v][k] = add(x[j][v][k], minus);
            }
            if (TPR < 32 ? __any_sync(0xffffffffu, any_far) : any_far) {   // (the same for all threads of a slot)
                float around[R], unused[R];
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    F2 d2 = f2(0.0f);
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        const int left = h - (v * TPR + t) * VEC;
                        F2 d[P];
#pragma unroll
                        for (int k = 0; k < P; ++k) d[k] = x[j][v][k];
                        if (left < VEC) ln_keep<P>(d, left);
#pragma unroll
                        for (int k = 0; k < P; ++k) d2 = fma(d[k], d[k], d2);
                    }
                    around[j] = lo(d2) + hi(d2);
                    unused[j] = 0.0f;
                }
                slot_sums<TPR, S::WARPS, R>(around, unused, t, slot, box[flip]);
                if constexpr (WIDE) cluster_sums<R>(around, unused, rank, parts, meet[flip]);
                flip ^= 1;
#pragma unroll
                for (int j = 0; j < R; ++j)
                    if (far[j]) var[j] = around[j] * inv_h;
            }
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const bool live = row_of(i, j) < count;
                const float rstd = rsqrtf(var[j] + a.eps);
                const F2 scale = f2(rstd);
                T *yj = y + j * a.y_row;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int c = (v * TPR + t) * VEC;
#pragma unroll
                    for (int k = 0; k < P; ++k) x[j][v][k] = fma(mul(x[j][v][k], scale), w[v][k], b[v][k]);
                    if (live && c < h) LnChunk<T>::write(WHOLE ? reinterpret_cast<char *>(yj + c) : px[j].result(v, t, stage), x[j][v]);
                }
                if (live && t == 0 && rank == 0) {
                    if (a.mean) a.mean[at + j] = mean[j];
                    if (a.rstd) a.rstd[at + j] = rstd;
                }
            }
            if constexpr (!WHOLE) {
                slot_sync<TPR>(slot);
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    if (row_of(i, j) < count) ln_store_row<T, NV, TPR>(y + j * a.y_row, px[j].ring + stage * S::STAGE_BYTES, t, h);
                    px[j].now += (uint32_t)x_step * (uint32_t)sizeof(T);
                }
            }
            y += y_step;
            at += SLOTS * R;
            stage = stage + 1 == S::STAGES ? 0 : stage + 1;
        }
        copy_wait<0>();
        if constexpr (!WHOLE) __syncthreads();   // the next group's rows go into the same ring
    }
    if constexpr (WIDE) cluster_sync();   // none may leave while another still hands it sums
}

template <typename T, bool WHOLE, bool WIDE = false>
struct LnForwardLaunch {
    LnForward a;
    cudaStream_t st;
    template <int TPR, int E, int SLOTS, int MINB>
    cudaError_t operator()() {
        constexpr int NV = E / LnChunk<T>::VEC;
        constexpr int R = E <= 16 ? 2 : 1;   // rows per turn: two where the registers hold them
        using S = LnShape<T, WHOLE, NV, TPR, SLOTS, MINB, R, 1>;
        static std::atomic<uint64_t> allowed{0};
        const auto kernel = ln_forward_kernel<T, WHOLE, WIDE, NV, TPR, SLOTS, MINB, R>;
        const cudaError_t e = ln_allow_smem(kernel, S::RING_BYTES, allowed);
        if (e != cudaSuccess) return e;
        const int parts = WIDE ? ln_parts(a.cols) : 1;
        a.part_cols = ln_part_cols(a.cols);
        // (one CTA per SM: a small share would leave its SM idle while it starts)
        a.share = ln_share((int64_t)a.groups * a.rows, SLOTS * R, ln_resident(MINB, parts), 1 << 30, MINB > 1);
        return ln_launch(kernel, a, a.share.ctas, parts, S::THREADS, S::RING_BYTES, st);
    }
};

template <typename T, bool WHOLE>
static cudaError_t forward_rows(const LnForward &a, cudaStream_t st) {
    if (ln_parts(a.cols) > 1) return ln_wide_shape(LnForwardLaunch<T, WHOLE, true>{a, st});
    return ln_forward_shape(a.cols, LnForwardLaunch<T, WHOLE>{a, st});
}

cudaError_t launch_layer_norm_forward(const LnForward &a, int dtype, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    const int esz = dtype == 0 ? 4 : 2;
    const bool whole = ln_whole(a.x, a.x_row, a.x_group, a.rows, a.groups, a.cols, esz) &&
                       ln_whole(a.y, a.y_row, a.y_group, a.rows, a.groups, a.cols, esz);
    if (dtype == 0) return whole ? forward_rows<float, true>(a, st) : forward_rows<float, false>(a, st);
    return whole ? forward_rows<__nv_bfloat16, true>(a, st) : forward_rows<__nv_bfloat16, false>(a, st);
}

}  // namespace liec

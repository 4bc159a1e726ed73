// Layer normalisation, backward pass.  Per row, with xh = (x - m) r and
// q = dy w:  dx = r (q - mean(q) - xh mean(q xh));  per worker  dw = sum over rows of dy xh,  db = sum over
// rows of dy.  x and dy cross HBM once: the column sums stay in the registers of the threads that own
// the columns, for all the rows of a CTA, and meet in two steps (slots of a CTA, then CTAs).
// Bfloat16, 32 x 4096 rows of 768: 105 us, of which 3 us the second step: 5.8 TB/s.  Wider rows are bound by the
// instructions of 12 to 16 warps per SM, all that the column sums leave registers for: 4 x 4096 of 4096 80 us
// = 5.0 TB/s with half of the issue slots in use, warps waiting for the row's exchange and for shared memory
// (measured beside it: 8 elements per thread and twice the threads 93 us, 32 per thread 85 us, two rows per exchange
// 95 us, three CTAs per SM with both rows read twice 88 us, SMs dealt rows by speed, which makes more pieces,
// 119 us).  Binary32, 4 x 8192 of 2048: 139 us = 5.8 TB/s.
#include "layer_norm_common.cuh"

namespace liec {

__device__ __forceinline__ void store_grad(void *base, int64_t at, int grad_dtype, float v) {
    if (grad_dtype == 0) ln_store(reinterpret_cast<float *>(base) + at, v);
    else ln_store(reinterpret_cast<__nv_bfloat16 *>(base) + at, v);
}

// A CTA takes its share of all groups * rows rows, group after group.  Its rows of one group leave their
// column sums as one piece; piece (b, group) lies at b + group, which no other pair on the staircase of
// CTAs over groups shares.  With a.direct a group is one CTA's and the sums are the gradient.
// With xc = x - m and g = dy r:  dx = g w - mean(g w) - xc r^2 mean(g w xc),  dw += g xc  (nine operations
// per element instead of the ten of xh and q).
template <typename T, bool WHOLE, bool WIDE, int NV, int TPR, int SLOTS, int MINB>
__global__ void __launch_bounds__(TPR * SLOTS, MINB) ln_backward_kernel(const __grid_constant__ LnBackward a) {
    using S = LnShape<T, WHOLE, NV, TPR, SLOTS, MINB, 1, 2>;
    constexpr int VEC = S::VEC, P = VEC / 2;
    constexpr bool KEEP = S::KEEP;   // x - m and g w stay in registers while the sums meet
    extern __shared__ __align__(16) char ln_ring[];
    __shared__ __align__(16) float box[2][SLOTS][S::WARPS][2];
    __shared__ float2 meet_rows[2][1][8];
    const int slot = threadIdx.x / TPR, t = threadIdx.x % TPR;
    // WIDE: this CTA's columns of the cluster's rows
    const int rank = WIDE ? cluster_rank() : 0, parts = WIDE ? cluster_size() : 1, c0 = WIDE ? rank * a.part_cols : 0;
    const int64_t cta = WIDE ? blockIdx.x / parts : blockIdx.x;
    const int h = WIDE ? min(a.part_cols, a.cols - c0) : a.cols;
    const float inv_h = 1.0f / (float)a.cols;
    if constexpr (WIDE) cluster_sync();   // (all have started: their shared memory may be written)
    LnPipe<T, S, WHOLE, NV, TPR> px, pd;
    px.place(ln_ring, slot);
    pd.place(ln_ring, SLOTS + slot);
    int flip = 0;
    const int64_t total = (int64_t)a.groups * a.rows;
    const int64_t u_end = min(total, a.share.first(cta + 1));
    for (int64_t u = a.share.first(cta); u < u_end;) {
        const int group = (int)(u / a.rows);
        const int64_t r0 = u - (int64_t)group * a.rows;
        const int count = (int)(min(a.rows, r0 + (u_end - u)) - r0);    // rows of this group
        u += count;
        const int turns = (count + SLOTS - 1) / SLOTS;
        const T *x_next = reinterpret_cast<const T *>(a.x) + group * a.x_group + (r0 + slot) * a.x_row + c0;       // the next row to fetch
        const T *dy_next = reinterpret_cast<const T *>(a.dy) + group * a.dy_group + (r0 + slot) * a.dy_row + c0;
        T *dx = reinterpret_cast<T *>(a.dx) + group * a.dx_group + (r0 + slot) * a.dx_row + c0;
        const int64_t x_step = (int64_t)SLOTS * a.x_row, dy_step = (int64_t)SLOTS * a.dy_row, dx_step = (int64_t)SLOTS * a.dx_row;
        const float *mean_at = a.mean + (int64_t)group * a.rows + r0 + slot, *rstd_at = a.rstd + (int64_t)group * a.rows + r0 + slot;
        if (h != S::COLS) {   // (at every group: the column sums of the last one lay here)
            ln_clear_tails<S, WHOLE>(ln_ring, h * (int)sizeof(T));
            __syncthreads();
        }
        struct Heads { LnHead x, dy; };
        auto fetch = [&](int turn, int stage, Heads &head) {
            head.x.to = head.dy.to = 0u;
            if (turn * SLOTS + slot < count) {
                px.fetch(x_next, t, h, stage, head.x);
                pd.fetch(dy_next, t, h, stage, head.dy);
            }
            x_next += x_step;
            dy_next += dy_step;
            copy_commit();
        };
        auto land = [&](const Heads &head) {
            px.land(head.x);
            px.land(head.dy);
        };
        px.now = (uint32_t)reinterpret_cast<uintptr_t>(x_next);
        pd.now = (uint32_t)reinterpret_cast<uintptr_t>(dy_next);
        Heads head[S::STAGES - 1];
#pragma unroll
        for (int s = 0; s < S::STAGES - 1; ++s) fetch(s, s, head[s]);
#pragma unroll
        for (int s = 0; s < S::STAGES - 2; ++s) land(head[s]);
        Heads &last = head[S::STAGES - 2];   // of the turn fetched last
        float mean_next, rstd_next;
        auto statistics = [&](int turn) {
            const bool live = turn * SLOTS + slot < count;
            mean_next = live ? __ldg(mean_at) : 0.0f;
            rstd_next = live ? __ldg(rstd_at) : 0.0f;
            mean_at += SLOTS;
            rstd_at += SLOTS;
        };
        statistics(0);
        F2 w[NV][P], gw[NV][P], gb[NV][P];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            ln_parameters<P>(a.weight, group * a.weight_stride + c0, (v * TPR + t) * VEC, h, 1.0f, w[v]);
#pragma unroll
            for (int k = 0; k < P; ++k) gw[v][k] = gb[v][k] = f2(0.0f);
        }
        for (int i = 0, stage = 0; i < turns; ++i) {
            const int ahead = i + S::STAGES - 1;                               // turn to fetch now
            const int into = stage == 0 ? S::STAGES - 1 : stage - 1;
            const bool live = i * SLOTS + slot < count;
            if constexpr (WHOLE) {
                fetch(ahead, into, last);
                copy_wait<S::STAGES - 1>();
            } else {
                copy_wait<S::STAGES - 2>();
                land(last);
                slot_sync<TPR>(slot);      // the rows of turn i are complete, and all are done with turn i - 1
                fetch(ahead, into, last);
            }
            const float rstd = rstd_next;
            const F2 minus = f2(-mean_next), scale = f2(rstd);
            statistics(i + 1);
            F2 along2 = f2(0.0f), level2 = f2(0.0f);
            F2 kept_x[KEEP ? NV : 1][P], kept_q[KEEP ? NV : 1][P];
            if (live) {   // (zeros beyond column h add nothing to any sum)
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    F2 dy[P], (&xc)[P] = kept_x[KEEP ? v : 0], (&q)[P] = kept_q[KEEP ? v : 0];
                    px.read(v, t, stage, xc);
                    pd.read(v, t, stage, dy);
#pragma unroll
                    for (int k = 0; k < P; ++k) {
                        xc[k] = add(xc[k], minus);
                        const F2 g = mul(dy[k], scale);
                        q[k] = mul(g, w[v][k]);
                        along2 = fma(q[k], xc[k], along2);
                        level2 = add(level2, q[k]);
                        gw[v][k] = fma(g, xc[k], gw[v][k]);
                        gb[v][k] = add(gb[v][k], dy[k]);
                    }
                }
            }
            if (a.dx) {
                float along[1] = {lo(along2) + hi(along2)}, level[1] = {lo(level2) + hi(level2)};
                slot_sums<TPR, S::WARPS, 1>(along, level, t, slot, box[flip]);
                if constexpr (WIDE) cluster_sums<1>(along, level, rank, parts, meet_rows[flip]);
                flip ^= 1;
                // !WHOLE: a finished row on its way out, in the place of its x once all have read that
                char *const result = KEEP ? px.ring + stage * S::STAGE_BYTES : ln_ring + S::RING_BYTES + slot * S::ROW_BYTES;
                if constexpr (!WHOLE && KEEP && S::WARPS == 1) __syncwarp();
                const F2 tilt = f2(-(along[0] * inv_h * rstd) * rstd), shift = f2(-level[0] * inv_h);
                if (live) {
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        const int c = (v * TPR + t) * VEC;
                        F2 (&xc)[P] = kept_x[KEEP ? v : 0], (&q)[P] = kept_q[KEEP ? v : 0];
                        if constexpr (!KEEP) {
                            px.read(v, t, stage, xc);
                            pd.read(v, t, stage, q);
                        }
#pragma unroll
                        for (int k = 0; k < P; ++k) {
                            if constexpr (!KEEP) {
                                xc[k] = add(xc[k], minus);
                                q[k] = rounded_mul(mul(q[k], scale), w[v][k]);
                            }
                            q[k] = fma(xc[k], tilt, add(q[k], shift));
                        }
                        if (c < h) LnChunk<T>::write(WHOLE ? reinterpret_cast<char *>(dx + c) : result + 16 + (v * TPR + t) * 16, q);
                    }
                }
                if constexpr (!WHOLE) {
                    slot_sync<TPR>(slot);
                    if (live) ln_store_row<T, NV, TPR>(dx, result, t, h);
                }
                dx += dx_step;
            }
            if constexpr (!WHOLE) {
                px.now += (uint32_t)x_step * (uint32_t)sizeof(T);
                pd.now += (uint32_t)dy_step * (uint32_t)sizeof(T);
            }
            stage = stage + 1 == S::STAGES ? 0 : stage + 1;
        }
        copy_wait<0>();
        if (u >= u_end) asm volatile("griddepcontrol.launch_dependents;");   // (the join may take its places)
        __syncthreads();   // the ring is free: for the sums of the slots and for the next group
        if (!a.dweight && !a.dbias) continue;
        // the slots' sums meet: lanes of one warp by shuffles, then halves of the CTA through shared memory
        if constexpr (TPR < 32) {
#pragma unroll
            for (int m = TPR; m < 32; m <<= 1)
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int k = 0; k < P; ++k) {
                        gw[v][k].v = add(gw[v][k], F2{__shfl_xor_sync(0xffffffffu, gw[v][k].v, m)}).v;
                        gb[v][k].v = add(gb[v][k], F2{__shfl_xor_sync(0xffffffffu, gb[v][k].v, m)}).v;
                    }
        }
        constexpr int TEAM = TPR < 32 ? 32 : TPR, TEAMS = S::THREADS / TEAM;   // threads that hold one set of sums
        const int team = threadIdx.x / TEAM, place = threadIdx.x % TEAM;
        F2 *meet = reinterpret_cast<F2 *>(ln_ring) + place;   // [TEAMS / 2][E pairs][TEAM]
#pragma unroll
        for (int half = TEAMS / 2; half >= 1; half /= 2) {
            if (team >= half && team < 2 * half) {
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int k = 0; k < P; ++k) {
                        meet[((team - half) * S::E + v * P + k) * TEAM] = gw[v][k];
                        meet[((team - half) * S::E + S::E / 2 + v * P + k) * TEAM] = gb[v][k];
                    }
            }
            __syncthreads();
            if (team < half) {
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int k = 0; k < P; ++k) {
                        gw[v][k] = add(gw[v][k], meet[(team * S::E + v * P + k) * TEAM]);
                        gb[v][k] = add(gb[v][k], meet[(team * S::E + S::E / 2 + v * P + k) * TEAM]);
                    }
            }
            __syncthreads();
        }
        if (team == 0 && (TPR >= 32 || place < TPR)) {
            const int64_t piece = (cta + group) * a.cols + c0;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    const int c = (v * TPR + t) * VEC + k;
                    const float sw = (k & 1) ? hi(gw[v][k / 2]) : lo(gw[v][k / 2]), sb = (k & 1) ? hi(gb[v][k / 2]) : lo(gb[v][k / 2]);
                    if (c < h) {
                        if (a.direct) {
                            if (a.dweight) store_grad(a.dweight, group * a.dweight_stride + c0 + c, a.grad_dtype, sw);
                            if (a.dbias) store_grad(a.dbias, group * a.dbias_stride + c0 + c, a.grad_dtype, sb);
                        } else {
                            a.part_w[piece + c] = sw;
                            a.part_b[piece + c] = sb;
                        }
                    }
                }
        }
    }
    if constexpr (WIDE) cluster_sync();   // none may leave while another still hands it sums
}

// Joins the pieces of a group (of all groups, where they share the gradient), in binary64 and in a fixed order, and
// rounds once to the gradient rows' type: 32 columns per CTA, four per thread, 32 threads per column.
__global__ void __launch_bounds__(256) ln_backward_join_kernel(const __grid_constant__ LnBackward a) {
    __shared__ double buf[8][32];
    const int group = blockIdx.y;
    const bool weight = blockIdx.z == 0;
    void *out = weight ? a.dweight : a.dbias;
    if (!out) return;   // (uniform; ends without the wait: it touches nothing)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, way = threadIdx.x >> 3;
    const int c = blockIdx.x * 32 + (threadIdx.x & 7) * 4;
    int64_t first = 0;   // pieces of the group: the parts of CTAs' shares
    int pieces = 0;
    if (a.rows > 0) {
        first = a.share.owner((int64_t)group * a.rows) + group;
        // (between two groups that meet where two shares meet lies a place without a piece: it holds zeros)
        const int end = a.shared ? a.groups : group + 1;
        pieces = (int)(a.share.owner((int64_t)end * a.rows - 1) + end - 1 - first) + 1;
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");   // the pieces are complete
    const float *p = (weight ? a.part_w : a.part_b) + (first + way) * a.cols + c;
    const int64_t step = (int64_t)32 * a.cols;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    if ((a.cols & 3) == 0 && c < a.cols) {
#pragma unroll 4
        for (int q = way; q < pieces; q += 32, p += step) {
            const float4 v = __ldcs(reinterpret_cast<const float4 *>(p));
            s[0] += (double)v.x; s[1] += (double)v.y; s[2] += (double)v.z; s[3] += (double)v.w;
        }
    } else {
        for (int q = way; q < pieces; q += 32, p += step)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (c + k < a.cols) s[k] += (double)__ldcs(p + k);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        s[k] += __shfl_xor_sync(0xffffffffu, s[k], 8);
        s[k] += __shfl_xor_sync(0xffffffffu, s[k], 16);
        if (lane < 8) buf[warp][lane * 4 + k] = s[k];
    }
    __syncthreads();
    const int cl = blockIdx.x * 32 + lane;
    if (warp == 0 && cl < a.cols) {
        const double t = ((buf[0][lane] + buf[1][lane]) + (buf[2][lane] + buf[3][lane])) + ((buf[4][lane] + buf[5][lane]) + (buf[6][lane] + buf[7][lane]));
        store_grad(out, group * (weight ? a.dweight_stride : a.dbias_stride) + cl, a.grad_dtype, (float)t);
    }
}

struct LnPlan {
    LnShare share;
    int64_t pieces;
    bool direct;
};

struct LnPlanner {
    int groups;
    int64_t rows;
    int parts;
    bool shared;
    template <int TPR, int E, int SLOTS, int MINB>
    LnPlan operator()() const {
        const int64_t total = (int64_t)groups * rows;
        const int resident = ln_resident(MINB, parts);
        LnPlan p;
        // one CTA (or cluster) per group and no second launch, which costs the host 2 us as well: up to four turns
        // (4 rows of 8192 binary32 columns, eight groups: 13.6 us, 15.8 us shared and joined; one group 13.5 and
        // 10.2 us; 16 rows of 768: 6.8 and 5.1 us, 32 rows 9.3 and 5.1 us); or with so many groups that their CTAs
        // fill the GPU several times over anyway
        p.direct = !shared && (rows <= 4 * SLOTS || (groups >= 4 * resident && rows <= (int64_t)SLOTS * LN_SUM_ROWS));
        p.share = p.direct ? LnShare{0, 0, rows, groups} : ln_share(total, SLOTS, resident, LN_SUM_ROWS, false);
        p.pieces = p.direct ? 0 : p.share.ctas + groups;
        return p;
    }
};

static LnPlan ln_plan(int groups, int64_t rows, int cols, bool shared) {
    const LnPlanner planner{groups, rows, ln_parts(cols), shared};
    return planner.parts > 1 ? ln_wide_shape(planner) : ln_backward_shape(cols, planner);
}

size_t layer_norm_workspace(int groups, int64_t rows, int cols, bool shared) {
    if (rows == 0) return 0;
    return sizeof(float) * 2 * (size_t)std::max<int64_t>(ln_plan(groups, rows, cols, shared).pieces, groups) * (size_t)cols;
}

template <typename T, bool WHOLE, bool WIDE = false>
struct LnBackwardLaunch {
    LnBackward a;
    cudaStream_t st;
    template <int TPR, int E, int SLOTS, int MINB>
    cudaError_t operator()() {
        constexpr int NV = E / LnChunk<T>::VEC;
        using S = LnShape<T, WHOLE, NV, TPR, SLOTS, MINB, 1, 2>;
        static_assert(S::THREADS <= 32 || S::RING_BYTES >= S::THREADS * S::E * 4, "half the CTA's column sums meet in the ring");
        static std::atomic<uint64_t> allowed{0};
        const auto kernel = ln_backward_kernel<T, WHOLE, WIDE, NV, TPR, SLOTS, MINB>;
        constexpr int SMEM = S::RING_BYTES + S::RESULT_BYTES;
        const cudaError_t e = ln_allow_smem(kernel, SMEM, allowed);
        if (e != cudaSuccess) return e;
        return ln_launch(kernel, a, a.share.ctas, WIDE ? ln_parts(a.cols) : 1, S::THREADS, SMEM, st);
    }
};

template <typename T, bool WHOLE>
static cudaError_t backward_rows(const LnBackward &a, cudaStream_t st) {
    if (ln_parts(a.cols) > 1) return ln_wide_shape(LnBackwardLaunch<T, WHOLE, true>{a, st});
    return ln_backward_shape(a.cols, LnBackwardLaunch<T, WHOLE>{a, st});
}

cudaError_t launch_layer_norm_backward(LnBackward a, int dtype, cudaStream_t st) {
    if (a.rows > 0) {
        const int esz = dtype == 0 ? 4 : 2;
        const bool whole = ln_whole(a.x, a.x_row, a.x_group, a.rows, a.groups, a.cols, esz) &&
                           ln_whole(a.dy, a.dy_row, a.dy_group, a.rows, a.groups, a.cols, esz) &&
                           (!a.dx || ln_whole(a.dx, a.dx_row, a.dx_group, a.rows, a.groups, a.cols, esz));
        const LnPlan p = ln_plan(a.groups, a.rows, a.cols, a.shared != 0);
        if (a.shared && (a.dweight || a.dbias)) {   // the places without a piece (all of it: 3 us of 107, 32 x 4096 of 768)
            const cudaError_t e = cudaMemsetAsync(a.part_w, 0, layer_norm_workspace(a.groups, a.rows, a.cols, true), st);
            if (e != cudaSuccess) return e;
        }
        a.share = p.share;
        a.direct = p.direct;
        a.part_cols = ln_part_cols(a.cols);
        const cudaError_t e = dtype == 0 ? whole ? backward_rows<float, true>(a, st) : backward_rows<float, false>(a, st)
                              : whole    ? backward_rows<__nv_bfloat16, true>(a, st)
                                         : backward_rows<__nv_bfloat16, false>(a, st);
        if (e != cudaSuccess) return e;
    }
    if ((a.dweight || a.dbias) && !a.direct) {
        // launched while the rows' kernel ends; it waits for that kernel's end before it reads
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((a.cols + 31) / 32, a.shared ? 1 : a.groups, 2);
        cfg.blockDim = dim3(256);
        cfg.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = a.rows > 0 ? 1 : 0;
        return cudaLaunchKernelEx(&cfg, ln_backward_join_kernel, a);
    }
    return cudaSuccess;
}

}  // namespace liec

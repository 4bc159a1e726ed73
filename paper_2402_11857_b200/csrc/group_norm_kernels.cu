// Group normalisation with an activation over N workers' images, channels last, forward and backward.  Images are
// cut into parts of their pixels; the parts' sums per channel go through the workspace.
#include "group_norm.cuh"

namespace liec {

struct GnPlace {   // what a CTA and its thread work on
    int64_t image, p0, n;   // first pixel of the part and their number
    int worker, sample, tile, part, chunk, lane, lanes, c;
    bool live;
    __device__ __forceinline__ GnPlace(const GnArgs &a, int vec) {
        int64_t b = blockIdx.x;
        part = (int)(b % a.parts);
        b /= a.parts;
        tile = (int)(b % a.tiles);
        image = b / a.tiles;
        worker = (int)(image / a.samples);
        sample = (int)(image - (int64_t)worker * a.samples);
        p0 = part * a.part_pixels;
        n = max((int64_t)0, min(a.part_pixels, a.pixels - p0));
        chunk = threadIdx.x % a.tile_chunks;
        lane = threadIdx.x / a.tile_chunks;
        lanes = GN_THREADS / a.tile_chunks;
        c = (tile * a.tile_chunks + chunk) * vec;
        live = lane < lanes && c < (a.channels + CK_BLOCK - 1) / CK_BLOCK * CK_BLOCK;
    }
};

// The channels' sums of all pixel lanes, in a fixed order: two per channel of the tile, through `box`.
template <int VEC>
__device__ __forceinline__ void gn_channel_sums(const GnPlace &at, int tile_chunks, const F2 (&s)[VEC / 2], const F2 (&t)[VEC / 2], float *box) {
    const int width = tile_chunks * VEC;
    if (at.live) {
#pragma unroll
        for (int k = 0; k < VEC / 2; ++k) {
            float *b = box + (at.lane * 2) * width + at.chunk * VEC + 2 * k;
            b[0] = lo(s[k]);
            b[1] = hi(s[k]);
            b[width] = lo(t[k]);
            b[width + 1] = hi(t[k]);
        }
    }
    __syncthreads();
    for (int q = threadIdx.x; q < 2 * width; q += GN_THREADS) {
        float v = 0.0f;
        for (int l = 0; l < at.lanes; ++l) v += box[l * 2 * width + q];
        box[q] = v;   // (own column: nobody else reads it)
    }
    __syncthreads();
}

// Mean and squares around it of every channel of a part, about the part's first pixel.
template <typename T>
__global__ void __launch_bounds__(GN_THREADS) gn_moments_kernel(const __grid_constant__ GnArgs a) {
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    __shared__ float box[GN_THREADS * 2 * VEC];
    const GnPlace at(a, VEC);
    F2 s[P] = {}, t[P] = {};
    if (at.live && at.n > 0) {
        const GnFromX<T> x(a, at.worker, at.sample, at.p0);
        F2 minus[P], d[P];
        const F2 none[P] = {};
        GnFromX<T>::centred(x.load(0, at.c, a.channels), none, minus);
#pragma unroll
        for (int k = 0; k < P; ++k) minus[k] = f2(-lo(minus[k]), -hi(minus[k]));
        for (int64_t p = at.lane; p < at.n; p += at.lanes) {
            GnFromX<T>::centred(x.load(p, at.c, a.channels), minus, d);
#pragma unroll
            for (int k = 0; k < P; ++k) {
                s[k] = add(s[k], d[k]);
                t[k] = fma(d[k], d[k], t[k]);
            }
        }
    }
    gn_channel_sums<VEC>(at, a.tile_chunks, s, t, box);
    const int width = a.tile_chunks * VEC, c0 = at.tile * width;
    float *out = a.part + (at.image * a.parts + at.part) * 2 * a.channels;
    const GnFromX<T> x(a, at.worker, at.sample, at.p0);
    for (int q = threadIdx.x; q < width && c0 + q < a.channels; q += GN_THREADS) {
        const float n = (float)at.n, mean = at.n > 0 ? box[q] / n : 0.0f;
        out[c0 + q] = at.n > 0 ? (float)x.row[c0 + q] + mean : 0.0f;
        out[a.channels + c0 + q] = at.n > 0 ? fmaxf(__fmaf_rn(-box[q], mean, box[width + q]), 0.0f) : 0.0f;
    }
}

// Joins a group's channels and parts: a warp per group, binary64, in a fixed order.
__global__ void __launch_bounds__(GN_THREADS) gn_statistics_kernel(const __grid_constant__ GnArgs a) {
    const int64_t g = ((int64_t)blockIdx.x * GN_THREADS + threadIdx.x) / 32, images = (int64_t)a.workers * a.samples;
    if (g >= images * a.groups) return;
    const int lane = threadIdx.x & 31, width = a.channels / a.groups, entries = width * a.parts;
    const int64_t image = g / a.groups;
    const float *part = a.part + image * a.parts * 2 * a.channels + (g - image * a.groups) * width;
    const double n = (double)a.pixels * width;
    double s = 0.0, t = 0.0;
    for (int i = lane; i < entries; i += 32) {
        const int q = i / width;
        s += (double)min(a.part_pixels, a.pixels - q * a.part_pixels) * part[(int64_t)q * 2 * a.channels + i % width];
    }
    const double mean = warp_sum(s) / n;
    for (int i = lane; i < entries; i += 32) {
        const int q = i / width;
        const float *at = part + (int64_t)q * 2 * a.channels + i % width;
        const double off = (double)at[0] - mean;
        t += (double)at[a.channels] + (double)min(a.part_pixels, a.pixels - q * a.part_pixels) * off * off;
    }
    const double var = warp_sum(t) / n;
    if (lane == 0) {
        a.mean[g] = (float)mean;
        a.rstd[g] = (float)(1.0 / sqrt(var + (double)a.eps));
    }
}

template <typename T, int ACT, bool COMPRESS>
__global__ void __launch_bounds__(GN_THREADS) gn_apply_kernel(const __grid_constant__ GnArgs a) {
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    const GnPlace at(a, VEC);
    if (!at.live) return;
    const GnFromX<T> x(a, at.worker, at.sample, at.p0);
    T *y = static_cast<T *>(a.y) + at.worker * a.y_worker + at.sample * a.y_sample + at.p0 * a.y_pixel;
    GnChannels<P> ch;
    ch.read(a, at.worker, at.image, at.c);
    const int64_t row0 = at.image * a.pixels + at.p0;
    for (int64_t p = at.lane; p < at.n; p += at.lanes) {
        const uint4 raw = x.load(p, at.c, a.channels);
        F2 d[P];
        if constexpr (COMPRESS) {
            LnChunk<T>::read(raw, d);
            gn_compress<T>(a, d, row0 + p, at.c);
        }
        GnFromX<T>::centred(raw, ch.minus, d);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            d[k] = gn_act<T, ACT>(fma(d[k], ch.scale[k], ch.bias[k]));
        }
        store_chunk(y + p * a.y_pixel, at.c, a.channels, d);
    }
}

// Backward: sums of dz and dz xh of every channel of a part.
template <typename T, typename X, int ACT>
__global__ void __launch_bounds__(GN_THREADS) gn_slopes_kernel(const __grid_constant__ GnArgs a) {
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    __shared__ float box[GN_THREADS * 2 * VEC];
    const GnPlace at(a, VEC);
    F2 s[P] = {}, t[P] = {};
    if (at.live) {
        const X x(a, at.worker, at.sample, at.p0);
        const T *dy = static_cast<const T *>(a.dy) + at.worker * a.y_worker + at.sample * a.y_sample + at.p0 * a.y_pixel;
        GnChannels<P> ch;
        ch.read(a, at.worker, at.image, at.c);
        for (int64_t p = at.lane; p < at.n; p += at.lanes) {
            const typename X::Raw raw = x.load(p, at.c, a.channels);
            F2 d[P], g[P];
            X::centred(raw, ch.minus, d);
            LnChunk<T>::read(load_chunk(dy + p * a.y_pixel, at.c, a.channels), g);
            gn_slope<T, ACT, X>(a, at.worker, at.image, at.c, ch, raw, d, g, g);
#pragma unroll
            for (int k = 0; k < P; ++k) {
                s[k] = add(s[k], g[k]);
                t[k] = fma(g[k], d[k], t[k]);
            }
        }
    }
    gn_channel_sums<VEC>(at, a.tile_chunks, s, t, box);
    const int width = a.tile_chunks * VEC, c0 = at.tile * width;
    float *out = a.part + (at.image * a.parts + at.part) * 2 * a.channels;
    for (int q = threadIdx.x; q < width && c0 + q < a.channels; q += GN_THREADS) {
        out[c0 + q] = box[q];
        out[a.channels + c0 + q] = box[width + q] * a.rstd[at.image * a.groups + (c0 + q) / (a.channels / a.groups)];
    }
}

// Per group: r mean(dz w) and r^2 mean(dz w xh).
__global__ void __launch_bounds__(GN_THREADS) gn_levels_kernel(const __grid_constant__ GnArgs a) {
    const int64_t g = ((int64_t)blockIdx.x * GN_THREADS + threadIdx.x) / 32, images = (int64_t)a.workers * a.samples;
    if (g >= images * a.groups) return;
    const int lane = threadIdx.x & 31, width = a.channels / a.groups, entries = width * a.parts;
    const int64_t image = g / a.groups;
    const int c0 = (int)(g - image * a.groups) * width, worker = (int)(image / a.samples);
    const float *part = a.part + image * a.parts * 2 * a.channels + c0;
    double s = 0.0, t = 0.0;
    for (int i = lane; i < entries; i += 32) {
        const int q = i / width, c = i % width;
        const double w = a.weight ? (double)a.weight[worker * a.weight_stride + c0 + c] : 1.0;
        const float *at = part + (int64_t)q * 2 * a.channels + c;
        s += w * at[0];
        t += w * at[a.channels];
    }
    s = warp_sum(s);
    t = warp_sum(t);
    if (lane == 0) {
        const double n = (double)a.pixels * width, r = (double)a.rstd[g];
        a.level[2 * g] = (float)(r * s / n);
        a.level[2 * g + 1] = (float)(r * r * t / n);
    }
}

// dx = A dz - r mean(dz w) - d r^2 mean(dz w xh)
template <typename T, typename X, int ACT>
__global__ void __launch_bounds__(GN_THREADS) gn_dx_kernel(const __grid_constant__ GnArgs a) {
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    const GnPlace at(a, VEC);
    if (!at.live || at.c >= a.channels) return;
    const X x(a, at.worker, at.sample, at.p0);
    const T *dy = static_cast<const T *>(a.dy) + at.worker * a.y_worker + at.sample * a.y_sample + at.p0 * a.y_pixel;
    T *dx = static_cast<T *>(a.dx) + at.worker * a.dx_worker + at.sample * a.dx_sample + at.p0 * a.dx_pixel;
    GnChannels<P> ch;
    ch.read(a, at.worker, at.image, at.c);
    F2 level[P], along[P];
#pragma unroll
    for (int k = 0; k < 2 * P; ++k) {
        const int64_t g = at.image * a.groups + min(at.c + k, a.channels - 1) / (a.channels / a.groups);
        GnChannels<P>::set(level[k / 2], k % 2, -a.level[2 * g]);
        GnChannels<P>::set(along[k / 2], k % 2, -a.level[2 * g + 1]);
    }
    for (int64_t p = at.lane; p < at.n; p += at.lanes) {
        const typename X::Raw raw = x.load(p, at.c, a.channels);
        F2 d[P], g[P];
        X::centred(raw, ch.minus, d);
        LnChunk<T>::read(load_chunk(dy + p * a.y_pixel, at.c, a.channels), g);
        gn_slope<T, ACT, X>(a, at.worker, at.image, at.c, ch, raw, d, g, g);
#pragma unroll
        for (int k = 0; k < P; ++k) d[k] = fma(g[k], ch.scale[k], fma(d[k], along[k], level[k]));
        store_chunk(dx + p * a.dx_pixel, at.c, a.channels, d);
    }
}

// dw and db: a worker's images and parts (all workers', where they share the gradient) in binary64, rounded once.  A
// warp takes 32 channels, eight warps share the parts.
__global__ void __launch_bounds__(GN_THREADS) gn_join_kernel(const __grid_constant__ GnArgs a) {
    __shared__ double box[GN_THREADS / 32][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, worker = blockIdx.y, c = blockIdx.x * 32 + lane;
    const bool weight = blockIdx.z == 0;
    void *out = weight ? a.dweight : a.dbias;
    if (!out) return;
    const int64_t rows = a.pixels == 0 ? 0 : (int64_t)(a.shared ? a.workers : 1) * a.samples * a.parts, first = a.shared ? 0 : (int64_t)worker * a.samples * a.parts;
    double s = 0.0;
    if (c < a.channels)
        for (int64_t i = warp; i < rows; i += GN_THREADS / 32) s += (double)a.part[((first + i) * 2 + (weight ? 1 : 0)) * a.channels + c];
    box[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < a.channels) {
        for (int w = 1; w < GN_THREADS / 32; ++w) s += box[w][lane];
        const int64_t at = worker * (weight ? a.dweight_stride : a.dbias_stride) + c;
        if (a.grad_dtype == LIEC_F32) static_cast<float *>(out)[at] = (float)s;
        else static_cast<__nv_bfloat16 *>(out)[at] = __float2bfloat16_rn((float)s);
    }
}

// ---- launches --------------------------------------------------------------------------------------------

static void gn_plan(GnArgs &a, int vec) {
    const int chunks = (int)(ck_cols(a.channels) / vec);
    a.tile_chunks = chunks < 64 ? chunks : 64;
    a.tiles = (chunks + a.tile_chunks - 1) / a.tile_chunks;
    const int lanes = GN_THREADS / a.tile_chunks;
    const int64_t images = (int64_t)a.workers * a.samples, places = images * a.tiles;
    const int64_t most = (a.pixels + 8 * lanes - 1) / (8 * lanes), want = (148 * 16 + places - 1) / std::max<int64_t>(places, 1);
    const int64_t parts = std::max<int64_t>(1, std::min(most, want));
    a.part_pixels = std::max<int64_t>(1, (a.pixels + parts - 1) / parts);
    a.parts = (int)std::max<int64_t>(1, (a.pixels + a.part_pixels - 1) / a.part_pixels);
}

static size_t gn_streamed_workspace(GnArgs a, int dtype, bool backward) {
    gn_plan(a, dtype == 0 ? 4 : 8);
    const size_t images = (size_t)a.workers * a.samples;
    return sizeof(float) * (images * a.parts * 2 * a.channels + (backward ? images * a.groups * 2 : 0));
}

size_t group_norm_workspace(const GnArgs &a, int dtype, bool backward) {
    size_t need = 0;
    for (int checkpoint = 0; checkpoint < (backward ? 2 : 1); ++checkpoint) {   // (a descriptor does not say which)
        GnArgs b = a;
        int smem;
        const bool resident = gn_resident_plan(b, dtype, backward, checkpoint != 0, smem);
        need = std::max(need, !resident ? gn_streamed_workspace(a, dtype, backward) : backward ? sizeof(float) * a.workers * a.samples * 2 * (size_t)a.channels : 0);
    }
    return need;
}

static bool gn_whole(const GnArgs &a, int dtype, const void *p, int64_t pixel, int64_t sample, int64_t worker) {
    uint64_t bits = reinterpret_cast<uintptr_t>(p);
    const uint64_t size = dtype == 0 ? 4 : 2;
    if (a.pixels > 1) bits |= (uint64_t)pixel * size;
    if (a.samples > 1) bits |= (uint64_t)sample * size;
    if (a.workers > 1) bits |= (uint64_t)worker * size;
    return (bits & 15u) == 0;
}

static unsigned gn_group_ctas(const GnArgs &a) {
    return (unsigned)(((int64_t)a.workers * a.samples * a.groups * 32 + GN_THREADS - 1) / GN_THREADS);
}

template <typename T>
struct GnForwardLaunch {
    const GnArgs &a;
    unsigned ctas;
    cudaStream_t st;
    template <int ACT>
    cudaError_t operator()() {
        gn_moments_kernel<T><<<ctas, GN_THREADS, 0, st>>>(a);
        gn_statistics_kernel<<<gn_group_ctas(a), GN_THREADS, 0, st>>>(a);
        if (a.q) gn_apply_kernel<T, ACT, true><<<ctas, GN_THREADS, 0, st>>>(a);
        else gn_apply_kernel<T, ACT, false><<<ctas, GN_THREADS, 0, st>>>(a);
        return cudaGetLastError();
    }
};

cudaError_t launch_group_norm_forward(GnArgs a, int dtype, cudaStream_t st) {
    if (a.samples == 0 || a.pixels == 0) return cudaSuccess;
    int smem;
    if (gn_resident_plan(a, dtype, false, false, smem)) {
        a.whole = gn_whole(a, dtype, a.x, a.x_pixel, a.x_sample, a.x_worker);
        a.whole_out = a.channels % (dtype == 0 ? 4 : 8) == 0 && gn_whole(a, dtype, a.y, a.y_pixel, a.y_sample, a.y_worker);
        return gn_resident_forward(a, dtype, smem, st);
    }
    gn_plan(a, dtype == 0 ? 4 : 8);
    const unsigned ctas = (unsigned)((int64_t)a.workers * a.samples * a.tiles * a.parts);
    return dtype == 0 ? gn_for_act(a.act, GnForwardLaunch<float>{a, ctas, st}) : gn_for_act(a.act, GnForwardLaunch<__nv_bfloat16>{a, ctas, st});
}

template <typename T, typename X>
struct GnBackwardLaunch {
    const GnArgs &a;
    unsigned ctas;
    cudaStream_t st;
    template <int ACT>
    cudaError_t operator()() {
        gn_slopes_kernel<T, X, ACT><<<ctas, GN_THREADS, 0, st>>>(a);
        if (a.dx) {
            gn_levels_kernel<<<gn_group_ctas(a), GN_THREADS, 0, st>>>(a);
            gn_dx_kernel<T, X, ACT><<<ctas, GN_THREADS, 0, st>>>(a);
        }
        return cudaGetLastError();
    }
};

template <typename T>
static cudaError_t gn_backward(const GnArgs &a, unsigned ctas, cudaStream_t st) {
    return a.x ? gn_for_act(a.act, GnBackwardLaunch<T, GnFromX<T>>{a, ctas, st}) : gn_for_act(a.act, GnBackwardLaunch<T, GnFromCheckpoint<T>>{a, ctas, st});
}

cudaError_t launch_group_norm_backward(GnArgs a, int dtype, cudaStream_t st) {
    int smem;
    if (a.samples == 0 || a.pixels == 0) {
        a.parts = 1;
    } else if (gn_resident_plan(a, dtype, true, !a.x, smem)) {
        a.whole = gn_whole(a, dtype, a.dy, a.y_pixel, a.y_sample, a.y_worker) && (!a.x || gn_whole(a, dtype, a.x, a.x_pixel, a.x_sample, a.x_worker));
        a.whole_out = a.channels % (dtype == 0 ? 4 : 8) == 0 && gn_whole(a, dtype, a.dx, a.dx_pixel, a.dx_sample, a.dx_worker);
        const cudaError_t e = gn_resident_backward(a, dtype, smem, st);
        if (e != cudaSuccess) return e;
        a.parts = 1;   // (the cluster's parts are one by now)
    } else {
        gn_plan(a, dtype == 0 ? 4 : 8);
        a.level = a.part + (int64_t)a.workers * a.samples * a.parts * 2 * a.channels;
        const unsigned ctas = (unsigned)((int64_t)a.workers * a.samples * a.tiles * a.parts);
        const cudaError_t e = dtype == 0 ? gn_backward<float>(a, ctas, st) : gn_backward<__nv_bfloat16>(a, ctas, st);
        if (e != cudaSuccess) return e;
    }
    if (a.dweight || a.dbias) {
        gn_join_kernel<<<dim3((a.channels + 31) / 32, a.shared ? 1 : a.workers, 2), GN_THREADS, 0, st>>>(a);
        return cudaGetLastError();
    }
    return cudaSuccess;
}

}  // namespace liec

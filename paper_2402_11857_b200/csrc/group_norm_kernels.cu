// Group normalisation with an activation over N workers' images, channels last, forward and backward: images of any size,
// read twice.  They are cut into tiles of channels and parts of pixels; a CTA's threads walk down the pixels of its part, and
// the parts' sums per channel go through the workspace.  The second reading takes the CTAs in the opposite order: what was
// read last is still in the L2 cache.
#include "group_norm.cuh"

namespace liec {

template <int VEC>
struct GnPlace {   // what a CTA and its thread work on
    int64_t image, p0, turns;   // the thread's first pixel and its chunks
    int worker, sample, part, chunk, lane, lanes, c, c0;
    __device__ __forceinline__ GnPlace(const GnArgs &a, bool backwards) {
        const uint32_t block = backwards ? gridDim.x - 1 - blockIdx.x : blockIdx.x, unit = block / (uint32_t)a.parts, picture = unit / (uint32_t)a.tiles;
        part = (int)(block - unit * a.parts);
        image = picture;
        worker = (int)(picture / (uint32_t)a.samples);
        sample = (int)(picture - (uint32_t)worker * a.samples);
        lane = (int)(threadIdx.x / (uint32_t)a.tile_chunks);
        chunk = (int)threadIdx.x - lane * a.tile_chunks;
        lanes = (int)(GN_THREADS / (uint32_t)a.tile_chunks);
        c0 = (int)(unit - picture * a.tiles) * a.tile_chunks * VEC;
        c = c0 + chunk * VEC;
        p0 = part * a.part_pixels + lane;
        const int64_t end = min((part + 1) * a.part_pixels, a.pixels);
        const bool live = lane < lanes && c < (a.channels + CK_BLOCK - 1) / CK_BLOCK * CK_BLOCK;
        turns = live && p0 < end ? (end - p0 + lanes - 1) / lanes : 0;
    }
};

// Two sums per channel over all pixel lanes, in a fixed order: out[which][channel].
template <int VEC>
__device__ __forceinline__ void gn_channel_sums(const GnPlace<VEC> &at, int tile_chunks, const F2 (&s)[VEC / 2], const F2 (&t)[VEC / 2], float *box) {
    const int width = tile_chunks * VEC;
    if (at.lane < at.lanes) {
        float4 *b = reinterpret_cast<float4 *>(box + at.lane * 2 * width + at.chunk * VEC);
#pragma unroll
        for (int k = 0; k < VEC / 2; k += 2) {
            b[k / 2] = make_float4(lo(s[k]), hi(s[k]), lo(s[k + 1]), hi(s[k + 1]));
            b[width / 4 + k / 2] = make_float4(lo(t[k]), hi(t[k]), lo(t[k + 1]), hi(t[k + 1]));
        }
    }
    __syncthreads();
    for (int q = threadIdx.x; q < 2 * width; q += GN_THREADS) {
        float v = 0.0f;
#pragma unroll 4
        for (int l = 0; l < at.lanes; ++l) v += box[l * 2 * width + q];
        box[q] = v;   // (own column: nobody else reads it)
    }
    __syncthreads();
}

__device__ __forceinline__ void gn_wait_for_kernel_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Sums over all pixel lanes of a column of N boxes, in a fixed order.
template <int N>
__device__ __forceinline__ void gn_column_sums(const float *box, int lanes, int width, int column, float (&sum)[N]) {
    float v[N][4] = {};
    int l = 0;
#pragma unroll 2
    for (; l + 4 <= lanes; l += 4)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < N; ++n) v[n][i] += box[(n * lanes + l + i) * width + column];
    for (; l < lanes; ++l)
#pragma unroll
        for (int n = 0; n < N; ++n) v[n][0] += box[(n * lanes + l) * width + column];
#pragma unroll
    for (int n = 0; n < N; ++n) sum[n] = (v[n][0] + v[n][1]) + (v[n][2] + v[n][3]);
}

// What the forward pass knows of a channel in a part of an image: its mean in two parts, the second what the first, a binary32
// number, leaves; and the squares around the mean.
constexpr int GN_FORWARD_PARTS = 3, GN_BACKWARD_PARTS = 2;

// A thread's entries about their own mean; then all threads' about one number per channel, their mean as far as it is known then.
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(GN_THREADS, WHOLE ? 4 : 3) gn_moments_kernel(const __grid_constant__ GnArgs a) {
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    extern __shared__ __align__(16) char gn_ring[];
    __shared__ __align__(16) float box[GN_THREADS * 2 * VEC];
    __shared__ __align__(16) float about[GN_THREADS * VEC];
    const GnPlace<VEC> at(a, false);
    const bool in = at.turns > 0 && at.c < a.channels;
    GnFromX<T, WHOLE> x(a, at.worker, at.sample, at.p0, at.lanes, at.c);
    GnMoments<P> m;
    if (in) m.template start<T>(load_chunk(x.row - at.c, at.c, a.channels));
    int done = 0;
    auto take = [&](uint4 chunk) {
        F2 v[P];
        LnChunk<T>::read(chunk, v);
        m.take(v);
    };
    auto after = [&](int n) {
        done += n;
        if (done == 4 || done == 16) m.move((float)done, done == 4 ? 0.25f : 0.0625f);
    };
    if constexpr (WHOLE) {
        const GnRing<16> ring(gn_ring);
        if (in) gn_ring_turns((int)at.turns, [&](int place) { ring.copy(place, x.row); x.next(); }, [&](int place, int) { take(ring.read(place)); }, after);
    } else {
        gn_turns<2>(at.turns, [&](int u) { return x.load(u); }, [&](int u, const typename GnFromX<T, WHOLE>::Raw &raw) { take(x.keep(raw, u)); }, [&](int n) { x.advance(n); after(n); });
    }
    const int width = a.tile_chunks * VEC;
    const float n = (float)at.turns, inverse = 1.0f / (float)(min((at.part + 1) * a.part_pixels, a.pixels) - at.part * a.part_pixels);
    float *out = a.part + (at.image * a.parts + at.part) * GN_FORWARD_PARTS * a.channels + at.c0;
    auto put = [&](int plane, auto &&value) {
        float4 *to = reinterpret_cast<float4 *>(box + (plane * at.lanes + at.lane) * width + at.chunk * VEC);
#pragma unroll
        for (int k = 0; k < P; k += 2) {
            const F2 v = value(k), w = value(k + 1);
            to[k / 2] = make_float4(lo(v), hi(v), lo(w), hi(w));
        }
    };
    if (at.lane < at.lanes) put(0, [&](int k) { return m.whole(k, n); });
    __syncthreads();
    for (int q = threadIdx.x; q < width; q += GN_THREADS) {
        float sum[1];
        gn_column_sums(box, at.lanes, width, q, sum);
        about[q] = sum[0] * inverse;
        if (at.c0 + q < a.channels) out[q] = about[q];
    }
    __syncthreads();
    if (at.lane < at.lanes) {
#pragma unroll
        for (int k = 0; k < P; ++k) m.move_to(k, f2(about[at.chunk * VEC + 2 * k], about[at.chunk * VEC + 2 * k + 1]), n);
        put(0, [&](int k) { return m.s[k]; });
        put(1, [&](int k) { return m.t[k]; });
    }
    __syncthreads();
    for (int q = threadIdx.x; q < width && at.c0 + q < a.channels; q += GN_THREADS) {
        float sum[2];
        gn_column_sums(box, at.lanes, width, q, sum);
        const float left = sum[0] * inverse;
        out[a.channels + q] = left;
        out[2 * a.channels + q] = fmaxf(__fmaf_rn(-sum[0], left, sum[1]), 0.0f);
    }
}

// f(image, group, lane) with LANES threads per group of an image.
template <int LANES, typename F>
__device__ __forceinline__ void gn_per_group(const GnArgs &a, F &&f) {
    const int64_t g = ((int64_t)blockIdx.x * GN_THREADS + threadIdx.x) / LANES;
    const uint32_t image = (uint32_t)(g / a.groups);
    f(g < (int64_t)a.workers * a.samples * a.groups, image, (uint32_t)(g - (int64_t)image * a.groups), (uint32_t)threadIdx.x % LANES);
}
template <int LANES>
__device__ __forceinline__ double gn_sum_lanes(double v) {
#pragma unroll
    for (int m = (LANES < 32 ? LANES : 32) / 2; m >= 1; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    if constexpr (LANES == GN_THREADS) {   // a CTA
        __shared__ double box[GN_THREADS / 32];
        __syncthreads();
        if (threadIdx.x % 32 == 0) box[threadIdx.x / 32] = v;
        __syncthreads();
        v = 0.0;
#pragma unroll
        for (int w = 0; w < GN_THREADS / 32; ++w) v += box[w];
    }
    return v;
}

// Joins a group's channels and parts, in binary64 and in a fixed order: about one of their means, which is one of `entries`, so the squares about
// it are at most that many times those about the mean of all.
template <int LANES>
__global__ void __launch_bounds__(GN_THREADS) gn_statistics_kernel(const __grid_constant__ GnArgs a) {
    gn_wait_for_kernel_before();
    gn_per_group<LANES>(a, [&](bool live, uint32_t image, uint32_t group, uint32_t lane) {
        const uint32_t width = (uint32_t)a.channels / (uint32_t)a.groups, entries = live ? width * a.parts : 0u;
        const float *part = a.part + (int64_t)image * a.parts * GN_FORWARD_PARTS * a.channels + group * width;
        const double n = (double)a.pixels * width, about = live ? (double)part[0] : 0.0;
        const double pixels = (double)a.part_pixels, last_pixels = (double)(a.pixels - (a.parts - 1) * a.part_pixels);
        double s = 0.0, t = 0.0;
        constexpr uint32_t BATCH = 4;   // entries whose loads are under way together
        for (uint32_t first = lane; first < entries; first += BATCH * LANES) {
            float mean[BATCH], left[BATCH], squares[BATCH];
            uint32_t q[BATCH];
#pragma unroll
            for (uint32_t k = 0; k < BATCH; ++k) {
                const uint32_t i = first + k * LANES;
                q[k] = i / width;
                if (i < entries) {
                    const float *at = part + (int64_t)q[k] * GN_FORWARD_PARTS * a.channels + (i - q[k] * width);
                    mean[k] = at[0];
                    left[k] = at[a.channels];
                    squares[k] = at[2 * a.channels];
                }
            }
#pragma unroll
            for (uint32_t k = 0; k < BATCH; ++k)
                if (first + k * LANES < entries) {
                    const double d = ((double)mean[k] - about) + (double)left[k], count = q[k] + 1 == (uint32_t)a.parts ? last_pixels : pixels;
                    s += count * d;
                    t += (double)squares[k] + count * d * d;
                }
        }
        s = gn_sum_lanes<LANES>(s);
        t = gn_sum_lanes<LANES>(t);
        if (live && lane == 0) {
            const double var = (t - s * s / n) / n;
            a.mean[(int64_t)image * a.groups + group] = (float)(about + s / n);
            a.rstd[(int64_t)image * a.groups + group] = 1.0f / sqrtf((var < 0.0 ? 0.0f : (float)var) + a.eps);   // (NaN stays)
        }
    });
}

template <typename T, bool WHOLE, int ACT, bool COMPRESS>
__global__ void __launch_bounds__(GN_THREADS, 3) gn_apply_kernel(const __grid_constant__ GnArgs a) {
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    extern __shared__ __align__(16) char gn_ring[];
    const GnPlace<VEC> at(a, true);
    GnFromX<T, WHOLE> x(a, at.worker, at.sample, at.p0, at.lanes, at.c);
    T *y = static_cast<T *>(a.y) + at.worker * a.y_worker + at.sample * a.y_sample + at.p0 * a.y_pixel;
    const int64_t y_step = at.lanes * a.y_pixel;
    GnCompressor<T> checkpoint(a, at.image * a.pixels + at.p0, at.lanes, at.c);
    gn_wait_for_kernel_before();
    if (at.turns == 0) return;
    GnChannels<P> ch;
    ch.read(a, at.worker, at.image, at.c);
    auto take = [&](uint4 chunk, int u) {
        if constexpr (COMPRESS) checkpoint.store(u, chunk);
        F2 d[P];
        GnFromX<T, WHOLE>::centred(chunk, ch.minus, d);
#pragma unroll
        for (int j = 0; j < P; ++j) d[j] = gn_act<T, ACT>(fma(d[j], ch.scale[j], ch.bias[j]));
        T *to = y + u * y_step;
        if (a.whole_out) {
            if (at.c < a.channels) LnChunk<T>::write(to + at.c, d);
        } else {
            store_chunk(to, at.c, a.channels, d);
        }
    };
    auto advance = [&](int n) {
        y += n * y_step;
        if constexpr (COMPRESS) checkpoint.advance(n);
    };
    if constexpr (WHOLE) {
        const GnRing<16> ring(gn_ring);
        const bool in = at.c < a.channels;
        // (threads beyond the last channel have zeros for the blocks that they share)
        gn_ring_turns((int)at.turns, [&](int place) { if (in) ring.copy(place, x.row); x.next(); },
                      [&](int place, int u) { take(in ? ring.read(place) : make_uint4(0u, 0u, 0u, 0u), u); }, advance);
    } else {
        gn_turns<2>(at.turns, [&](int u) { return x.load(u); }, [&](int u, const typename GnFromX<T, WHOLE>::Raw &raw) { take(x.keep(raw, u), u); },
                    [&](int n) { x.advance(n); advance(n); });
    }
}

// take(x, chunk of dy, u) for all turns of a backward kernel, u of them before the next advance(n).
template <typename T, bool WHOLE, typename X, typename F, typename A>
__device__ __forceinline__ void gn_backward_turns(const GnArgs &a, const GnPlace<Bits<T>::VEC> &at, X &x, GnReader<T, WHOLE> &dy, char *memory, F &&take, A &&advance) {
    if constexpr (WHOLE) {
        if (at.c >= a.channels) return;
        constexpr int X_BYTES = X::CHECKPOINT ? Bits<T>::VEC : 16;
        const GnRing<16> dy_ring(memory);
        const GnRing<X_BYTES> x_ring(memory + GnRing<16>::SIZE);
        typename X::Powers powers = x.powers((int)at.turns);
        gn_ring_turns((int)at.turns,
                      [&](int place) {
                          dy_ring.copy(place, dy.row);
                          dy.row += dy.step;
                          x_ring.copy(place, x.place());
                          x.announce(powers, 0);
                          x.next();
                      },
                      [&](int place, int u) { take(X::kept(x_ring.read(place), powers, u), dy_ring.read(place), u); },
                      [&](int n) {
                          X::walk(powers, n);
                          advance(n);
                      });
    } else {
        struct Raw { typename X::Raw x; typename GnReader<T, WHOLE>::Raw dy; };
        gn_turns<2>(at.turns, [&](int u) { return Raw{x.load(u), dy.load(u)}; }, [&](int u, const Raw &raw) { take(x.keep(raw.x, u), dy.chunk(raw.dy, u), u); },
                    [&](int n) { x.advance(n); dy.advance(n); advance(n); });
    }
}

// Backward: sums of dz and dz xh of every channel of a part.
template <typename T, bool WHOLE, typename X, int ACT>
__global__ void __launch_bounds__(GN_THREADS, 2) gn_slopes_kernel(const __grid_constant__ GnArgs a) {
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    extern __shared__ __align__(16) char gn_ring[];
    __shared__ __align__(16) float box[GN_THREADS * 2 * VEC];
    const GnPlace<VEC> at(a, false);
    F2 s[P] = {}, t[P] = {};
    if (at.turns > 0) {
        X x(a, at.worker, at.sample, at.p0, at.lanes, at.c);
        GnReader<T, WHOLE> dy(static_cast<const T *>(a.dy) + at.worker * a.y_worker + at.sample * a.y_sample + at.p0 * a.y_pixel, at.lanes * a.y_pixel, at.c,
                                    a.channels);
        GnChannels<P> ch;
        ch.read(a, at.worker, at.image, at.c);
        auto take = [&](const typename X::Kept &kept, uint4 chunk) {
            F2 d[P], g[P];
            X::centred(kept, ch.minus, d);
            LnChunk<T>::read(chunk, g);
            gn_slope<T, ACT>(a, at.worker, at.image, at.c, ch, [&](F2 (&v)[P]) { const F2 none[P] = {}; X::centred(kept, none, v); }, d, g, g);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                s[j] = add(s[j], g[j]);
                t[j] = fma(g[j], d[j], t[j]);
            }
        };
        gn_backward_turns<T, WHOLE>(a, at, x, dy, gn_ring, [&](const typename X::Kept &kept, uint4 chunk, int) { take(kept, chunk); }, [](int) {});
    }
    gn_channel_sums<VEC>(at, a.tile_chunks, s, t, box);
    const int width = a.tile_chunks * VEC;
    float *out = a.part + (at.image * a.parts + at.part) * GN_BACKWARD_PARTS * a.channels + at.c0;
    for (int q = threadIdx.x; q < width && at.c0 + q < a.channels; q += GN_THREADS) {
        out[q] = box[q];
        out[a.channels + q] = box[width + q] * a.rstd[at.image * a.groups + (uint32_t)(at.c0 + q) / (uint32_t)(a.channels / a.groups)];
    }
}

// dw and db: a worker's images and parts (all workers', where they share the gradient) in binary64, rounded once.  A
// warp takes 32 channels, eight warps share the parts.
__device__ __forceinline__ void gn_join(const GnArgs &a, uint32_t block) {
    __shared__ double box[GN_THREADS / 32][32];
    const uint32_t columns = (uint32_t)(a.channels + 31) / 32, pair = block / columns;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, worker = (int)(pair >> 1), c = (int)(block - pair * columns) * 32 + lane;
    const bool weight = (pair & 1) == 0;
    void *out = weight ? a.dweight : a.dbias;
    if (!out) return;
    const int64_t rows = a.pixels == 0 ? 0 : (int64_t)(a.shared ? a.workers : 1) * a.samples * a.parts, first = a.shared ? 0 : (int64_t)worker * a.samples * a.parts;
    double s = 0.0;
    if (c < a.channels) {
        const float *from = a.part + (first * 2 + (weight ? 1 : 0)) * a.channels + c;
#pragma unroll 4
        for (int64_t i = warp; i < rows; i += GN_THREADS / 32) s += (double)from[i * 2 * a.channels];
    }
    box[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < a.channels) {
        for (int w = 1; w < GN_THREADS / 32; ++w) s += box[w][lane];
        const int64_t at = worker * (weight ? a.dweight_stride : a.dbias_stride) + c;
        if (a.grad_dtype == LIEC_F32) static_cast<float *>(out)[at] = (float)s;
        else static_cast<__nv_bfloat16 *>(out)[at] = __float2bfloat16_rn((float)s);
    }
}

// The first `level_ctas` CTAs: per group r mean(dz w) and r^2 mean(dz w xh).  The others: dw and db.
template <int LANES>
__global__ void __launch_bounds__(GN_THREADS) gn_levels_kernel(const __grid_constant__ GnArgs a, uint32_t level_ctas) {
    gn_wait_for_kernel_before();
    if (blockIdx.x >= level_ctas) {
        gn_join(a, blockIdx.x - level_ctas);
        return;
    }
    gn_per_group<LANES>(a, [&](bool live, uint32_t image, uint32_t group, uint32_t lane) {
        const uint32_t width = (uint32_t)a.channels / (uint32_t)a.groups, entries = live ? width * a.parts : 0u, worker = image / (uint32_t)a.samples;
        const float *part = a.part + (int64_t)image * a.parts * GN_BACKWARD_PARTS * a.channels + group * width;
        const float *weight = a.weight ? a.weight + worker * a.weight_stride + group * width : nullptr;
        double s = 0.0, t = 0.0;
#pragma unroll 4
        for (uint32_t i = lane; i < entries; i += LANES) {
            const uint32_t q = i / width, c = i - q * width;
            const double w = weight ? (double)weight[c] : 1.0;
            const float *at = part + (int64_t)q * GN_BACKWARD_PARTS * a.channels + c;
            s += w * at[0];
            t += w * at[a.channels];
        }
        s = gn_sum_lanes<LANES>(s);
        t = gn_sum_lanes<LANES>(t);
        if (live && lane == 0) {
            const int64_t g = (int64_t)image * a.groups + group;
            const double n = (double)a.pixels * width, r = (double)a.rstd[g];
            a.level[2 * g] = (float)(-r * s / n);
            a.level[2 * g + 1] = (float)(-r * r * t / n);
        }
    });
}

// dx = A dz - r mean(dz w) - d r^2 mean(dz w xh)
template <typename T, bool WHOLE, typename X, int ACT>
__global__ void __launch_bounds__(GN_THREADS, 2) gn_dx_kernel(const __grid_constant__ GnArgs a) {
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    extern __shared__ __align__(16) char gn_ring[];
    const GnPlace<VEC> at(a, true);
    X x(a, at.worker, at.sample, at.p0, at.lanes, at.c);
    GnReader<T, WHOLE> dy(static_cast<const T *>(a.dy) + at.worker * a.y_worker + at.sample * a.y_sample + at.p0 * a.y_pixel, at.lanes * a.y_pixel, at.c, a.channels);
    T *dx = static_cast<T *>(a.dx) + at.worker * a.dx_worker + at.sample * a.dx_sample + at.p0 * a.dx_pixel;
    const int64_t dx_step = at.lanes * a.dx_pixel;
    GnChannels<P> ch;
    if (at.turns > 0) ch.read(a, at.worker, at.image, at.c);
    gn_wait_for_kernel_before();
    if (at.turns == 0 || at.c >= a.channels) return;
    F2 level[P], along[P];
    const uint32_t width = (uint32_t)a.channels / (uint32_t)a.groups;
    GnGroup group(at.c, width);
    const float *levels = a.level + at.image * a.groups * 2;
#pragma unroll
    for (int k = 0; k < 2 * P; ++k, group.next(width)) {
        const bool in = at.c + k < a.channels;
        GnChannels<P>::set(level[k / 2], k % 2, in ? levels[2 * group.group] : 0.0f);
        GnChannels<P>::set(along[k / 2], k % 2, in ? levels[2 * group.group + 1] : 0.0f);
    }
    gn_backward_turns<T, WHOLE>(a, at, x, dy, gn_ring, [&](const typename X::Kept &kept, uint4 chunk, int u) {
        F2 d[P], g[P];
        X::centred(kept, ch.minus, d);
        LnChunk<T>::read(chunk, g);
        gn_slope<T, ACT>(a, at.worker, at.image, at.c, ch, [&](F2 (&v)[P]) { const F2 none[P] = {}; X::centred(kept, none, v); }, d, g, g);
#pragma unroll
        for (int j = 0; j < P; ++j) d[j] = fma(g[j], ch.scale[j], fma(d[j], along[j], level[j]));
        if (a.whole_out) LnChunk<T>::write(dx + u * dx_step + at.c, d);
        else store_chunk(dx + u * dx_step, at.c, a.channels, d);
    }, [&](int n) { dx += n * dx_step; });
}

// ---- launches --------------------------------------------------------------------------------------------

// Threads of a CTA share the chunks of a tile, so that few images still give a thread 16 pixels or more (4 of a part); parts of an
// image's pixels as there are places for CTAs (forward four on an SM, backward two), twice as many while a thread keeps
// 64 pixels (8 x 32 images of 56 x 56 x 64 backward with six on an SM: 117 us, two: 107; 4 of 256 x 256 x 128: 94 and 76).
// Never more than GN_CHAIN pixels to a thread, however many images there are: its sums are chains of binary32 additions, which lose up
// to 2^-24 in each (600 images of 65,536 x 128 with 4096: a constant dy came to 7e-5 less than it is).
constexpr int GN_CHAIN = 64;
static void gn_plan(GnArgs &a, int vec, bool backward) {
    const int places_per_sm = backward ? 2 : 4;
    const int chunks = (int)(ck_cols(a.channels) / vec), step = CK_BLOCK / vec;
    int64_t lanes = std::max<int64_t>(1, std::min<int64_t>(GN_THREADS / step, a.pixels / 16));
    a.tile_chunks = (int)std::min<int64_t>(chunks, std::max<int64_t>(std::min(chunks, 32), GN_THREADS / lanes / step * step));
    a.tiles = (chunks + a.tile_chunks - 1) / a.tile_chunks;
    a.tile_chunks = ((chunks + a.tiles - 1) / a.tiles + step - 1) / step * step;
    lanes = GN_THREADS / a.tile_chunks;
    const int64_t places = (int64_t)a.workers * a.samples * a.tiles;
    const int64_t few = std::min((LN_SMS * places_per_sm + places - 1) / places, a.pixels / (lanes * 4));
    const int64_t many = std::min((LN_SMS * 2 * places_per_sm + places - 1) / places, a.pixels / (lanes * 64));
    const int64_t again = std::max({int64_t(1), few, many}), parts = std::max(again, (a.pixels + lanes * GN_CHAIN - 1) / (lanes * GN_CHAIN));
    const auto cut = [&](int64_t into, int64_t &pixels, int32_t &number) {
        pixels = std::max<int64_t>(1, (a.pixels + into - 1) / into);
        number = (int32_t)std::max<int64_t>(1, (a.pixels + pixels - 1) / pixels);
    };
    cut(parts, a.part_pixels, a.parts);
    cut(again, a.again_pixels, a.again_parts);
}
// What the kernels of the second reading get; it sums nothing, so its parts may be long.
static GnArgs gn_again(GnArgs a) {
    a.parts = a.again_parts;
    a.part_pixels = a.again_pixels;
    return a;
}
static int64_t gn_ctas(const GnArgs &a) { return (int64_t)a.workers * a.samples * a.tiles * a.parts; }

static size_t gn_streamed_workspace(GnArgs a, int dtype, bool backward) {
    gn_plan(a, dtype == 0 ? 4 : 8, backward);
    const size_t images = (size_t)a.workers * a.samples;
    return sizeof(float) * (images * a.parts * (backward ? GN_BACKWARD_PARTS : GN_FORWARD_PARTS) * a.channels + (backward ? images * a.groups * 2 : 0));
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
    bits |= (uint64_t)a.channels * size;
    if (a.pixels > 1) bits |= (uint64_t)pixel * size;
    if (a.samples > 1) bits |= (uint64_t)sample * size;
    if (a.workers > 1) bits |= (uint64_t)worker * size;
    return (bits & 15u) == 0;
}

template <auto KERNEL>
static cudaError_t gn_allow(int memory) {
    static std::atomic<uint64_t> allowed{0};
    return ln_allow_smem(KERNEL, memory, allowed);
}

// after: starts while the kernel before ends, and waits for it where it needs it.
template <typename... A>
static cudaError_t gn_launch(void (*kernel)(A...), int64_t ctas, int memory, bool after, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.dynamicSmemBytes = (size_t)memory;
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(GN_THREADS);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = after ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Threads that join a group: eight, a warp where it has many channels and parts, a CTA where very many.
static int gn_group_lanes(const GnArgs &a) {
    const int64_t entries = (int64_t)(a.channels / a.groups) * a.parts;
    return entries > 512 ? GN_THREADS : entries > 64 ? 32 : 8;
}
template <int LANES> using GnLanes = std::integral_constant<int, LANES>;
template <typename F>
static cudaError_t gn_for_lanes(int lanes, F &&f) { return lanes == 8 ? f(GnLanes<8>{}) : lanes == 32 ? f(GnLanes<32>{}) : f(GnLanes<GN_THREADS>{}); }
static int64_t gn_group_ctas(const GnArgs &a) { return ((int64_t)a.workers * a.samples * a.groups * gn_group_lanes(a) + GN_THREADS - 1) / GN_THREADS; }
static int64_t gn_join_ctas(const GnArgs &a) { return a.dweight || a.dbias ? (int64_t)((a.channels + 31) / 32) * (a.shared ? 1 : a.workers) * 2 : 0; }

template <typename T, bool WHOLE>
struct GnForwardLaunch {
    const GnArgs &a;
    cudaStream_t st;
    template <int ACT>
    cudaError_t operator()() {
        constexpr int RING = WHOLE ? GnRing<16>::SIZE : 0;
        constexpr auto moments = gn_moments_kernel<T, WHOLE>;
        const GnArgs again = gn_again(a);
        cudaError_t e = gn_allow<moments>(RING + 40 * 1024);
        if (e == cudaSuccess) e = gn_launch(moments, gn_ctas(a), RING, false, st, a);
        if (e == cudaSuccess) e = gn_for_lanes(gn_group_lanes(a), [&](auto lanes) { return gn_launch(gn_statistics_kernel<decltype(lanes)::value>, gn_group_ctas(a), 0, true, st, a); });
        if (e != cudaSuccess) return e;
        return gn_launch(a.q ? gn_apply_kernel<T, WHOLE, ACT, true> : gn_apply_kernel<T, WHOLE, ACT, false>, gn_ctas(again), RING, true, st, again);
    }
};

cudaError_t launch_group_norm_forward(GnArgs a, int dtype, cudaStream_t st) {
    if (a.samples == 0 || a.pixels == 0) return cudaSuccess;
    int smem;
    a.whole = gn_whole(a, dtype, a.x, a.x_pixel, a.x_sample, a.x_worker);
    a.whole_out = gn_whole(a, dtype, a.y, a.y_pixel, a.y_sample, a.y_worker);
    if (gn_resident_plan(a, dtype, false, false, smem)) return gn_resident_forward(a, dtype, smem, st);
    gn_plan(a, dtype == 0 ? 4 : 8, false);
    if (dtype == 0) return a.whole ? gn_for_act(a.act, GnForwardLaunch<float, true>{a, st}) : gn_for_act(a.act, GnForwardLaunch<float, false>{a, st});
    return a.whole ? gn_for_act(a.act, GnForwardLaunch<__nv_bfloat16, true>{a, st}) : gn_for_act(a.act, GnForwardLaunch<__nv_bfloat16, false>{a, st});
}

template <typename T, bool WHOLE, typename X>
struct GnBackwardLaunch {
    const GnArgs &a;
    cudaStream_t st;
    template <int ACT>
    cudaError_t operator()() {
        constexpr int RING = WHOLE ? GnRing<16>::SIZE + GnRing<X::CHECKPOINT ? Bits<T>::VEC : 16>::SIZE : 0;
        constexpr auto slopes = gn_slopes_kernel<T, WHOLE, X, ACT>;
        constexpr auto dx = gn_dx_kernel<T, WHOLE, X, ACT>;
        const GnArgs again = gn_again(a);
        const int64_t levels = a.dx ? gn_group_ctas(a) : 0;
        cudaError_t e = gn_allow<slopes>(RING + 40 * 1024);
        if (e == cudaSuccess) e = gn_allow<dx>(RING + 40 * 1024);
        if (e == cudaSuccess) e = gn_launch(slopes, gn_ctas(a), RING, false, st, a);
        if (e == cudaSuccess) 
            e = gn_for_lanes(gn_group_lanes(a), [&](auto lanes) { return gn_launch(gn_levels_kernel<decltype(lanes)::value>, levels + gn_join_ctas(a), 0, true, st, a, (uint32_t)levels); });
        if (e == cudaSuccess && a.dx) e = gn_launch(dx, gn_ctas(again), RING, true, st, again);
        return e;
    }
};

template <typename T, bool WHOLE>
static cudaError_t gn_backward(const GnArgs &a, cudaStream_t st) {
    return a.x ? gn_for_act(a.act, GnBackwardLaunch<T, WHOLE, GnFromX<T, WHOLE>>{a, st}) : gn_for_act(a.act, GnBackwardLaunch<T, WHOLE, GnFromCheckpoint<T>>{a, st});
}

cudaError_t launch_group_norm_backward(GnArgs a, int dtype, cudaStream_t st) {
    int smem;
    if (a.samples == 0 || a.pixels == 0) {
        a.parts = 1;
        return gn_launch(gn_levels_kernel<8>, gn_join_ctas(a), 0, false, st, a, 0u);
    }
    a.whole = gn_whole(a, dtype, a.dy, a.y_pixel, a.y_sample, a.y_worker) && (!a.x || gn_whole(a, dtype, a.x, a.x_pixel, a.x_sample, a.x_worker));
    a.whole_out = gn_whole(a, dtype, a.dx, a.dx_pixel, a.dx_sample, a.dx_worker);
    if (gn_resident_plan(a, dtype, true, !a.x, smem)) {
        const cudaError_t e = gn_resident_backward(a, dtype, smem, st);
        if (e != cudaSuccess || gn_join_ctas(a) == 0) return e;
        a.parts = 1;
        return gn_launch(gn_levels_kernel<8>, gn_join_ctas(a), 0, true, st, a, 0u);
    }
    gn_plan(a, dtype == 0 ? 4 : 8, true);
    a.level = a.part + (int64_t)a.workers * a.samples * a.parts * GN_BACKWARD_PARTS * a.channels;
    if (dtype == 0) return a.whole ? gn_backward<float, true>(a, st) : gn_backward<float, false>(a, st);
    return a.whole ? gn_backward<__nv_bfloat16, true>(a, st) : gn_backward<__nv_bfloat16, false>(a, st);
}

}  // namespace liec

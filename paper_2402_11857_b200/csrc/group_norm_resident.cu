// Group normalisation of images that a cluster of CTAs holds in shared memory: every element crosses HBM once each way,
// in one launch (backward: a second one joins the images' gradients of weight and bias).
//
// A cluster takes the channels of some groups of one image, a CTA a part of the pixels.  Its threads copy their chunks
// (16 bytes of a pixel's channels) into places that they alone read again, sum them per channel, and the sums of all
// CTAs meet: each CTA hands its own to every other, and all add them in the same order.
#include "group_norm.cuh"

namespace liec {

// What lies in dynamic shared memory, in bytes: planes of chunks ([turn][thread]), then the exchange.
template <typename T, bool CHECKPOINT, int DZ_PLANES>
struct GnMemory {
    static constexpr int VEC = Bits<T>::VEC, X_BYTES = CHECKPOINT ? VEC : 16;
    __host__ __device__ static int x_plane(int turns) { return turns * GN_THREADS * X_BYTES; }
    __host__ __device__ static int powers(int turns) { return CHECKPOINT ? turns * GN_THREADS : 0; }
    __host__ __device__ static int dz_plane(int turns) { return turns * GN_THREADS * 16; }
    __host__ __device__ static int planes(int turns) { return x_plane(turns) + DZ_PLANES * dz_plane(turns) + powers(turns); }
    __host__ __device__ static int exchange(int ranks, int width) { return ranks * 2 * width * 4; }   // [rank][sum][channel]
    __host__ __device__ static int total(int turns, int ranks, int width) {
        return planes(turns) + exchange(ranks, width) + GN_THREADS * VEC * 4 + 2 * width * 4;          // box; two values per group
    }
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Where this CTA and thread are.
template <int VEC>
struct GnSpot {
    int64_t image, p0;
    int worker, sample, tile, rank, ranks, chunk, lane, lanes, c, c0, width, n;   // n: pixels of this CTA
    bool live;
    __device__ __forceinline__ GnSpot(const GnArgs &a) {
        ranks = a.parts;
        rank = (int)(blockIdx.x % ranks);
        const int64_t unit = blockIdx.x / ranks;
        tile = (int)(unit % a.tiles);
        image = unit / a.tiles;
        worker = (int)(image / a.samples);
        sample = (int)(image - (int64_t)worker * a.samples);
        p0 = rank * a.part_pixels;
        n = (int)max((int64_t)0, min(a.part_pixels, a.pixels - p0));
        chunk = threadIdx.x % a.tile_chunks;
        lane = threadIdx.x / a.tile_chunks;
        lanes = GN_THREADS / a.tile_chunks;
        width = a.tile_chunks * VEC;
        c0 = tile * width;
        c = c0 + chunk * VEC;
        live = lane < lanes && c < (a.channels + CK_BLOCK - 1) / CK_BLOCK * CK_BLOCK;
    }
    __device__ __forceinline__ int channels(const GnArgs &a) const { return min(width, a.channels - c0); }   // of the tile
};

// The channels' sums over the CTA's pixel lanes, then over the cluster: every CTA ends up with sums[rank][which][channel].
template <int VEC>
__device__ __forceinline__ void gn_exchange(const GnSpot<VEC> &at, const F2 (&v)[VEC / 2], int which, float *box, float *sums, bool last) {
    const int width = at.width;
    if (at.lane < at.lanes) {
#pragma unroll
        for (int k = 0; k < VEC / 2; k += 2)
            *reinterpret_cast<float4 *>(box + at.lane * width + at.chunk * VEC + 2 * k) = make_float4(lo(v[k]), hi(v[k]), lo(v[k + 1]), hi(v[k + 1]));
    }
    __syncthreads();
    // 256 / width threads share a channel, then one adds their sums
    const int ways = max(1, GN_THREADS / width), way = threadIdx.x / width, column = threadIdx.x - way * width;
    float s = 0.0f;
    for (int q = threadIdx.x; q < width; q += GN_THREADS) {   // (tiles wider than the CTA: a thread takes several channels)
        if (width <= GN_THREADS) break;
        float t = 0.0f;
        for (int l = 0; l < at.lanes; ++l) t += box[l * width + q];
        for (int r = 0; r < at.ranks; ++r) {
            uint32_t to;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(sums + (at.rank * 2 + which) * width + q)), "r"(r));
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(t) : "memory");
        }
    }
    if (width <= GN_THREADS) {
        if (way < ways)
            for (int l = way; l < at.lanes; l += ways) s += box[l * width + column];
        __syncthreads();
        if (way < ways && way > 0) box[way * width + column] = s;
        __syncthreads();
        if (way == 0) {
            for (int w = 1; w < ways; ++w) s += box[w * width + column];
            for (int r = 0; r < at.ranks; ++r) {
                uint32_t to;
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(sums + (at.rank * 2 + which) * width + column)), "r"(r));
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(s) : "memory");
            }
        }
    }
    if (!last) __syncthreads();   // the box is used again
}

constexpr int GN_PHASES = 4;   // a thread's chunks are summed in four goes, each as its copies are in

template <typename T, int ACT, bool COMPRESS>
__global__ void __launch_bounds__(GN_THREADS, 3) gn_resident_forward_kernel(const __grid_constant__ GnArgs a) {
    using M = GnMemory<T, false, 0>;
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    extern __shared__ __align__(16) char gn_memory[];
    const GnSpot<VEC> at(a);
    float *sums = reinterpret_cast<float *>(gn_memory + M::planes(a.turns)), *box = sums + at.ranks * 2 * at.width, *value = box + GN_THREADS * VEC;
    uint4 *place = reinterpret_cast<uint4 *>(gn_memory) + threadIdx.x;
    const uint32_t place_u32 = (uint32_t)__cvta_generic_to_shared(place);
    cluster_arrive();
    const T *image = static_cast<const T *>(a.x) + at.worker * a.x_worker + at.sample * a.x_sample, *x = image + (at.p0 + at.lane) * a.x_pixel;
    const int per = (a.turns + GN_PHASES - 1) / GN_PHASES, turns = at.live ? (at.n - at.lane + at.lanes - 1) / at.lanes : 0;   // (at.n - at.lane <= 0: none)
    const int64_t step = at.lanes * a.x_pixel;
#pragma unroll
    for (int q = 0; q < GN_PHASES; ++q) {
        for (int k = q * per; k < min((q + 1) * per, turns); ++k) gn_fetch(a, place_u32 + k * GN_THREADS * 16, x + k * step, at.c);
        copy_commit();
    }
    // sums about the image's first pixel
    F2 s[P] = {}, t[P] = {}, minus[P] = {};
    if (at.live && at.c < a.channels) {
        F2 v[P];
        LnChunk<T>::read(load_chunk(image, at.c, a.channels), v);
#pragma unroll
        for (int k = 0; k < P; ++k) minus[k] = f2(-lo(v[k]), -hi(v[k]));
    }
    auto go = [&](int q) {
#pragma unroll 2
        for (int k = q * per; k < min((q + 1) * per, turns); ++k) {
            F2 d[P];
            LnChunk<T>::read(place[k * GN_THREADS], d);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                d[j] = add(d[j], minus[j]);
                s[j] = add(s[j], d[j]);
                t[j] = fma(d[j], d[j], t[j]);
            }
        }
    };
    copy_wait<3>(); go(0);
    copy_wait<2>(); go(1);
    copy_wait<1>(); go(2);
    copy_wait<0>(); go(3);
    cluster_wait();                                     // all CTAs of the cluster are there
    gn_exchange<VEC>(at, s, 0, box, sums, false);
    gn_exchange<VEC>(at, t, 1, box, sums, true);
    cluster_arrive();
    cluster_wait();
    // every channel's mean and squares around it, then the groups'
    const int channels = at.channels(a), width = a.channels / a.groups, groups = channels / width;
    float *mean_c = sums, *square_c = sums + at.width;   // (rank 0's sums, read and written by the same thread)
    for (int q = threadIdx.x; q < channels; q += GN_THREADS) {
        float v = 0.0f, w = 0.0f;
        for (int r = 0; r < at.ranks; ++r) {
            v += sums[r * 2 * at.width + q];
            w += sums[(r * 2 + 1) * at.width + q];
        }
        const float m = v / (float)a.pixels;
        box[q] = m;                                      // mean about the first pixel
        mean_c[q] = (float)image[at.c0 + q];
        square_c[q] = fmaxf(__fmaf_rn(-v, m, w), 0.0f);
    }
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int g = warp; g < groups; g += GN_THREADS / 32) {
        double v = 0.0, w = 0.0;
        for (int q = lane; q < width; q += 32) v += (double)mean_c[g * width + q] + (double)box[g * width + q];
        const double mean = warp_sum(v) / width;
        for (int q = lane; q < width; q += 32) {
            const double off = (double)mean_c[g * width + q] + (double)box[g * width + q] - mean;
            w += (double)square_c[g * width + q] + (double)a.pixels * off * off;
        }
        const double var = warp_sum(w) / ((double)a.pixels * width);
        if (lane == 0) {
            const float m = (float)mean, r = (float)(1.0 / sqrt(var + (double)a.eps));
            value[2 * g] = m;
            value[2 * g + 1] = r;
            if (at.rank == 0) {
                const int64_t to = at.image * a.groups + at.c0 / width + g;
                a.mean[to] = m;
                a.rstd[to] = r;
            }
        }
    }
    __syncthreads();
    if (!at.live) return;
    GnChannels<P> ch;
    ch.read(a, at.worker, at.c, [&](int c, float &m, float &r) {
        const int g = (c - at.c0) / width;
        m = value[2 * g];
        r = value[2 * g + 1];
    });
    T *y = static_cast<T *>(a.y) + at.worker * a.y_worker + at.sample * a.y_sample + (at.p0 + at.lane) * a.y_pixel;
    const int64_t y_step = at.lanes * a.y_pixel, row0 = at.image * a.pixels + at.p0 + at.lane;
#pragma unroll 2
    for (int k = 0; k < turns; ++k) {
        F2 d[P];
        LnChunk<T>::read(place[k * GN_THREADS], d);
        if constexpr (COMPRESS) gn_compress<T>(a, d, row0 + (int64_t)k * at.lanes, at.c);
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const F2 z = fma(add(d[j], ch.minus[j]), ch.scale[j], ch.bias[j]);
            d[j] = f2(gn_act<T, ACT>(lo(z)), gn_act<T, ACT>(hi(z)));
        }
        store_chunk(y + k * y_step, at.c, a.channels, d);
    }
}

// dz is kept for the second go: as dy's type where it is dy or zero, else in binary32.
template <typename T, typename X, int ACT>
__global__ void __launch_bounds__(GN_THREADS, 2) gn_resident_backward_kernel(const __grid_constant__ GnArgs a) {
    constexpr bool CHECKPOINT = X::CHECKPOINT, WIDE = ACT == LIEC_ACT_SILU && sizeof(T) == 2;
    using M = GnMemory<T, CHECKPOINT, WIDE ? 2 : 1>;
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    extern __shared__ __align__(16) char gn_memory[];
    const GnSpot<VEC> at(a);
    uint4 *dz_place = reinterpret_cast<uint4 *>(gn_memory) + threadIdx.x;
    const int plane = a.turns * GN_THREADS;   // chunks of a plane
    char *x_place = gn_memory + M::dz_plane(a.turns) * (WIDE ? 2 : 1) + threadIdx.x * M::X_BYTES;
    uint8_t *power_place = reinterpret_cast<uint8_t *>(gn_memory) + M::dz_plane(a.turns) * (WIDE ? 2 : 1) + M::x_plane(a.turns) + threadIdx.x;
    float *sums = reinterpret_cast<float *>(gn_memory + M::planes(a.turns)), *box = sums + at.ranks * 2 * at.width, *value = box + GN_THREADS * VEC;
    cluster_arrive();
    const T *dy = static_cast<const T *>(a.dy) + at.worker * a.y_worker + at.sample * a.y_sample + (at.p0 + at.lane) * a.y_pixel;
    const int per = (a.turns + GN_PHASES - 1) / GN_PHASES, turns = at.live ? (at.n - at.lane + at.lanes - 1) / at.lanes : 0;
    const int64_t step = at.lanes * a.y_pixel;
    const X x(a, at.worker, at.sample, at.p0 + at.lane);
    const uint32_t dz_u32 = (uint32_t)__cvta_generic_to_shared(dz_place), x_u32 = (uint32_t)__cvta_generic_to_shared(x_place);
#pragma unroll
    for (int q = 0; q < GN_PHASES; ++q) {
        for (int k = q * per; k < min((q + 1) * per, turns); ++k) {
            gn_fetch(a, dz_u32 + k * GN_THREADS * 16, dy + k * step, at.c);
            x.fetch(a, x_u32 + k * GN_THREADS * M::X_BYTES, power_place + k * GN_THREADS, (int64_t)k * at.lanes, at.c);
        }
        copy_commit();
    }
    GnChannels<P> ch;
    if (at.live) ch.read(a, at.worker, at.image, at.c);
    F2 s[P] = {}, t[P] = {};
    auto go = [&](int q) {
#pragma unroll 2
        for (int k = q * per; k < min((q + 1) * per, turns); ++k) {
            const typename X::Raw raw = X::kept(x_place + k * GN_THREADS * M::X_BYTES, power_place + k * GN_THREADS);
            F2 d[P], g[P];
            X::centred(raw, ch.minus, d);
            LnChunk<T>::read(dz_place[k * GN_THREADS], g);
            gn_slope<T, ACT, X>(a, at.worker, at.image, at.c, ch, raw, d, g, g);
            if constexpr (WIDE) {
                LnChunk<float>::write(dz_place + k * GN_THREADS, {g[0], g[1]});
                LnChunk<float>::write(dz_place + plane + k * GN_THREADS, {g[2], g[3]});
            } else if constexpr (ACT != LIEC_ACT_NONE) {
                LnChunk<T>::write(dz_place + k * GN_THREADS, g);
            }
#pragma unroll
            for (int j = 0; j < P; ++j) {
                s[j] = add(s[j], g[j]);
                t[j] = fma(g[j], d[j], t[j]);
            }
        }
    };
    copy_wait<3>(); go(0);
    copy_wait<2>(); go(1);
    copy_wait<1>(); go(2);
    copy_wait<0>(); go(3);
    cluster_wait();
    gn_exchange<VEC>(at, s, 0, box, sums, false);
    gn_exchange<VEC>(at, t, 1, box, sums, true);
    cluster_arrive();
    cluster_wait();
    const int channels = at.channels(a), width = a.channels / a.groups, groups = channels / width;
    for (int q = threadIdx.x; q < channels; q += GN_THREADS) {
        float v = 0.0f, w = 0.0f;
        for (int r = 0; r < at.ranks; ++r) {
            v += sums[r * 2 * at.width + q];
            w += sums[(r * 2 + 1) * at.width + q];
        }
        w *= a.rstd[at.image * a.groups + (at.c0 + q) / width];
        if (at.rank == 0 && a.part) {   // the image's share of db and dw
            a.part[at.image * 2 * a.channels + at.c0 + q] = v;
            a.part[(at.image * 2 + 1) * a.channels + at.c0 + q] = w;
        }
        const float weight = a.weight ? __ldg(a.weight + at.worker * a.weight_stride + at.c0 + q) : 1.0f;
        sums[q] = v * weight;
        sums[at.width + q] = w * weight;
    }
    if (!a.dx) return;
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int g = warp; g < groups; g += GN_THREADS / 32) {
        double v = 0.0, w = 0.0;
        for (int q = lane; q < width; q += 32) {
            v += (double)sums[g * width + q];
            w += (double)sums[at.width + g * width + q];
        }
        v = warp_sum(v);
        w = warp_sum(w);
        if (lane == 0) {
            const double n = (double)a.pixels * width, r = (double)a.rstd[at.image * a.groups + at.c0 / width + g];
            value[2 * g] = (float)(-r * v / n);
            value[2 * g + 1] = (float)(-r * r * w / n);
        }
    }
    __syncthreads();
    if (!at.live || at.c >= a.channels) return;
    F2 level[P], along[P];
#pragma unroll
    for (int k = 0; k < 2 * P; ++k) {
        const int g = (min(at.c + k, a.channels - 1) - at.c0) / width;
        GnChannels<P>::set(level[k / 2], k % 2, value[2 * g]);
        GnChannels<P>::set(along[k / 2], k % 2, value[2 * g + 1]);
    }
    T *dx = static_cast<T *>(a.dx) + at.worker * a.dx_worker + at.sample * a.dx_sample + (at.p0 + at.lane) * a.dx_pixel;
    const int64_t dx_step = at.lanes * a.dx_pixel;
#pragma unroll 2
    for (int k = 0; k < turns; ++k) {
        const typename X::Raw raw = X::kept(x_place + k * GN_THREADS * M::X_BYTES, power_place + k * GN_THREADS);
        F2 d[P], g[P];
        X::centred(raw, ch.minus, d);
        if constexpr (WIDE) {
            F2 low[2], high[2];
            LnChunk<float>::read(dz_place[k * GN_THREADS], low);
            LnChunk<float>::read(dz_place[plane + k * GN_THREADS], high);
            g[0] = low[0]; g[1] = low[1]; g[2] = high[0]; g[3] = high[1];
        } else {
            LnChunk<T>::read(dz_place[k * GN_THREADS], g);
        }
#pragma unroll
        for (int j = 0; j < P; ++j) d[j] = fma(g[j], ch.scale[j], fma(d[j], along[j], level[j]));
        store_chunk(dx + k * dx_step, at.c, a.channels, d);
    }
}

// ---- launches --------------------------------------------------------------------------------------------

constexpr int GN_MAX_MEMORY = 224 * 1024;

template <auto KERNEL>
static cudaError_t gn_resident_launch(const GnArgs &a, int smem, cudaStream_t st) {
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = ln_allow_smem(KERNEL, GN_MAX_MEMORY, allowed);
    if (e != cudaSuccess) return e;
    return ln_launch(KERNEL, a, (int64_t)a.workers * a.samples * a.tiles, a.parts, GN_THREADS, smem, st);
}

template <typename T>
struct GnResidentForward {
    const GnArgs &a;
    int smem;
    cudaStream_t st;
    template <int ACT>
    cudaError_t operator()() {
        return a.q ? gn_resident_launch<gn_resident_forward_kernel<T, ACT, true>>(a, smem, st) : gn_resident_launch<gn_resident_forward_kernel<T, ACT, false>>(a, smem, st);
    }
};
cudaError_t gn_resident_forward(const GnArgs &a, int dtype, int smem, cudaStream_t st) {
    return dtype == 0 ? gn_for_act(a.act, GnResidentForward<float>{a, smem, st}) : gn_for_act(a.act, GnResidentForward<__nv_bfloat16>{a, smem, st});
}

template <typename T>
struct GnResidentBackward {
    const GnArgs &a;
    int smem;
    cudaStream_t st;
    template <int ACT>
    cudaError_t operator()() {
        return a.x ? gn_resident_launch<gn_resident_backward_kernel<T, GnFromX<T>, ACT>>(a, smem, st)
                   : gn_resident_launch<gn_resident_backward_kernel<T, GnFromCheckpoint<T>, ACT>>(a, smem, st);
    }
};
cudaError_t gn_resident_backward(const GnArgs &a, int dtype, int smem, cudaStream_t st) {
    return dtype == 0 ? gn_for_act(a.act, GnResidentBackward<float>{a, smem, st}) : gn_for_act(a.act, GnResidentBackward<__nv_bfloat16>{a, smem, st});
}

template <typename T>
static int gn_memory_bytes(bool backward, bool checkpoint, int act, int turns, int ranks, int width) {
    if (!backward) return GnMemory<T, false, 0>::total(turns, ranks, width);
    const bool wide = act == LIEC_ACT_SILU && sizeof(T) == 2;
    if (checkpoint) return wide ? GnMemory<T, true, 2>::total(turns, ranks, width) : GnMemory<T, true, 1>::total(turns, ranks, width);
    return wide ? GnMemory<T, false, 2>::total(turns, ranks, width) : GnMemory<T, false, 1>::total(turns, ranks, width);
}

// Channels per cluster: whole groups and whole blocks of a checkpoint, at least 128 bytes of a pixel (or all of it); more while an image
// is small and there are CTAs enough.  CTAs per cluster: as few as leave room for three CTAs on an SM,
// then two, then one, so that the copies of one hide behind the sums and stores of the others; more, down to two
// turns per thread, while SMs are idle.
bool gn_resident_plan(GnArgs &a, int dtype, bool backward, bool checkpoint, int &smem) {
    const int vec = dtype == 0 ? 4 : 8, group = a.channels / a.groups;
    int unit = group;
    while (unit % CK_BLOCK != 0) unit += group;
    const int64_t images = (int64_t)a.workers * a.samples;
    const int most = 8;
    auto fits = [&](int channels, int ranks, int budget) {
        const int chunks = (int)(ck_cols(channels) / vec);
        if (chunks > GN_THREADS) return false;
        a.tile_chunks = chunks;
        a.tiles = (a.channels + channels - 1) / channels;
        a.part_pixels = (a.pixels + ranks - 1) / ranks;
        a.parts = ranks;
        const int lanes = GN_THREADS / chunks;
        const int64_t turns = (a.part_pixels + lanes - 1) / lanes;
        if (turns > 1024) return false;
        a.turns = (int)turns;
        smem = dtype == 0 ? gn_memory_bytes<float>(backward, checkpoint, a.act, a.turns, ranks, chunks * vec)
                          : gn_memory_bytes<__nv_bfloat16>(backward, checkpoint, a.act, a.turns, ranks, chunks * vec);
        return smem <= budget;
    };
    int channels = std::min(unit, a.channels);
    auto wider = [&]() {
        if (channels >= a.channels) return false;
        channels = 2 * channels >= a.channels ? a.channels : 2 * channels;
        return true;
    };
    while (channels * (16 / vec) < 128 && wider()) {}
    // (a range that is doubled is still a multiple of the unit, or all channels)
    while (channels < a.channels && channels * 2 <= 32 * vec && a.pixels * channels <= 4 * GN_THREADS * vec && images * ((a.channels + channels - 1) / channels) > 4 * LN_SMS)
        wider();
    const int budgets[3] = {75 * 1024, 112 * 1024, GN_MAX_MEMORY};
    for (int budget : budgets)
        for (int ranks = 1; ranks <= most; ++ranks) {
            if (ranks > 1 && ranks > a.pixels) break;
            if (!fits(channels, ranks, budget)) continue;
            int better = ranks;
            while (better < most && images * a.tiles * better * 2 <= LN_SMS && a.turns > 2) {
                better = std::min(2 * better, most);
                if (better > a.pixels || !fits(channels, better, budget)) break;
                ranks = better;
            }
            return fits(channels, ranks, budget) && images * a.tiles * a.parts < (int64_t(1) << 31);
        }
    return false;
}

}  // namespace liec

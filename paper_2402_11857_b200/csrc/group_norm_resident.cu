// Group normalisation of small images in one launch: a CTA holds some groups' channels of an image in shared memory, so
// every element crosses HBM once each way (backward: a second launch joins the images' gradients of weight and bias).  Its
// threads copy their chunks into places that they alone read again.
#include "group_norm.cuh"

namespace liec {

constexpr int GR_THREADS = 128;   // few threads with many chunks each: what is done once per thread is as much as a dozen chunks cost

// What lies in dynamic shared memory, in bytes: planes of chunks ([turn][thread]), the channels' two sums, those of the pixel
// lanes on their way there, and per channel and group what follows from them.
template <typename T, bool CHECKPOINT, int DZ_PLANES>
struct GnMemory {
    static constexpr int VEC = Bits<T>::VEC, X_BYTES = CHECKPOINT ? VEC : 16;
    __host__ __device__ static int x_plane(int turns) { return turns * GR_THREADS * X_BYTES; }
    __host__ __device__ static int powers(int turns) { return CHECKPOINT ? turns * GR_THREADS : 0; }
    __host__ __device__ static int dz_plane(int turns) { return turns * GR_THREADS * 16; }
    __host__ __device__ static int planes(int turns) { return x_plane(turns) + DZ_PLANES * dz_plane(turns) + powers(turns); }
    __host__ __device__ static int total(int turns, int width) { return planes(turns) + 2 * width * 4 + GR_THREADS * VEC * 4 + 3 * width * 4; }
};

// Where this CTA and thread are.
template <int VEC>
struct GnSpot {
    int64_t image, p0;   // p0: the thread's first pixel
    int worker, sample, chunk, lane, lanes, c, c0, width, turns;   // turns: the thread's chunks
    __device__ __forceinline__ GnSpot(const GnArgs &a) {
        const uint32_t picture = blockIdx.x / (uint32_t)a.tiles;
        image = picture;
        worker = (int)(picture / (uint32_t)a.samples);
        sample = (int)(picture - (uint32_t)worker * a.samples);
        lane = (int)(threadIdx.x / (uint32_t)a.tile_chunks);
        chunk = (int)threadIdx.x - lane * a.tile_chunks;
        lanes = (int)(GR_THREADS / (uint32_t)a.tile_chunks);
        width = a.tile_chunks * VEC;
        c0 = (int)(blockIdx.x - picture * a.tiles) * width;
        c = c0 + chunk * VEC;
        p0 = lane;
        const bool live = lane < lanes && c < (a.channels + CK_BLOCK - 1) / CK_BLOCK * CK_BLOCK;
        turns = live && lane < a.pixels ? ((int)a.pixels - lane + lanes - 1) / lanes : 0;
    }
    __device__ __forceinline__ int channels(const GnArgs &a) const { return min(width, a.channels - c0); }   // of the tile
};

// A sum per channel over the pixel lanes, complete for all threads.
template <int VEC>
__device__ __forceinline__ void gn_add_lanes(const GnSpot<VEC> &at, const F2 (&mine)[VEC / 2], float *box, float *sums) {
    const int width = at.width;
    if (at.lane < at.lanes) {
#pragma unroll
        for (int k = 0; k < VEC / 2; k += 2)
            *reinterpret_cast<float4 *>(box + at.lane * width + at.chunk * VEC + 2 * k) = make_float4(lo(mine[k]), hi(mine[k]), lo(mine[k + 1]), hi(mine[k + 1]));
    }
    __syncthreads();
    if (2 * width > GR_THREADS) {   // a thread per channel, or several channels
        for (int q = threadIdx.x; q < width; q += GR_THREADS) {
            float s = 0.0f;
            for (int l = 0; l < at.lanes; ++l) s += box[l * width + q];
            sums[q] = s;
        }
    } else {                        // several threads per channel, then one adds their sums
        const uint32_t ways = GR_THREADS / (uint32_t)width, way = threadIdx.x / (uint32_t)width;
        const int column = (int)(threadIdx.x - way * width);
        float s = 0.0f;
        if (way < ways)
#pragma unroll 4
            for (int l = way; l < at.lanes; l += ways) s += box[l * width + column];
        __syncthreads();
        if (way < ways && way > 0) box[way * width + column] = s;
        __syncthreads();
        if (way == 0) {
            for (uint32_t w = 1; w < ways; ++w) s += box[w * width + column];
            sums[column] = s;
        }
    }
    __syncthreads();   // the box is used again
}
// Sums over a warp's pixel lanes, in all of its threads: 4, 8 or 16 chunks, so that lanes are neighbours in it.
template <int P>
__device__ __forceinline__ void gn_add_warp_lanes(F2 (&v)[P], int chunks) {
#pragma unroll
    for (int m = 4; m < 32; m <<= 1)
        if (m >= chunks)
#pragma unroll
            for (int k = 0; k < P; ++k) v[k] = add(v[k], F2{__shfl_xor_sync(0xffffffffu, v[k].v, m)});
}
// The channels' two sums: sums[which][channel].
template <int VEC>
__device__ __forceinline__ void gn_add_lanes(const GnSpot<VEC> &at, const F2 (&a)[VEC / 2], const F2 (&b)[VEC / 2], float *box, float *sums) {
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        F2 mine[VEC / 2];
#pragma unroll
        for (int k = 0; k < VEC / 2; ++k) mine[k] = which ? b[k] : a[k];
        gn_add_lanes<VEC>(at, mine, box, sums + which * at.width);
    }
}

// f(group, its sum) for every group of the tile: a thread adds the channels of a narrow one, a warp those of a wide one.
template <int N, typename S, typename V, typename F>
__device__ __forceinline__ void gn_over_groups(int channels, int width, V &&values, F &&f) {
    const int groups = (int)((uint32_t)channels / (uint32_t)width);
    if (width <= 16) {
        for (int g = threadIdx.x; g < groups; g += GR_THREADS) {
            S s[N] = {};
            for (int q = g * width; q < (g + 1) * width; ++q) values(g, q, s);
            f(g, s);
        }
    } else {
        const int lane = threadIdx.x & 31;
        for (int g = threadIdx.x >> 5; g < groups; g += GR_THREADS / 32) {
            S s[N] = {};
            for (int q = g * width + lane; q < (g + 1) * width; q += 32) values(g, q, s);
#pragma unroll
            for (int m = 16; m >= 1; m >>= 1)
#pragma unroll
                for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], m);
            f(g, s);   // (the same in every lane)
        }
    }
}

constexpr int GN_PHASES = 4;   // a thread's chunks are summed in four goes, each as its copies are in

__device__ __forceinline__ void gn_wait_phase(int q) {
    if (q == 0) copy_wait<3>();
    else if (q == 1) copy_wait<2>();
    else if (q == 2) copy_wait<1>();
    else copy_wait<0>();
}

// One array's chunks of a thread on their way to its places, asynchronously where rows start on 16 bytes: turns from to to
// end - 1.
template <typename T>
__device__ __forceinline__ void gn_fetch(const GnArgs &a, uint32_t place, const T *first, int64_t step, int c, int from, int end) {
    if (a.whole) {
        const int bytes = c < a.channels ? 16 : 0;
        const T *p = (bytes > 0 ? first + c : first) + from * step;
        for (int k = from; k < end; ++k, p += step) copy_async(place + k * (GR_THREADS * 16), p, bytes);
    } else {
#pragma unroll 4
        for (int k = from; k < end; ++k) {
            const uint4 v = c < a.channels ? load_chunk(first + k * step, c, a.channels) : make_uint4(0u, 0u, 0u, 0u);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(place + k * (GR_THREADS * 16)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
        }
    }
}

// Results of a thread's chunks: results(k, d) for every turn, stored 16 bytes at a time where all rows start there.
template <typename T, typename F>
__device__ __forceinline__ void gn_store(const GnArgs &a, T *first, int64_t step, int c, int turns, F &&results) {
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    T *p = first + c;
    if (a.whole_out) {   // (the same way for all threads: those of a checkpoint's block find its maximum in results())
#pragma unroll 2
        for (int k = 0; k < turns; ++k, p += step) {
            F2 d[P];
            results(k, d);
            if (c < a.channels) LnChunk<T>::write(p, d);
        }
    } else {
        for (int k = 0; k < turns; ++k) {
            F2 d[P];
            results(k, d);
            store_chunk(first + k * step, c, a.channels, d);
        }
    }
}

// (Registers for seven CTAs on an SM: with 82, for five, 256 images of 64 x 256 took 13.5 us, now 10.7.)
template <typename T, int ACT, bool COMPRESS>
__global__ void __launch_bounds__(GR_THREADS, 7) gn_resident_forward_kernel(const __grid_constant__ GnArgs a) {
    using M = GnMemory<T, false, 0>;
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    extern __shared__ __align__(16) char gn_memory[];
    const GnSpot<VEC> at(a);
    float *sums = reinterpret_cast<float *>(gn_memory + M::planes(a.turns)), *box = sums + 2 * at.width;
    float *origin = box + GR_THREADS * VEC;
    const uint4 *place = reinterpret_cast<const uint4 *>(gn_memory) + threadIdx.x;
    const uint32_t place_u32 = (uint32_t)__cvta_generic_to_shared(place);
    const T *image = static_cast<const T *>(a.x) + at.worker * a.x_worker + at.sample * a.x_sample, *x = image + at.p0 * a.x_pixel;
    const int per = (a.turns + GN_PHASES - 1) / GN_PHASES, turns = at.turns;
#pragma unroll 1
    for (int q = 0; q < GN_PHASES; ++q) {
        gn_fetch(a, place_u32, x, at.lanes * a.x_pixel, at.c, q * per, min((q + 1) * per, turns));
        copy_commit();
    }
    // a thread's entries about their own mean; then all threads' about one number per channel, their mean as far as it is known then
    GnMoments<P> m;
#pragma unroll 1
    for (int q = 0; q < GN_PHASES; ++q) {
        gn_wait_phase(q);
        if (q == 0 && turns > 0) m.template start<T>(place[0]);
        const int end = min((q + 1) * per, turns);
#pragma unroll 2
        for (int k = q * per; k < end; ++k) {
            F2 v[P];
            LnChunk<T>::read(place[k * GR_THREADS], v);
            m.take(v);
        }
        if (q < 2 && end > 1) m.move((float)end, __fdividef(1.0f, (float)end));   // (the second half about the first half's mean)
    }
    const float entries = (float)turns, pixels = (float)a.pixels, inverse = 1.0f / pixels;
    F2 whole[P];
#pragma unroll
    for (int k = 0; k < P; ++k) whole[k] = m.whole(k, entries);
    const int channels = at.channels(a), width = (int)((uint32_t)a.channels / (uint32_t)a.groups);
    // every channel's mean (about its number) and squares around it
    auto channel = [&](int q, float left, float squares) {
        const float mean = left * inverse;
        sums[q] = mean;
        sums[at.width + q] = fmaxf(__fmaf_rn(-left, mean, squares), 0.0f);
    };
    const int chunks = a.tile_chunks;
    if (chunks == 4 || chunks == 8 || chunks == 16) {   // a warp's lanes meet by shuffles: two or three barriers in place of a dozen
        constexpr int WARPS = GR_THREADS / 32;
        const int warp = threadIdx.x / 32, first = at.chunk * VEC;
        const bool writes = (int)(threadIdx.x & 31) < chunks;
        auto put = [&](float *plane, const F2 (&v)[P]) {
#pragma unroll
            for (int k = 0; k < P; k += 2)
                if (writes) *reinterpret_cast<float4 *>(plane + warp * at.width + first + 2 * k) = make_float4(lo(v[k]), hi(v[k]), lo(v[k + 1]), hi(v[k + 1]));
        };
        gn_add_warp_lanes(whole, chunks);
        put(box, whole);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < P; ++k) {
            F2 sum = f2(0.0f);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float2 v = *reinterpret_cast<const float2 *>(box + w * at.width + first + 2 * k);
                sum = add(sum, f2(v.x, v.y));
            }
            sum = mul(sum, f2(inverse));
            if (at.lane == 0) *reinterpret_cast<float2 *>(origin + first + 2 * k) = make_float2(lo(sum), hi(sum));
            m.move_to(k, sum, entries);
        }
        float *planes = box + WARPS * at.width;   // (three of them, where they fit)
        if (chunks > 8) {
            planes = box;
            __syncthreads();
        }
        gn_add_warp_lanes(m.s, chunks);
        gn_add_warp_lanes(m.t, chunks);
        put(planes, m.s);
        put(planes + WARPS * at.width, m.t);
        __syncthreads();
        for (int q = threadIdx.x; q < channels; q += GR_THREADS) {
            float left = 0.0f, squares = 0.0f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                left += planes[w * at.width + q];
                squares += planes[(WARPS + w) * at.width + q];
            }
            channel(q, left, squares);
        }
    } else {
        gn_add_lanes<VEC>(at, whole, box, origin);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const float2 sum = *reinterpret_cast<const float2 *>(origin + at.chunk * VEC + 2 * k);
            m.move_to(k, f2(sum.x * inverse, sum.y * inverse), entries);
        }
        gn_add_lanes<VEC>(at, m.s, m.t, box, sums);
        for (int q = threadIdx.x; q < at.width; q += GR_THREADS) origin[q] *= inverse;   // (as above)
        for (int q = threadIdx.x; q < channels; q += GR_THREADS) channel(q, sums[q], sums[at.width + q]);
    }
    __syncthreads();
    // the groups', in binary64 about their first channel's number
    gn_over_groups<2, double>(channels, width,
                              [&](int g, int q, double (&v)[2]) {
                                  const double d = ((double)origin[q] - (double)origin[g * width]) + (double)sums[q];
                                  v[0] += d;
                                  v[1] += (double)sums[at.width + q] + (double)pixels * d * d;
                              },
                              [&](int g, double (&v)[2]) {
                                  const double off = v[0] / width, var = v[1] / ((double)pixels * width) - off * off;
                                  const float mean = (float)((double)origin[g * width] + off), r = 1.0f / sqrtf((var < 0.0 ? 0.0f : (float)var) + a.eps);   // (NaN stays)
                                  if (width <= 16 || (threadIdx.x & 31) == 0) {
                                      box[2 * g] = mean;
                                      box[2 * g + 1] = r;
                                      const int64_t to = at.image * a.groups + (int)((uint32_t)at.c0 / (uint32_t)width) + g;
                                      a.mean[to] = mean;
                                      a.rstd[to] = r;
                                  }
                              });
    __syncthreads();
    if (turns == 0) return;
    GnChannels<P> ch;
    const uint32_t first_group = (uint32_t)at.c0 / (uint32_t)width;
    ch.read(a, at.worker, at.c, [&](uint32_t g, float &m, float &r) {
        m = box[2 * (g - first_group)];
        r = box[2 * (g - first_group) + 1];
    });
    T *y = static_cast<T *>(a.y) + at.worker * a.y_worker + at.sample * a.y_sample + at.p0 * a.y_pixel;
    const GnCompressor<T> checkpoint(a, at.image * a.pixels + at.p0, at.lanes, at.c);
    gn_store<T>(a, y, at.lanes * a.y_pixel, at.c, turns, [&](int k, F2 (&d)[P]) {
        const uint4 chunk = place[k * GR_THREADS];
        LnChunk<T>::read(chunk, d);
        if constexpr (COMPRESS) checkpoint.store(k, chunk);
#pragma unroll
        for (int j = 0; j < P; ++j) d[j] = gn_act<T, ACT>(fma(add(d[j], ch.minus[j]), ch.scale[j], ch.bias[j]));
    });
}

// dz is kept for the second go: as dy's type where it is dy or zero, else in binary32.
template <typename T, typename X, int ACT>
__global__ void __launch_bounds__(GR_THREADS, 4) gn_resident_backward_kernel(const __grid_constant__ GnArgs a) {
    constexpr bool CHECKPOINT = X::CHECKPOINT, WIDE = ACT == LIEC_ACT_SILU && sizeof(T) == 2;
    using M = GnMemory<T, CHECKPOINT, WIDE ? 2 : 1>;
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2;
    extern __shared__ __align__(16) char gn_memory[];
    const GnSpot<VEC> at(a);
    uint4 *dz_place = reinterpret_cast<uint4 *>(gn_memory) + threadIdx.x;
    const int plane = a.turns * GR_THREADS;   // chunks of a plane
    char *x_place = gn_memory + M::dz_plane(a.turns) * (WIDE ? 2 : 1) + threadIdx.x * M::X_BYTES;
    uint8_t *power_place = reinterpret_cast<uint8_t *>(gn_memory) + M::dz_plane(a.turns) * (WIDE ? 2 : 1) + M::x_plane(a.turns) + threadIdx.x;
    float *sums = reinterpret_cast<float *>(gn_memory + M::planes(a.turns)), *box = sums + 2 * at.width, *value = box + GR_THREADS * VEC;
    const T *dy = static_cast<const T *>(a.dy) + at.worker * a.y_worker + at.sample * a.y_sample + at.p0 * a.y_pixel;
    const int per = (a.turns + GN_PHASES - 1) / GN_PHASES, turns = at.turns;
    const X x(a, at.worker, at.sample, at.p0, at.lanes, at.c);
    const uint32_t dz_u32 = (uint32_t)__cvta_generic_to_shared(dz_place), x_u32 = (uint32_t)__cvta_generic_to_shared(x_place);
#pragma unroll 1
    for (int q = 0; q < GN_PHASES; ++q) {
        const int end = min((q + 1) * per, turns);
        gn_fetch(a, dz_u32, dy, at.lanes * a.y_pixel, at.c, q * per, end);
        if constexpr (CHECKPOINT) {
            const int64_t power_step = x.step, step = power_step * CK_BLOCK;
            const int8_t *from = x.q + q * per * step;
            for (int k = q * per; k < end; ++k, from += step)
                asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(x_u32 + k * (GR_THREADS * M::X_BYTES)), "l"(from), "n"(M::X_BYTES) : "memory");
            const uint8_t *power = x.scales + q * per * power_step;
#pragma unroll 4
            for (int k = q * per; k < end; ++k) power_place[k * GR_THREADS] = __ldg(power + (k - q * per) * power_step);
        } else {
            gn_fetch(a, x_u32, x.row - at.c, x.step, at.c, q * per, end);
        }
        copy_commit();
    }
    const int channels = at.channels(a), width = (int)((uint32_t)a.channels / (uint32_t)a.groups);
    const float *rstd = a.rstd + at.image * a.groups, *weight = a.weight ? a.weight + at.worker * a.weight_stride : nullptr;
    const uint32_t first_group = (uint32_t)at.c0 / (uint32_t)width;
    GnChannels<P> ch;
    if (turns > 0) ch.read(a, at.worker, at.image, at.c);
    F2 s[P] = {}, t[P] = {};
#pragma unroll 1
    for (int q = 0; q < GN_PHASES; ++q) {
        gn_wait_phase(q);
#pragma unroll 2
        for (int k = q * per; k < min((q + 1) * per, turns); ++k) {
            const typename X::Kept raw = X::kept(x_place + k * GR_THREADS * M::X_BYTES, power_place + k * GR_THREADS);
            F2 d[P], g[P];
            X::centred(raw, ch.minus, d);
            LnChunk<T>::read(dz_place[k * GR_THREADS], g);
            gn_slope<T, ACT>(a, at.worker, at.image, at.c, ch, [&](F2 (&v)[P]) { const F2 none[P] = {}; X::centred(raw, none, v); }, d, g, g);
            if constexpr (WIDE) {
                LnChunk<float>::write(dz_place + k * GR_THREADS, {g[0], g[1]});
                LnChunk<float>::write(dz_place + plane + k * GR_THREADS, {g[2], g[3]});
            } else if constexpr (ACT != LIEC_ACT_NONE) {
                LnChunk<T>::write(dz_place + k * GR_THREADS, g);
            }
#pragma unroll
            for (int j = 0; j < P; ++j) {
                s[j] = add(s[j], g[j]);
                t[j] = fma(g[j], d[j], t[j]);
            }
        }
    }
    // (loaded while the sums meet)
    const float my_rstd = (int)threadIdx.x < channels ? __ldg(rstd + (at.c0 + threadIdx.x) / (uint32_t)width) : 0.0f;
    const float my_weight = (int)threadIdx.x < channels && weight ? __ldg(weight + at.c0 + threadIdx.x) : 1.0f;
    gn_add_lanes<VEC>(at, s, t, box, sums);
    for (int q = threadIdx.x; q < channels; q += GR_THREADS) {
        const float v = sums[q];
        float w = sums[at.width + q];
        const bool mine = q == (int)threadIdx.x;
        w *= mine ? my_rstd : __ldg(rstd + (uint32_t)(at.c0 + q) / (uint32_t)width);
        a.part[at.image * 2 * a.channels + at.c0 + q] = v;   // the image's share of db and dw
        a.part[(at.image * 2 + 1) * a.channels + at.c0 + q] = w;
        const float by = mine || !weight ? my_weight : __ldg(weight + at.c0 + q);
        box[q] = v * by;
        box[at.width + q] = w * by;
    }
    if (!a.dx) return;
    __syncthreads();
    gn_over_groups<2, float>(channels, width, [&](int, int q, float (&v)[2]) { v[0] += box[q]; v[1] += box[at.width + q]; },
                      [&](int g, float (&v)[2]) {
                          const float r = __ldg(rstd + first_group + g), by = r / ((float)a.pixels * (float)width);
                          if (width <= 16 || (threadIdx.x & 31) == 0) {
                              value[2 * g] = -by * v[0];
                              value[2 * g + 1] = -by * r * v[1];
                          }
                      });
    __syncthreads();
    if (turns == 0 || at.c >= a.channels) return;
    F2 level[P], along[P];
    GnGroup group(at.c - at.c0, width);
#pragma unroll
    for (int k = 0; k < 2 * P; ++k, group.next(width)) {
        const bool in = at.c + k < a.channels;
        GnChannels<P>::set(level[k / 2], k % 2, in ? value[2 * group.group] : 0.0f);
        GnChannels<P>::set(along[k / 2], k % 2, in ? value[2 * group.group + 1] : 0.0f);
    }
    T *dx = static_cast<T *>(a.dx) + at.worker * a.dx_worker + at.sample * a.dx_sample + at.p0 * a.dx_pixel;
    gn_store<T>(a, dx, at.lanes * a.dx_pixel, at.c, turns, [&](int k, F2 (&d)[P]) {
        const typename X::Kept raw = X::kept(x_place + k * GR_THREADS * M::X_BYTES, power_place + k * GR_THREADS);
        F2 g[P];
        X::centred(raw, ch.minus, d);
        if constexpr (WIDE) {
            F2 low[2], high[2];
            LnChunk<float>::read(dz_place[k * GR_THREADS], low);
            LnChunk<float>::read(dz_place[plane + k * GR_THREADS], high);
            g[0] = low[0]; g[1] = low[1]; g[2] = high[0]; g[3] = high[1];
        } else {
            LnChunk<T>::read(dz_place[k * GR_THREADS], g);
        }
#pragma unroll
        for (int j = 0; j < P; ++j) d[j] = fma(g[j], ch.scale[j], fma(d[j], along[j], level[j]));
    });
}

// ---- launches --------------------------------------------------------------------------------------------

constexpr int GN_MAX_MEMORY = 112 * 1024;
// Beyond, reading twice is faster backward, which is most of the two passes: its threads walk down many more pixels for what each does once
// (forward / backward from the checkpoint, SiLU, held and read twice: 32 images of 196 pixels x 128 bfloat16 6 / 10 and 10 / 12 us, 256 of
// 64 x 256 11 / 21 and 17 / 29, 256 of 256 x 256 19 / 52 and 30 / 52; 256 of 196 x 1024 54 / 135 and 60 / 117).
constexpr int64_t GN_RESIDENT_ELEMENTS = 1 << 24;

template <auto KERNEL>
static cudaError_t gn_resident_launch(const GnArgs &a, int smem, cudaStream_t st) {
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = ln_allow_smem(KERNEL, GN_MAX_MEMORY, allowed);
    if (e != cudaSuccess) return e;
    return ln_launch(KERNEL, a, (int64_t)a.workers * a.samples * a.tiles, 1, GR_THREADS, smem, st);
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
        return a.x ? gn_resident_launch<gn_resident_backward_kernel<T, GnFromX<T, true>, ACT>>(a, smem, st)
                   : gn_resident_launch<gn_resident_backward_kernel<T, GnFromCheckpoint<T>, ACT>>(a, smem, st);
    }
};
cudaError_t gn_resident_backward(const GnArgs &a, int dtype, int smem, cudaStream_t st) {
    return dtype == 0 ? gn_for_act(a.act, GnResidentBackward<float>{a, smem, st}) : gn_for_act(a.act, GnResidentBackward<__nv_bfloat16>{a, smem, st});
}

template <typename T>
static int gn_memory_bytes(bool backward, bool checkpoint, int act, int turns, int width) {
    if (!backward) return GnMemory<T, false, 0>::total(turns, width);
    const bool wide = act == LIEC_ACT_SILU && sizeof(T) == 2;
    if (checkpoint) return wide ? GnMemory<T, true, 2>::total(turns, width) : GnMemory<T, true, 1>::total(turns, width);
    return wide ? GnMemory<T, false, 2>::total(turns, width) : GnMemory<T, false, 1>::total(turns, width);
}

// Channels per CTA: whole groups and whole blocks of a checkpoint, at least 64 bytes of a pixel (or all of it); more, to 128
// bytes and then to a thread per pixel and chunk, while there are CTAs enough.
bool gn_resident_plan(GnArgs &a, int dtype, bool backward, bool checkpoint, int &smem) {
    const int vec = dtype == 0 ? 4 : 8, group = a.channels / a.groups;
    const int64_t images = (int64_t)a.workers * a.samples;
    if (a.pixels > 4096 || images * a.pixels * a.channels > GN_RESIDENT_ELEMENTS) return false;
    int unit = group;
    while (unit % CK_BLOCK != 0) unit += group;
    auto fits = [&](int channels) {
        const int chunks = (int)(ck_cols(channels) / vec);
        if (chunks > GR_THREADS / 2) return false;
        a.tile_chunks = chunks;
        a.tiles = (a.channels + channels - 1) / channels;
        const int lanes = GR_THREADS / chunks;
        a.turns = (int)((a.pixels + lanes - 1) / lanes);
        smem = dtype == 0 ? gn_memory_bytes<float>(backward, checkpoint, a.act, a.turns, chunks * vec)
                          : gn_memory_bytes<__nv_bfloat16>(backward, checkpoint, a.act, a.turns, chunks * vec);
        return smem <= GN_MAX_MEMORY;
    };
    // (a range that is doubled is still a multiple of the unit, or all channels)
    int channels = std::min(unit, a.channels);
    while (channels < a.channels && channels * (16 / vec) < 64) channels = std::min(2 * channels, a.channels);
    while (channels < a.channels) {
        const int wider = std::min(2 * channels, a.channels);
        if (images * ((a.channels + wider - 1) / wider) < 4 * LN_SMS || !fits(wider) || (a.turns > 16 && channels * (16 / vec) >= 128)) break;
        channels = wider;
    }
    return fits(channels);
}

}  // namespace liec

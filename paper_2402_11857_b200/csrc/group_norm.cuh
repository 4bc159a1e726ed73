// Group normalisation with an activation, channels last: what the kernels share.
//
// z = (x - m) A + b with A = r w is evaluated from d = x - m (rounded once, so a far mean costs no digits), one fused
// operation more.  A thread owns one 16-byte chunk of channels and walks down the pixels, so what belongs to a channel
// stays in registers and a channel's sums are the thread's until they meet those of the other pixels.
#pragma once
#include <type_traits>

#include "activation.cuh"

namespace liec {

constexpr int GN_THREADS = 256;

// A thread's chunks of one array, walked pixel by pixel (`step` elements): load(u) is u turns ahead.  Raw is what a load leaves in
// registers, so that several can be under way; rows off the 16-byte grid (not WHOLE) give two granules each, cut when
// they are used.
template <typename T, bool WHOLE>
struct GnReader {
    static constexpr int VEC = Bits<T>::VEC;
    struct Pair { uint4 a, b; };
    struct One { uint4 a; };
    using Raw = std::conditional_t<WHOLE, One, Pair>;
    const T *row;   // this turn's chunk
    int64_t step;
    int c, cols;
    __device__ __forceinline__ GnReader(const T *first, int64_t step, int c, int cols) : row(first + c), step(step), c(c), cols(cols) {}
    __device__ __forceinline__ void advance(int turns) { row += turns * step; }
    __device__ __forceinline__ const void *place() const { return row; }
    __device__ __forceinline__ bool inside(const T *now, uint32_t &shift) const {   // two whole granules hold the chunk
        shift = (uint32_t)reinterpret_cast<uintptr_t>(now) & 15u;
        const int back = (int)shift / (int)sizeof(T);
        return c >= back && c - back + 2 * VEC <= cols;
    }
    __device__ __forceinline__ Raw load(int u) const {
        Raw r;
        const T *now = row + u * step;
        if constexpr (WHOLE) {   // (cols is a multiple of a chunk)
            r.a = c < cols ? __ldg(reinterpret_cast<const uint4 *>(now)) : make_uint4(0u, 0u, 0u, 0u);
        } else {
            uint32_t shift;
            if (inside(now, shift)) {
                const uint4 *g = reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(now) & ~uintptr_t(15));
                r.a = __ldg(g);
                r.b = __ldg(g + 1);
            } else {   // at a row's ends, element by element, put together in chunk(): nothing waits here
                uint32_t w[8] = {};
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (c + e < cols) {
                        if constexpr (sizeof(T) == 4) w[e] = __ldg(reinterpret_cast<const unsigned *>(now) + e);
                        else w[e] = __ldg(reinterpret_cast<const unsigned short *>(now) + e);
                    }
                r.a = make_uint4(w[0], w[1], w[2], w[3]);
                r.b = make_uint4(w[4], w[5], w[6], w[7]);
            }
        }
        return r;
    }
    __device__ __forceinline__ uint4 chunk(const Raw &r, int u) const {
        if constexpr (!WHOLE) {
            uint32_t shift;
            if (inside(row + u * step, shift)) return cut_granules<(int)sizeof(T)>(r.a, r.b, shift);
            if constexpr (sizeof(T) == 2) return make_uint4(r.a.x | r.a.y << 16, r.a.z | r.a.w << 16, r.b.x | r.b.y << 16, r.b.z | r.b.w << 16);
        }
        return r.a;
    }
};

// Where x comes from: the activations themselves, or their checkpoint.
template <typename T, bool WHOLE>
struct GnFromX : GnReader<T, WHOLE> {
    static constexpr bool CHECKPOINT = false;
    using Raw = typename GnReader<T, WHOLE>::Raw;
    using Kept = uint4;
    __device__ __forceinline__ GnFromX(const GnArgs &a, int worker, int sample, int64_t p, int lanes, int c)
        : GnReader<T, WHOLE>(static_cast<const T *>(a.x) + worker * a.x_worker + sample * a.x_sample + p * a.x_pixel, lanes * a.x_pixel, c, a.channels) {}
    __device__ __forceinline__ Kept keep(const Raw &r, int u) const { return this->chunk(r, u); }
    struct Powers {};   // nothing but the chunk itself is needed
    __device__ __forceinline__ Powers powers(int) const { return {}; }
    static __device__ __forceinline__ void announce(const Powers &, int) {}
    static __device__ __forceinline__ Kept kept(uint4 chunk, const Powers &, int) { return chunk; }
    static __device__ __forceinline__ void walk(Powers &, int) {}
    __device__ __forceinline__ void next() { this->row += this->step; }
    static __device__ __forceinline__ Kept kept(const char *place, const uint8_t *) { return *reinterpret_cast<const uint4 *>(place); }
    template <int P>
    static __device__ __forceinline__ void centred(const Kept &chunk, const F2 (&minus)[P], F2 (&d)[P]) {
        LnChunk<T>::read(chunk, d);
#pragma unroll
        for (int k = 0; k < P; ++k) d[k] = add(d[k], minus[k]);
    }
};

template <typename T>
struct GnFromCheckpoint {
    static constexpr bool CHECKPOINT = true;
    static constexpr int VEC = Bits<T>::VEC;
    struct Raw { uint32_t w[VEC / 4]; uint32_t byte; };
    using Kept = Raw;
    const int8_t *q;
    const uint8_t *scales;
    int64_t step;
    __device__ __forceinline__ GnFromCheckpoint(const GnArgs &a, int worker, int sample, int64_t p, int lanes, int c) {
        const int64_t cols = (a.channels + CK_BLOCK - 1) / CK_BLOCK * CK_BLOCK, row = ((int64_t)worker * a.samples + sample) * a.pixels + p;
        q = a.q + row * cols + c;
        scales = a.scales + row * (cols / CK_BLOCK) + c / CK_BLOCK;
        step = lanes * (cols / CK_BLOCK);   // of the powers
    }
    __device__ __forceinline__ void advance(int turns) {
        q += turns * (step * CK_BLOCK);
        scales += turns * step;
    }
    __device__ __forceinline__ const void *place() const { return q; }
    __device__ __forceinline__ Raw load(int u) const {
        Raw r;
        const int8_t *at = q + u * (step * CK_BLOCK);
        if constexpr (VEC == 8) {
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(at));
            r.w[0] = v.x;
            r.w[1] = v.y;
        } else {
            r.w[0] = __ldg(reinterpret_cast<const uint32_t *>(at));
        }
        r.byte = __ldg(scales + u * step);
        return r;
    }
    __device__ __forceinline__ Kept keep(const Raw &r, int) const { return r; }
    // A byte among few: no copy of its own brings it to the ring.  It is announced to the L2 cache when its chunk's copy
    // starts and loaded one stage before it is used.
    struct Powers {
        const uint8_t *at;   // of the stage after the present one
        int64_t step;
        int left;            // turns from there on
        uint32_t now[2], next[2];
        __device__ __forceinline__ void load() {
            next[0] = left > 0 ? (uint32_t)__ldg(at) : 127u;
            next[1] = left > 1 ? (uint32_t)__ldg(at + step) : 127u;
        }
    };
    __device__ __forceinline__ Powers powers(int turns) const {
        Powers p{scales, step, turns, {}, {}};
        p.load();
        walk(p, 2);
        return p;
    }
    static __device__ __forceinline__ void walk(Powers &p, int n) {   // a stage on; single turns only at the end
        if (n == 2) {
            p.now[0] = p.next[0];
            p.now[1] = p.next[1];
            p.at += 2 * p.step;
            p.left -= 2;
            p.load();
        } else {
            p.now[0] = p.now[1];
            p.now[1] = p.next[0];
            p.next[0] = p.next[1];
            p.at += p.step;
            p.left -= 1;
            p.next[1] = p.left > 1 ? (uint32_t)__ldg(p.at + p.step) : 127u;
        }
    }
    __device__ __forceinline__ void announce(const Powers &, int) const { asm volatile("prefetch.global.L2 [%0];" ::"l"(scales)); }
    static __device__ __forceinline__ Kept kept(uint4 chunk, const Powers &p, int u) {
        Raw r;
        r.w[0] = chunk.x;
        if constexpr (VEC == 8) r.w[1] = chunk.y;
        r.byte = p.now[u];
        return r;
    }
    __device__ __forceinline__ void next() {
        q += step * CK_BLOCK;
        scales += step;
    }
    static __device__ __forceinline__ Kept kept(const char *place, const uint8_t *power) {
        Raw r;
        if constexpr (VEC == 8) {
            const uint2 v = *reinterpret_cast<const uint2 *>(place);
            r.w[0] = v.x;
            r.w[1] = v.y;
        } else {
            r.w[0] = *reinterpret_cast<const uint32_t *>(place);
        }
        r.byte = *power;
        return r;
    }
    template <int P>
    static __device__ __forceinline__ void centred(const Kept &raw, const F2 (&minus)[P], F2 (&d)[P]) {
        const F2 power = f2(ck_power(raw.byte));
#pragma unroll
        for (int k = 0; k < P; k += 2) ck_unpack(raw.w[k / 2], d[k], d[k + 1]);
#pragma unroll
        for (int k = 0; k < P; ++k) d[k] = fma(d[k], power, minus[k]);   // (q 2^e is exact: one rounding)
    }
};

// use(u, raw) for all turns, the loads of N of them issued together; advance(n) then walks n turns on.
template <int N, typename L, typename U, typename A>
__device__ __forceinline__ void gn_turns(int64_t turns, L &&load, U &&use, A &&advance) {
#pragma unroll 1
    for (; turns >= N; turns -= N) {
        decltype(load(0)) raw[N];
#pragma unroll
        for (int u = 0; u < N; ++u) raw[u] = load(u);
#pragma unroll
        for (int u = 0; u < N; ++u) use(u, raw[u]);
        advance(N);
    }
#pragma unroll 1
    for (; turns > 0; --turns) {
        use(0, load(0));
        advance(1);
    }
}

// ---- a thread's ring in shared memory: its chunks of the next turns on their way, at no cost of registers ----
//
// Two turns make a stage.  Only the thread that copies a chunk reads it again, so no barrier guards the ring.
constexpr int GN_STAGES = 4;
template <int BYTES>
struct GnRing {
    static constexpr int SIZE = GN_STAGES * 2 * GN_THREADS * BYTES;
    uint32_t place;
    __device__ __forceinline__ explicit GnRing(char *memory) : place((uint32_t)__cvta_generic_to_shared(memory) + threadIdx.x * BYTES) {}
    __device__ __forceinline__ void copy(int at, const void *from) const {
        const uint32_t to = place + at * BYTES;
        if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
    }
    __device__ __forceinline__ uint4 read(int turn) const {
        const uint32_t at = place + turn * BYTES;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if constexpr (BYTES == 16) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
        else if constexpr (BYTES == 8) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
        else asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v.x) : "r"(at) : "memory");
        return v;
    }
};

// copy(place) for every turn in order, each a few stages before its use(place, u); place: bytes from the ring's start for chunks of one
// byte, u = 0 or 1 within a stage; after(n) ends a stage of n turns.
template <typename C, typename U, typename A>
__device__ __forceinline__ void gn_ring_turns(int turns, C &&copy, U &&use, A &&after) {
    constexpr int TURN = GN_THREADS, RING = 2 * GN_STAGES * TURN;
    static_assert((RING & (RING - 1)) == 0, "places wrap by a mask");
    int ahead = 0;   // turns whose copies are under way
#pragma unroll
    for (int s = 0; s < GN_STAGES - 1; ++s) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (ahead + u < turns) copy((2 * s + u) * TURN);
        ahead += 2;
        copy_commit();
    }
    int now = 0;
    // while both turns of the stage to copy are there, so are those to use
#pragma unroll 1
    for (; ahead + 1 < turns; ahead += 2) {
        const int fill = (now + 2 * (GN_STAGES - 1) * TURN) & (RING - 1);
        copy(fill);
        copy(fill + TURN);
        copy_commit();
        copy_wait<GN_STAGES - 1>();
        use(now, 0);
        use(now + TURN, 1);
        after(2);
        now = (now + 2 * TURN) & (RING - 1);
    }
    const int left = turns - (ahead - 2 * (GN_STAGES - 1));
    if (ahead < turns) copy((now + 2 * (GN_STAGES - 1) * TURN) & (RING - 1));
    copy_commit();
    copy_wait<0>();
#pragma unroll 1
    for (int k = 0; k < left; ++k) {
        use(now, 0);
        after(1);
        now = (now + TURN) & (RING - 1);
    }
}

// SiLU of a pair.  Results in bfloat16 take the hardware's exponential and reciprocal as they are (relative errors of
// (|z| + 2) 2^-23, far below a bfloat16 step wherever the gate is not zero; an infinite exponential gives a gate of zero).
__device__ __forceinline__ float gn_exp2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float gn_reciprocal(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
template <typename T>
__device__ __forceinline__ F2 gn_exp(F2 z) {   // exp(-z)
    if constexpr (sizeof(T) == 4) return f2(fminf(expf(-lo(z)), 1e30f), fminf(expf(-hi(z)), 1e30f));
    const F2 t = mul(z, f2(-1.44269504f));
    return f2(gn_exp2(lo(t)), gn_exp2(hi(t)));
}
template <typename T>
__device__ __forceinline__ F2 gn_gate(F2 e) {   // 1 / (1 + e)
    const F2 u = add(e, f2(1.0f));
    if constexpr (sizeof(T) == 4) return f2(__fdividef(1.0f, lo(u)), __fdividef(1.0f, hi(u)));
    return f2(gn_reciprocal(lo(u)), gn_reciprocal(hi(u)));
}

template <typename T, int ACT>
__device__ __forceinline__ F2 gn_act(F2 z) {
    if constexpr (ACT == LIEC_ACT_RELU) return f2(lo(z) < 0.0f ? 0.0f : lo(z), hi(z) < 0.0f ? 0.0f : hi(z));   // (NaN stays)
    if constexpr (ACT == LIEC_ACT_SILU) return mul(z, gn_gate<T>(gn_exp<T>(z)));
    return z;
}

// silu'(z) = s (1 + z (1 - s)).  1 - s = exp(-z) s keeps its digits where s is near one; in bfloat16 the difference has
// enough of them.
template <typename T>
__device__ __forceinline__ F2 gn_silu_slope(F2 z) {
    const F2 e = gn_exp<T>(z), s = gn_gate<T>(e);
    const F2 rest = sizeof(T) == 4 ? mul(e, s) : fma(s, f2(-1.0f), f2(1.0f));
    return mul(s, fma(z, rest, f2(1.0f)));
}

// z from its definition in binary64.
static __device__ __noinline__ bool gn_positive(const GnArgs &a, int worker, int64_t image, int c, float x) {
    const int64_t g = image * a.groups + c / (a.channels / a.groups);
    const double w = a.weight ? (double)a.weight[worker * a.weight_stride + c] : 1.0, b = a.bias ? (double)a.bias[worker * a.bias_stride + c] : 0.0;
    return ((double)x - (double)a.mean[g]) * (double)a.rstd[g] * w + b > 0.0;
}

// The group of a channel, channel after channel.
struct GnGroup {
    uint32_t group, rest;
    __device__ __forceinline__ GnGroup(uint32_t c, uint32_t width) : group(c / width), rest(c - c / width * width) {}
    __device__ __forceinline__ void next(uint32_t width) {
        if (++rest == width) {
            rest = 0;
            ++group;
        }
    }
};

// What belongs to a thread's channels: -m, A = r w, b; zeros beyond the last channel.
template <int P>
struct GnChannels {
    F2 minus[P], scale[P], bias[P];
    // statistics(group, m, r)
    template <typename F>
    __device__ __forceinline__ void read(const GnArgs &a, int worker, int c, F &&statistics) {
        const uint32_t width = (uint32_t)a.channels / (uint32_t)a.groups;
        GnGroup g(c, width);
#pragma unroll
        for (int k = 0; k < 2 * P; ++k, g.next(width)) {
            float m = 0.0f, s = 0.0f, b = 0.0f;
            if (c + k < a.channels) {
                statistics(g.group, m, s);
                s *= a.weight ? __ldg(a.weight + worker * a.weight_stride + c + k) : 1.0f;
                b = a.bias ? __ldg(a.bias + worker * a.bias_stride + c + k) : 0.0f;
            }
            set(minus[k / 2], k % 2, -m);
            set(scale[k / 2], k % 2, s);
            set(bias[k / 2], k % 2, b);
        }
    }
    __device__ __forceinline__ void read(const GnArgs &a, int worker, int64_t image, int c) {
        const float *mean = a.mean + image * a.groups, *rstd = a.rstd + image * a.groups;
        read(a, worker, c, [&](uint32_t g, float &m, float &r) {
            m = __ldg(mean + g);
            r = __ldg(rstd + g);
        });
    }
    static __device__ __forceinline__ void set(F2 &p, int odd, float v) { p = odd ? f2(lo(p), v) : f2(v, 0.0f); }
};

// dz = dy act'(z) from d = x - m.  The sign of z decides for ReLU: z carries at most 4 2^-24 (|b| + |z|) of rounding, so
// where |z| is above 2^-20 |b| its sign is right; elsewhere it is taken from binary64.
template <typename T, int ACT, int P, typename E>
__device__ __forceinline__ void gn_slope(const GnArgs &a, int worker, int64_t image, int c, const GnChannels<P> &ch, E &&exact,
                                         const F2 (&d)[P], const F2 (&dy)[P], F2 (&dz)[P]) {
    if constexpr (ACT == LIEC_ACT_NONE) {
#pragma unroll
        for (int k = 0; k < P; ++k) dz[k] = dy[k];
        return;
    }
    F2 z[P];
#pragma unroll
    for (int k = 0; k < P; ++k) z[k] = fma(d[k], ch.scale[k], ch.bias[k]);
    if constexpr (ACT == LIEC_ACT_SILU) {
#pragma unroll
        for (int k = 0; k < P; ++k) dz[k] = mul(gn_silu_slope<T>(z[k]), dy[k]);
    }
    if constexpr (ACT == LIEC_ACT_RELU) {
        constexpr float NEAR = 9.5367431640625e-7f;
        bool near = false;
        F2 kept[P];   // (dz may be dy)
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const float l = lo(z[k]), h = hi(z[k]);
            near |= fabsf(l) <= NEAR * fabsf(lo(ch.bias[k]));
            near |= fabsf(h) <= NEAR * fabsf(hi(ch.bias[k]));
            kept[k] = dy[k];
            dz[k] = f2(l > 0.0f ? lo(dy[k]) : 0.0f, h > 0.0f ? hi(dy[k]) : 0.0f);
        }
        if (near) {
            F2 x[P];
            exact(x);   // x itself
#pragma unroll
            for (int k = 0; k < P; ++k) {
                float v[2] = {lo(dz[k]), hi(dz[k])};
                const float each[2] = {lo(x[k]), hi(x[k])}, was[2] = {lo(kept[k]), hi(kept[k])}, at[2] = {lo(z[k]), hi(z[k])}, b[2] = {lo(ch.bias[k]), hi(ch.bias[k])};
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (fabsf(at[e]) <= NEAR * fabsf(b[e]) && c + 2 * k + e < a.channels) v[e] = gn_positive(a, worker, image, c + 2 * k + e, each[e]) ? was[e] : 0.0f;
                dz[k] = f2(v[0], v[1]);
            }
        }
    }
}

// Mean and squares of a thread's entries in one pass: sums s of d and t of d^2 about an origin (minus is its negative) that
// starts as the thread's own first entry and moves to the mean so far as the entries become more.  N entries that lie about
// their mean and n further ones about that mean: the squares of the n are at most n / N times those of all about their common
// mean, so nothing is lost however far the first entry, or any other, lies from the rest.
template <int P>
struct GnMoments {
    F2 minus[P] = {}, s[P] = {}, t[P] = {};   // (minus is zero without entries)
    template <typename T>
    __device__ __forceinline__ void start(uint4 first) {
        LnChunk<T>::read(first, minus);
#pragma unroll
        for (int k = 0; k < P; ++k) minus[k] = mul(minus[k], f2(-1.0f));
    }
    __device__ __forceinline__ void take(const F2 (&x)[P]) {
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const F2 d = add(x[k], minus[k]);
            s[k] = add(s[k], d);
            t[k] = fma(d, d, t[k]);
        }
    }
    // Sums about an origin h further on: n entries.
    static __device__ __forceinline__ void moved(F2 &s, F2 &t, F2 h, F2 minus_n) {
        const F2 was = s;
        s = fma(minus_n, h, s);
        t = fma(mul(h, f2(-1.0f)), add(was, s), t);
    }
    // To the mean of the n entries taken; inverse is about 1 / n.
    __device__ __forceinline__ void move(float n, float inverse) {
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const F2 to = fma(s[k], f2(-inverse), minus[k]), h = fma(to, f2(-1.0f), minus[k]);
            minus[k] = to;
            moved(s[k], t[k], h, f2(-n));
        }
    }
    // To an origin that the threads of a channel share.
    __device__ __forceinline__ void move_to(int k, F2 origin, float n) { moved(s[k], t[k], add(origin, minus[k]), f2(-n)); }
    // The sum of the n entries themselves.
    __device__ __forceinline__ F2 whole(int k, float n) const { return fma(minus[k], f2(-n), s[k]); }
};

// The checkpoint of a thread's chunks: the 4 or 8 threads of a block are neighbours in a warp and come here together.
template <typename T>
struct GnCompressor {
    static constexpr int VEC = Bits<T>::VEC, P = VEC / 2, LANES = CK_BLOCK / VEC;
    int8_t *q;
    uint8_t *scales;
    int64_t step;
    uint32_t mates;
    bool first;
    __device__ __forceinline__ GnCompressor(const GnArgs &a, int64_t row, int lanes, int c) {
        const int64_t cols = (a.channels + CK_BLOCK - 1) / CK_BLOCK * CK_BLOCK;
        q = a.q + row * cols + c;
        scales = a.scales + row * (cols / CK_BLOCK) + c / CK_BLOCK;
        step = lanes * (cols / CK_BLOCK);
        mates = ((1u << LANES) - 1u) << (threadIdx.x & 31 & ~(LANES - 1));
        first = c % CK_BLOCK == 0;
    }
    __device__ __forceinline__ void advance(int turns) {
        q += turns * (step * CK_BLOCK);
        scales += turns * step;
    }
    __device__ __forceinline__ void store(int u, uint4 chunk) const {
        uint32_t top = ck_top<T>(chunk);
#pragma unroll
        for (int m = LANES / 2; m >= 1; m >>= 1) top = ck_larger<T>(top, __shfl_xor_sync(mates, top, m));
        const uint32_t byte = ck_scale_byte(__uint_as_float(ck_top_bits<T>(top)));
        F2 v[P];
        LnChunk<T>::read(chunk, v);
        uint32_t words[P / 2];
        ck_bytes<P>(v, byte, words);
        int8_t *to = q + u * (step * CK_BLOCK);
        if constexpr (VEC == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(words[0], words[1]);
        else *reinterpret_cast<uint32_t *>(to) = words[0];
        if (first) scales[u * step] = (uint8_t)byte;
    }
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    return v;
}

// Images that CTAs hold in shared memory (group_norm_resident.cu): sets the launch's sizes, or says no.
bool gn_resident_plan(GnArgs &a, int dtype, bool backward, bool checkpoint, int &smem);
cudaError_t gn_resident_forward(const GnArgs &a, int dtype, int smem, cudaStream_t st);
cudaError_t gn_resident_backward(const GnArgs &a, int dtype, int smem, cudaStream_t st);

template <typename F>
cudaError_t gn_for_act(int act, F &&f) {
    if (act == LIEC_ACT_RELU) return f.template operator()<LIEC_ACT_RELU>();
    if (act == LIEC_ACT_SILU) return f.template operator()<LIEC_ACT_SILU>();
    return f.template operator()<LIEC_ACT_NONE>();
}

}  // namespace liec

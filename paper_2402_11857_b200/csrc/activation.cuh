// Chunks of 16 bytes of activations (4 binary32 or 8 bfloat16) of rows of any place, and the blocks of an 8-bit
// checkpoint.
#pragma once
#include "activation.h"
#include "granule.cuh"
#include "layer_norm_common.cuh"

namespace liec {

template <typename T> struct Bits;
template <> struct Bits<float> { static constexpr int VEC = 4; };
template <> struct Bits<__nv_bfloat16> { static constexpr int VEC = 8; };

// Element by element, zeros from column cols on.
template <typename T>
__device__ __noinline__ uint4 load_chunk_edge(const T *p, int left) {
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < Bits<T>::VEC; ++e)
        if (e < left) {
            if constexpr (sizeof(T) == 4) w[e] = __ldg(reinterpret_cast<const unsigned *>(p) + e);
            else w[e / 2] |= (uint32_t)__ldg(reinterpret_cast<const unsigned short *>(p) + e) << (e % 2 * 16);
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Columns c .. c + VEC - 1 of a row of cols elements; zeros beyond.  Rows off the 16-byte grid are read as whole
// granules where those lie within the row.
template <typename T>
__device__ __forceinline__ uint4 load_chunk(const T *row, int c, int cols) {
    constexpr int VEC = Bits<T>::VEC;
    const T *p = row + c;
    const int shift = (int)(reinterpret_cast<uintptr_t>(p) & 15u), back = shift / (int)sizeof(T);
    if (shift == 0 && c + VEC <= cols) return __ldg(reinterpret_cast<const uint4 *>(p));
    if (shift != 0 && c >= back && c - back + 2 * VEC <= cols) {
        const uint4 *g = reinterpret_cast<const uint4 *>(p - back);
        return cut_granules<(int)sizeof(T)>(__ldg(g), __ldg(g + 1), (uint32_t)shift);
    }
    return load_chunk_edge(p, cols - c);
}

template <typename T>
__device__ __forceinline__ void store_chunk(T *row, int c, int cols, const F2 (&v)[Bits<T>::VEC / 2]) {
    constexpr int VEC = Bits<T>::VEC;
    T *p = row + c;
    if ((reinterpret_cast<uintptr_t>(p) & 15u) == 0 && c + VEC <= cols) {
        LnChunk<T>::write(p, v);
        return;
    }
#pragma unroll
    for (int k = 0; k < VEC / 2; ++k) {
        if (c + 2 * k < cols) ln_store(p + 2 * k, lo(v[k]));
        if (c + 2 * k + 1 < cols) ln_store(p + 2 * k + 1, hi(v[k]));
    }
}

// ---- a checkpoint's block: 32 signed bytes q and the byte e + 127 of a power of two; stands for q 2^e ----
//
// e is the least exponent from -126 on for which the largest magnitude a rounds to at most 127: a 2^-e < 127.5.  With
// a = 1.m 2^E that is e = E - 6, and E - 5 where 1.m >= 127.5 / 64, which is where adding 2^16 to the bits of a carries
// into the exponent.  Next to the end of the range e stays at 121 and q is held to 127, so that q 2^e is finite.  An
// infinity or NaN in the block: byte 255, q = 0, which gives NaN when multiplied out.
constexpr uint32_t CK_TOP_BYTE = 248u;
__device__ __forceinline__ uint32_t ck_scale_byte(float a) {
    const uint32_t bits = __float_as_uint(a);
    return bits >= 0x7f800000u ? 255u : (uint32_t)min(max((int)((bits + 0x10000u) >> 23) - 6, 1), (int)CK_TOP_BYTE);
}
__device__ __forceinline__ float ck_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }   // 2^-e
__device__ __forceinline__ float ck_power(uint32_t byte) { return __uint_as_float(byte << 23); }
constexpr float CK_ROUND = 12582912.0f;   // 1.5 2^23: x + this has the integer nearest to x (even at halves) in its last bits

// Two values' bytes, in the last byte of each half; the fused operation rounds x 2^-e once, to the integer.
__device__ __forceinline__ F2 ck_round(F2 x, F2 inverse) { return fma(x, inverse, f2(CK_ROUND)); }
__device__ __forceinline__ uint32_t ck_pack(F2 a, F2 b) {
    const uint32_t l = __byte_perm((uint32_t)a.v, (uint32_t)(a.v >> 32), 0x0040), h = __byte_perm((uint32_t)b.v, (uint32_t)(b.v >> 32), 0x0040);
    return __byte_perm(l, h, 0x5410);
}
// The bytes of a chunk whose block has the scale byte `byte`.
template <int P>
__device__ __forceinline__ void ck_bytes(F2 (&x)[P], uint32_t byte, uint32_t (&words)[P / 2]) {
    if (byte == CK_TOP_BYTE) {
        const float most = 127.0f * 2658455991569831745807614120560689152.0f;   // 127 2^121
#pragma unroll
        for (int k = 0; k < P; ++k) x[k] = f2(fminf(fmaxf(lo(x[k]), -most), most), fminf(fmaxf(hi(x[k]), -most), most));
    }
    const F2 inverse = f2(ck_inverse(byte));
#pragma unroll
    for (int k = 0; k < P; k += 2) words[k / 2] = byte == 255u ? 0u : ck_pack(ck_round(x[k], inverse), ck_round(x[k + 1], inverse));
}
// Four bytes as numbers: 2^23 + (q + 128) has q + 128 as its last byte.
__device__ __forceinline__ void ck_unpack(uint32_t w, F2 &a, F2 &b) {
    const uint32_t u = w ^ 0x80808080u;
    const F2 off = f2(-8388736.0f);
    a = add(f2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7441))), off);
    b = add(f2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7442)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7443))), off);
}

// Largest magnitude of a chunk, as bits: those of magnitudes order like the numbers, NaN above infinity.  Bfloat16: two at
// a time, the two halves apart until ck_top_bits.
template <typename T>
__device__ __forceinline__ uint32_t ck_larger(uint32_t a, uint32_t b) {
    if constexpr (sizeof(T) == 4) return max(a, b);
    else return __vmaxu2(a, b);
}
template <typename T>
__device__ __forceinline__ uint32_t ck_top(uint4 q) {
    constexpr uint32_t MAGNITUDE = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
    return ck_larger<T>(ck_larger<T>(q.x & MAGNITUDE, q.y & MAGNITUDE), ck_larger<T>(q.z & MAGNITUDE, q.w & MAGNITUDE));
}
template <typename T>
__device__ __forceinline__ uint32_t ck_top_bits(uint32_t top) {
    if constexpr (sizeof(T) == 4) return top;
    else return max(top & 0xffff0000u, top << 16);
}

}  // namespace liec

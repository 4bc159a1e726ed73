// 8-bit checkpoints of activations: every 32 consecutive channels of a row become 32 signed bytes and one power of
// two, and come back as bytes times power, which is exact in binary32 and in bfloat16.
#include "activation.cuh"

namespace liec {

constexpr int CK_THREADS = 256;

// A thread takes one 16-byte chunk of x; the 4 (bfloat16) or 8 (binary32) threads of a block find its largest
// magnitude by shuffles.  Chunks are numbered through the padded rows, so a block never crosses a warp.
template <typename T>
__global__ void __launch_bounds__(CK_THREADS) ck_compress_kernel(const __grid_constant__ CkArgs a, int64_t row_chunks, int64_t chunks) {
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2, LANES = CK_BLOCK / VEC;
    const int64_t i = (int64_t)blockIdx.x * CK_THREADS + threadIdx.x;
    const int64_t row = i / row_chunks;
    const int c = (int)(i - row * row_chunks) * VEC;
    const bool live = i < chunks;
    uint4 chunk = make_uint4(0u, 0u, 0u, 0u);
    if (live) {
        const int64_t w = row / a.rows;
        chunk = load_chunk(static_cast<const T *>(a.in) + w * a.x_worker + (row - w * a.rows) * a.x_row, c, a.cols);
    }
    uint32_t top = ck_top<T>(chunk);
#pragma unroll
    for (int m = LANES / 2; m >= 1; m >>= 1) top = ck_larger<T>(top, __shfl_xor_sync(0xffffffffu, top, m));
    const uint32_t byte = ck_scale_byte(__uint_as_float(ck_top_bits<T>(top)));
    F2 x[P];
    LnChunk<T>::read(chunk, x);
    if (!live) return;
    uint32_t words[P / 2];
    ck_bytes<P>(x, byte, words);
    int8_t *q = a.q + i * VEC;
    if constexpr (VEC == 8) *reinterpret_cast<uint2 *>(q) = make_uint2(words[0], words[1]);
    else *reinterpret_cast<uint32_t *>(q) = words[0];
    if (i % LANES == 0) a.scales[i / LANES] = (uint8_t)byte;
}

template <typename T>
__global__ void __launch_bounds__(CK_THREADS) ck_restore_kernel(const __grid_constant__ CkArgs a, int64_t row_chunks, int64_t chunks) {
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2, LANES = CK_BLOCK / VEC;
    const int64_t i = (int64_t)blockIdx.x * CK_THREADS + threadIdx.x;
    if (i >= chunks) return;
    const int64_t row = i / row_chunks, w = row / a.rows;
    const int c = (int)(i - row * row_chunks) * VEC;
    if (c >= a.cols) return;
    const F2 power = f2(ck_power(__ldg(a.scales + i / LANES)));
    const int8_t *q = a.q + i * VEC;
    F2 x[P];
    if constexpr (VEC == 8) {
        const uint2 v = __ldg(reinterpret_cast<const uint2 *>(q));
        ck_unpack(v.x, x[0], x[1]);
        ck_unpack(v.y, x[2], x[3]);
    } else {
        ck_unpack(__ldg(reinterpret_cast<const uint32_t *>(q)), x[0], x[1]);
    }
#pragma unroll
    for (int k = 0; k < P; ++k) x[k] = mul(x[k], power);
    store_chunk(static_cast<T *>(a.x) + w * a.x_worker + (row - w * a.rows) * a.x_row, c, a.cols, x);
}

template <typename K>
static cudaError_t ck_launch(K kernel, const CkArgs &a, int vec, cudaStream_t st) {
    const int64_t row_chunks = ck_cols(a.cols) / vec, chunks = row_chunks * a.rows * a.workers;
    if (chunks == 0) return cudaSuccess;
    kernel<<<(unsigned)((chunks + CK_THREADS - 1) / CK_THREADS), CK_THREADS, 0, st>>>(a, row_chunks, chunks);
    return cudaGetLastError();
}

cudaError_t launch_activation_compress(CkArgs a, int dtype, cudaStream_t st) {
    return dtype == 0 ? ck_launch(ck_compress_kernel<float>, a, 4, st) : ck_launch(ck_compress_kernel<__nv_bfloat16>, a, 8, st);
}
cudaError_t launch_activation_restore(CkArgs a, int dtype, cudaStream_t st) {
    return dtype == 0 ? ck_launch(ck_restore_kernel<float>, a, 4, st) : ck_launch(ck_restore_kernel<__nv_bfloat16>, a, 8, st);
}

}  // namespace liec

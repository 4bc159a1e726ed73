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

// A row's chunks, each with its neighbour in the warp: chunks off the 16-byte grid leave as granules, put together from the end
// of the chunk before and the start of this one; what has no neighbour goes element by element.  Whole warps.  (Bfloat16, 32 x
// 4096 rows of 767: 100 us, all element by element 225.  Binary32 has half the elements per chunk: 8 x 8192 rows of 1001
// 108 us, element by element 90.)
__device__ __forceinline__ void store_chunks(__nv_bfloat16 *row, int c, int cols, uint4 chunk, bool live) {
    constexpr int VEC = 8, SIZE = 2;
    const int lane = threadIdx.x & 31, shift = live ? (int)(reinterpret_cast<uintptr_t>(row + c) & 15u) : 0, head = (16 - shift) / SIZE;   // elements up to the next granule
    uint4 before;
    before.x = __shfl_up_sync(0xffffffffu, chunk.x, 1);
    before.y = __shfl_up_sync(0xffffffffu, chunk.y, 1);
    before.z = __shfl_up_sync(0xffffffffu, chunk.z, 1);
    before.w = __shfl_up_sync(0xffffffffu, chunk.w, 1);
    if (!live || c >= cols) return;
    char *to = reinterpret_cast<char *>(row + c);
    int first = 0, end = min(VEC, cols - c);   // elements that are left
    if (shift == 0) {
        if (end == VEC) {
            *reinterpret_cast<uint4 *>(to) = chunk;
            return;
        }
    } else {
        if (lane > 0 && c > 0 && c + head <= cols) {
            *reinterpret_cast<uint4 *>(to - shift) = cut_granules<SIZE>(before, chunk, (uint32_t)(16 - shift));
            first = head;
        }
        if (lane < 31 && c + VEC + head <= cols) end = head;   // the next thread takes them
    }
    const uint32_t words[4] = {chunk.x, chunk.y, chunk.z, chunk.w};
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        if (e >= first && e < end) reinterpret_cast<unsigned short *>(to)[e] = (unsigned short)(words[e / 2] >> (e % 2 * 16));
}

// Rows of any width and place.
template <typename T>
__global__ void __launch_bounds__(CK_THREADS) ck_restore_kernel(const __grid_constant__ CkArgs a, int64_t row_chunks, int64_t chunks) {
    constexpr int VEC = Bits<T>::VEC, P = VEC / 2, LANES = CK_BLOCK / VEC;
    const int64_t i = (int64_t)blockIdx.x * CK_THREADS + threadIdx.x;
    const bool live = i < chunks;
    const int64_t row = live ? i / row_chunks : 0, w = row / a.rows;
    const int c = (int)(i - row * row_chunks) * VEC;
    uint4 chunk = make_uint4(0u, 0u, 0u, 0u);
    if (live) {
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
        if constexpr (VEC == 8) chunk = make_uint4(LnChunk<T>::word(x[0]), LnChunk<T>::word(x[1]), LnChunk<T>::word(x[2]), LnChunk<T>::word(x[3]));
        else if (c < a.cols) store_chunk(static_cast<T *>(a.x) + w * a.x_worker + (row - w * a.rows) * a.x_row, c, a.cols, x);
    }
    if constexpr (VEC == 8) store_chunks(static_cast<T *>(a.x) + w * a.x_worker + (row - w * a.rows) * a.x_row, c, a.cols, chunk, live);
}

// Rows of whole blocks that start on 32 bytes: a thread takes a block, in 32-byte pieces, so that no threads have to meet and a
// warp's powers are 32 bytes that lie together.  HBM bounds it: 32 x 4096 rows of 768 bfloat16 51 us each way (6.0 TB/s; four
// threads per block and 16-byte pieces: 71).
struct Piece { uint32_t w[8]; };
__device__ __forceinline__ Piece load_piece(const void *p) {
    Piece r;
    asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7]) : "l"(p));
    return r;
}
__device__ __forceinline__ void store_piece(void *p, const Piece &r) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7]) : "memory");
}

// Element offset of block i in x; rows that follow one another without a gap are one row.
__device__ __forceinline__ int64_t ck_place(const CkArgs &a, int64_t i, int64_t row_blocks) {
    if (row_blocks == 0) return i * CK_BLOCK;
    const int64_t row = i / row_blocks, w = row / a.rows;
    return w * a.x_worker + (row - w * a.rows) * a.x_row + (i - row * row_blocks) * CK_BLOCK;
}

template <typename T>
__global__ void __launch_bounds__(CK_THREADS) ck_compress_blocks_kernel(const __grid_constant__ CkArgs a, int64_t row_blocks, int64_t blocks) {
    constexpr int PIECES = CK_BLOCK * (int)sizeof(T) / 32, P = CK_BLOCK / 2;
    const int64_t i = (int64_t)blockIdx.x * CK_THREADS + threadIdx.x;
    if (i >= blocks) return;
    const char *from = reinterpret_cast<const char *>(static_cast<const T *>(a.in) + ck_place(a, i, row_blocks));
    Piece x[PIECES];
#pragma unroll
    for (int k = 0; k < PIECES; ++k) x[k] = load_piece(from + 32 * k);
    uint32_t top = 0u;
    F2 v[P];
#pragma unroll
    for (int k = 0; k < PIECES; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 chunk = make_uint4(x[k].w[4 * h], x[k].w[4 * h + 1], x[k].w[4 * h + 2], x[k].w[4 * h + 3]);
            top = ck_larger<T>(top, ck_top<T>(chunk));
            constexpr int EACH = 8 / (int)sizeof(T);   // pairs of a chunk
            F2 pair[EACH];
            LnChunk<T>::read(chunk, pair);
#pragma unroll
            for (int e = 0; e < EACH; ++e) v[(2 * k + h) * EACH + e] = pair[e];
        }
    const uint32_t byte = ck_scale_byte(__uint_as_float(ck_top_bits<T>(top)));
    Piece q;
    ck_bytes<P>(v, byte, q.w);
    store_piece(a.q + i * CK_BLOCK, q);
    a.scales[i] = (uint8_t)byte;
}

template <typename T>
__global__ void __launch_bounds__(CK_THREADS) ck_restore_blocks_kernel(const __grid_constant__ CkArgs a, int64_t row_blocks, int64_t blocks) {
    constexpr int PIECES = CK_BLOCK * (int)sizeof(T) / 32, WORDS = 8 / PIECES;   // words of q per piece of x
    const int64_t i = (int64_t)blockIdx.x * CK_THREADS + threadIdx.x;
    if (i >= blocks) return;
    const Piece q = load_piece(a.q + i * CK_BLOCK);
    const F2 power = f2(ck_power(__ldg(a.scales + i)));
    char *to = reinterpret_cast<char *>(static_cast<T *>(a.x) + ck_place(a, i, row_blocks));
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        Piece x;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            F2 v[2];
            ck_unpack(q.w[k * WORDS + w], v[0], v[1]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                v[e] = mul(v[e], power);
                if constexpr (sizeof(T) == 4) {
                    x.w[4 * w + 2 * e] = __float_as_uint(lo(v[e]));
                    x.w[4 * w + 2 * e + 1] = __float_as_uint(hi(v[e]));
                } else {
                    x.w[2 * w + e] = LnChunk<T>::word(v[e]);
                }
            }
        }
        store_piece(to + 32 * k, x);
    }
}

// Blocks per row if a thread can take a whole one (0: all rows follow one another), -1 if not.
static int64_t ck_row_blocks(const CkArgs &a, const void *x, int size) {
    uint64_t bits = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(a.q);
    if (a.rows > 1) bits |= (uint64_t)a.x_row * size;
    if (a.workers > 1) bits |= (uint64_t)a.x_worker * size;
    if ((bits & 31u) != 0 || a.cols % CK_BLOCK != 0) return -1;
    const bool joined = (a.rows == 1 || a.x_row == a.cols) && (a.workers == 1 || a.x_worker == a.rows * a.cols);
    return joined ? 0 : a.cols / CK_BLOCK;
}

template <typename K>
static cudaError_t ck_launch(K kernel, const CkArgs &a, int64_t row_items, int64_t items, cudaStream_t st) {
    if (items == 0) return cudaSuccess;
    kernel<<<(unsigned)((items + CK_THREADS - 1) / CK_THREADS), CK_THREADS, 0, st>>>(a, row_items, items);
    return cudaGetLastError();
}

cudaError_t launch_activation_compress(CkArgs a, int dtype, cudaStream_t st) {
    const int64_t rows = a.rows * a.workers, cols = ck_cols(a.cols), row_blocks = ck_row_blocks(a, a.in, dtype == 0 ? 4 : 2);
    if (row_blocks >= 0)
        return ck_launch(dtype == 0 ? ck_compress_blocks_kernel<float> : ck_compress_blocks_kernel<__nv_bfloat16>, a, row_blocks, rows * (cols / CK_BLOCK), st);
    return dtype == 0 ? ck_launch(ck_compress_kernel<float>, a, cols / 4, rows * (cols / 4), st) : ck_launch(ck_compress_kernel<__nv_bfloat16>, a, cols / 8, rows * (cols / 8), st);
}
cudaError_t launch_activation_restore(CkArgs a, int dtype, cudaStream_t st) {
    const int64_t rows = a.rows * a.workers, cols = ck_cols(a.cols), row_blocks = ck_row_blocks(a, a.x, dtype == 0 ? 4 : 2);
    if (row_blocks >= 0)
        return ck_launch(dtype == 0 ? ck_restore_blocks_kernel<float> : ck_restore_blocks_kernel<__nv_bfloat16>, a, row_blocks, rows * (cols / CK_BLOCK), st);
    return dtype == 0 ? ck_launch(ck_restore_kernel<float>, a, cols / 4, rows * (cols / 4), st) : ck_launch(ck_restore_kernel<__nv_bfloat16>, a, cols / 8, rows * (cols / 8), st);
}

}  // namespace liec

// Norm of every worker's gradient over all its tensors, and clipping.  For worker i with entries g_j:
//   norm_i = sqrt(sum_j g_j^2),  c_i = max_norm / norm_i if norm_i > max_norm, else 1,  out_j = round(c_i g_j)
// The squares are exact in binary64; a tile's sum is the balanced tree over its 8192 entries, and the
// row's sum the balanced tree over the row's tile sums in tile order, zero-padded to a power of two, so
// that the norm does not depend on how the tiles are spread over CTAs.  The gradients come as rows
// [N][d] or as N*T separate tensors (a table of pointers); a missing tensor counts as zeros.
#include "device_common.cuh"
#include "kernels.h"

namespace liec {

constexpr int ROW_MAX_CHUNKS = 512;   // chunks of FIN_CHUNK tiles in a row: 2^32 / TILE + 65535 tiles at most

template <typename ST>
__device__ __forceinline__ const ST *source_tile(const Params &p, const ClipArgs &a, int row, const TileInfo &ti) {
    if (a.table) {
        const ST *t = reinterpret_cast<const ST *>(a.table[(int64_t)row * p.T + ti.t]);
        return t ? t + ti.rel : nullptr;
    }
    return reinterpret_cast<const ST *>(a.rows) + (int64_t)row * p.d + ti.seg_beg + ti.rel;
}

__device__ __forceinline__ void store1(float *ptr, float v) { *ptr = v; }
__device__ __forceinline__ void store1(__nv_bfloat16 *ptr, float v) { *ptr = __float2bfloat16_rn(v); }

template <typename ST>
__global__ void __launch_bounds__(THREADS) clip_sumsq_kernel(const __grid_constant__ Params p, const __grid_constant__ ClipArgs a) {
    __shared__ double warp_sums[8];
    const int row = blockIdx.y;
    const TileInfo ti = locate_tile(p, blockIdx.x);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const ST *src = source_tile<ST>(p, a, row, ti);
    const int len = src ? ti.len : 0;
    const bool fast = (len == TILE) && ((reinterpret_cast<uintptr_t>(src) & (4 * sizeof(ST) - 1)) == 0);
    double leaf[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float v[4];
        if (fast) load4_cached(src + tile_pos(warp, lane, j), v);
        else load4_guarded(src, tile_pos(warp, lane, j), len, v);
        leaf[j] = leaf4_sq(v);
    }
    const double s = cta_tree_reduce(warp_tree_reduce8(leaf, lane), warp_sums);
    if (threadIdx.x == 0) a.partials[(int64_t)row * p.TT + blockIdx.x] = s;
}

// One CTA per row: the tree over the tile sums, the norm and the factor.
__global__ void __launch_bounds__(THREADS) clip_norm_kernel(const __grid_constant__ Params p, const __grid_constant__ ClipArgs a) {
    __shared__ double buf[FIN_CHUNK];
    __shared__ double chunk_sums[ROW_MAX_CHUNKS];
    const int row = blockIdx.x;
    const double total = tree_reduce_partials(a.partials + (int64_t)row * p.TT, p.TT, buf, chunk_sums);
    if (threadIdx.x == 0) {
        const double norm = sqrt(total);
        if (a.norms) a.norms[row] = (float)norm;
        a.factor[row] = norm > (double)a.max_norm ? (float)((double)a.max_norm / norm) : 1.0f;
        a.clear[row] = a.zero_nonfinite && !isfinite(norm);
    }
}

template <typename ST, typename DT>
__global__ void __launch_bounds__(THREADS) clip_scale_kernel(const __grid_constant__ Params p, const __grid_constant__ ClipArgs a) {
    const int row = blockIdx.y;
    const float c = a.factor[row];
    const bool clear = a.clear[row] != 0;
    if (a.in_place && c == 1.0f && !clear) return;   // the row stays as it is
    const TileInfo ti = locate_tile(p, blockIdx.x);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const ST *src = source_tile<ST>(p, a, row, ti);
    const int len = src && !clear ? ti.len : 0;
    DT *dst = reinterpret_cast<DT *>(a.out) + (int64_t)row * p.d + ti.seg_beg + ti.rel;
    const bool fast = (len == TILE) && ((reinterpret_cast<uintptr_t>(src) & (4 * sizeof(ST) - 1)) == 0);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int pos = tile_pos(warp, lane, j);
        float v[4];
        if (fast) load4_cached(src + pos, v);
        else load4_guarded(src, pos, len, v);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (pos + q < ti.len) store1(dst + pos + q, __fmul_rn(v[q], c));
    }
}

// The pointer table travels as kernel arguments: the call is ordered on the stream, can be captured,
// and leaves no host buffer behind that a later call could overwrite too early.
template <int CAP>
struct PointerBlock { const void *ptr[CAP]; };

template <int CAP>
__global__ void upload_pointers_kernel(const __grid_constant__ PointerBlock<CAP> block, const void **table, int count) {
    for (int q = threadIdx.x; q < count; q += blockDim.x) table[q] = block.ptr[q];
}

template <int CAP>
static cudaError_t upload_block(const void *const *tensors, const void **table, int count, cudaStream_t st) {
    PointerBlock<CAP> block;
    for (int q = 0; q < count; ++q) block.ptr[q] = tensors[q];
    upload_pointers_kernel<CAP><<<1, THREADS, 0, st>>>(block, table, count);
    return cudaGetLastError();
}

// Arguments of up to 4 KB are the cheap kind; longer tables go in blocks of 31 KB, near the 32,764-byte limit.
cudaError_t launch_upload_pointers(const void *const *tensors, const void **table, int64_t count, cudaStream_t st, int64_t *launches) {
    constexpr int SMALL = 480, LARGE = 3968;
    for (int64_t at = 0; at < count;) {
        const int64_t left = count - at;
        const int here = (int)(left < LARGE ? left : LARGE);
        const cudaError_t e = here <= SMALL ? upload_block<SMALL>(tensors + at, table + at, here, st)
                                            : upload_block<LARGE>(tensors + at, table + at, here, st);
        if (e != cudaSuccess) return e;
        ++*launches;
        at += here;
    }
    return cudaSuccess;
}

template <typename ST>
static cudaError_t launch_clip_t(const Params &p, const ClipArgs &a, cudaStream_t st, int64_t *launches) {
    const dim3 grid(p.TT, p.N);
    clip_sumsq_kernel<ST><<<grid, THREADS, 0, st>>>(p, a);
    clip_norm_kernel<<<p.N, THREADS, 0, st>>>(p, a);
    if (p.gdt == DT_F32) clip_scale_kernel<ST, float><<<grid, THREADS, 0, st>>>(p, a);
    else clip_scale_kernel<ST, __nv_bfloat16><<<grid, THREADS, 0, st>>>(p, a);
    *launches += 3;
    return cudaGetLastError();
}

cudaError_t launch_clip(const Params &p, const ClipArgs &a, cudaStream_t st, int64_t *launches) {
    return a.src_dtype == DT_F32 ? launch_clip_t<float>(p, a, st, launches) : launch_clip_t<__nv_bfloat16>(p, a, st, launches);
}

}  // namespace liec

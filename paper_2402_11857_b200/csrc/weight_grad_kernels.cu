// Weight gradient of a linear layer from the 8-bit checkpoint of its input: dW[o][c] = sum over tokens of
// dy[t][o] x^[t][c], for N workers.
#include "activation.cuh"

namespace liec {

constexpr int WG_TILE = 64, WG_DEPTH = 16;

__device__ __forceinline__ float wg_value(float x) { return x; }
__device__ __forceinline__ float wg_value(__nv_bfloat16 x) { return __bfloat162float(x); }

template <typename T>
__global__ void __launch_bounds__(256) wg_kernel(const __grid_constant__ WgArgs a, int64_t q_cols) {
    __shared__ float dy[WG_DEPTH][WG_TILE], x[WG_DEPTH][WG_TILE];
    const int worker = blockIdx.z, o0 = blockIdx.y * WG_TILE, c0 = blockIdx.x * WG_TILE, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    for (int64_t t0 = 0; t0 < a.rows; t0 += WG_DEPTH) {
        for (int i = threadIdx.x; i < WG_DEPTH * WG_TILE; i += 256) {
            const int t = i / WG_TILE, k = i % WG_TILE;
            const int64_t row = t0 + t, at = worker * a.rows + row;
            const bool live = row < a.rows;
            dy[t][k] = live && o0 + k < a.out ? wg_value(static_cast<const T *>(a.dy)[worker * a.dy_worker + row * a.dy_row + o0 + k]) : 0.0f;
            x[t][k] = live && c0 + k < a.in ? (float)a.q[at * q_cols + c0 + k] * ck_power(a.scales[at * (q_cols / CK_BLOCK) + (c0 + k) / CK_BLOCK]) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < WG_DEPTH; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __fmaf_rn(dy[t][ty * 4 + i], x[t][tx * 4 + j], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int o = o0 + ty * 4 + i, c = c0 + tx * 4 + j;
            if (o >= a.out || c >= a.in) continue;
            const int64_t at = worker * a.dw_worker + o * a.dw_row + c;
            if (a.grad_dtype == 0) static_cast<float *>(a.dweight)[at] = acc[i][j];
            else static_cast<__nv_bfloat16 *>(a.dweight)[at] = __float2bfloat16_rn(acc[i][j]);
        }
}

size_t weight_grad_workspace(const WgArgs &, int) { return 0; }

cudaError_t launch_weight_grad(WgArgs a, int dtype, cudaStream_t st) {
    const dim3 grid((a.in + WG_TILE - 1) / WG_TILE, (a.out + WG_TILE - 1) / WG_TILE, a.workers);
    if (dtype == 0) wg_kernel<float><<<grid, 256, 0, st>>>(a, ck_cols(a.in));
    else wg_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(a, ck_cols(a.in));
    return cudaGetLastError();
}

}  // namespace liec

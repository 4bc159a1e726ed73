// Layer normalisation of N workers' activations at once, and its backward pass.  Per row x of h
// elements, with the worker's own weight w and bias b:
//   m = mean(x),  r = 1 / sqrt(mean((x - m)^2) + eps),  xh = (x - m) r,  y = xh w + b
//   dx = r (dy w - mean(dy w) - xh mean(dy w xh)),  dw = sum over rows of dy xh,  db = sum over rows of dy
// Sums are binary32 over at most a few hundred terms per accumulator, joined in binary64; the variance
// is taken around the mean (never as a difference of squares).  The order of every sum is fixed by the
// sizes alone: no atomics.
#include "layer_norm.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>

namespace liec {

__device__ __forceinline__ float ln_load(const float *p) { return __ldg(p); }
__device__ __forceinline__ float ln_load(const __nv_bfloat16 *p) {
    return __uint_as_float((uint32_t)__ldg(reinterpret_cast<const unsigned short *>(p)) << 16);
}
__device__ __forceinline__ void ln_store(float *p, float v) { *p = v; }
__device__ __forceinline__ void ln_store(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    return v;
}

constexpr int LN_THREADS = 256;

__device__ __forceinline__ float cta_sum(float v, float *buf /*[8]*/) {
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < LN_THREADS / 32; ++w) s += buf[w];
    __syncthreads();
    return s;
}

template <typename T>
__global__ void __launch_bounds__(LN_THREADS) ln_forward_rows_kernel(const __grid_constant__ LnForward a) {
    __shared__ float buf[LN_THREADS / 32];
    const int group = blockIdx.y;
    const float inv_h = 1.0f / (float)a.cols;
    const float *w = a.weight ? a.weight + (int64_t)group * a.weight_stride : nullptr;
    const float *b = a.bias ? a.bias + (int64_t)group * a.bias_stride : nullptr;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = reinterpret_cast<const T *>(a.x) + group * a.x_group + row * a.x_row;
        T *y = reinterpret_cast<T *>(a.y) + group * a.y_group + row * a.y_row;
        float s = 0.0f;
        for (int c = threadIdx.x; c < a.cols; c += LN_THREADS) s += ln_load(x + c);
        const float mean = cta_sum(s, buf) * inv_h;
        float q = 0.0f;
        for (int c = threadIdx.x; c < a.cols; c += LN_THREADS) {
            const float t = ln_load(x + c) - mean;
            q = __fmaf_rn(t, t, q);
        }
        const float rstd = 1.0f / sqrtf(cta_sum(q, buf) * inv_h + a.eps);
        for (int c = threadIdx.x; c < a.cols; c += LN_THREADS)
            ln_store(y + c, __fmaf_rn((ln_load(x + c) - mean) * rstd, w ? w[c] : 1.0f, b ? b[c] : 0.0f));
        if (threadIdx.x == 0) {
            const int64_t at = (int64_t)group * a.rows + row;
            if (a.mean) a.mean[at] = mean;
            if (a.rstd) a.rstd[at] = rstd;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(LN_THREADS) ln_backward_rows_kernel(const __grid_constant__ LnBackward a) {
    __shared__ float buf[LN_THREADS / 32];
    const int group = blockIdx.y;
    const float inv_h = 1.0f / (float)a.cols;
    const float *w = a.weight ? a.weight + (int64_t)group * a.weight_stride : nullptr;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = reinterpret_cast<const T *>(a.x) + group * a.x_group + row * a.x_row;
        const T *dy = reinterpret_cast<const T *>(a.dy) + group * a.dy_group + row * a.dy_row;
        T *dx = reinterpret_cast<T *>(a.dx) + group * a.dx_group + row * a.dx_row;
        const float mean = a.mean[(int64_t)group * a.rows + row], rstd = a.rstd[(int64_t)group * a.rows + row];
        float along = 0.0f, level = 0.0f;
        for (int c = threadIdx.x; c < a.cols; c += LN_THREADS) {
            const float t = ln_load(dy + c) * (w ? w[c] : 1.0f);
            along = __fmaf_rn(t, (ln_load(x + c) - mean) * rstd, along);
            level += t;
        }
        along = cta_sum(along, buf) * inv_h;
        level = cta_sum(level, buf) * inv_h;
        for (int c = threadIdx.x; c < a.cols; c += LN_THREADS) {
            const float t = ln_load(dy + c) * (w ? w[c] : 1.0f), xh = (ln_load(x + c) - mean) * rstd;
            ln_store(dx + c, rstd * __fmaf_rn(-xh, along, t - level));
        }
    }
}

// Column sums of one run of rows: 32 columns per CTA, a warp per row, eight rows at a time.
template <typename T>
__global__ void __launch_bounds__(LN_THREADS) ln_backward_columns_kernel(const __grid_constant__ LnBackward a) {
    __shared__ float sw[LN_THREADS / 32][32], sb[LN_THREADS / 32][32];
    const int group = blockIdx.z, run = blockIdx.y;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = blockIdx.x * 32 + lane;
    const int64_t first = (int64_t)run * a.run_rows;
    const int64_t last = min(a.rows, first + a.run_rows);
    float gw = 0.0f, gb = 0.0f;
    if (c < a.cols) {
        for (int64_t row = first + warp; row < last; row += LN_THREADS / 32) {
            const float dy = ln_load(reinterpret_cast<const T *>(a.dy) + group * a.dy_group + row * a.dy_row + c);
            const float x = ln_load(reinterpret_cast<const T *>(a.x) + group * a.x_group + row * a.x_row + c);
            const int64_t at = (int64_t)group * a.rows + row;
            gw = __fmaf_rn(dy, (x - a.mean[at]) * a.rstd[at], gw);
            gb += dy;
        }
    }
    sw[warp][lane] = gw;
    sb[warp][lane] = gb;
    __syncthreads();
    if (warp == 0 && c < a.cols) {
        float tw = 0.0f, tb = 0.0f;
#pragma unroll
        for (int q = 0; q < LN_THREADS / 32; ++q) { tw += sw[q][lane]; tb += sb[q][lane]; }
        const int64_t at = ((int64_t)group * a.runs + run) * a.cols + c;
        a.part_w[at] = tw;
        a.part_b[at] = tb;
    }
}

// Joins the runs in run order, in binary64, and rounds once to the gradient rows' type.
template <typename GT>
__global__ void __launch_bounds__(LN_THREADS) ln_backward_join_kernel(const __grid_constant__ LnBackward a) {
    const int group = blockIdx.y;
    const int c = blockIdx.x * LN_THREADS + threadIdx.x;
    if (c >= a.cols) return;
    double tw = 0.0, tb = 0.0;
    for (int run = 0; run < a.runs; ++run) {
        const int64_t at = ((int64_t)group * a.runs + run) * a.cols + c;
        tw += (double)a.part_w[at];
        tb += (double)a.part_b[at];
    }
    if (a.dweight) ln_store(reinterpret_cast<GT *>(a.dweight) + (int64_t)group * a.dweight_stride + c, (float)tw);
    if (a.dbias) ln_store(reinterpret_cast<GT *>(a.dbias) + (int64_t)group * a.dbias_stride + c, (float)tb);
}

// Rows whose column sums one CTA takes: 1024, i.e. 128 terms per binary32 accumulator, and more only
// where there would be more than 32768 runs (grid y).
static int64_t ln_run_rows(int64_t rows) {
    const int64_t even = (rows + 32767) / 32768;
    return even > 1024 ? even : 1024;
}
static int64_t ln_runs(int64_t rows) { return (rows + ln_run_rows(rows) - 1) / ln_run_rows(rows); }

template <typename T>
static cudaError_t forward_t(const LnForward &a, cudaStream_t st) {
    const dim3 grid((unsigned)(a.rows < 65536 ? a.rows : 65536), a.groups);
    ln_forward_rows_kernel<T><<<grid, LN_THREADS, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_layer_norm_forward(const LnForward &a, int dtype, cudaStream_t st) {
    if (a.rows == 0) return cudaSuccess;
    return dtype == 0 ? forward_t<float>(a, st) : forward_t<__nv_bfloat16>(a, st);
}

template <typename T>
static cudaError_t backward_t(const LnBackward &a, int grad_dtype, cudaStream_t st) {
    if (a.rows > 0 && a.dx) {
        const dim3 grid((unsigned)(a.rows < 65536 ? a.rows : 65536), a.groups);
        ln_backward_rows_kernel<T><<<grid, LN_THREADS, 0, st>>>(a);
    }
    if (a.dweight || a.dbias) {
        if (a.rows > 0)
            ln_backward_columns_kernel<T><<<dim3((a.cols + 31) / 32, (unsigned)a.runs, a.groups), LN_THREADS, 0, st>>>(a);
        const dim3 grid((a.cols + LN_THREADS - 1) / LN_THREADS, a.groups);
        if (grad_dtype == 0) ln_backward_join_kernel<float><<<grid, LN_THREADS, 0, st>>>(a);
        else ln_backward_join_kernel<__nv_bfloat16><<<grid, LN_THREADS, 0, st>>>(a);
    }
    return cudaGetLastError();
}

cudaError_t launch_layer_norm_backward(LnBackward a, int dtype, int grad_dtype, cudaStream_t st) {
    a.run_rows = ln_run_rows(a.rows);
    a.runs = (int)ln_runs(a.rows);
    return dtype == 0 ? backward_t<float>(a, grad_dtype, st) : backward_t<__nv_bfloat16>(a, grad_dtype, st);
}

size_t layer_norm_workspace(int groups, int64_t rows, int cols) {
    return sizeof(float) * 2 * (size_t)groups * (size_t)ln_runs(rows) * (size_t)cols;
}

}  // namespace liec

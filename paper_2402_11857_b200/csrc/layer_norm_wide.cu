// Layer normalisation of rows wider than 8192 columns: a CTA sweeps a row three times (twice in the backward
// pass), the later sweeps out of L1 and L2; the column sums of the backward pass are a kernel of their own.
#include "layer_norm_common.cuh"

namespace liec {

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


// Rows whose column sums one CTA of ln_backward_columns_kernel takes: 1024, i.e. 128 terms per binary32
// accumulator, and more only where there would be more than 32768 runs (grid y).
static int64_t run_rows(int64_t rows) {
    const int64_t even = (rows + 32767) / 32768;
    return even > 1024 ? even : 1024;
}
int64_t ln_wide_runs(int64_t rows) { return (rows + run_rows(rows) - 1) / run_rows(rows); }

cudaError_t launch_layer_norm_forward_wide(const LnForward &a, int dtype, cudaStream_t st) {
    const dim3 grid((unsigned)std::min<int64_t>(a.rows, 65536), a.groups);
    if (dtype == 0) ln_forward_rows_kernel<float><<<grid, LN_THREADS, 0, st>>>(a);
    else ln_forward_rows_kernel<__nv_bfloat16><<<grid, LN_THREADS, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename T>
static cudaError_t backward_wide_t(const LnBackward &a, cudaStream_t st) {
    if (a.dx) ln_backward_rows_kernel<T><<<dim3((unsigned)std::min<int64_t>(a.rows, 65536), a.groups), LN_THREADS, 0, st>>>(a);
    if (a.dweight || a.dbias)
        ln_backward_columns_kernel<T><<<dim3((a.cols + 31) / 32, (unsigned)a.runs, a.groups), LN_THREADS, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_layer_norm_backward_wide(LnBackward &a, int dtype, cudaStream_t st) {
    a.run_rows = run_rows(a.rows);
    a.runs = (int)ln_wide_runs(a.rows);
    return dtype == 0 ? backward_wide_t<float>(a, st) : backward_wide_t<__nv_bfloat16>(a, st);
}

}  // namespace liec

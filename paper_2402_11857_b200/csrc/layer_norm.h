// Layer normalisation over N workers: arguments of the kernels and their launchers.
#pragma once
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace liec {

// Strides in elements; group = worker.  NULL weight: ones; NULL bias: zeros.
struct LnForward {
    const void *x;
    const float *weight, *bias;
    void *y;
    float *mean, *rstd;   // [groups][rows], or NULL
    int64_t rows, x_row, x_group, y_row, y_group, weight_stride, bias_stride;
    int32_t groups, cols;
    float eps;
};

struct LnBackward {
    const void *dy, *x;
    const float *mean, *rstd, *weight;
    void *dx, *dweight, *dbias;   // any may be NULL
    float *part_w, *part_b;       // [groups][runs][cols] column sums of runs of rows
    int64_t rows, x_row, x_group, dy_row, dy_group, dx_row, dx_group, weight_stride, dweight_stride, dbias_stride;
    int64_t run_rows;
    int32_t groups, cols, runs;
};

cudaError_t launch_layer_norm_forward(const LnForward &a, int dtype, cudaStream_t st);
cudaError_t launch_layer_norm_backward(LnBackward a, int dtype, int grad_dtype, cudaStream_t st);
size_t layer_norm_workspace(int groups, int64_t rows, int cols);   // bytes of part_w and part_b together

}  // namespace liec

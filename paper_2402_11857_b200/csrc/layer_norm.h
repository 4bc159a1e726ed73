// Layer normalisation over N workers: arguments of the kernels and their launchers.
#pragma once
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace liec {

// How the rows, numbered through all groups, are dealt to CTAs: the first `large` CTAs take large_rows
// consecutive rows each, the others small_rows.
struct LnShare {
    int64_t large, large_rows, small_rows, ctas;
#ifdef __CUDACC__
    __host__ __device__
#endif
    int64_t first(int64_t cta) const { return cta <= large ? cta * large_rows : large * large_rows + (cta - large) * small_rows; }
#ifdef __CUDACC__
    __host__ __device__
#endif
    int64_t owner(int64_t row) const { return row < large * large_rows ? row / large_rows : large + (row - large * large_rows) / small_rows; }
};

// Strides in elements; group = worker.  NULL weight: ones; NULL bias: zeros.
struct LnForward {
    const void *x;
    const float *weight, *bias;
    void *y;
    float *mean, *rstd;   // [groups][rows], or NULL
    int64_t rows, x_row, x_group, y_row, y_group, weight_stride, bias_stride;
    LnShare share;
    int32_t groups, cols, part_cols;   // part_cols: columns per CTA of a row
    float eps;
};

struct LnBackward {
    const void *dy, *x;
    const float *mean, *rstd, *weight;
    void *dx, *dweight, *dbias;   // any may be NULL
    float *part_w, *part_b;       // column sums of pieces of a group's rows, [piece][cols]
    int64_t rows, x_row, x_group, dy_row, dy_group, dx_row, dx_group, weight_stride, dweight_stride, dbias_stride;
    LnShare share;
    int32_t groups, cols, part_cols, grad_dtype;
    int32_t direct;               // every group is one CTA's: it writes the gradient itself
    int32_t shared;               // one gradient vector for all groups: the pieces of all of them are joined
};

cudaError_t launch_layer_norm_forward(const LnForward &a, int dtype, cudaStream_t st);
cudaError_t launch_layer_norm_backward(LnBackward a, int dtype, cudaStream_t st);
size_t layer_norm_workspace(int groups, int64_t rows, int cols, bool shared);   // bytes of part_w and part_b together

}  // namespace liec

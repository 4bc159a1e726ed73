// Activations of N workers: 8-bit checkpoints, group normalisation, weight gradients from checkpoints.
// Arguments of the kernels and their launchers.
#pragma once
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/liec.h"

namespace liec {

constexpr int CK_BLOCK = LIEC_ACTIVATION_BLOCK;
inline int64_t ck_cols(int64_t cols) { return (cols + CK_BLOCK - 1) / CK_BLOCK * CK_BLOCK; }

// The message behind liec_last_error(NULL); returns st.
liec_status refuse(liec_status st, const char *text);

struct CkArgs {   // x: [workers][rows][cols] with strides in elements; q, scales without gaps
    const void *in;
    void *x;
    int8_t *q;
    uint8_t *scales;
    int64_t rows, x_row, x_worker;
    int32_t workers, cols;
};
cudaError_t launch_activation_compress(CkArgs a, int dtype, cudaStream_t st);
cudaError_t launch_activation_restore(CkArgs a, int dtype, cudaStream_t st);

struct GnArgs {   // an image is a worker's sample; strides in elements
    const void *x, *dy;           // x NULL: from q and scales
    const float *weight, *bias;
    void *y, *dx, *dweight, *dbias;
    int8_t *q;
    uint8_t *scales;
    float *mean, *rstd;           // [workers][samples][groups]
    float *part;                  // per channel of every part of an image: forward three numbers, backward two, [image][part][2 or 3][channels]
    float *level;                 // backward: r mean(dz w) and r^2 mean(dz w xh), [image][groups][2]
    int64_t x_pixel, x_sample, x_worker, y_pixel, y_sample, y_worker, dx_pixel, dx_sample, dx_worker;   // y: of dy in the backward pass
    int64_t weight_stride, bias_stride, dweight_stride, dbias_stride;
    int64_t pixels;
    int32_t workers, samples, channels, groups, act, grad_dtype, shared;
    float eps;
    int32_t parts, tiles, tile_chunks;   // of an image's pixels; of its channels, each of tile_chunks 16-byte chunks
    int64_t part_pixels;
    int32_t again_parts;          // as cut for the second reading
    int64_t again_pixels;
    int32_t whole, whole_out;     // rows that are read, rows that are written, start on 16 bytes
    int32_t turns;                // resident images: chunks of a thread
};
cudaError_t launch_group_norm_forward(GnArgs a, int dtype, cudaStream_t st);
cudaError_t launch_group_norm_backward(GnArgs a, int dtype, cudaStream_t st);
size_t group_norm_workspace(const GnArgs &a, int dtype, bool backward);

struct WgArgs {
    const void *dy;
    const int8_t *q;
    const uint8_t *scales;
    void *dweight;
    float *part;      // workspace: the runs' sums, [run][worker][out][in], and
    void *packed;     // dy in rows of whole 16 bytes, where its own are not
    int64_t rows, dy_row, dy_worker, dw_row, dw_worker;
    int32_t workers, in, out, grad_dtype;
};
cudaError_t launch_weight_grad(WgArgs a, int dtype, cudaStream_t st);
size_t weight_grad_workspace(const WgArgs &a, int dtype);

}  // namespace liec

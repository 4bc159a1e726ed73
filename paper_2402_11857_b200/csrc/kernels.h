// Launchers of the CUDA kernels (one translation unit per kernel family).
#pragma once
#include <cuda_runtime.h>

#include "plan.h"

namespace liec {

// scaled sign
cudaError_t launch_sign_uplink(const Params &p, cudaStream_t st);
cudaError_t launch_scale_finalize(const Params &p, bool uplink, cudaStream_t st);
cudaError_t launch_server_dense(const Params &p, cudaStream_t st);
cudaError_t launch_sign_error(const Params &p, cudaStream_t st);
cudaError_t launch_identity_downlink(const Params &p, cudaStream_t st);

// top-k (launch counters are bumped per kernel)
cudaError_t launch_topk_hist1(const Params &p, bool uplink, cudaStream_t st, int64_t *launches);
cudaError_t launch_topk_select(const Params &p, bool uplink, cudaStream_t st, int64_t *launches);
cudaError_t launch_topk_small_segments(const Params &p, bool uplink, cudaStream_t st, int64_t *launches);
cudaError_t launch_server_topk(const Params &p, cudaStream_t st, int64_t *launches);
cudaError_t configure_topk_kernels();  // opt-in shared memory sizes; call once per device

// random-k: messages gathered at the caller's subsets, per-tile offsets into them
cudaError_t launch_randk_compress(const Params &p, bool uplink, cudaStream_t st, int64_t *launches);

// model-averaging iteration and mean model
cudaError_t launch_average_step(const Params &p, float lr, cudaStream_t st);
cudaError_t launch_mean_params(const Params &p, float *out, cudaStream_t st);
cudaError_t configure_average_kernels();  // opt-in shared memory sizes; call once per device

// squared norms (monitoring)
cudaError_t launch_sumsq(const Params &p, const void *src, int64_t row_stride, int rows, bool bf16, cudaStream_t st);
cudaError_t launch_sum_finalize(const Params &p, const double *partials, int rows, double *out, cudaStream_t st);

// norm of every worker's gradient and clipping
struct ClipArgs {
    const void *rows;          // [N][d] of src_dtype, used when table is NULL
    const void *const *table;  // device, [N][T] pointers to the tensors (NULL entry: zeros) and a word that says of
                               // what type they are (TABLE_F32, TABLE_BF16), or NULL
    void *out;                 // [N][d] of the context's gradient type
    float *norms;              // [N] or NULL
    // for rows that go through the streaming kernel, one block of CLIP_STREAM_BYTES:
    double *partials;                    // [N][TT] sums of squares
    unsigned long long *answer;          // [N] a row's factor
    unsigned long long *gave_up;         // [1] a wait ran out
    unsigned long long *sum_ticket, *scale_ticket; // [1] tiles handed out for their sums, for scaling
    float max_norm;
    int32_t src_dtype, in_place, zero_nonfinite;
    // set by the launcher
    int32_t norms_only;            // nothing to write
    int32_t batch;                 // tiles per ticket
};
// The word behind a table: 0 while there is none.  The host's knowledge of the type is not enough: a replayed graph
// writes the table again without the host, and a captured call has not written it yet.
constexpr unsigned long long TABLE_F32 = DT_F32 + 1, TABLE_BF16 = DT_BF16 + 1;
constexpr size_t CLIP_STREAM_BYTES(size_t N, size_t TT) { return 8 * (N * TT + N + 3); }
cudaError_t configure_clip_kernels();  // opt-in shared memory sizes; call once per device
cudaError_t launch_clip(const Params &p, const ClipArgs &a, cudaStream_t st, int64_t *launches);
cudaError_t launch_upload_pointers(const void *const *tensors, int dtype, const void **table, int64_t count, cudaStream_t st, int64_t *launches);

// worker update
cudaError_t launch_worker_update(const Params &p, float lr, cudaStream_t st);

}  // namespace liec

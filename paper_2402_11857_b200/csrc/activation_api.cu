// C ABI of the operators on activations: checks of arguments, then the launch.
#include <cmath>

#include "activation.h"
#include "axes.h"

using namespace liec;

namespace {

constexpr int64_t MAX_ROWS = int64_t(1) << 31, MAX_STRIDE = int64_t(1) << 40;

liec_status invalid(const char *text) { return refuse(LIEC_ERR_INVALID_ARG, text); }
liec_status unsupported(const char *text) { return refuse(LIEC_ERR_UNSUPPORTED, text); }
liec_status launched(cudaError_t e) { return e == cudaSuccess ? LIEC_OK : refuse(LIEC_ERR_CUDA, cudaGetErrorString(e)); }

int size_of(int32_t dtype) { return dtype == LIEC_BF16 ? 2 : 4; }
bool known(int32_t dtype) { return dtype == LIEC_F32 || dtype == LIEC_BF16; }
bool aligned(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
bool strides_ok(std::initializer_list<int64_t> strides) {
    for (int64_t s : strides)
        if (s < 0 || s > MAX_STRIDE) return false;
    return true;
}

// The two arrays of a checkpoint of `rows` rows.
Axes bytes_of(const int8_t *q, int64_t rows, int64_t cols) { return axes_of(q, rows * ck_cols(cols), 1, {}, {}); }
Axes powers_of(const uint8_t *scales, int64_t rows, int64_t cols) { return axes_of(scales, rows * (ck_cols(cols) / CK_BLOCK), 1, {}, {}); }

liec_status check(const liec_activation_desc *d) {
    if (!d) return invalid("activation: desc is NULL");
    if (d->workers < 1 || d->rows < 0 || d->cols < 1) return invalid("activation: workers and cols must be >= 1, rows >= 0");
    if (d->workers > 65535) return unsupported("activation: workers above 65535");
    if (d->cols > LIEC_ACTIVATION_MAX_COLS) return unsupported("activation: cols above LIEC_ACTIVATION_MAX_COLS");
    if (d->rows >= MAX_ROWS) return unsupported("activation: rows must be below 2^31");
    if (d->workers * d->rows * (ck_cols(d->cols) / CK_BLOCK) > int64_t(1) << 35) return unsupported("activation: more than 2^40 elements (launch grid)");
    if (!known(d->dtype)) return invalid("activation: unknown dtype");
    if (!strides_ok({d->x_row_stride, d->x_worker_stride})) return invalid("activation: strides must be >= 0 (and at most 2^40)");
    return LIEC_OK;
}

liec_status activation_call(const liec_activation_desc *d, const void *x, const int8_t *q, const uint8_t *scales, bool restore, CkArgs &a) {
    const liec_status st = check(d);
    if (st != LIEC_OK || d->rows == 0) return st;
    if (!x || !q || !scales) return invalid("activation: x, q and scales must be non-NULL");
    if (!aligned(x, size_of(d->dtype))) return invalid("activation: x is not aligned to its element size");
    if (!aligned(q, 16)) return invalid("activation: q must be 16-byte aligned");
    const Axes xa = axes_of(x, d->cols, size_of(d->dtype), {d->workers, d->rows}, {d->x_worker_stride, d->x_row_stride});
    const int64_t rows = d->workers * d->rows;
    const Axes qa = bytes_of(q, rows, d->cols), sa = powers_of(scales, rows, d->cols);
    if (restore && !disjoint(d->cols, {d->workers, d->rows}, {d->x_worker_stride, d->x_row_stride})) return invalid("activation: the rows of x overlap");
    if (meet(xa, qa) || meet(xa, sa) || (!restore && meet(qa, sa))) return invalid("activation: x, q and scales overlap");
    a.rows = d->rows; a.workers = d->workers; a.cols = d->cols;
    a.x_row = d->x_row_stride; a.x_worker = d->x_worker_stride;
    a.q = const_cast<int8_t *>(q);
    a.scales = const_cast<uint8_t *>(scales);
    return LIEC_OK;
}

liec_status check(const liec_group_norm_desc *d) {
    if (!d) return invalid("group norm: desc is NULL");
    if (d->workers < 1 || d->samples < 0 || d->pixels < 0 || d->channels < 1 || d->groups < 1)
        return invalid("group norm: workers, channels and groups must be >= 1, samples and pixels >= 0");
    if (d->channels > LIEC_GROUP_NORM_MAX_CHANNELS) return unsupported("group norm: channels above LIEC_GROUP_NORM_MAX_CHANNELS");
    if (d->channels % d->groups != 0) return invalid("group norm: groups must divide channels");
    if (d->workers > 65535) return unsupported("group norm: workers above 65535");
    if (d->pixels >= MAX_ROWS) return unsupported("group norm: pixels must be below 2^31");
    if ((int64_t)d->workers * d->samples > ((int64_t(1) << 31) - (d->channels == 1)) / d->channels) return unsupported("group norm: images times channels above 2^31, or 2^31 images (launch grid)");
    if ((int64_t)d->workers * d->samples > 0 && d->pixels > (int64_t(1) << 40) / ((int64_t)d->workers * d->samples * d->channels))
        return unsupported("group norm: more than 2^40 elements");
    if (!known(d->dtype) || !known(d->grad_dtype)) return invalid("group norm: unknown dtype");
    if (d->activation < LIEC_ACT_NONE || d->activation > LIEC_ACT_SILU) return invalid("group norm: unknown activation");
    if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return invalid("group norm: eps must be finite and >= 0");
    if (!strides_ok({d->x_pixel_stride, d->x_sample_stride, d->x_worker_stride, d->y_pixel_stride, d->y_sample_stride, d->y_worker_stride,
                     d->dx_pixel_stride, d->dx_sample_stride, d->dx_worker_stride, d->weight_stride, d->bias_stride, d->dweight_stride, d->dbias_stride}))
        return invalid("group norm: strides must be >= 0 (and at most 2^40)");
    return LIEC_OK;
}

Axes images(const liec_group_norm_desc *d, const void *base, int64_t worker, int64_t sample, int64_t pixel) {
    return axes_of(base, d->channels, size_of(d->dtype), {d->workers, d->samples, d->pixels}, {worker, sample, pixel});
}
bool images_disjoint(const liec_group_norm_desc *d, int64_t worker, int64_t sample, int64_t pixel) {
    return disjoint(d->channels, {d->workers, d->samples, d->pixels}, {worker, sample, pixel});
}
Axes vectors(const void *base, int64_t worker_stride, int count, int channels, int size) { return axes_of(base, channels, size, {count}, {worker_stride}); }

liec_status apart(const Axes *out, int outs, const Axes *in, int ins) {
    for (int i = 0; i < outs; ++i) {
        for (int j = 0; j < ins; ++j)
            if (meet(out[i], in[j])) return invalid("group norm: an output overlaps an input");
        for (int j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return invalid("group norm: outputs overlap");
    }
    return LIEC_OK;
}

GnArgs gn_args(const liec_group_norm_desc *d) {
    GnArgs a{};
    a.x_pixel = d->x_pixel_stride; a.x_sample = d->x_sample_stride; a.x_worker = d->x_worker_stride;
    a.y_pixel = d->y_pixel_stride; a.y_sample = d->y_sample_stride; a.y_worker = d->y_worker_stride;
    a.dx_pixel = d->dx_pixel_stride; a.dx_sample = d->dx_sample_stride; a.dx_worker = d->dx_worker_stride;
    a.weight_stride = d->weight_stride; a.bias_stride = d->bias_stride; a.dweight_stride = d->dweight_stride; a.dbias_stride = d->dbias_stride;
    a.pixels = d->pixels; a.workers = d->workers; a.samples = d->samples; a.channels = d->channels; a.groups = d->groups;
    a.act = d->activation; a.grad_dtype = d->grad_dtype; a.eps = d->eps;
    a.shared = d->shared_grads != 0 && d->workers > 1;
    return a;
}

liec_status workspace_ok(size_t need, const void *workspace, size_t bytes, const char *bad, const char *small) {
    if (need == 0) return LIEC_OK;
    if (!workspace || !aligned(workspace, 16)) return invalid(bad);
    return bytes < need ? refuse(LIEC_ERR_WORKSPACE, small) : LIEC_OK;
}

liec_status check(const liec_weight_grad_desc *d) {
    if (!d) return invalid("weight grad: desc is NULL");
    if (d->workers < 1 || d->rows < 0 || d->in < 1 || d->out < 1) return invalid("weight grad: workers, in and out must be >= 1, rows >= 0");
    if (d->workers > 65535) return unsupported("weight grad: workers above 65535");
    if (d->in > LIEC_ACTIVATION_MAX_COLS || d->out > LIEC_ACTIVATION_MAX_COLS) return unsupported("weight grad: in or out above LIEC_ACTIVATION_MAX_COLS");
    if (d->rows >= MAX_ROWS) return unsupported("weight grad: rows must be below 2^31");
    if ((int64_t)d->workers * d->in * d->out > int64_t(1) << 38) return unsupported("weight grad: more than 2^38 weights (launch grid)");
    if (!known(d->dtype) || !known(d->grad_dtype)) return invalid("weight grad: unknown dtype");
    if (!strides_ok({d->dy_row_stride, d->dy_worker_stride, d->dweight_row_stride, d->dweight_worker_stride}))
        return invalid("weight grad: strides must be >= 0 (and at most 2^40)");
    return LIEC_OK;
}

WgArgs wg_args(const liec_weight_grad_desc *d) {
    WgArgs a{};
    a.rows = d->rows; a.workers = d->workers; a.in = d->in; a.out = d->out; a.grad_dtype = d->grad_dtype;
    a.dy_row = d->dy_row_stride; a.dy_worker = d->dy_worker_stride;
    a.dw_row = d->dweight_row_stride; a.dw_worker = d->dweight_worker_stride;
    return a;
}

}  // namespace

extern "C" {

int64_t liec_activation_cols(int64_t cols) { return cols < 1 || cols > LIEC_ACTIVATION_MAX_COLS ? 0 : ck_cols(cols); }

liec_status liec_activation_compress(const liec_activation_desc *d, const void *x, int8_t *q, uint8_t *scales, void *stream) {
    CkArgs a{};
    const liec_status st = activation_call(d, x, q, scales, false, a);
    if (st != LIEC_OK || d->rows == 0) return st;
    a.in = x;
    return launched(launch_activation_compress(a, d->dtype, static_cast<cudaStream_t>(stream)));
}

liec_status liec_activation_restore(const liec_activation_desc *d, const int8_t *q, const uint8_t *scales, void *x, void *stream) {
    CkArgs a{};
    const liec_status st = activation_call(d, x, q, scales, true, a);
    if (st != LIEC_OK || d->rows == 0) return st;
    a.x = x;
    return launched(launch_activation_restore(a, d->dtype, static_cast<cudaStream_t>(stream)));
}

size_t liec_group_norm_workspace_bytes(const liec_group_norm_desc *d, int32_t backward) {
    if (check(d) != LIEC_OK || d->samples == 0 || d->pixels == 0) return 0;
    return (group_norm_workspace(gn_args(d), d->dtype, backward != 0) + 255) / 256 * 256;
}

liec_status liec_group_norm_forward(const liec_group_norm_desc *d, const void *x, const float *weight, const float *bias, void *y, float *mean,
                                    float *rstd, int8_t *q, uint8_t *scales, void *workspace, size_t workspace_bytes, void *stream) {
    liec_status st = check(d);
    if (st != LIEC_OK) return st;
    if (d->samples == 0 || d->pixels == 0) return LIEC_OK;
    if (!x || !y || !mean || !rstd) return invalid("group norm: x, y, mean and rstd must be non-NULL");
    if (!q != !scales) return invalid("group norm: q and scales must be given together");
    const int size = size_of(d->dtype);
    if (!aligned(x, size) || !aligned(y, size) || !aligned(weight, 4) || !aligned(bias, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
        return invalid("group norm: a pointer is not aligned to its element size");
    if (!aligned(q, 16)) return invalid("group norm: q must be 16-byte aligned");
    if (!images_disjoint(d, d->y_worker_stride, d->y_sample_stride, d->y_pixel_stride)) return invalid("group norm: the rows of y overlap");
    GnArgs a = gn_args(d);
    st = workspace_ok(group_norm_workspace(a, d->dtype, false), workspace, workspace_bytes, "group norm: workspace must be non-NULL and 16-byte aligned",
                      "workspace smaller than liec_group_norm_workspace_bytes()");
    if (st != LIEC_OK) return st;
    const int64_t rows = (int64_t)d->workers * d->samples * d->pixels, stats = (int64_t)d->workers * d->samples * d->groups;
    Axes in[3];
    int ins = 0;
    in[ins++] = images(d, x, d->x_worker_stride, d->x_sample_stride, d->x_pixel_stride);
    if (weight) in[ins++] = vectors(weight, d->weight_stride, d->workers, d->channels, 4);
    if (bias) in[ins++] = vectors(bias, d->bias_stride, d->workers, d->channels, 4);
    Axes out[5] = {images(d, y, d->y_worker_stride, d->y_sample_stride, d->y_pixel_stride), axes_of(mean, stats, 4, {}, {}), axes_of(rstd, stats, 4, {}, {})};
    int outs = 3;
    if (q) {
        out[outs++] = bytes_of(q, rows, d->channels);
        out[outs++] = powers_of(scales, rows, d->channels);
    }
    st = apart(out, outs, in, ins);
    if (st != LIEC_OK) return st;
    a.x = x; a.weight = weight; a.bias = bias; a.y = y; a.mean = mean; a.rstd = rstd; a.q = q; a.scales = scales;
    a.part = static_cast<float *>(workspace);
    return launched(launch_group_norm_forward(a, d->dtype, static_cast<cudaStream_t>(stream)));
}

liec_status liec_group_norm_backward(const liec_group_norm_desc *d, const void *dy, const void *x, const int8_t *q, const uint8_t *scales,
                                     const float *mean, const float *rstd, const float *weight, const float *bias, void *dx, void *dweight, void *dbias,
                                     void *workspace, size_t workspace_bytes, void *stream) {
    liec_status st = check(d);
    if (st != LIEC_OK) return st;
    const bool any = d->samples > 0 && d->pixels > 0;
    if (!dweight && !dbias && (!dx || !any)) return LIEC_OK;
    if (any && (!dy || !mean || !rstd)) return invalid("group norm: dy, mean and rstd must be non-NULL");
    if (any && (x ? q || scales : !q || !scales)) return invalid("group norm: either x or q and scales must be given");
    const int size = size_of(d->dtype), grad = size_of(d->grad_dtype);
    if (!aligned(x, size) || !aligned(dy, size) || !aligned(dx, size) || !aligned(weight, 4) || !aligned(bias, 4) || !aligned(mean, 4) || !aligned(rstd, 4) ||
        !aligned(dweight, grad) || !aligned(dbias, grad))
        return invalid("group norm: a pointer is not aligned to its element size");
    if (!aligned(q, 16)) return invalid("group norm: q must be 16-byte aligned");
    if (dx && any && !images_disjoint(d, d->dx_worker_stride, d->dx_sample_stride, d->dx_pixel_stride)) return invalid("group norm: the rows of dx overlap");
    GnArgs a = gn_args(d);
    const int count = a.shared ? 1 : d->workers;
    if ((dweight && !disjoint(d->channels, {count}, {d->dweight_stride})) || (dbias && !disjoint(d->channels, {count}, {d->dbias_stride})))
        return invalid("group norm: the workers' rows of dweight or dbias overlap");
    if (any) {
        st = workspace_ok(group_norm_workspace(a, d->dtype, true), workspace, workspace_bytes, "group norm: workspace must be non-NULL and 16-byte aligned",
                          "workspace smaller than liec_group_norm_workspace_bytes()");
        if (st != LIEC_OK) return st;
    }
    Axes in[7], out[3];   // (x, or q and scales)
    int ins = 0, outs = 0;
    const int64_t rows = (int64_t)d->workers * d->samples * d->pixels, stats = (int64_t)d->workers * d->samples * d->groups;
    if (any) {
        in[ins++] = images(d, dy, d->y_worker_stride, d->y_sample_stride, d->y_pixel_stride);
        if (x) in[ins++] = images(d, x, d->x_worker_stride, d->x_sample_stride, d->x_pixel_stride);
        else {
            in[ins++] = bytes_of(q, rows, d->channels);
            in[ins++] = powers_of(scales, rows, d->channels);
        }
        if (weight) in[ins++] = vectors(weight, d->weight_stride, d->workers, d->channels, 4);
        if (bias) in[ins++] = vectors(bias, d->bias_stride, d->workers, d->channels, 4);
        in[ins++] = axes_of(mean, stats, 4, {}, {});
        in[ins++] = axes_of(rstd, stats, 4, {}, {});
        if (dx) out[outs++] = images(d, dx, d->dx_worker_stride, d->dx_sample_stride, d->dx_pixel_stride);
    }
    if (dweight) out[outs++] = vectors(dweight, d->dweight_stride, count, d->channels, grad);
    if (dbias) out[outs++] = vectors(dbias, d->dbias_stride, count, d->channels, grad);
    st = apart(out, outs, in, ins);
    if (st != LIEC_OK) return st;
    a.dy = dy; a.x = x; a.q = const_cast<int8_t *>(q); a.scales = const_cast<uint8_t *>(scales);
    a.mean = const_cast<float *>(mean); a.rstd = const_cast<float *>(rstd); a.weight = weight; a.bias = bias;
    a.dx = dx; a.dweight = dweight; a.dbias = dbias;
    a.part = static_cast<float *>(workspace);
    return launched(launch_group_norm_backward(a, d->dtype, static_cast<cudaStream_t>(stream)));
}

size_t liec_weight_grad_workspace_bytes(const liec_weight_grad_desc *d, const void *dy) {
    if (check(d) != LIEC_OK) return 0;
    WgArgs a = wg_args(d);
    a.dy = dy;
    return (weight_grad_workspace(a, d->dtype) + 255) / 256 * 256;
}

liec_status liec_weight_grad(const liec_weight_grad_desc *d, const void *dy, const int8_t *q, const uint8_t *scales, void *dweight, void *workspace,
                             size_t workspace_bytes, void *stream) {
    liec_status st = check(d);
    if (st != LIEC_OK) return st;
    if (!dweight) return invalid("weight grad: dweight must be non-NULL");
    if (d->rows > 0 && (!dy || !q || !scales)) return invalid("weight grad: dy, q and scales must be non-NULL");
    if (!aligned(dy, size_of(d->dtype)) || !aligned(dweight, size_of(d->grad_dtype))) return invalid("weight grad: a pointer is not aligned to its element size");
    if (!aligned(q, 16)) return invalid("weight grad: q must be 16-byte aligned");
    if (!disjoint(d->in, {d->workers, d->out}, {d->dweight_worker_stride, d->dweight_row_stride})) return invalid("weight grad: the rows of dweight overlap");
    WgArgs a = wg_args(d);
    a.dy = dy;
    st = workspace_ok(weight_grad_workspace(a, d->dtype), workspace, workspace_bytes, "weight grad: workspace must be non-NULL and 16-byte aligned",
                      "workspace smaller than liec_weight_grad_workspace_bytes()");
    if (st != LIEC_OK) return st;
    if (d->rows > 0) {
        const Axes out = axes_of(dweight, d->in, size_of(d->grad_dtype), {d->workers, d->out}, {d->dweight_worker_stride, d->dweight_row_stride});
        const int64_t rows = d->workers * d->rows;
        if (meet(out, axes_of(dy, d->out, size_of(d->dtype), {d->workers, d->rows}, {d->dy_worker_stride, d->dy_row_stride})) ||
            meet(out, bytes_of(q, rows, d->in)) || meet(out, powers_of(scales, rows, d->in)))
            return invalid("weight grad: dweight overlaps an input");
    }
    a.q = q; a.scales = scales; a.dweight = dweight;
    a.part = static_cast<float *>(workspace);
    return launched(launch_weight_grad(a, d->dtype, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"

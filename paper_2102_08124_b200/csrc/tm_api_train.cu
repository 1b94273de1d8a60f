// C ABI of the operators of the training step around the masked layers (see include/tm.h): argument checks and dispatch.
#include <cfloat>
#include <cmath>

#include "../../include/tm.h"
#include "tm_launch.h"

namespace {

constexpr size_t kWorkspaceAlign = 256;

bool good_dtype(int dtype) { return dtype == TM_F32 || dtype == TM_BF16; }
size_t elem_bytes(int dtype) { return dtype == TM_F32 ? 4 : 2; }
bool off(const void* p, size_t bytes) { return (uintptr_t)p % bytes != 0; }
bool good_rows(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 0; }
// a matrix's leading dimension: rows must not overlap, and offsets must stay inside 63 bits
bool good_ld(int64_t rows, int64_t cols, int64_t ld) { return ld >= cols && (rows == 0 || ld <= (INT64_MAX / 8) / rows); }

// logits are scaled by log2(e) / T: below the normal range that has no fp32 value
bool good_temperature(float t) { return t >= FLT_MIN && std::isfinite(t); }

int finish(cudaError_t e) {
    if (e == cudaSuccess) return TM_OK;
    cudaGetLastError();
    return TM_ERR_CUDA;
}

struct Lists {
    const float* values; const int32_t* ids; int k; const float* teacher_lse; const float* row_weight; float temperature, scale;
};

int check_distill(const void* logits, int dtype, int64_t rows, int64_t vocab, int64_t ld, const Lists& l, const int* status) {
    if (!good_dtype(dtype)) return TM_ERR_DTYPE;
    if (!good_rows(rows, vocab) || !good_ld(rows, vocab, ld) || vocab > TM_VOCAB_MAX) return TM_ERR_SHAPE;
    if (l.k < 0 || l.k > TM_TOP_MAX || !good_temperature(l.temperature) || !std::isfinite(l.scale)) return TM_ERR_RANGE;
    if (rows == 0) return TM_OK;
    if ((vocab > 0 && !logits) || (l.k > 0 && (!l.values || !l.ids))) return TM_ERR_NULL;
    if (off(logits, elem_bytes(dtype)) || off(l.values, 4) || off(l.ids, 4) || off(l.teacher_lse, 4) || off(l.row_weight, 4) || off(status, 4)) return TM_ERR_ALIGN;
    return TM_OK;
}

int run_distill(const void* logits, int dtype, int64_t rows, int64_t vocab, int64_t ld, const Lists& l, float* loss, float* stats,
                const float* grad_loss, void* dlogits, int64_t ld_d, bool want_loss, bool want_grad, int* status, void* stream) {
    int sms = 0;
    const int rc = tmask::device_sms(&sms);
    if (rc != TM_OK) return rc;
    tmask::DistillArgs a;
    a.logits = logits; a.rows = rows; a.vocab = vocab; a.ld = ld; a.ld_d = ld_d;
    a.values = l.values; a.ids = l.ids; a.k = l.k; a.teacher_lse = l.teacher_lse; a.row_weight = l.row_weight;
    a.temperature = l.temperature; a.scale = l.scale;
    a.loss = loss; a.stats = stats; a.grad_loss = grad_loss; a.dlogits = dlogits; a.status = status;
    return finish(tmask::launch_distill(a, dtype, want_loss, want_grad, sms, static_cast<cudaStream_t>(stream)));
}

}  // namespace

static_assert(TM_TOP_MAX == tmask::kTopMax && TM_DEV_BADID == tmask::kDevBadId, "include/tm.h and the kernels agree");

extern "C" {

int tm_layer_norm(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, int dtype, int64_t rows, int64_t cols,
                  const void* weight, const void* bias, int weight_dtype, float eps, void* sum_out, int64_t ld_sum, void* y, int64_t ld_y,
                  float* mean_out, float* rstd_out, void* cuda_stream) {
    if (!good_dtype(dtype) || !good_dtype(weight_dtype)) return TM_ERR_DTYPE;
    if (!good_rows(rows, cols) || !good_ld(rows, cols, ld_x) || !good_ld(rows, cols, ld_y) || (residual && !good_ld(rows, cols, ld_residual)) ||
        (sum_out && !good_ld(rows, cols, ld_sum))) return TM_ERR_SHAPE;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return TM_ERR_RANGE;
    if (rows == 0 || cols == 0) return TM_OK;
    if (!x || !y) return TM_ERR_NULL;
    const size_t e = elem_bytes(dtype), w = elem_bytes(weight_dtype);
    if (off(x, e) || off(residual, e) || off(sum_out, e) || off(y, e) || off(weight, w) || off(bias, w) || off(mean_out, 4) || off(rstd_out, 4)) return TM_ERR_ALIGN;
    int sms = 0;
    const int rc = tmask::device_sms(&sms);
    if (rc != TM_OK) return rc;
    tmask::NormArgs a = {};
    a.x = x; a.residual = residual; a.rows = rows; a.cols = cols; a.ld_x = ld_x; a.ld_residual = ld_residual; a.ld_sum = ld_sum; a.ld_y = ld_y;
    a.weight = weight; a.bias = bias; a.weight_f32 = weight_dtype == TM_F32; a.eps = eps; a.sum = sum_out; a.y = y; a.mean = mean_out; a.rstd = rstd_out;
    return finish(tmask::launch_norm_forward(a, dtype, sms, static_cast<cudaStream_t>(cuda_stream)));
}

size_t tm_layer_norm_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0) return kWorkspaceAlign;
    const size_t bytes = (size_t)tmask::norm_partial_rows(rows, cols) * 2 * sizeof(float) * (size_t)cols;
    return (bytes + kWorkspaceAlign - 1) / kWorkspaceAlign * kWorkspaceAlign;
}

int tm_layer_norm_backward(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h, int dtype, int64_t rows, int64_t cols,
                           const void* weight, int weight_dtype, const float* mean, const float* rstd, const void* dsum, int64_t ld_dsum,
                           void* dx, int64_t ld_dx, void* dweight_out, void* dbias_out, void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
    if (!good_dtype(dtype) || !good_dtype(weight_dtype)) return TM_ERR_DTYPE;
    if (!good_rows(rows, cols) || !good_ld(rows, cols, ld_dy) || !good_ld(rows, cols, ld_h) || !good_ld(rows, cols, ld_dx) ||
        (dsum && !good_ld(rows, cols, ld_dsum))) return TM_ERR_SHAPE;
    if (cols == 0) return TM_OK;
    if (rows > 0 && (!dy || !h || !mean || !rstd || !dx)) return TM_ERR_NULL;
    const size_t e = elem_bytes(dtype), w = elem_bytes(weight_dtype);
    if (off(dy, e) || off(h, e) || off(dsum, e) || off(dx, e) || off(weight, w) || off(dweight_out, w) || off(dbias_out, w) || off(mean, 4) || off(rstd, 4)) return TM_ERR_ALIGN;
    if ((dweight_out || dbias_out) && rows > 0 &&
        (!workspace_dev || off(workspace_dev, kWorkspaceAlign) || workspace_bytes < tm_layer_norm_workspace_bytes(rows, cols))) return TM_ERR_WORKSPACE;
    if (rows == 0 && !dweight_out && !dbias_out) return TM_OK;
    int sms = 0;
    const int rc = tmask::device_sms(&sms);
    if (rc != TM_OK) return rc;
    tmask::NormBackArgs a = {};
    a.dy = dy; a.h = h; a.dsum = dsum; a.rows = rows; a.cols = cols; a.ld_dy = ld_dy; a.ld_h = ld_h; a.ld_dsum = ld_dsum; a.ld_dx = ld_dx;
    a.weight = weight; a.weight_f32 = weight_dtype == TM_F32; a.mean = mean; a.rstd = rstd; a.dx = dx; a.partials = static_cast<float*>(workspace_dev);
    return finish(tmask::launch_norm_backward(a, dtype, dweight_out, dbias_out, sms, static_cast<cudaStream_t>(cuda_stream)));
}

int tm_top_logits(const void* logits, int dtype, int64_t rows, int64_t vocab, int64_t ld, int k, float temperature,
                  float* values_out, int32_t* ids_out, float* lse_out, int* status_dev, void* cuda_stream) {
    if (!good_dtype(dtype)) return TM_ERR_DTYPE;
    if (!good_rows(rows, vocab) || !good_ld(rows, vocab, ld) || vocab > TM_VOCAB_MAX) return TM_ERR_SHAPE;
    if (k < 1 || k > TM_TOP_MAX || !good_temperature(temperature)) return TM_ERR_RANGE;
    if (rows == 0) return TM_OK;
    if ((vocab > 0 && !logits) || !values_out || !ids_out) return TM_ERR_NULL;
    if (off(logits, elem_bytes(dtype)) || off(values_out, 4) || off(ids_out, 4) || off(lse_out, 4) || off(status_dev, 4)) return TM_ERR_ALIGN;
    int sms = 0;
    const int rc = tmask::device_sms(&sms);
    if (rc != TM_OK) return rc;
    tmask::TopArgs a;
    a.logits = logits; a.rows = rows; a.vocab = vocab; a.ld = ld; a.k = k; a.temperature = temperature;
    a.values = values_out; a.ids = ids_out; a.lse = lse_out; a.status = status_dev;
    return finish(tmask::launch_top(a, dtype, sms, static_cast<cudaStream_t>(cuda_stream)));
}

int tm_distill_loss(const void* logits, int dtype, int64_t rows, int64_t vocab, int64_t ld, const float* top_values, const int32_t* top_ids, int k,
                    const float* teacher_lse, const float* row_weight, float temperature, float scale, float* loss_out, float* stats_out,
                    int* status_dev, void* cuda_stream) {
    const Lists l = {top_values, top_ids, k, teacher_lse, row_weight, temperature, scale};
    const int rc = check_distill(logits, dtype, rows, vocab, ld, l, status_dev);
    if (rc != TM_OK || rows == 0) return rc;
    if (!loss_out) return TM_ERR_NULL;
    if (off(loss_out, 4) || off(stats_out, 4)) return TM_ERR_ALIGN;
    return run_distill(logits, dtype, rows, vocab, ld, l, loss_out, stats_out, nullptr, nullptr, 0, true, false, status_dev, cuda_stream);
}

int tm_distill_grad(const void* logits, int dtype, int64_t rows, int64_t vocab, int64_t ld, const float* top_values, const int32_t* top_ids, int k,
                    const float* teacher_lse, const float* row_weight, float temperature, float scale, const float* stats, const float* grad_loss,
                    void* dlogits, int64_t ld_d, int* status_dev, void* cuda_stream) {
    const Lists l = {top_values, top_ids, k, teacher_lse, row_weight, temperature, scale};
    const int rc = check_distill(logits, dtype, rows, vocab, ld, l, status_dev);
    if (rc != TM_OK) return rc;
    if (!good_ld(rows, vocab, ld_d)) return TM_ERR_SHAPE;
    if (rows == 0) return TM_OK;
    if (!stats || (vocab > 0 && !dlogits)) return TM_ERR_NULL;
    if (off(stats, 4) || off(grad_loss, 4) || off(dlogits, elem_bytes(dtype))) return TM_ERR_ALIGN;
    return run_distill(logits, dtype, rows, vocab, ld, l, nullptr, const_cast<float*>(stats), grad_loss, dlogits, ld_d, false, true, status_dev, cuda_stream);
}

int tm_distill_loss_grad(const void* logits, int dtype, int64_t rows, int64_t vocab, int64_t ld, const float* top_values, const int32_t* top_ids, int k,
                         const float* teacher_lse, const float* row_weight, float temperature, float scale, float* loss_out, void* dlogits,
                         int64_t ld_d, int* status_dev, void* cuda_stream) {
    const Lists l = {top_values, top_ids, k, teacher_lse, row_weight, temperature, scale};
    const int rc = check_distill(logits, dtype, rows, vocab, ld, l, status_dev);
    if (rc != TM_OK) return rc;
    if (!good_ld(rows, vocab, ld_d)) return TM_ERR_SHAPE;
    if (rows == 0) return TM_OK;
    if (!loss_out || (vocab > 0 && !dlogits)) return TM_ERR_NULL;
    if (off(loss_out, 4) || off(dlogits, elem_bytes(dtype))) return TM_ERR_ALIGN;
    return run_distill(logits, dtype, rows, vocab, ld, l, loss_out, nullptr, nullptr, dlogits, ld_d, true, true, status_dev, cuda_stream);
}

}  // extern "C"

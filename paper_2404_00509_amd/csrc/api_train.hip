// C ABI of the operators around the encoder: layer norm, dropout, the linear loss, the gradients of the
// patch embedding.  Host-side validation of the caller's descriptors, then kernel launches.
#include "../../include/mae_hip.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "api_common.hpp"
#include "mae_device.hpp"
#include "mae_kernels.hpp"

namespace {

using mae::aligned;
using mae::have_device;

bool is_dtype(int32_t t) { return t == MAE_F32 || t == MAE_BF16; }
size_t size_of(int32_t t) { return t == MAE_BF16 ? 2 : 4; }

// a workspace of at least `need` bytes
bool has_workspace(const void* p, size_t bytes, size_t need) { return p && aligned(p, 256) && bytes >= need; }

int validate_norm(const mae_norm_desc* d) {
  if (!d) return MAE_ERR_NULL;
  if (!d->x) return MAE_ERR_NULL;
  if (d->M <= 0 || d->D <= 0) return MAE_ERR_SHAPE;
  if (d->M > (int64_t(1) << 28) || d->D > 8192) return MAE_ERR_RANGE;
  if (!(d->eps >= 0.0f) || !isfinite(d->eps)) return MAE_ERR_RANGE;
  if (!is_dtype(d->x_dtype) || !is_dtype(d->y_dtype)) return MAE_ERR_DTYPE;
  if (!aligned(d->x, size_of(d->x_dtype)) || !aligned(d->weight, 4) || !aligned(d->bias, 4)) return MAE_ERR_RANGE;
  return MAE_OK;
}

mae::NormArgs norm_args(const mae_norm_desc* d) {
  mae::NormArgs a{};
  a.M = d->M;
  a.D = d->D;
  a.padded = (d->D + 3) & ~3;
  a.x_bf16 = d->x_dtype == MAE_BF16;
  a.y_bf16 = d->y_dtype == MAE_BF16;
  a.eps = d->eps;
  a.x = d->x;
  a.weight = d->weight;
  a.bias = d->bias;
  return a;
}

int validate_dropout(const mae_dropout_desc* d) {
  if (!d) return MAE_ERR_NULL;
  if (!d->x) return MAE_ERR_NULL;
  if (d->M <= 0 || d->D <= 0) return MAE_ERR_SHAPE;
  if (d->M > (int64_t(1) << 28) || d->D > 8192) return MAE_ERR_RANGE;
  if (!is_dtype(d->dtype)) return MAE_ERR_DTYPE;
  if (!(d->p >= 0.0f && d->p <= 1.0f)) return MAE_ERR_RANGE;
  if (d->rows_per_draw < 0) return MAE_ERR_RANGE;
  if (d->row_base > (uint64_t(1) << 48)) return MAE_ERR_RANGE;  // every index stays below 2^62
  if (!aligned(d->x, size_of(d->dtype)) || !aligned(d->residual, size_of(d->dtype))) return MAE_ERR_RANGE;
  return MAE_OK;
}

int validate_class(const mae_class_desc* d) {
  if (!d) return MAE_ERR_NULL;
  if (!d->tokens || !d->weight || !d->labels) return MAE_ERR_NULL;
  if (d->M <= 0 || d->D <= 0 || d->V <= 0) return MAE_ERR_SHAPE;
  if (d->D % 8 != 0) return MAE_ERR_SHAPE;
  if (d->M > (int64_t(1) << 24) || d->D > 8192 || d->V > (1 << 20)) return MAE_ERR_RANGE;
  if (d->M * d->V > (int64_t(1) << 38)) return MAE_ERR_RANGE;  // keeps every grid below 2^32 threads
  if (!(d->smoothing >= 0.0f && d->smoothing <= 1.0f) || !isfinite(d->grad_scale)) return MAE_ERR_RANGE;
  if (!aligned(d->tokens, 16) || !aligned(d->weight, 16) || !aligned(d->bias, 4) || !aligned(d->labels, 4))
    return MAE_ERR_RANGE;
  return MAE_OK;
}

constexpr int kMaxPosRows = 8192;  // the work of grad_pos grows with it

int validate_embed_grad(const mae_embed_desc* d) {
  const int rc = mae::validate_embed(d);
  if (rc != MAE_OK) return rc;
  if (d->out_dtype != MAE_BF16) return MAE_ERR_DTYPE;
  if (d->pos && d->L > kMaxPosRows) return MAE_ERR_RANGE;
  return MAE_OK;
}

}  // namespace

extern "C" {

int mae_layer_norm(const mae_norm_desc* d, void* y, float* mean, float* rstd, void* hip_stream) {
  int rc = validate_norm(d);
  if (rc != MAE_OK) return rc;
  if (!y) return MAE_ERR_NULL;
  if (!aligned(y, size_of(d->y_dtype)) || !aligned(mean, 4) || !aligned(rstd, 4)) return MAE_ERR_RANGE;
  rc = have_device();
  if (rc != MAE_OK) return rc;
  mae::NormArgs a = norm_args(d);
  a.y = y;
  a.mean_out = mean;
  a.rstd_out = rstd;
  return mae::launch_layer_norm(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MAE_OK : MAE_ERR_HIP;
}

size_t mae_layer_norm_workspace_bytes(const mae_norm_desc* d) {
  if (validate_norm(d) != MAE_OK) return 0;
  return (size_t)mae::norm_partials(d->M, d->D) * 2 * (size_t)((d->D + 3) & ~3) * sizeof(float);
}

int mae_layer_norm_grad(const mae_norm_desc* d, const void* grad_y, const float* mean, const float* rstd, void* grad_x,
                        float* grad_weight, float* grad_bias, void* workspace, size_t workspace_bytes,
                        void* hip_stream) {
  int rc = validate_norm(d);
  if (rc != MAE_OK) return rc;
  if (!grad_y || !mean || !rstd || (!grad_x && !grad_weight && !grad_bias)) return MAE_ERR_NULL;
  if (!aligned(grad_y, size_of(d->y_dtype)) || !aligned(grad_x, size_of(d->x_dtype)) || !aligned(mean, 4) ||
      !aligned(rstd, 4) || !aligned(grad_weight, 4) || !aligned(grad_bias, 4))
    return MAE_ERR_RANGE;
  const bool params = grad_weight || grad_bias;
  if (params && !has_workspace(workspace, workspace_bytes, mae_layer_norm_workspace_bytes(d)))
    return MAE_ERR_WORKSPACE;
  rc = have_device();
  if (rc != MAE_OK) return rc;
  mae::NormArgs a = norm_args(d);
  a.grad_y = grad_y;
  a.mean = mean;
  a.rstd = rstd;
  a.grad_x = grad_x;
  a.grad_weight = grad_weight;
  a.grad_bias = grad_bias;
  a.partials = params ? static_cast<float*>(workspace) : nullptr;
  a.num_partials = mae::norm_partials(d->M, d->D);
  return mae::launch_layer_norm_grad(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MAE_OK : MAE_ERR_HIP;
}

int mae_dropout(const mae_dropout_desc* d, void* y, void* hip_stream) {
  int rc = validate_dropout(d);
  if (rc != MAE_OK) return rc;
  if (!y) return MAE_ERR_NULL;
  if (!aligned(y, size_of(d->dtype))) return MAE_ERR_RANGE;
  rc = have_device();
  if (rc != MAE_OK) return rc;
  mae::DropoutArgs a{};
  a.count = d->M * d->D;
  const uint64_t word = ((uint64_t)d->layer << 32) | ((uint64_t)mae::kDropout << 24);
  a.key = mae::mix64(mae::batch_key(d->seed, d->batch_index) + mae::kGamma * (word + 1));
  const double p = (double)d->p;
  a.threshold = (uint64_t)floor(p * 4294967296.0 + 0.5);
  a.scale = p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.0f;
  a.bf16 = d->dtype == MAE_BF16;
  a.x = d->x;
  a.residual = d->residual;
  a.y = y;
  if (d->rows_per_draw) {
    a.span = (uint64_t)d->rows_per_draw * (uint64_t)d->D;
    a.group0 = d->row_base / (uint64_t)d->rows_per_draw;
    a.first = d->row_base % (uint64_t)d->rows_per_draw * (uint64_t)d->D;
  } else {
    a.first = d->row_base * (uint64_t)d->D;
  }
  return mae::launch_dropout(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MAE_OK : MAE_ERR_HIP;
}

size_t mae_class_loss_workspace_bytes(const mae_class_desc* d, int32_t with_grad) {
  if (validate_class(d) != MAE_OK) return 0;
  return mae::class_plan(d->M, d->D, d->V, d->bias != nullptr, d->smoothing > 0.0f, with_grad != 0).bytes;
}

int mae_class_loss(const mae_class_desc* d, float* loss, float* row_loss, void* grad_tokens, void* grad_weight,
                   float* grad_bias, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = validate_class(d);
  if (rc != MAE_OK) return rc;
  if (!loss) return MAE_ERR_NULL;
  if (grad_bias && !d->bias) return MAE_ERR_NULL;
  if (!aligned(loss, 4) || !aligned(row_loss, 4) || !aligned(grad_tokens, 16) || !aligned(grad_weight, 16) ||
      !aligned(grad_bias, 4))
    return MAE_ERR_RANGE;
  const bool grad = grad_tokens || grad_weight || grad_bias;
  const mae::ClassPlan p = mae::class_plan(d->M, d->D, d->V, d->bias != nullptr, d->smoothing > 0.0f, grad);
  if (!has_workspace(workspace, workspace_bytes, p.bytes)) return MAE_ERR_WORKSPACE;
  rc = have_device();
  if (rc != MAE_OK) return rc;
  char* ws = static_cast<char*>(workspace);
  const auto at = [&](size_t offset, auto* type) { return reinterpret_cast<decltype(type)>(ws + offset); };
  mae::ClassArgs a{};
  a.M = d->M;
  a.D = d->D;
  a.V = d->V;
  a.smoothing = d->smoothing;
  a.grad_scale = d->grad_scale;
  a.tokens = d->tokens;
  a.weight = d->weight;
  a.bias = d->bias;
  a.labels = d->labels;
  a.loss = loss;
  a.row_loss = row_loss;
  a.grad_tokens = grad_tokens;
  a.grad_weight = grad_weight;
  a.grad_bias = grad_bias;
  a.stats = at(p.stats, (float*)nullptr);
  a.logit_sums = d->smoothing > 0.0f ? at(p.logit_sums, (float*)nullptr) : nullptr;
  a.label_logit = at(p.label_logit, (float*)nullptr);
  if (p.few) {  // the tokens and labels as they are
    a.packed = const_cast<uint16_t*>(static_cast<const uint16_t*>(d->tokens));
    a.label_of = const_cast<int32_t*>(d->labels);
  } else {
    a.count = at(p.count, (int32_t*)nullptr);
    a.label_of = at(p.label_of, (int32_t*)nullptr);
    a.row_of = at(p.row_of, (int32_t*)nullptr);
    a.packed = at(p.packed, (uint16_t*)nullptr);
    a.partials = at(p.partials, (double*)nullptr);
  }
  if (grad) {
    a.ranges = at(p.ranges, (uint32_t*)nullptr);
    a.wide = at(p.wide, (int32_t*)nullptr);
    a.row_max = at(p.row_max, (float*)nullptr);
    a.row_inv = at(p.row_inv, (float*)nullptr);
    a.half_tokens = at(p.half_tokens, (uint16_t*)nullptr);
    a.half_weight = at(p.half_weight, (uint16_t*)nullptr);
    a.g = at(p.g, (uint16_t*)nullptr);
    a.logits = at(p.logits, (float*)nullptr);
    a.tops = at(p.tops, (float*)nullptr);
    a.column_sums = at(p.column_sums, (float*)nullptr);
    a.tokens_acc = at(p.tokens_acc, (float*)nullptr);
    a.weight_acc = at(p.weight_acc, (float*)nullptr);
  }
  return mae::launch_class_loss(a, p, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MAE_OK : MAE_ERR_HIP;
}

size_t mae_patch_embed_grad_workspace_bytes(const mae_embed_desc* d) {
  if (validate_embed_grad(d) != MAE_OK) return 0;
  return mae::embed_grad_plan(d->M, d->D, d->E, d->pos ? d->L : 1).bytes;
}

int mae_patch_embed_grad(const mae_embed_desc* d, const void* grad_tokens, float* grad_weight, float* grad_bias,
                         float* grad_pos, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = validate_embed_grad(d);
  if (rc != MAE_OK) return rc;
  if (!grad_tokens || (!grad_weight && !grad_bias && !grad_pos) || (grad_pos && !d->pos)) return MAE_ERR_NULL;
  if (!aligned(grad_tokens, 16) || !aligned(grad_weight, 16) || !aligned(grad_bias, 4) || !aligned(grad_pos, 4))
    return MAE_ERR_RANGE;
  if (!has_workspace(workspace, workspace_bytes, mae_patch_embed_grad_workspace_bytes(d))) return MAE_ERR_WORKSPACE;
  rc = have_device();
  if (rc != MAE_OK) return rc;
  mae::EmbedGradArgs a{};
  a.M = d->M;
  a.D = d->D;
  a.E = d->E;
  a.pos_columns = grad_pos ? d->L : grad_bias ? 1 : 0;
  const mae::EmbedGradPlan p = mae::embed_grad_plan(d->M, d->D, d->E, d->pos ? d->L : 1);
  char* ws = static_cast<char*>(workspace);
  a.g = static_cast<const uint16_t*>(grad_tokens);
  a.visible = static_cast<const uint16_t*>(d->visible);
  a.ids = grad_pos ? d->ids_keep : nullptr;
  a.grad_weight = grad_weight;
  a.grad_bias = grad_bias;
  a.grad_pos = grad_pos;
  a.weight_acc = reinterpret_cast<float*>(ws + p.weight_acc);
  a.pos_acc = reinterpret_cast<float*>(ws + p.pos_acc);
  return mae::launch_embed_grad(a, p, reinterpret_cast<uint16_t*>(ws + p.padded),
                                static_cast<hipStream_t>(hip_stream)) == hipSuccess
             ? MAE_OK
             : MAE_ERR_HIP;
}

}  // extern "C"

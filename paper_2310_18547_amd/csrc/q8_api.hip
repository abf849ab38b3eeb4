// C ABI of the 8-bit backbone: argument checks and dispatch (include/sgmv.h, last section).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/sgmv.h"
#include "launch.h"
#include "q8.h"
#include "spans.h"

namespace {

using namespace sgmv;

int check_rows(int32_t dtype, int32_t n_tokens, int32_t h) {
  if (dtype != SGMV_F16 && dtype != SGMV_BF16) return SGMV_ERR_UNSUPPORTED;
  if (n_tokens < 0 || h <= 0) return SGMV_ERR_SHAPE;
  if (h % 8 != 0 || h > kRowsMostWidth) return SGMV_ERR_UNSUPPORTED;
  return SGMV_OK;
}

// The two parts of an 8-bit result go together; `must`: they cannot be left out.
int check_q8(const int8_t* q, const float* q_scales, bool must) {
  if ((q == nullptr) != (q_scales == nullptr) || (must && q == nullptr)) return SGMV_ERR_NULL;
  if (!aligned(q, 16) || !aligned(q_scales, 4)) return SGMV_ERR_ALIGN;
  return SGMV_OK;
}

// Whether a row call would overwrite what it still reads, or one of its outputs another.  A thread reads its part of every input
// before it stores, so a 16-bit output may be an input as a whole; 8-bit rows lie elsewhere than the 16-bit ones they come from.
bool rows_overlap(const RowsArgs& a) {
  const size_t n = (size_t)a.n_tokens, values = n * (size_t)a.h;
  const Span written[] = {{a.out, 2 * values}, {a.sum, 2 * values}, {a.q, values}, {a.q_scales, 4 * n}};
  const Span read[] = {{a.x, 2 * values}, {a.other, 2 * values}, {a.weight, 2 * (size_t)a.h}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < i; ++j)
      if (overlap(written[i], written[j])) return true;
    for (int j = 0; j < 3; ++j)
      if (overlap(written[i], read[j]) && !(i < 2 && j < 2 && written[i].at == read[j].at)) return true;
  }
  return false;
}

// The same of a dense call with that many bytes of partial sums.
bool dense_overlap(const DenseArgs& a, size_t partials) {
  const size_t n = (size_t)a.n_tokens, h_in = (size_t)a.h_in;
  const Span q = {a.q, n * h_in}, q_scales = {a.q_scales, 4 * n}, scratch = {partials > 0 ? a.workspace : nullptr, partials};
  if (overlap(scratch, q) || overlap(scratch, q_scales)) return true;
  for (int i = 0; i < a.n_proj; ++i) {
    const size_t channels = (size_t)a.h_out[i];
    const Span y = {a.y[i], 2 * n * channels}, w = {a.w[i], channels * h_in}, w_scales = {a.w_scales[i], 4 * channels};
    if (overlap(y, q) || overlap(y, q_scales) || overlap(y, scratch) || overlap(scratch, w) || overlap(scratch, w_scales)) return true;
    for (int j = 0; j < a.n_proj; ++j) {
      const size_t others = (size_t)a.h_out[j];
      if (overlap(y, {a.w[j], others * h_in}) || overlap(y, {a.w_scales[j], 4 * others})) return true;
      if (j < i && overlap(y, {a.y[j], 2 * n * others})) return true;
    }
  }
  return false;
}

// What a dense call and its plan refuse alike; `*nothing`: the call has nothing to do.
int check_dense(int32_t dtype, int32_t n_proj, int32_t n_tokens, int32_t h_in, const int32_t* h_outs, const void* workspace,
                size_t workspace_bytes, bool* nothing) {
  *nothing = n_proj == 0 || n_tokens == 0;
  if (dtype != SGMV_F16 && dtype != SGMV_BF16) return SGMV_ERR_UNSUPPORTED;
  if (n_proj < 0 || n_proj > kDenseMostProjections || n_tokens < 0 || h_in <= 0) return SGMV_ERR_SHAPE;
  if (workspace_bytes > SIZE_MAX / 2) return SGMV_ERR_SHAPE;  // a negative number of the caller's
  if (h_in % 8 != 0 || h_in > kDenseMostHin || n_tokens > kDenseMostTokens) return SGMV_ERR_UNSUPPORTED;
  if (n_proj > 0 && h_outs == nullptr) return SGMV_ERR_NULL;
  long long channels = 0;
  for (int i = 0; i < n_proj; ++i) {
    if (h_outs[i] <= 0) return SGMV_ERR_SHAPE;
    if (h_outs[i] % 8 != 0 || h_outs[i] > kDenseMostHout) return SGMV_ERR_UNSUPPORTED;
    channels += h_outs[i];
  }
  if (n_tokens * channels > kDenseMostValues) return SGMV_ERR_UNSUPPORTED;
  return aligned(workspace, 256) ? SGMV_OK : SGMV_ERR_ALIGN;
}

DenseArgs dense_shape(int32_t dtype, int32_t n_proj, int32_t n_tokens, int32_t h_in, const int32_t* h_outs, void* workspace,
                      size_t workspace_bytes) {
  DenseArgs a = {};
  a.bf16 = dtype == SGMV_BF16;
  a.n_tokens = n_tokens;
  a.h_in = h_in;
  a.n_proj = n_proj;
  for (int i = 0; i < n_proj; ++i) a.h_out[i] = h_outs[i];
  a.workspace = workspace;
  a.workspace_bytes = workspace == nullptr ? 0 : workspace_bytes;
  return a;
}

int launch(const RowsArgs& a, void* stream) {
  if (rows_overlap(a)) return SGMV_ERR_SHAPE;
  return launch_rows(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SGMV_OK : SGMV_ERR_LAUNCH;
}

}  // namespace

extern "C" {

int sgmv_rms_norm_q8(int32_t dtype, void* out, int8_t* q, float* q_scales, void* sum, const void* x, const void* residual,
                     const void* weight, float eps, int32_t n_tokens, int32_t h, void* stream) {
  int rc = check_rows(dtype, n_tokens, h);
  if (rc != SGMV_OK) return rc;
  if (!(eps >= 0.0f) || !(eps < __builtin_inff())) return SGMV_ERR_UNSUPPORTED;
  if (n_tokens == 0) return SGMV_OK;
  if (x == nullptr || weight == nullptr || (out == nullptr && q == nullptr)) return SGMV_ERR_NULL;
  rc = check_q8(q, q_scales, false);
  if (rc != SGMV_OK) return rc;
  if (!aligned(out, 16) || !aligned(sum, 16) || !aligned(x, 16) || !aligned(residual, 16) || !aligned(weight, 16)) return SGMV_ERR_ALIGN;
  return launch(RowsArgs{kRowsNorm, dtype == SGMV_BF16, n_tokens, h, eps, x, residual, weight, sum, out, q, q_scales}, stream);
}

int sgmv_silu_mul_q8(int32_t dtype, void* out, int8_t* q, float* q_scales, const void* gate, const void* up, int32_t n_tokens,
                     int32_t h, void* stream) {
  int rc = check_rows(dtype, n_tokens, h);
  if (rc != SGMV_OK) return rc;
  if (n_tokens == 0) return SGMV_OK;
  if (gate == nullptr || up == nullptr || (out == nullptr && q == nullptr)) return SGMV_ERR_NULL;
  rc = check_q8(q, q_scales, false);
  if (rc != SGMV_OK) return rc;
  if (!aligned(out, 16) || !aligned(gate, 16) || !aligned(up, 16)) return SGMV_ERR_ALIGN;
  return launch(RowsArgs{kRowsSiluMul, dtype == SGMV_BF16, n_tokens, h, 0.0f, gate, up, nullptr, nullptr, out, q, q_scales}, stream);
}

int sgmv_quantize_q8(int32_t dtype, int8_t* q, float* q_scales, const void* x, int32_t n_tokens, int32_t h, void* stream) {
  int rc = check_rows(dtype, n_tokens, h);
  if (rc != SGMV_OK) return rc;
  if (n_tokens == 0) return SGMV_OK;
  if (x == nullptr) return SGMV_ERR_NULL;
  rc = check_q8(q, q_scales, true);
  if (rc != SGMV_OK) return rc;
  if (!aligned(x, 16)) return SGMV_ERR_ALIGN;
  return launch(RowsArgs{kRowsQuantize, dtype == SGMV_BF16, n_tokens, h, 0.0f, x, nullptr, nullptr, nullptr, nullptr, q, q_scales}, stream);
}

int sgmv_dense_q8(int32_t dtype, int32_t n_proj, void* const* ys, const int8_t* q, const float* q_scales, const int8_t* const* ws,
                  const float* const* w_scales, int32_t n_tokens, int32_t h_in, const int32_t* h_outs, void* workspace,
                  size_t workspace_bytes, void* stream) {
  bool nothing = false;
  const int rc = check_dense(dtype, n_proj, n_tokens, h_in, h_outs, workspace, workspace_bytes, &nothing);
  if (rc != SGMV_OK || nothing) return rc;
  if (ys == nullptr || q == nullptr || q_scales == nullptr || ws == nullptr || w_scales == nullptr) return SGMV_ERR_NULL;
  if (!aligned(q, 16) || !aligned(q_scales, 4)) return SGMV_ERR_ALIGN;
  DenseArgs a = dense_shape(dtype, n_proj, n_tokens, h_in, h_outs, workspace, workspace_bytes);
  a.q = q;
  a.q_scales = q_scales;
  for (int i = 0; i < n_proj; ++i) {
    if (ys[i] == nullptr || ws[i] == nullptr || w_scales[i] == nullptr) return SGMV_ERR_NULL;
    if (!aligned(ys[i], 16) || !aligned(ws[i], 16) || !aligned(w_scales[i], 16)) return SGMV_ERR_ALIGN;
    a.w[i] = ws[i];
    a.w_scales[i] = w_scales[i];
    a.y[i] = ys[i];
  }
  DensePlan plan;
  plan_dense(a, compute_units(), &plan);
  size_t channels = 0;
  for (int i = 0; i < n_proj; ++i) channels += (size_t)h_outs[i];
  if (dense_overlap(a, plan.splits > 1 ? 4 * channels * n_tokens * plan.splits : 0)) return SGMV_ERR_SHAPE;
  return launch_dense(a, plan, static_cast<hipStream_t>(stream)) == hipSuccess ? SGMV_OK : SGMV_ERR_LAUNCH;
}

int sgmv_plan_dense_q8(int32_t dtype, int32_t n_proj, int32_t n_tokens, int32_t h_in, const int32_t* h_outs,
                       const void* workspace, size_t workspace_bytes, sgmv_plan* plan) {
  if (plan == nullptr) return SGMV_ERR_NULL;
  *plan = sgmv_plan{};
  bool nothing = false;
  const int rc = check_dense(dtype, n_proj, n_tokens, h_in, h_outs, workspace, workspace_bytes, &nothing);
  if (rc != SGMV_OK || nothing) return rc;
  DensePlan d;
  plan_dense(dense_shape(dtype, n_proj, n_tokens, h_in, h_outs, const_cast<void*>(workspace), workspace_bytes), compute_units(), &d);
  plan->kernel = d.family == kDenseFew ? SGMV_KERNEL_DENSE_FEW : d.family == kDenseSmall ? SGMV_KERNEL_DENSE_SMALL : SGMV_KERNEL_DENSE_LARGE;
  plan->launches = d.splits > 1 ? 2 : (n_tokens + d.tokens - 1LL) / d.tokens;
  plan->slices = d.splits;
  plan->workgroups = (int32_t)d.workgroups;
  plan->lds_bytes = d.lds;
  return SGMV_OK;
}

}  // extern "C"

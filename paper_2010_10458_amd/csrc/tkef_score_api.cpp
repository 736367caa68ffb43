// Host side of the scores of given tokens (include/tkef.h, "scores of tokens"): plans,
// argument checks, the launch of the kernels in tkef_score.hip.
#include <new>

#include "tkef.h"
#include "tkef_rows.h"
#include "tkef_rows_host.h"

struct tkef_score_plan_s : RowPlan {};

namespace {

tkef::ScoreArgs score_args(const RowPlan& p, const void* z, int64_t ld, int64_t rows,
                           const int32_t* tokens, uint32_t* status) {
  tkef::ScoreArgs a{};
  a.z = z;
  a.ld = ld;
  a.rows = rows;
  a.V = (int32_t)p.vocab;
  a.dtype = p.dtype;
  a.a = (float)(kLog2e / p.temperature);
  a.inv_t = (float)(1.0 / p.temperature);
  a.tokens = tokens;
  a.status = status;
  return a;
}

}  // namespace

extern "C" {

int tkef_score_plan_create(int64_t rows, int64_t vocab, int64_t k, int32_t dtype,
                           double temperature, tkef_score_plan* plan_out) {
  if (plan_out == nullptr) return TKEF_EINVAL;
  *plan_out = nullptr;
  const int rc = check_sizes(rows, vocab, dtype, temperature);
  if (rc != TKEF_OK) return rc;
  if (k < 0 || k > vocab || k > TKEF_SCORE_MAX_K) return TKEF_ERANGE;
  tkef_score_plan p = new (std::nothrow) tkef_score_plan_s;
  if (p == nullptr) return TKEF_ENOMEM;
  p->rows = rows;
  p->vocab = vocab;
  p->k = k;
  p->dtype = dtype;
  p->temperature = temperature;
  p->ws_bytes = (tkef::score_workspace(rows, vocab, k, dtype) + 255) & ~(size_t)255;
  *plan_out = p;
  return TKEF_OK;
}

int tkef_score_plan_destroy(tkef_score_plan plan) {
  if (plan == nullptr) return TKEF_EINVAL;
  delete plan;
  return TKEF_OK;
}

int tkef_score_plan_info(tkef_score_plan plan, size_t* workspace_bytes) {
  if (plan == nullptr) return TKEF_EINVAL;
  if (workspace_bytes != nullptr) *workspace_bytes = plan->ws_bytes;
  return TKEF_OK;
}

int tkef_score_forward(tkef_score_plan plan, const void* logits, int64_t row_stride, int64_t rows,
                       const int32_t* tokens, float* logp, float* entropy, int32_t* idx_out,
                       float* val_out, float* stats, void* ws, size_t ws_bytes, uint32_t* status,
                       hipStream_t stream) {
  if (plan == nullptr) return TKEF_EINVAL;
  int rc = check_rows(*plan, logits, row_stride, rows);
  if (rc == TKEF_OK) rc = check_ws(plan->ws_bytes, ws, ws_bytes);
  if (rc != TKEF_OK || rows == 0) return rc;
  if (tokens == nullptr || logp == nullptr || (idx_out == nullptr) != (val_out == nullptr))
    return TKEF_EINVAL;
  if (!aligned(tokens, 4) || !aligned(logp, 4) || !aligned(entropy, 4) || !aligned(idx_out, 4) ||
      !aligned(val_out, 4) || !aligned(stats, 16) || !aligned(status, 4))
    return TKEF_EINVAL;
  tkef::ScoreArgs a = score_args(*plan, logits, row_stride, rows, tokens, status);
  a.k = idx_out != nullptr ? (int32_t)plan->k : 0;
  a.logp = logp;
  a.entropy = entropy;
  a.idx = idx_out;
  a.val = val_out;
  a.stats = reinterpret_cast<float4*>(stats);
  return done(tkef::launch_score_forward(a, ws, stream));
}

int tkef_score_backward(tkef_score_plan plan, const void* logits, int64_t row_stride, int64_t rows,
                        const int32_t* tokens, const float* stats, const float* dlogp,
                        const float* dentropy, void* grad, int64_t grad_stride, uint32_t* status,
                        hipStream_t stream) {
  if (plan == nullptr) return TKEF_EINVAL;
  int rc = check_rows(*plan, logits, row_stride, rows);
  if (rc != TKEF_OK || rows == 0) return rc;
  rc = check_grad(*plan, logits, row_stride, rows, grad, grad_stride);
  if (rc != TKEF_OK) return rc;
  if (tokens == nullptr || stats == nullptr || (dlogp == nullptr && dentropy == nullptr))
    return TKEF_EINVAL;
  if (!aligned(tokens, 4) || !aligned(stats, 16) || !aligned(dlogp, 4) || !aligned(dentropy, 4) ||
      !aligned(status, 4))
    return TKEF_EINVAL;
  tkef::ScoreArgs a = score_args(*plan, logits, row_stride, rows, tokens, status);
  a.stats = reinterpret_cast<float4*>(const_cast<float*>(stats));
  a.dlogp = dlogp;
  a.dentropy = dentropy;
  a.grad = grad;
  a.gld = grad_stride;
  return done(tkef::launch_score_backward(a, stream));
}

}  // extern "C"

// Host side of the row operators (include/tkef.h, "Rows of logits"): plans,
// argument checks, the launch of the kernels in tkef_rows.hip.
#include <math.h>

#include <new>

#include "tkef.h"
#include "tkef_internal.h"
#include "tkef_rows.h"

namespace {

struct RowPlan {
  int64_t rows = 0, vocab = 0, k = 0;
  int32_t dtype = 0, val_format = 0;
  double temperature = 1.0;
  size_t ws_bytes = 0;
};

constexpr double kLog2e = 1.4426950408889634074;
constexpr int64_t kMaxStride = (int64_t)1 << 40;  // elements: byte offsets stay below 2^63

size_t elem_size(int32_t dtype) { return dtype == TKEF_DTYPE_F32 ? 4 : 2; }

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int check_sizes(int64_t rows, int64_t vocab, int32_t dtype, double temperature) {
  if (dtype != TKEF_DTYPE_F32 && dtype != TKEF_DTYPE_F16 && dtype != TKEF_DTYPE_BF16)
    return TKEF_EINVAL;
  if (rows < 1 || rows > TKEF_ROWS_MAX_ROWS || vocab < 1 || vocab > TKEF_ROWS_MAX_VOCAB)
    return TKEF_ERANGE;
  if (!(temperature >= 1e-6 && temperature <= 1e6)) return TKEF_ERANGE;
  return TKEF_OK;
}

int check_list(int64_t vocab, int64_t k, int32_t val_format) {
  if (val_format != TKEF_VAL_F32 && val_format != TKEF_VAL_F16) return TKEF_EINVAL;
  return k < 1 || k > vocab || k > TKEF_ROWS_MAX_K ? TKEF_ERANGE : TKEF_OK;
}

int check_ws(size_t need, const void* ws, size_t ws_bytes) {
  if (need == 0) return TKEF_OK;
  return ws == nullptr || ws_bytes < need || !aligned(ws, 256) ? TKEF_EWORKSPACE : TKEF_OK;
}

int check_rows(const RowPlan& p, const void* z, int64_t ld, int64_t rows) {
  if (rows < 0 || rows > p.rows) return TKEF_ERANGE;
  if (ld > kMaxStride) return TKEF_ERANGE;
  if (rows > 0 && (z == nullptr || !aligned(z, elem_size(p.dtype)) || ld < p.vocab))
    return TKEF_EINVAL;
  return TKEF_OK;
}

int check_lists(const RowPlan& p, const int32_t* idx, const void* val, const float* tail,
                const int32_t* count, const float* weight, const uint32_t* status) {
  if (idx == nullptr || val == nullptr) return TKEF_EINVAL;
  if (!aligned(idx, 4) || !aligned(val, p.val_format == TKEF_VAL_F16 ? 2 : 4) ||
      !aligned(tail, 4) || !aligned(count, 4) || !aligned(weight, 4) || !aligned(status, 4))
    return TKEF_EINVAL;
  return TKEF_OK;
}

// grad is the logits themselves or does not touch them: it lies before or after all of
// their rows, or between them at their stride
int check_grad(const RowPlan& p, const void* z, int64_t ld, int64_t rows, const void* g,
               int64_t gld) {
  if (gld > kMaxStride) return TKEF_ERANGE;
  if (g == nullptr || !aligned(g, elem_size(p.dtype)) || gld < p.vocab) return TKEF_EINVAL;
  if (g == z && gld == ld) return TKEF_OK;
  const size_t e = elem_size(p.dtype), row = (size_t)p.vocab * e, step = (size_t)ld * e;
  const uintptr_t za = reinterpret_cast<uintptr_t>(z), ga = reinterpret_cast<uintptr_t>(g);
  const uintptr_t ze = za + (size_t)(rows - 1) * step + row;
  const uintptr_t ge = ga + (size_t)(rows - 1) * (size_t)gld * e + row;
  if (za >= ge || ga >= ze) return TKEF_OK;
  if (gld != ld) return TKEF_EINVAL;
  // where a row of grad begins behind the row of logits before it
  const size_t at = ga >= za ? (ga - za) % step : (step - (za - ga) % step) % step;
  return at >= row && at + row <= step ? TKEF_OK : TKEF_EINVAL;
}

int done(hipError_t e) { return e == hipSuccess ? TKEF_OK : TKEF_EHIP; }

}  // namespace

struct tkef_top_plan_s : RowPlan {};
struct tkef_distill_plan_s : RowPlan {};
struct tkef_verify_plan_s : RowPlan {  // rows: the batch
  int64_t draft = 0;
};

namespace {

tkef::DistillArgs distill_args(const RowPlan& p, const void* z, int64_t ld, int64_t rows,
                               const int32_t* idx, const void* val, const float* tail,
                               const int32_t* count, const float* weight, uint32_t* status) {
  tkef::DistillArgs a{};
  a.z = z;
  a.ld = ld;
  a.rows = rows;
  a.V = (int32_t)p.vocab;
  a.k = (int32_t)p.k;
  a.dtype = p.dtype;
  a.val_format = p.val_format;
  a.a = (float)(kLog2e / p.temperature);
  a.inv_t = (float)(1.0 / p.temperature);
  a.inv_t_lo = (float)(1.0 / p.temperature - (double)a.inv_t);
  a.temperature = (float)p.temperature;
  a.idx = idx;
  a.val = val;
  a.tail = tail;
  a.count = count;
  a.weight = weight;
  a.status = status;
  return a;
}

}  // namespace

extern "C" {

int tkef_top_plan_create(int64_t rows, int64_t vocab, int64_t k, int32_t dtype,
                         int32_t val_format, double temperature, tkef_top_plan* plan_out) {
  if (plan_out == nullptr) return TKEF_EINVAL;
  *plan_out = nullptr;
  int rc = check_sizes(rows, vocab, dtype, temperature);
  if (rc == TKEF_OK) rc = check_list(vocab, k, val_format);
  if (rc != TKEF_OK) return rc;
  tkef_top_plan p = new (std::nothrow) tkef_top_plan_s;
  if (p == nullptr) return TKEF_ENOMEM;
  p->rows = rows;
  p->vocab = vocab;
  p->k = k;
  p->dtype = dtype;
  p->val_format = val_format;
  p->temperature = temperature;
  p->ws_bytes = (tkef::top_workspace(rows, vocab, k, dtype) + 255) & ~(size_t)255;
  *plan_out = p;
  return TKEF_OK;
}

int tkef_top_plan_destroy(tkef_top_plan plan) {
  if (plan == nullptr) return TKEF_EINVAL;
  delete plan;
  return TKEF_OK;
}

int tkef_top_plan_info(tkef_top_plan plan, size_t* workspace_bytes) {
  if (plan == nullptr) return TKEF_EINVAL;
  if (workspace_bytes != nullptr) *workspace_bytes = plan->ws_bytes;
  return TKEF_OK;
}

int tkef_top_execute(tkef_top_plan plan, const void* logits, int64_t row_stride, int64_t rows,
                     int32_t* idx_out, void* val_out, float* tail_out, void* ws,
                     size_t ws_bytes, uint32_t* status, hipStream_t stream) {
  if (plan == nullptr) return TKEF_EINVAL;
  int rc = check_rows(*plan, logits, row_stride, rows);
  if (rc == TKEF_OK) rc = check_ws(plan->ws_bytes, ws, ws_bytes);
  if (rc != TKEF_OK || rows == 0) return rc;
  if (idx_out == nullptr || val_out == nullptr || !aligned(idx_out, 4) ||
      !aligned(val_out, plan->val_format == TKEF_VAL_F16 ? 2 : 4) || !aligned(tail_out, 4) ||
      !aligned(status, 4))
    return TKEF_EINVAL;
  tkef::TopArgs a{};
  a.z = logits;
  a.ld = row_stride;
  a.rows = rows;
  a.V = (int32_t)plan->vocab;
  a.k = (int32_t)plan->k;
  a.dtype = plan->dtype;
  a.val_format = plan->val_format;
  a.a = (float)(kLog2e / plan->temperature);
  a.inv_t = (float)(1.0 / plan->temperature);
  a.idx = idx_out;
  a.val = val_out;
  a.tail = tail_out;
  a.status = status;
  return done(tkef::launch_top(a, ws, stream));
}

int tkef_distill_plan_create(int64_t rows, int64_t vocab, int64_t k, int32_t dtype,
                             int32_t val_format, double temperature,
                             tkef_distill_plan* plan_out) {
  if (plan_out == nullptr) return TKEF_EINVAL;
  *plan_out = nullptr;
  int rc = check_sizes(rows, vocab, dtype, temperature);
  if (rc == TKEF_OK) rc = check_list(vocab, k, val_format);
  if (rc != TKEF_OK) return rc;
  tkef_distill_plan p = new (std::nothrow) tkef_distill_plan_s;
  if (p == nullptr) return TKEF_ENOMEM;
  p->rows = rows;
  p->vocab = vocab;
  p->k = k;
  p->dtype = dtype;
  p->val_format = val_format;
  p->temperature = temperature;
  const int chunks = tkef::distill_chunks(vocab, dtype, rows, false);  // (a step has no more)
  if (chunks > 1)
    p->ws_bytes = ((size_t)rows * (size_t)chunks * tkef::kPartBytes + 255) & ~(size_t)255;
  *plan_out = p;
  return TKEF_OK;
}

int tkef_distill_plan_destroy(tkef_distill_plan plan) {
  if (plan == nullptr) return TKEF_EINVAL;
  delete plan;
  return TKEF_OK;
}

int tkef_distill_plan_info(tkef_distill_plan plan, size_t* workspace_bytes) {
  if (plan == nullptr) return TKEF_EINVAL;
  if (workspace_bytes != nullptr) *workspace_bytes = plan->ws_bytes;
  return TKEF_OK;
}

int tkef_distill_forward(tkef_distill_plan plan, const void* logits, int64_t row_stride,
                         int64_t rows, const int32_t* idx, const void* val, const float* tail,
                         const int32_t* count, const float* weight, float* loss, float* stats,
                         void* ws, size_t ws_bytes, uint32_t* status, hipStream_t stream) {
  if (plan == nullptr) return TKEF_EINVAL;
  int rc = check_rows(*plan, logits, row_stride, rows);
  if (rc == TKEF_OK) rc = check_ws(plan->ws_bytes, ws, ws_bytes);
  if (rc != TKEF_OK || rows == 0) return rc;
  rc = check_lists(*plan, idx, val, tail, count, weight, status);
  if (rc != TKEF_OK) return rc;
  if (loss == nullptr || !aligned(loss, 4) || !aligned(stats, 16)) return TKEF_EINVAL;
  tkef::DistillArgs a =
      distill_args(*plan, logits, row_stride, rows, idx, val, tail, count, weight, status);
  a.loss = loss;
  a.stats = reinterpret_cast<float4*>(stats);
  return done(tkef::launch_distill_forward(a, ws, stream));
}

int tkef_distill_backward(tkef_distill_plan plan, const void* logits, int64_t row_stride,
                          int64_t rows, const int32_t* idx, const void* val, const float* tail,
                          const int32_t* count, const float* weight, const float* stats,
                          const float* dloss, void* grad, int64_t grad_stride, void* /*ws*/,
                          size_t /*ws_bytes*/, uint32_t* status, hipStream_t stream) {
  if (plan == nullptr) return TKEF_EINVAL;
  int rc = check_rows(*plan, logits, row_stride, rows);
  if (rc != TKEF_OK || rows == 0) return rc;
  rc = check_lists(*plan, idx, val, tail, count, weight, status);
  if (rc == TKEF_OK) rc = check_grad(*plan, logits, row_stride, rows, grad, grad_stride);
  if (rc != TKEF_OK) return rc;
  if (stats == nullptr || !aligned(stats, 16) || !aligned(dloss, 4)) return TKEF_EINVAL;
  tkef::DistillArgs a =
      distill_args(*plan, logits, row_stride, rows, idx, val, tail, count, weight, status);
  a.stats = reinterpret_cast<float4*>(const_cast<float*>(stats));
  a.dloss = dloss;
  a.grad = grad;
  a.gld = grad_stride;
  return done(tkef::launch_distill_backward(a, stream));
}

int tkef_distill_step(tkef_distill_plan plan, const void* logits, int64_t row_stride,
                      int64_t rows, const int32_t* idx, const void* val, const float* tail,
                      const int32_t* count, const float* weight, float* loss, void* grad,
                      int64_t grad_stride, void* ws, size_t ws_bytes, uint32_t* status,
                      hipStream_t stream) {
  if (plan == nullptr) return TKEF_EINVAL;
  int rc = check_rows(*plan, logits, row_stride, rows);
  if (rc == TKEF_OK) rc = check_ws(plan->ws_bytes, ws, ws_bytes);
  if (rc != TKEF_OK || rows == 0) return rc;
  rc = check_lists(*plan, idx, val, tail, count, weight, status);
  if (rc == TKEF_OK) rc = check_grad(*plan, logits, row_stride, rows, grad, grad_stride);
  if (rc != TKEF_OK) return rc;
  if (loss == nullptr || !aligned(loss, 4)) return TKEF_EINVAL;
  tkef::DistillArgs a =
      distill_args(*plan, logits, row_stride, rows, idx, val, tail, count, weight, status);
  a.loss = loss;
  a.grad = grad;
  a.gld = grad_stride;
  return done(tkef::launch_distill_step(a, ws, stream));
}

int tkef_verify_plan_create(int64_t batch, int64_t draft, int64_t vocab, int32_t dtype,
                            double temperature, tkef_verify_plan* plan_out) {
  if (plan_out == nullptr) return TKEF_EINVAL;
  *plan_out = nullptr;
  const int rc = check_sizes(batch, vocab, dtype, temperature);
  if (rc != TKEF_OK) return rc;
  if (batch > TKEF_VERIFY_MAX_BATCH || draft < 1 || draft > TKEF_VERIFY_MAX_DRAFT ||
      !tkef::verify_fits(batch, draft, vocab, dtype))
    return TKEF_ERANGE;
  tkef_verify_plan p = new (std::nothrow) tkef_verify_plan_s;
  if (p == nullptr) return TKEF_ENOMEM;
  p->rows = batch;
  p->draft = draft;
  p->vocab = vocab;
  p->dtype = dtype;
  p->temperature = temperature;
  p->ws_bytes = tkef::verify_layout(batch, draft, vocab, dtype).bytes;
  *plan_out = p;
  return TKEF_OK;
}

int tkef_verify_plan_destroy(tkef_verify_plan plan) {
  if (plan == nullptr) return TKEF_EINVAL;
  delete plan;
  return TKEF_OK;
}

int tkef_verify_plan_info(tkef_verify_plan plan, size_t* workspace_bytes) {
  if (plan == nullptr) return TKEF_EINVAL;
  if (workspace_bytes != nullptr) *workspace_bytes = plan->ws_bytes;
  return TKEF_OK;
}

int tkef_verify_plan_bind(tkef_verify_plan plan, void* ws, size_t ws_bytes,
                          hipStream_t stream) {
  if (plan == nullptr) return TKEF_EINVAL;
  const int rc = check_ws(plan->ws_bytes, ws, ws_bytes);
  if (rc != TKEF_OK) return rc;
  const tkef::VerifyLayout l =
      tkef::verify_layout(plan->rows, plan->draft, plan->vocab, plan->dtype);
  return done(tkef::launch_fill_u32(static_cast<uint32_t*>(ws), 0u, (int64_t)(l.zeroed / 4),
                                    stream));
}

int tkef_verify_execute(tkef_verify_plan plan, const void* target, int64_t target_batch_stride,
                        int64_t target_stride, const void* drafts, int64_t draft_batch_stride,
                        int64_t draft_stride, int64_t batch, const int32_t* tokens,
                        const float* uniform, const float* noise, int64_t noise_stride,
                        const int32_t* length, int32_t* accepted, int32_t* tokens_out,
                        float* logp_out, void* ws, size_t ws_bytes, uint32_t* status,
                        hipStream_t stream) {
  if (plan == nullptr) return TKEF_EINVAL;
  int rc = check_rows(*plan, target, target_stride, batch);
  if (rc == TKEF_OK) rc = check_rows(*plan, drafts, draft_stride, batch);
  if (rc == TKEF_OK) rc = check_ws(plan->ws_bytes, ws, ws_bytes);
  if (rc != TKEF_OK || batch == 0) return rc;
  // any distance between sequences whose rows do not run into the negative
  if (target_batch_stride < 0 || draft_batch_stride < 0 || noise_stride < plan->vocab)
    return TKEF_EINVAL;
  if (target_batch_stride > kMaxStride || draft_batch_stride > kMaxStride ||
      noise_stride > kMaxStride)
    return TKEF_ERANGE;
  if (tokens == nullptr || uniform == nullptr || noise == nullptr || accepted == nullptr ||
      tokens_out == nullptr)
    return TKEF_EINVAL;
  if (!aligned(tokens, 4) || !aligned(uniform, 4) || !aligned(noise, 4) || !aligned(length, 4) ||
      !aligned(accepted, 4) || !aligned(tokens_out, 4) || !aligned(logp_out, 4) ||
      !aligned(status, 4))
    return TKEF_EINVAL;
  tkef::VerifyArgs a{};
  a.target = target;
  a.drafts = drafts;
  a.tb = target_batch_stride;
  a.ti = target_stride;
  a.db = draft_batch_stride;
  a.di = draft_stride;
  a.batch = (int32_t)batch;
  a.draft = (int32_t)plan->draft;
  a.V = (int32_t)plan->vocab;
  a.dtype = plan->dtype;
  a.a = (float)(kLog2e / plan->temperature);
  a.inv_t = (float)(1.0 / plan->temperature);
  a.tokens = tokens;
  a.uniform = uniform;
  a.noise = noise;
  a.noise_ld = noise_stride;
  a.length = length;
  a.accepted = accepted;
  a.tokens_out = tokens_out;
  a.logp = logp_out;
  a.status = status;
  const tkef::VerifyLayout l =
      tkef::verify_layout(plan->rows, plan->draft, plan->vocab, plan->dtype);
  char* base = static_cast<char*>(ws);
  tkef::VerifyScratch w;
  w.best = reinterpret_cast<uint64_t*>(base + l.best);
  w.rejected = reinterpret_cast<uint32_t*>(base + l.rejected);
  w.raced = reinterpret_cast<uint32_t*>(base + l.raced);
  w.arrived = reinterpret_cast<uint32_t*>(base + l.arrived);
  w.sums = reinterpret_cast<float4*>(base + l.sums);
  w.parts = reinterpret_cast<float2*>(base + l.parts);
  return done(tkef::launch_verify(a, w, stream));
}

}  // extern "C"

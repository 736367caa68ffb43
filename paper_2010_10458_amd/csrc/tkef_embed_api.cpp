// Host side of the embedding of tokens (include/tkef.h, "Embedding of tokens"): plans,
// argument checks, the launch of the kernels in tkef_embed.hip.
#include <math.h>

#include <new>

#include "tkef.h"
#include "tkef_embed.h"
#include "tkef_rows_host.h"

struct tkef_embed_plan_s {
  int64_t rows = 0, vocab = 0, width = 0;
  int32_t dtype = 0, out_dtype = 0, grad_dtype = 0, val_format = 0;
  float scale = 1.f;
  size_t ws_bytes = 0;
};

namespace {

bool is_dtype(int32_t t) {
  return t == TKEF_DTYPE_F32 || t == TKEF_DTYPE_F16 || t == TKEF_DTYPE_BF16;
}

// rows of the plan's width and of a type, `ld` apart
int check_block(const tkef_embed_plan_s& p, const void* x, int64_t ld, int32_t dtype) {
  if (ld > kMaxStride) return TKEF_ERANGE;
  return x == nullptr || !aligned(x, elem_size(dtype)) || ld < p.width ? TKEF_EINVAL : TKEF_OK;
}

bool apart_blocks(const tkef_embed_plan_s& p, const void* x, int64_t ld, int32_t dtype,
                  int64_t rows, const void* y, int64_t yld, int32_t ydtype, int64_t yrows) {
  const size_t e = elem_size(dtype), f = elem_size(ydtype);
  return apart(x, (size_t)p.width * e, (size_t)ld * e, rows, y, (size_t)p.width * f,
               (size_t)yld * f, yrows);
}

int check_tokens(const tkef_embed_plan_s& p, const int32_t* tokens, int64_t rows,
                 const uint32_t* status) {
  if (rows < 0 || rows > p.rows) return TKEF_ERANGE;
  return (rows > 0 && tokens == nullptr) || !aligned(tokens, 4) || !aligned(status, 4)
             ? TKEF_EINVAL
             : TKEF_OK;
}

tkef::EmbedArgs embed_args(const tkef_embed_plan_s& p, const int32_t* tokens, int64_t rows,
                           uint32_t* status) {
  tkef::EmbedArgs a{};
  a.tokens = tokens;
  a.n = rows;
  a.V = (int32_t)p.vocab;
  a.width = (int32_t)p.width;
  a.scale = p.scale;
  a.dtype = p.dtype;
  a.out_dtype = p.out_dtype;
  a.grad_dtype = p.grad_dtype;
  a.val_format = p.val_format;
  a.status = status;
  return a;
}

}  // namespace

extern "C" {

int tkef_embed_plan_create(int64_t rows, int64_t vocab, int64_t width, int32_t dtype,
                           int32_t out_dtype, int32_t grad_dtype, int32_t val_format,
                           double scale, tkef_embed_plan* plan_out) {
  if (plan_out == nullptr) return TKEF_EINVAL;
  *plan_out = nullptr;
  if (!is_dtype(dtype) || !is_dtype(out_dtype) || !is_dtype(grad_dtype) ||
      (val_format != TKEF_VAL_F32 && val_format != TKEF_VAL_F16))
    return TKEF_EINVAL;
  if (rows < 1 || rows > TKEF_EMBED_MAX_ROWS || vocab < 1 || vocab > TKEF_ROWS_MAX_VOCAB ||
      width < 1 || width > TKEF_EMBED_MAX_WIDTH || !isfinite((float)scale))
    return TKEF_ERANGE;
  tkef_embed_plan p = new (std::nothrow) tkef_embed_plan_s;
  if (p == nullptr) return TKEF_ENOMEM;
  p->rows = rows;
  p->vocab = vocab;
  p->width = width;
  p->dtype = dtype;
  p->out_dtype = out_dtype;
  p->grad_dtype = grad_dtype;
  p->val_format = val_format;
  p->scale = (float)scale;
  p->ws_bytes = tkef::embed_layout(rows, vocab, width).bytes;
  *plan_out = p;
  return TKEF_OK;
}

int tkef_embed_plan_destroy(tkef_embed_plan plan) {
  if (plan == nullptr) return TKEF_EINVAL;
  delete plan;
  return TKEF_OK;
}

int tkef_embed_plan_info(tkef_embed_plan plan, size_t* workspace_bytes) {
  if (plan == nullptr) return TKEF_EINVAL;
  if (workspace_bytes != nullptr) *workspace_bytes = plan->ws_bytes;
  return TKEF_OK;
}

int tkef_embed_forward(tkef_embed_plan plan, const void* table, int64_t table_stride,
                       const int32_t* tokens, int64_t rows, void* out, int64_t out_stride,
                       uint32_t* status, hipStream_t stream) {
  if (plan == nullptr) return TKEF_EINVAL;
  int rc = check_tokens(*plan, tokens, rows, status);
  if (rc != TKEF_OK || rows == 0) return rc;
  rc = check_block(*plan, table, table_stride, plan->dtype);
  if (rc == TKEF_OK) rc = check_block(*plan, out, out_stride, plan->out_dtype);
  if (rc != TKEF_OK) return rc;
  if (!apart_blocks(*plan, table, table_stride, plan->dtype, plan->vocab, out, out_stride,
                    plan->out_dtype, rows))
    return TKEF_EINVAL;
  tkef::EmbedArgs a = embed_args(*plan, tokens, rows, status);
  a.table = table;
  a.table_ld = table_stride;
  a.out = out;
  a.out_ld = out_stride;
  return done(tkef::launch_embed_forward(a, stream));
}

int tkef_embed_backward(tkef_embed_plan plan, const int32_t* tokens, int64_t rows,
                        const void* dout, int64_t dout_stride, const void* add,
                        int64_t add_stride, void* grad, int64_t grad_stride, void* ws,
                        size_t ws_bytes, uint32_t* status, hipStream_t stream) {
  if (plan == nullptr) return TKEF_EINVAL;
  const tkef_embed_plan_s& p = *plan;
  int rc = check_tokens(p, tokens, rows, status);
  if (rc == TKEF_OK) rc = check_ws(p.ws_bytes, ws, ws_bytes);
  if (rc == TKEF_OK && rows > 0) rc = check_block(p, dout, dout_stride, p.out_dtype);
  if (rc == TKEF_OK) rc = check_block(p, grad, grad_stride, p.grad_dtype);
  if (rc == TKEF_OK && add != nullptr) rc = check_block(p, add, add_stride, p.grad_dtype);
  if (rc != TKEF_OK) return rc;
  const bool in_place = add == grad && add_stride == grad_stride;
  if (rows > 0 && !apart_blocks(p, dout, dout_stride, p.out_dtype, rows, grad, grad_stride,
                                p.grad_dtype, p.vocab))
    return TKEF_EINVAL;
  if (add != nullptr && !in_place &&
      !apart_blocks(p, add, add_stride, p.grad_dtype, p.vocab, grad, grad_stride, p.grad_dtype,
                    p.vocab))
    return TKEF_EINVAL;
  tkef::EmbedArgs a = embed_args(p, tokens, rows, status);
  a.dout = dout;
  a.out_ld = dout_stride;
  a.add = add;
  a.add_ld = add_stride;
  a.grad = grad;
  a.grad_ld = grad_stride;
  return done(tkef::launch_embed_backward(a, ws, stream));
}

int tkef_embed_lists(tkef_embed_plan plan, const int32_t* tokens, int64_t rows, const void* dout,
                     int64_t dout_stride, int64_t offset, int32_t* idx_out, void* val_out,
                     int32_t* nnz_out, void* ws, size_t ws_bytes, uint32_t* status,
                     hipStream_t stream) {
  if (plan == nullptr) return TKEF_EINVAL;
  const tkef_embed_plan_s& p = *plan;
  int rc = check_tokens(p, tokens, rows, status);
  if (rc == TKEF_OK) rc = check_ws(p.ws_bytes, ws, ws_bytes);
  if (rc == TKEF_OK && rows > 0) rc = check_block(p, dout, dout_stride, p.out_dtype);
  if (rc != TKEF_OK) return rc;
  if (offset < 0 || offset > INT32_MAX || offset + p.vocab * p.width > INT32_MAX)
    return TKEF_ERANGE;
  if (nnz_out == nullptr || !aligned(nnz_out, 4) ||
      (rows > 0 && (idx_out == nullptr || val_out == nullptr)) || !aligned(idx_out, 4) ||
      !aligned(val_out, p.val_format == TKEF_VAL_F16 ? 2 : 4))
    return TKEF_EINVAL;
  tkef::EmbedArgs a = embed_args(p, tokens, rows, status);
  a.dout = dout;
  a.out_ld = dout_stride;
  a.offset = offset;
  a.idx = idx_out;
  a.val = val_out;
  a.nnz = nnz_out;
  return done(tkef::launch_embed_backward(a, ws, stream));
}

}  // extern "C"

// Host code that the operators on rows share: plans, argument checks.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "tkef.h"

namespace {

struct RowPlan {
  int64_t rows = 0, vocab = 0, k = 0;
  int32_t dtype = 0, val_format = 0;
  double temperature = 1.0;
  size_t ws_bytes = 0;
};

constexpr double kLog2e = 1.4426950408889634074;
constexpr int64_t kMaxStride = (int64_t)1 << 40;  // elements: byte offsets stay below 2^63

inline size_t elem_size(int32_t dtype) { return dtype == TKEF_DTYPE_F32 ? 4 : 2; }

inline bool aligned(const void* p, size_t n) {
  return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0;
}

inline int check_sizes(int64_t rows, int64_t vocab, int32_t dtype, double temperature) {
  if (dtype != TKEF_DTYPE_F32 && dtype != TKEF_DTYPE_F16 && dtype != TKEF_DTYPE_BF16)
    return TKEF_EINVAL;
  if (rows < 1 || rows > TKEF_ROWS_MAX_ROWS || vocab < 1 || vocab > TKEF_ROWS_MAX_VOCAB)
    return TKEF_ERANGE;
  if (!(temperature >= 1e-6 && temperature <= 1e6)) return TKEF_ERANGE;
  return TKEF_OK;
}

inline int check_ws(size_t need, const void* ws, size_t ws_bytes) {
  if (need == 0) return TKEF_OK;
  return ws == nullptr || ws_bytes < need || !aligned(ws, 256) ? TKEF_EWORKSPACE : TKEF_OK;
}

inline int check_rows(const RowPlan& p, const void* z, int64_t ld, int64_t rows) {
  if (rows < 0 || rows > p.rows) return TKEF_ERANGE;
  if (ld > kMaxStride) return TKEF_ERANGE;
  if (rows > 0 && (z == nullptr || !aligned(z, elem_size(p.dtype)) || ld < p.vocab))
    return TKEF_EINVAL;
  return TKEF_OK;
}

// Whether rows of `row` bytes, `step` apart, do not touch others: they lie before or
// after all of them, or between them at their step.
inline bool apart(const void* z, size_t row, size_t step, int64_t rows, const void* g, size_t grow,
                  size_t gstep, int64_t grows) {
  if (rows < 1 || grows < 1) return true;
  const uintptr_t za = reinterpret_cast<uintptr_t>(z), ga = reinterpret_cast<uintptr_t>(g);
  const uintptr_t ze = za + (size_t)(rows - 1) * step + row;
  const uintptr_t ge = ga + (size_t)(grows - 1) * gstep + grow;
  if (za >= ge || ga >= ze) return true;
  if (gstep != step) return false;
  // where a row of g begins behind the row of z before it
  const size_t at = ga >= za ? (ga - za) % step : (step - (za - ga) % step) % step;
  return at >= row && at + grow <= step;
}

// grad is the logits themselves or does not touch them
inline int check_grad(const RowPlan& p, const void* z, int64_t ld, int64_t rows, const void* g,
                      int64_t gld) {
  if (gld > kMaxStride) return TKEF_ERANGE;
  if (g == nullptr || !aligned(g, elem_size(p.dtype)) || gld < p.vocab) return TKEF_EINVAL;
  if (g == z && gld == ld) return TKEF_OK;
  const size_t e = elem_size(p.dtype), row = (size_t)p.vocab * e;
  return apart(z, row, (size_t)ld * e, rows, g, row, (size_t)gld * e, rows) ? TKEF_OK : TKEF_EINVAL;
}

inline int done(hipError_t e) { return e == hipSuccess ? TKEF_OK : TKEF_EHIP; }

}  // namespace

// Internal interface of the row operators (top logits, distillation, draft
// verification, scores of tokens): argument blocks the host fills and the gfx950
// kernels read.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

namespace tkef {

// A temperature enters the kernels as a = log2(e) / temperature and as inv_t
// (+ inv_t_lo, what its rounding leaves) = 1 / temperature.
struct TopArgs {
  const void* z;
  int64_t ld, rows;
  int32_t V, k, dtype, val_format;
  float a, inv_t;
  int32_t* idx;
  void* val;
  float* tail;     // may be null
  uint32_t* status;  // may be null
};

struct DistillArgs {
  const void* z;
  int64_t ld, rows;
  int32_t V, k, dtype, val_format;
  float a, inv_t, inv_t_lo, temperature;
  const int32_t* idx;
  const void* val;
  const float* tail;      // may be null
  const int32_t* count;   // may be null
  const float* weight;    // may be null
  float* loss;            // forward, step
  float4* stats;          // forward: out (may be null); backward: in
  const float* dloss;     // backward; may be null
  void* grad;             // backward, step
  int64_t gld;
  uint32_t* status;       // may be null
};

struct VerifyArgs {
  const void* target;
  const void* drafts;
  int64_t tb, ti, db, di;  // strides: target batch, target row, draft batch, draft row
  int32_t batch, draft, V, dtype;
  float a, inv_t;
  const int32_t* tokens;
  const float* uniform;
  const float* noise;
  int64_t noise_ld;
  const int32_t* length;  // may be null
  int32_t* accepted;
  int32_t* tokens_out;
  float* logp;            // may be null
  uint32_t* status;       // may be null
};

struct ScoreArgs {
  const void* z;
  int64_t ld, rows;
  int32_t V, k, dtype;    // k: alternatives, 0: none asked for
  float a, inv_t;
  const int32_t* tokens;
  float* logp;
  float* entropy;         // may be null
  int32_t* idx;
  float* val;
  float4* stats;          // forward: out (may be null); backward: in
  const float* dlogp;     // backward; may be null
  const float* dentropy;  // backward; may be null
  void* grad;
  int64_t gld;
  uint32_t* status;       // may be null
};

// Bytes of ws that launch_top uses (0: rows short enough for one workgroup).
size_t top_workspace(int64_t rows, int64_t V, int64_t k, int32_t dtype);
hipError_t launch_top(const TopArgs& a, void* ws, hipStream_t s);
// A row that is too long for one workgroup is taken in this many chunks (1:
// whole) for its loss, and for its loss and gradient (then never more);
// ws then holds kPartBytes for each.
constexpr size_t kPartBytes = 32;
int distill_chunks(int64_t V, int32_t dtype, int64_t rows, bool gradient);
hipError_t launch_distill_forward(const DistillArgs& a, void* ws, hipStream_t s);
hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t s);
hipError_t launch_distill_step(const DistillArgs& a, void* ws, hipStream_t s);
// Offsets into a verification's workspace. Everything below `zeroed` is zero
// between executions.
struct VerifyLayout {
  size_t best, rejected, raced, arrived, zeroed, sums, parts, bytes;
};
// Whether the grid over places and units of 32 KB stays within a launch's limits.
bool verify_fits(int64_t batch, int64_t draft, int64_t V, int32_t dtype);
VerifyLayout verify_layout(int64_t batch, int64_t draft, int64_t V, int32_t dtype);

struct VerifyScratch {
  uint64_t* best;       // per sequence: the race's best key of the residual, of the target
  uint32_t* rejected;   // per sequence: 64 - place of the first rejection, 0: none
  uint32_t* raced;      // per sequence: chunks of the race that have ended
  uint32_t* arrived;    // per sequence and place: chunks of the sums that have ended
  float4* sums;         // per sequence and place: target (m, S), draft (m, S)
  float2* parts;        // per sequence, place and chunk: the same of a chunk, as two pairs
};
hipError_t launch_verify(const VerifyArgs& a, const VerifyScratch& w, hipStream_t s);


// Bytes of ws that launch_score_forward uses for calls with up to k alternatives
// (0: rows short enough for one workgroup).
size_t score_workspace(int64_t rows, int64_t V, int64_t k, int32_t dtype);
hipError_t launch_score_forward(const ScoreArgs& a, void* ws, hipStream_t s);
hipError_t launch_score_backward(const ScoreArgs& a, hipStream_t s);

}  // namespace tkef

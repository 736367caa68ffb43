// Internal interface of the embedding of tokens and its gradient: argument
// blocks the host fills and the gfx950 kernels read.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

namespace tkef {

struct EmbedArgs {
  const int32_t* tokens;
  int64_t n;              // tokens of the call
  int32_t V, width;
  float scale;
  int32_t dtype, out_dtype, grad_dtype, val_format;
  const void* table;      // forward
  int64_t table_ld;
  void* out;              // forward
  const void* dout;       // backward, lists
  int64_t out_ld;         // of out, of dout
  const void* add;        // backward; may be null, may be grad
  int64_t add_ld;
  void* grad;             // backward
  int64_t grad_ld;
  int64_t offset;         // lists
  int32_t* idx;           // (null where a list has no tokens)
  void* val;
  int32_t* nnz;
  uint32_t* status;       // may be null
};

// Offsets into the workspace of a gradient, for up to `rows` tokens.
struct EmbedLayout {
  size_t sorted, slots, first, bins, before, partial, part, ends, bytes;
};
EmbedLayout embed_layout(int64_t rows, int64_t V, int64_t width);

hipError_t launch_embed_forward(const EmbedArgs& a, hipStream_t s);
// the table's gradient, or (a.nnz not null) its lists
hipError_t launch_embed_backward(const EmbedArgs& a, void* ws, hipStream_t s);

}  // namespace tkef

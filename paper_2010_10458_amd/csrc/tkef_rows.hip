// gfx950 kernels for rows of logits over a vocabulary: a teacher's top logits,
// distillation on them (loss and gradient), verification of drafted tokens.
//
// All exponentials are taken in base 2: exp(s x) = 2^(x a) with a = log2(e) / temperature.
// A sum of exponentials is held as a pair (m, S), meaning S * 2^(m a), with m
// its largest logit: each term is 2^((x - m) a). The difference is taken
// before the product, so logits at the lowest value of their type (a common
// mask) neither overflow nor lose their order.
#include <hip/hip_runtime.h>

#include "tkef.h"
#include "tkef_rows.h"

#pragma clang fp contract(off)

namespace tkef {

namespace {

constexpr float kInf = __builtin_huge_valf();
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLog2e = 1.4426950408889634074f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }

// 2^((m - top) a) for two maxima, 0 for an empty sum (m = -inf, also below top = -inf)
__device__ __forceinline__ float rescale(float m, float top, float a) {
  return m == -kInf ? 0.f : exp2_((m - top) * a);
}

template <typename T>
__device__ __forceinline__ float load1(const T* p, int64_t i) {
  return (float)p[i];
}

// value j of a list in the wire format (binary32 or binary16)
__device__ __forceinline__ float load_val(const void* p, int format, int64_t j) {
  return format == TKEF_VAL_F16 ? (float)static_cast<const _Float16*>(p)[j]
                                : static_cast<const float*>(p)[j];
}

// unsigned key whose order is the order of x: -0 equals +0; a NaN lies beyond
// the infinity of its sign
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x);
  if (b == 0x80000000u) return 0x80000000u;
  return (b >> 31) ? ~b : (b | 0x80000000u);
}

__device__ __forceinline__ float key_value(uint32_t key) {
  return __uint_as_float((key >> 31) ? (key & 0x7FFFFFFFu) : ~key);
}

// Reductions over the NT threads of a workgroup; every thread gets the result.
// red: NT / 64 floats of LDS; the first barrier lets it be reused from call to call.
template <int NT, typename F>
__device__ __forceinline__ float block_reduce(float x, float* red, F op) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x = op(x, __shfl_xor(x, d));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  float r = red[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) r = op(r, red[i]);
  return r;
}

// larger of two values; a NaN wins
struct MaxOp {
  __device__ float operator()(float a, float b) const {
    return (a > b || a != a) ? a : b;
  }
};
struct AddOp {
  __device__ float operator()(float a, float b) const { return a + b; }
};

__device__ __forceinline__ uint32_t wave_incl(uint32_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// Exclusive prefix over the workgroup; *total gets the sum. Two barriers.
template <int NT>
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* red, uint32_t* total) {
  const uint32_t inc = wave_incl(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) red[threadIdx.x >> 6] = inc;
  __syncthreads();
  uint32_t base = 0u, all = 0u;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) {
    const uint32_t t = red[i];
    base += i < (int)(threadIdx.x >> 6) ? t : 0u;
    all += t;
  }
  *total = all;
  return base + inc - x;
}

__device__ __forceinline__ void raise_status(uint32_t* status, uint32_t bits) {
  if (status != nullptr && bits != 0u) atomicOr(status, bits);
}

constexpr int kNT = 256;

// ----------------------------------------------------------------------------
// top logits, one workgroup per row: radix select of the k-th largest order
// key over four 8-bit digits, then the ordered compaction and the rest's sum.
// Takes any row; reads it seven times.
template <typename T>
__global__ __launch_bounds__(kNT) void k_top_radix(TopArgs A) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t red[kNT / 64];
  __shared__ float fred[kNT / 64];
  __shared__ uint32_t pick[2];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* p = static_cast<const T*>(A.z) + row * A.ld;
  const int V = A.V;
  uint32_t prefix = 0u, need = (uint32_t)A.k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    hist[tid] = 0u;
    __syncthreads();
    for (int i = tid; i < V; i += kNT) {
      const uint32_t key = order_key(load1(p, i));
      if (shift == 24 || (key >> (shift + 8)) == prefix)
        atomicAdd(&hist[(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    // digit 255 - tid: the exclusive prefix counts the keys in higher digits
    const uint32_t mine = hist[255 - tid];
    uint32_t total;
    const uint32_t above = block_scan<kNT>(mine, red, &total);
    if (above < need && need <= above + mine) {
      pick[0] = 255u - (uint32_t)tid;
      pick[1] = need - above;
    }
    __syncthreads();
    prefix = (prefix << 8) | pick[0];
    need = pick[1];
  }
  // the k-th key, and how many of its class are taken (the lowest words)
  const uint32_t kth = prefix, quota = need;
  uint32_t done_gt = 0u, done_eq = 0u;
  float top = -kInf;
  bool nan = false;
  for (int base = 0; base < V; base += kNT) {
    const int i = base + tid;
    const float x = i < V ? load1(p, i) : 0.f;
    const uint32_t key = i < V ? order_key(x) : 0u;
    const bool gt = i < V && key > kth, eq = i < V && key == kth;
    uint32_t tot_gt, tot_eq;
    const uint32_t r_gt = done_gt + block_scan<kNT>(gt, red, &tot_gt);
    const uint32_t r_eq = done_eq + block_scan<kNT>(eq, red, &tot_eq);
    const bool take = gt || (eq && r_eq < quota);
    if (take) {
      const int64_t o = row * A.k + r_gt + (r_eq < quota ? r_eq : quota);
      A.idx[o] = i;
      if (A.val_format == TKEF_VAL_F16)
        static_cast<_Float16*>(A.val)[o] = (_Float16)x;
      else
        static_cast<float*>(A.val)[o] = x;
    } else if (i < V) {
      top = x > top ? x : top;
    }
    nan |= i < V && x != x;
    done_gt += tot_gt;
    done_eq += tot_eq;
  }
  nan = __syncthreads_or(nan);
  if (nan && tid == 0) raise_status(A.status, TKEF_STATUS_NAN);
  if (A.tail == nullptr) return;
  top = block_reduce<kNT>(top, fred, MaxOp());
  const float m = top == -kInf ? 0.f : top;
  float sum = 0.f;
  for (int i = tid; i < V; i += kNT) {
    const float x = load1(p, i);
    if (order_key(x) < kth) sum += exp2_((x - m) * A.a);
  }
  sum = block_reduce<kNT>(sum, fred, AddOp());
  if (tid == 0) {
    // the class of the k-th key that was not taken
    const float tie = key_value(kth);
    if (done_eq > quota && tie > -kInf)
      sum += (float)(done_eq - quota) * exp2_((tie - m) * A.a);
    const float tail = top == kInf ? kInf : sum > 0.f ? m * A.inv_t + kLn2 * log2_(sum) : -kInf;
    A.tail[row] = nan ? __uint_as_float(0x7FC00000u) : tail;
  }
}

// ----------------------------------------------------------------------------
// distillation

// a sum of exponentials S * 2^(m a)
struct LogSum {
  float m = -kInf, S = 0.f;
  __device__ void add(float x, float a) {
    if (x == -kInf) return;
    if (x > m || x != x) {
      S = S * rescale(m, x, a) + exp2_((x - x) * a);  // (1, or NaN)
      m = x;
    } else {
      S += exp2_((x - m) * a);
    }
  }
};

template <int NT>
__device__ __forceinline__ LogSum block_join(LogSum v, float a, float* red) {
  LogSum r;
  r.m = block_reduce<NT>(v.m, red, MaxOp());
  r.S = block_reduce<NT>(v.S * rescale(v.m, r.m, a), red, AddOp());
  return r;
}

// log2 of (2^(tau log2 e) / 2^(m a)), with 1 / temperature in two parts so
// that the product's rounding does not enter
__device__ __forceinline__ float tail_over(float tau, float m, float inv_t, float inv_t_lo) {
  return (__builtin_fmaf(-m, inv_t, tau) - m * inv_t_lo) * kLog2e;
}

// The teacher's side of a row: the list's sum, with the tail's mass.
struct Teacher {
  float m, S, inv;  // p_j = 2^((t - m) a) * inv, inv = 1 / S
  float tau, p_rest;
};

__device__ __forceinline__ Teacher teacher_of(LogSum list, const DistillArgs& A, int64_t row) {
  Teacher t;
  t.tau = A.tail != nullptr ? A.tail[row] : -kInf;
  const float tail_m = t.tau * A.temperature;
  t.m = list.m > tail_m ? list.m : tail_m;
  const float rest =
      t.tau == -kInf ? 0.f : exp2_(tail_over(t.tau, t.m, A.inv_t, A.inv_t_lo));
  t.S = list.S * rescale(list.m, t.m, A.a) + rest;
  t.inv = 1.f / t.S;
  t.p_rest = rest * t.inv;
  return t;
}

// false for a list without mass, or with infinite or NaN logits
__device__ __forceinline__ bool has_mass(const Teacher& t) { return t.S > 0.f && t.S < kInf; }

// p_j of a listed logit v
__device__ __forceinline__ float teacher_prob(float v, float a, const Teacher& t) {
  return exp2_((v - t.m) * a) * t.inv;
}

// Whether entry j of a row's list counts: inside [0, V) and above the entry before it.
__device__ __forceinline__ bool entry_ok(const int32_t* idx, int j, int V, uint32_t* bits) {
  const int32_t i = idx[j];
  if (i < 0 || i >= V) {
    *bits |= TKEF_STATUS_INDEX_RANGE;
    return false;
  }
  if (j > 0 && idx[j - 1] >= i) {
    *bits |= TKEF_STATUS_UNSORTED;
    return false;
  }
  return true;
}

constexpr int kTileWords = 1024;                // LDS bitmap of listed words
constexpr int kTileElems = kTileWords * 32;

// loss and the student's sums, one workgroup per row, reading it in tiles
template <typename T>
__global__ __launch_bounds__(kNT) void k_distill_loss(DistillArgs A) {
  __shared__ uint32_t listed[kTileWords];
  __shared__ float red[kNT / 64];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* p = static_cast<const T*>(A.z) + row * A.ld;
  const int32_t* idx = A.idx + row * A.k;
  int cnt = A.k;
  if (A.count != nullptr) cnt = A.count[row] < 0 ? 0 : A.count[row] < A.k ? A.count[row] : A.k;
  const float w = A.weight != nullptr ? A.weight[row] : 1.f;
  if (cnt == 0 || w == 0.f) {
    if (tid == 0) {
      if (A.loss != nullptr) A.loss[row] = 0.f;
      if (A.stats != nullptr) A.stats[row] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    return;
  }
  uint32_t bits = 0u;
  LogSum teach, zl;
  for (int j = tid; j < cnt; j += kNT) {
    if (!entry_ok(idx, j, A.V, &bits)) continue;
    const float t = load_val(A.val, A.val_format, row * A.k + j);
    teach.add(t, A.a);
    zl.add(load1(p, idx[j]), A.a);
  }
  raise_status(A.status, bits);
  teach = block_join<kNT>(teach, A.a, red);
  zl = block_join<kNT>(zl, A.a, red);
  LogSum rest;
  for (int base = 0; base < A.V; base += kTileElems) {
    for (int i = tid; i < kTileWords; i += kNT) listed[i] = 0u;
    __syncthreads();
    for (int j = tid; j < cnt; j += kNT) {
      uint32_t ignore = 0u;
      const int32_t i = idx[j] - base;
      if (entry_ok(idx, j, A.V, &ignore) && i >= 0 && i < kTileElems)
        atomicOr(&listed[i >> 5], 1u << (i & 31));
    }
    __syncthreads();
    const int end = A.V - base < kTileElems ? A.V - base : kTileElems;
    for (int i = tid; i < end; i += kNT)
      if (!((listed[i >> 5] >> (i & 31)) & 1u)) rest.add(load1(p, base + i), A.a);
    __syncthreads();
  }
  rest = block_join<kNT>(rest, A.a, red);
  const Teacher t = teacher_of(teach, A, row);
  LogSum all;
  all.m = rest.m > zl.m ? rest.m : zl.m;
  all.S = rest.S * rescale(rest.m, all.m, A.a) + zl.S * rescale(zl.m, all.m, A.a);
  // sum_j p_j (log p_j - log q_j) = sum_j p_j s (t_j - z_j) + (LZ - LT) sum_j p_j
  float cross = 0.f;
  for (int j = tid; j < cnt; j += kNT) {
    uint32_t ignore = 0u;
    if (!entry_ok(idx, j, A.V, &ignore)) continue;
    const float v = load_val(A.val, A.val_format, row * A.k + j);
    const float pj = teacher_prob(v, A.a, t);
    if (pj > 0.f) cross += pj * ((v - load1(p, idx[j])) * A.a);
  }
  cross = block_reduce<kNT>(cross, red, AddOp());
  if (tid == 0) {
    float loss = cross + ((all.m - t.m) * A.a + (log2_(all.S) - log2_(t.S)));
    if (t.p_rest > 0.f)
      loss += rest.S == 0.f
                  ? kInf
                  : t.p_rest * (tail_over(t.tau, rest.m, A.inv_t, A.inv_t_lo) - log2_(rest.S));
    if (!(all.S > 0.f) || !has_mass(t)) loss = __uint_as_float(0x7FC00000u);
    if (A.loss != nullptr) A.loss[row] = loss * (kLn2 * w) * (A.temperature * A.temperature);
    if (A.stats != nullptr) A.stats[row] = make_float4(rest.m, rest.S, zl.m, zl.S);
  }
}

// gradient from the student's sums, one workgroup per row
template <typename T>
__global__ __launch_bounds__(kNT) void k_distill_grad(DistillArgs A) {
  __shared__ float red[kNT / 64];
  __shared__ float patch[TKEF_ROWS_MAX_K];  // gradients of the listed words
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* p = static_cast<const T*>(A.z) + row * A.ld;
  T* g = static_cast<T*>(A.grad) + row * A.gld;
  const int32_t* idx = A.idx + row * A.k;
  int cnt = A.k;
  if (A.count != nullptr) cnt = A.count[row] < 0 ? 0 : A.count[row] < A.k ? A.count[row] : A.k;
  const float w = A.weight != nullptr ? A.weight[row] : 1.f;
  if (cnt == 0 || w == 0.f) {
    for (int i = tid; i < A.V; i += kNT) g[i] = (T)0.f;
    return;
  }
  uint32_t bits = 0u;
  LogSum teach;
  for (int j = tid; j < cnt; j += kNT) {
    if (!entry_ok(idx, j, A.V, &bits)) continue;
    const float t = load_val(A.val, A.val_format, row * A.k + j);
    teach.add(t, A.a);
  }
  raise_status(A.status, bits);
  teach = block_join<kNT>(teach, A.a, red);
  const Teacher t = teacher_of(teach, A, row);
  const float4 st = A.stats[row];  // rest (m, S), listed (m, S)
  const float top = st.x > st.z ? st.x : st.z;
  const float s_rest = rescale(st.x, top, A.a), s_list = rescale(st.z, top, A.a);
  const float total = st.y * s_rest + st.w * s_list;
  const float inv = 1.f / total;
  const float up = w * A.temperature * (A.dloss != nullptr ? A.dloss[row] : 1.f);
  // q_i (1 - p_r / q_r) = 2^((x - m) a) (s_rest / total - p_r / S)
  float coef = s_rest * inv - (t.p_rest > 0.f && st.y > 0.f ? t.p_rest / st.y : 0.f);
  coef *= up;
  if (!(total > 0.f) || !has_mass(t)) coef = __uint_as_float(0x7FC00000u);
  for (int j = tid; j < cnt; j += kNT) {
    uint32_t ignore = 0u;
    if (!entry_ok(idx, j, A.V, &ignore)) continue;
    const float v = load_val(A.val, A.val_format, row * A.k + j);
    const float pj = teacher_prob(v, A.a, t);
    const float z = load1(p, idx[j]);
    const float q = z == -kInf ? 0.f * inv : exp2_((z - st.z) * A.a) * (s_list * inv);
    patch[j] = up * (q - pj);
  }
  __syncthreads();
  const float m = st.x == -kInf ? 0.f : st.x;
  for (int i = tid; i < A.V; i += kNT)
    g[i] = (T)(exp2_((load1(p, i) - m) * A.a) * coef);
  __syncthreads();
  for (int j = tid; j < cnt; j += kNT) {
    uint32_t ignore = 0u;
    if (entry_ok(idx, j, A.V, &ignore)) g[idx[j]] = (T)patch[j];
  }
}

// ----------------------------------------------------------------------------
// verification, one workgroup per sequence, row by row

struct Best {
  float score = 0.f;
  int word = -1;
  __device__ void offer(float s, int w) {
    if (s > score || (s == score && s > 0.f && w < word)) {
      score = s;
      word = w;
    }
  }
};

template <int NT>
__device__ __forceinline__ Best block_best(Best v, uint64_t* red) {
  // larger score first, then the lower word
  uint64_t key = v.word < 0 ? 0ull
                            : ((uint64_t)__float_as_uint(v.score) << 32) | (0xFFFFFFFFu - v.word);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)key, d);
    key = o > key ? o : key;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = key;
  __syncthreads();
  for (int i = 0; i < NT / 64; ++i) key = red[i] > key ? red[i] : key;
  Best r;
  if (key != 0ull) {
    r.score = __uint_as_float((uint32_t)(key >> 32));
    r.word = (int)(0xFFFFFFFFu - (uint32_t)key);
  }
  return r;
}

// probability of logit x in a row whose sum is v
__device__ __forceinline__ float prob(float x, float a, LogSum v) {
  if (v.m == -kInf) return 0.f;  // (an empty row)
  return exp2_((x - v.m) * a) / v.S;
}

template <typename T>
__global__ __launch_bounds__(kNT) void k_verify_rows(VerifyArgs A) {
  __shared__ float red[kNT / 64];
  __shared__ uint64_t red64[kNT / 64];
  const int tid = threadIdx.x;
  const int64_t b = blockIdx.x;
  const T* target = static_cast<const T*>(A.target) + b * A.tb;
  const T* drafts = static_cast<const T*>(A.drafts) + b * A.db;
  int len = A.draft;
  if (A.length != nullptr)
    len = A.length[b] < 0 ? 0 : A.length[b] < A.draft ? A.length[b] : A.draft;
  int32_t* out = A.tokens_out + b * (A.draft + 1);
  float* logp = A.logp != nullptr ? A.logp + b * (A.draft + 1) : nullptr;
  LogSum pt, qt;
  const T *tp = target, *dp = nullptr;
  int n = 0;
  for (;; ++n) {
    tp = target + n * A.ti;
    dp = n < len ? drafts + n * A.di : nullptr;
    pt = LogSum();
    qt = LogSum();
    for (int i = tid; i < A.V; i += kNT) {
      pt.add(load1(tp, i), A.a);
      if (dp != nullptr) qt.add(load1(dp, i), A.a);
    }
    pt = block_join<kNT>(pt, A.a, red);
    qt = block_join<kNT>(qt, A.a, red);
    if (n == len) break;
    const int x = A.tokens[b * A.draft + n];
    if (x < 0 || x >= A.V) {
      if (tid == 0) raise_status(A.status, TKEF_STATUS_INDEX_RANGE);
      break;
    }
    const float zt = load1(tp, x);
    if (!(A.uniform[b * A.draft + n] * prob(load1(dp, x), A.a, qt) < prob(zt, A.a, pt))) break;
    if (tid == 0) {
      out[n] = x;
      if (logp != nullptr)
        logp[n] = (zt - pt.m) * A.inv_t - kLn2 * log2_(pt.S);
    }
  }
  Best over, plain;
  const float* noise = A.noise + b * A.noise_ld;
  for (int i = tid; i < A.V; i += kNT) {
    const float pi = prob(load1(tp, i), A.a, pt), e = noise[i];
    const float r = dp != nullptr ? pi - prob(load1(dp, i), A.a, qt) : pi;
    if (r > 0.f) over.offer(r / e, i);
    if (pi > 0.f) plain.offer(pi / e, i);
  }
  over = block_best<kNT>(over, red64);
  plain = block_best<kNT>(plain, red64);
  const int word = over.word >= 0 ? over.word : plain.word;
  if (tid == 0) {
    if (pt.S != pt.S || qt.S != qt.S) raise_status(A.status, TKEF_STATUS_NAN);
    A.accepted[b] = n;
    out[n] = word;
    if (logp != nullptr)
      logp[n] = word < 0 ? 0.f
                         : (load1(tp, word) - pt.m) * A.inv_t - kLn2 * log2_(pt.S);
  }
  for (int i = n + 1 + tid; i <= A.draft; i += kNT) {
    out[i] = -1;
    if (logp != nullptr) logp[i] = 0.f;
  }
}

// f(T*) for the logits' type
template <typename F>
hipError_t by_dtype(int32_t dtype, F f) {
  switch (dtype) {
    case TKEF_DTYPE_F32: f(static_cast<float*>(nullptr)); break;
    case TKEF_DTYPE_F16: f(static_cast<_Float16*>(nullptr)); break;
    default: f(static_cast<__bf16*>(nullptr)); break;
  }
  return hipGetLastError();
}

template <typename P>
struct Pointee;
template <typename T>
struct Pointee<T*> {
  using type = T;
};

}  // namespace

hipError_t launch_top(const TopArgs& a, hipStream_t s) {
  return by_dtype(a.dtype, [&](auto* t) {
    using T = typename Pointee<decltype(t)>::type;
    k_top_radix<T><<<dim3((unsigned)a.rows), dim3(kNT), 0, s>>>(a);
  });
}

hipError_t launch_distill_forward(const DistillArgs& a, hipStream_t s) {
  return by_dtype(a.dtype, [&](auto* t) {
    using T = typename Pointee<decltype(t)>::type;
    k_distill_loss<T><<<dim3((unsigned)a.rows), dim3(kNT), 0, s>>>(a);
  });
}

hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t s) {
  return by_dtype(a.dtype, [&](auto* t) {
    using T = typename Pointee<decltype(t)>::type;
    k_distill_grad<T><<<dim3((unsigned)a.rows), dim3(kNT), 0, s>>>(a);
  });
}

hipError_t launch_distill_step(const DistillArgs& a, hipStream_t s) {
  const hipError_t e = launch_distill_forward(a, s);
  return e != hipSuccess ? e : launch_distill_backward(a, s);
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t s) {
  return by_dtype(a.dtype, [&](auto* t) {
    using T = typename Pointee<decltype(t)>::type;
    k_verify_rows<T><<<dim3((unsigned)a.batch), dim3(kNT), 0, s>>>(a);
  });
}

}  // namespace tkef

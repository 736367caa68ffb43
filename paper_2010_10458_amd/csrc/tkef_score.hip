// gfx950 kernels for scores of given tokens: log-probability, the row's entropy,
// its greatest words in descending order, and the gradient of the first two.
// Exponentials, sums and vectors of rows: tkef_rows_device.h.
#include <type_traits>

#include <hip/hip_runtime.h>

#include "tkef.h"
#include "tkef_rows.h"
#include "tkef_rows_device.h"

#pragma clang fp contract(off)

namespace tkef {

namespace {

constexpr uint32_t kNaNBits = 0x7FC00000u;

// What a part of a row (a thread's share, a wave's, a chunk's) adds to its sums,
// with y = (x - m) a the exponent of a word from the part's maximum m:
//   S = sum 2^y,  T = sum 2^y y
// Of a whole row: log p of a logit x = (x - m) / temperature - ln S, and the entropy
//   H = -sum p log p = ln 2 (log2 S - T / S),
// both terms of which are positive: nothing cancels.
struct ScorePart {
  float m, S, T, pad;
};

// A word without probability has a term of 0 whatever its exponent; -1000 in place of -inf
// keeps the product finite.
constexpr float kFar = -1000.f;
__device__ __forceinline__ float near(float y) { return fmaxf(y, kFar); }

__device__ __forceinline__ void move_to(ScorePart& p, float top, float a) {
  const float f = rescale(p.m, top, a);
  p.T = f * (p.T + (p.S != 0.f && p.m != top ? p.S * near((p.m - top) * a) : 0.f));
  p.S *= f;
  p.m = top;
}

__device__ __forceinline__ ScorePart wave_join(ScorePart p, float a) {
  move_to(p, wave_max(p.m), a);
  p.S = wave_sum(p.S);
  p.T = wave_sum(p.T);
  return p;
}

struct RowScore {
  float m, log_sum, entropy, S;
  bool valid;  // false: NaN, +inf, or nothing but -inf
};

__device__ __forceinline__ RowScore row_score(const ScorePart& p) {
  RowScore r;
  r.m = p.m;
  r.S = p.S;
  r.valid = p.S > 0.f && p.S < kInf;
  const float log2_s = log2_(p.S);
  r.log_sum = kLn2 * log2_s;
  r.entropy = kLn2 * (log2_s - p.T / p.S);
  return r;
}

// (a difference beyond the largest binary32 number, which a temperature may bring back, is
// taken in halves)
__device__ __forceinline__ float log_prob(float x, const RowScore& r, float inv_t) {
  const float d = x - r.m;
  const float z = d == -kInf ? (0.5f * x - 0.5f * r.m) * (2.f * inv_t) : d * inv_t;
  return z - r.log_sum;
}

// one row's results but the alternatives, by one thread
__device__ __forceinline__ void put_score(const ScoreArgs& A, int64_t row, int32_t token,
                                          const RowScore& r) {
  const float nan = __uint_as_float(kNaNBits);
  const float x = load1_of(A.z, A.dtype, row * A.ld + token);
  A.logp[row] = r.valid ? log_prob(x, r, A.inv_t) : nan;
  if (A.entropy != nullptr) A.entropy[row] = r.valid ? r.entropy : nan;
  if (A.stats != nullptr)
    A.stats[row] = make_float4(r.m, r.valid ? r.S : nan, r.valid ? r.entropy : nan, 0.f);
  if (!r.valid) raise_status(A.status, TKEF_STATUS_NAN);
}

// A row without a token, by threads tid, tid + step ...
__device__ __forceinline__ void put_none(const ScoreArgs& A, int64_t row, int32_t token, int tid,
                                         int step) {
  if (tid == 0) {
    A.logp[row] = 0.f;
    if (A.entropy != nullptr) A.entropy[row] = 0.f;
    if (A.stats != nullptr) A.stats[row] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (token != -1) raise_status(A.status, TKEF_STATUS_INDEX_RANGE);
  }
  for (int j = tid; j < A.k; j += step) {
    A.idx[row * A.k + j] = -1;
    A.val[row * A.k + j] = 0.f;
  }
}

// alternative j of a row
template <typename T>
__device__ __forceinline__ void put_alternative(const ScoreArgs& A, int64_t row, int j, uint64_t c,
                                                const RowScore& r) {
  A.idx[row * A.k + j] = r.valid ? word_of(c) : -1;
  A.val[row * A.k + j] = r.valid ? log_prob(value_of<T>(c), r, A.inv_t) : __uint_as_float(kNaNBits);
}

// A thread's words of a row's chunk: vectors v0 + i * TPB + tid, and an extra
template <typename T, int TPB, int NV>
struct Share {
  const Span<T>& s;
  int v0, tid;
  bool has_ex;
  float ex;
  // the greatest candidate below a limit, 0: none
  __device__ uint64_t best_below(uint64_t limit) const {
    constexpr int N = Span<T>::N;
    const T* type = nullptr;
    uint64_t best = 0ull;
    const auto look = [&](float x, int32_t word) {
      const uint64_t c = candidate<T>(order_key(x), word);
      best = c < limit && c > best ? c : best;
    };
    if (has_ex) look(ex, s.extra(tid));
    for (int i = 0; i < NV; ++i) {
      const int v = v0 + i * TPB + tid;
      if (v >= s.nvec) break;
      float x[N];
      unpack(load16<false>(s.vec(v)), x, type);
#pragma unroll
      for (int n = 0; n < N; ++n) look(x[n], s.head + v * N + n);
    }
    return best;
  }
};

// The k first words of a workgroup's share in descending order, zeros behind
// them where there are fewer: the greatest of the threads' best candidates, k times.
template <typename T, int TPB, int NV>
__device__ __forceinline__ void extract(const Share<T, TPB, NV>& mine, int k, uint64_t* picked,
                                        uint64_t (*top)[TPB / 64]) {
  constexpr int NW = TPB / 64;
  const int tid = threadIdx.x;
  uint64_t best = mine.best_below(~0ull);
  for (int j = 0; j < k; ++j) {
    uint64_t c = wave_max64(best);
    if ((tid & 63) == 0) top[j & 1][tid >> 6] = c;
    __syncthreads();
    c = 0ull;
#pragma unroll
    for (int w = 0; w < NW; ++w) c = top[j & 1][w] > c ? top[j & 1][w] : c;
    if (tid == 0) picked[j] = c;
    if (best == c && c != 0ull) best = mine.best_below(c);
  }
}

// LDS of a selection. kVecs vectors of 16 bytes, kCand candidates: the words of a row with
// fewer than TKEF_SCORE_MAX_K vectors fit (63 of eight, and 14 extras).
constexpr int kVecs = 192, kCand = 576;
struct SelectLds {
  alignas(16) uint4 vec[kVecs];
  alignas(16) uint64_t cand[kCand + 8];
  int32_t word[kVecs];
  uint32_t group[256];
  uint32_t bound, vecs, count, scan[4];
  uint64_t top[2][4];
};

struct Nothing {};
template <bool ALT>
using Maybe = std::conditional_t<ALT, SelectLds, Nothing>;

// The k first words of a workgroup's share, which its threads hold in registers (r: vectors v0
// + i * 256 + tid; m: their greatest), in descending order, zeros behind them where there are
// fewer.
//   1. The k-th greatest of the threads' own greatest words, bisected on order keys by one wave,
//      is at most the k-th greatest word, and few others reach it (of 32,000 words, k = 20:
//      some 21).
//   2. Vectors that have a word which does go to LDS, and their words that do become candidates.
//   3. A candidate's place is the number of better ones.
// Where more reach the bound than LDS holds, they mostly do so by ties (rows with fewer
// unmasked words than k, constant rows): the words above it are the candidates then, and the
// lowest at it fill up. Where even those are too many (the greatest words in few threads'
// shares), they are taken one after the other.
template <typename T, int NV>
__device__ __forceinline__ void select(uint4 (&r)[NV], float m, const Share<T, 256, NV>& mine, int k,
                                       uint64_t* picked, SelectLds& L) {
  constexpr int N = Span<T>::N, TPB = 256;
  const int tid = threadIdx.x, lane = tid & 63;
  const T* type = nullptr;
  const Span<T>& s = mine.s;
  L.group[tid] = order_key(m);
  if (tid < k) picked[tid] = 0ull;
  if (tid == 0) L.vecs = L.count = 0u;
  __syncthreads();
  if (tid < 64) {
    uint32_t g[4], lo = 0xFFFFFFFFu, hi = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      g[i] = L.group[i * 64 + lane];
      lo = g[i] < lo ? g[i] : lo;
      hi = g[i] > hi ? g[i] : hi;
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      const uint32_t a = __shfl_xor(lo, d), b = __shfl_xor(hi, d);
      lo = a < lo ? a : lo;
      hi = b > hi ? b : hi;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi) + 1u;
    // at least k keys are >= lo, fewer than k are >= hi
    const uint32_t least = 1u << key_shift(type), enough = (uint32_t)k + ((uint32_t)k >> 3) + 1u;
    while (hi - lo > least) {
      const uint32_t mid = lo + (hi - lo) / 2u;
      uint32_t c = 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) c += (uint32_t)__popcll(__ballot(g[i] >= mid));
      if (c >= (uint32_t)k) {
        lo = mid;
        if (c <= enough) break;
      } else {
        hi = mid;
      }
    }
    // the least key at or above lo that a value of the type has: ties lie at the bound
    lo = (lo >> 31) ? (lo + least - 1u) & ~(least - 1u) : lo | (least - 1u);
    if (lane == 0) L.bound = lo;
  }
  __syncthreads();
  const float bound = key_value(L.bound);
  // words that reach the bound, or lie above it
  const auto collect = [&](bool strict) {
    const auto reaches = [&](float x) { return strict ? x > bound : x >= bound; };
    const auto put = [&](float x, int32_t word) {
      const uint32_t at = atomicAdd(&L.count, 1u);
      if (at < (uint32_t)kCand) L.cand[at] = candidate<T>(order_key(x), word);
    };
    const int tid2 = renew(tid);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = mine.v0 + i * TPB + tid2;
      renew(r[i]);
      const bool above = reaches(max_packed(-kInf, r[i], type)) && v < s.nvec;
      const uint64_t who = __ballot(above);
      if (who == 0ull) continue;
      uint32_t at = 0u;
      if (lane == 0) at = atomicAdd(&L.vecs, (uint32_t)__popcll(who));
      at = __builtin_amdgcn_readfirstlane(at) +
           __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32),
                                     __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
      if (above && at < (uint32_t)kVecs) {
        L.vec[at] = r[i];
        L.word[at] = s.head + v * N;
      }
    }
    if (mine.has_ex && reaches(mine.ex)) put(mine.ex, s.extra(tid));
    __syncthreads();
    const uint32_t vecs = L.vecs;
    if (vecs <= (uint32_t)kVecs)
      for (int e = tid; e < (int)vecs * N; e += TPB) {
        const float x = (float)reinterpret_cast<const T*>(&L.vec[e / N])[e % N];
        if (reaches(x)) put(x, L.word[e / N] + e % N);
      }
    __syncthreads();
    return vecs <= (uint32_t)kVecs && L.count <= (uint32_t)kCand ? (int)L.count : -1;
  };
  int C = collect(false);
  if (C < 0) {  // (the same for the whole workgroup, as all that is decided here)
    __syncthreads();
    if (tid == 0) L.vecs = L.count = 0u;
    __syncthreads();
    C = collect(true);
    if (C < 0) {
      extract<T, TPB, NV>(mine, k, picked, L.top);
      return;
    }
    // the lowest words at the bound, in rounds over the share in ascending order
    const int wanted = C < k ? k - C : 0;
    int done = 0;
    const auto round = [&](bool valid, int32_t word) {
      const bool tie = valid && load1(s.p, word) == bound;
      uint32_t total;
      const int at = done + (int)block_scan<TPB>(tie ? 1u : 0u, L.scan, &total);
      if (tie && at < wanted) L.cand[C + at] = candidate<T>(L.bound, word);
      done += (int)total;
    };
    const bool edges = mine.v0 == 0;
    const int end = s.nvec - mine.v0 < TPB * NV ? s.nvec - mine.v0 : TPB * NV;
    const int32_t first = s.head + mine.v0 * N, behind = s.head + s.nvec * N;
    if (edges && wanted > 0) round(tid < s.head, tid);
    for (int i = 0; i < end * N && done < wanted; i += TPB) round(i + tid < end * N, first + i + tid);
    if (edges && done < wanted) round(behind + tid < (int)(s.extras - s.head) + behind, behind + tid);
    C += done < wanted ? done : wanted;
  }
  if (tid < 8) L.cand[C + tid] = 0ull;
  __syncthreads();
  for (int q = tid; q < C; q += TPB) {
    const uint64_t c = L.cand[q];
    int rank = 0;
    for (int j = 0; j < C; j += 8) {  // (zeros follow; all reads before the first use)
      ulonglong2 o[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) o[u] = *reinterpret_cast<const ulonglong2*>(&L.cand[j + 2 * u]);
#pragma unroll
      for (int u = 0; u < 4; ++u) rank += (o[u].x > c ? 1 : 0) + (o[u].y > c ? 1 : 0);
    }
    if (rank < k) picked[rank] = c;
  }
}

// One workgroup takes a row, or one of a row's chunks (PART, blockIdx.y), and holds it
// in registers: NV vectors a thread, loaded once. Reads bound it: 8,192 x 32,000 bfloat16 (an eighth
// without a token) in 73 us, 6.3 TB/s; 509 x 131,071 binary32 in chunks in 43 us, 6.2 TB/s. With
// alternatives, 2,048 x 131,071 binary16 and k = 5 in 92 us, 5.5 TB/s: the selection's chain is
// hidden by three other workgroups of a compute unit. One row of 32,000 takes 5.8 us without, 8.1 with
// one and 9.4 with twenty of them; 1,024 threads for such a row: 5.5 and 9.3 us.
template <typename T, int TPB, int NV, bool ALT, bool PART>
__global__ __launch_bounds__(TPB) void k_score_row(ScoreArgs A, ScorePart* parts, uint64_t* lists) {
  constexpr int N = Span<T>::N, NW = TPB / 64;
  __shared__ ScorePart red[NW];
  __shared__ uint64_t picked[ALT ? TKEF_SCORE_MAX_K : 1];
  __shared__ Maybe<ALT> L;
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t row = blockIdx.x;
  const int32_t token = A.tokens[row];
  if (token < 0 || token >= A.V) {
    if constexpr (!PART) put_none(A, row, token, tid, TPB);
    return;
  }
  const Span<T> s(static_cast<const T*>(A.z) + row * A.ld, A.V);
  const int v0 = PART ? (int)blockIdx.y * (TPB * NV) : 0;
  const bool edges = !PART || blockIdx.y == 0;
  const T* type = nullptr;
  uint4 r[NV];
  load_slots<T, TPB, NV, true>(r, s, v0);
  const bool has_ex = edges && tid < s.extras;
  const float ex = has_ex ? (float)s.p[s.extra(tid)] : -kInf;
  ScorePart part;
  float m = ex;
#pragma unroll
  for (int i = 0; i < NV; ++i) m = max_packed(m, r[i], type);
  // exponents of the fused form y' = y - g, whose rounding g enters both sums at their end
  const Product ref(m, A.a);
  float S = 0.f, T_ = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float x[N];
    renew(r[i]);
    unpack(r[i], x, type);
    float e = 0.f, t = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float y = ref.exponent(x[n]), p = exp2_(y);
      e += p;
      t = __builtin_fmaf(p, near(y), t);
    }
    S += e;
    T_ += t;
  }
  const float g = -__builtin_fmaf(ref.m, ref.a, -ref.c), back = exp2_(g);
  const float ye = (ex - ref.m) * A.a, pe = exp2_(ye);
  part.m = m;
  part.S = S * back + pe;
  part.T = (T_ + S * g) * back + pe * near(ye);
  part.pad = 0.f;
  part = wave_join(part, A.a);
  if (lane == 0) red[tid >> 6] = part;
  __syncthreads();
  part = red[lane < NW ? lane : 0];
  if (lane >= NW) part.S = part.T = 0.f;
  part = wave_join(part, A.a);
  if (!Product::fits(part.m, A.a)) {  // (the same for the whole workgroup)
    // nothing but far logits: again, by the difference
    ScorePart q = {part.m, 0.f, 0.f, 0.f};
    const auto add = [&](float x) {
      const float y = (x - part.m) * A.a, p = exp2_(y);
      q.S += p;
      q.T += p * near(y);
    };
    const int end = s.nvec - v0 < TPB * NV ? s.nvec - v0 : TPB * NV;
    for (int i = tid; i < end * N; i += TPB) add((float)s.vec(v0)[i]);
    if (has_ex) add(ex);
    q = wave_join(q, A.a);
    __syncthreads();
    if (lane == 0) red[tid >> 6] = q;
    __syncthreads();
    q = red[lane < NW ? lane : 0];
    if (lane >= NW) q.S = q.T = 0.f;
    part = wave_join(q, A.a);
  }
  if constexpr (ALT) {
    if (!(part.S != part.S)) {
      const Share<T, TPB, NV> mine = {s, v0, tid, has_ex, ex};
      select<T, NV>(r, m, mine, A.k, picked, L);
    }
    __syncthreads();
  }
  if constexpr (PART) {
    const int64_t at = row * gridDim.y + blockIdx.y;
    if (tid == 0) parts[at] = part;
    if constexpr (ALT)
      for (int j = tid; j < A.k; j += TPB) lists[at * A.k + j] = picked[j];
  } else {
    const RowScore score = row_score(part);
    if (tid == 0) put_score(A, row, token, score);
    if constexpr (ALT)
      for (int j = tid; j < A.k; j += TPB) put_alternative<T>(A, row, j, picked[j], score);
  }
}

// A row from its chunks, one wave a row. Lane l goes through the list of chunk l: the k
// first of the row are the greatest of the lists' heads, k times (2,048 rows: 6 us for
// k = 5, 38 for k = 64).
template <typename T, bool ALT>
__global__ __launch_bounds__(64) void k_score_join(ScoreArgs A, const ScorePart* parts,
                                                   const uint64_t* lists, int chunks) {
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x;
  const int32_t token = A.tokens[row];
  if (token < 0 || token >= A.V) {
    put_none(A, row, token, lane, 64);
    return;
  }
  ScorePart p = {-kInf, 0.f, 0.f, 0.f};
  for (int i = lane; i < chunks; i += 64) {
    ScorePart q = parts[row * chunks + i];
    const float top = fmaxf(p.m, q.m);
    move_to(p, top, A.a);
    move_to(q, top, A.a);
    p.S += q.S;
    p.T += q.T;
  }
  p = wave_join(p, A.a);
  const RowScore score = row_score(p);
  if (lane == 0) put_score(A, row, token, score);
  if constexpr (ALT) {
    const uint64_t* list = lists + (row * chunks + lane) * A.k;
    int at = 0;
    uint64_t head = lane < chunks && score.valid ? list[0] : 0ull;
    for (int j = 0; j < A.k; ++j) {
      const uint64_t c = wave_max64(head);
      if (lane == 0) put_alternative<T>(A, row, j, c, score);
      if (head == c && c != 0ull) {
        ++at;
        head = at < A.k ? list[at] : 0ull;
      }
    }
  }
}

// Gradient of one chunk (blockIdx.y of gridDim.y) of a row, from the saved sums. With
// y = (x_i - m) a:  q_i = 2^y / S,  log q_i = ln 2 y - ln S, so
//   dlogp (1{i = t} - q_i) - dentropy q_i (log q_i + H)
//     = 1{i = t} dlogp + 2^y (P + Q y)
// over the temperature, with P and Q the row's. Reads and writes bound it: 8,192 x 32,000 bfloat16 in
// 173 us, 5.7 TB/s.
template <typename T, int TPB, int NV>
__global__ __launch_bounds__(TPB) void k_score_grad(ScoreArgs A) {
  constexpr int N = Span<T>::N;
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  T* grad = static_cast<T*>(A.grad) + row * A.gld;
  const int32_t token = A.tokens[row];
  const float dl = A.dlogp != nullptr ? A.dlogp[row] : 0.f;
  const float dh = A.dentropy != nullptr ? A.dentropy[row] : 0.f;
  const bool none = token < 0 || token >= A.V;
  if (none || (dl == 0.f && dh == 0.f)) {
    if (none && token != -1 && blockIdx.y == 0 && tid == 0)
      raise_status(A.status, TKEF_STATUS_INDEX_RANGE);
    zero_row<T, TPB>(grad, A.V, (int)blockIdx.y, (int)gridDim.y);
    return;
  }
  const Span<T> s(static_cast<const T*>(A.z) + row * A.ld, A.V);
  const int v0 = (int)blockIdx.y * (TPB * NV);
  const T* type = nullptr;
  uint4 r[NV];
  load_slots<T, TPB, NV, true>(r, s, v0);
  const bool has_ex = blockIdx.y == 0 && tid < s.extras;
  const float ex = has_ex ? (float)s.p[s.extra(tid)] : -kInf;
  const float4 st = A.stats[row];
  const float m = st.x, scale = A.inv_t / st.y;
  const float up = dl * A.inv_t;
  float Q = -scale * dh * kLn2;
  float P = -scale * (dl + dh * (st.z - kLn2 * log2_(st.y)));
  if (!(st.y > 0.f && st.y < kInf)) P = Q = __uint_as_float(kNaNBits);
  const auto of = [&](float x) {
    const float y = near((x - m) * A.a);
    return exp2_(y) * __builtin_fmaf(Q, y, P);
  };
  // the token's vector and place in it
  const int e = token - s.head;
  const int tv = e >= 0 && e < s.nvec * N ? e / N : -1;
  const int tid2 = renew(tid);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = v0 + i * TPB + tid2;
    float x[N];
    unpack(r[i], x, type);
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = of(x[n]);
    if (v == tv) {
#pragma unroll
      for (int n = 0; n < N; ++n) x[n] += n == e % N ? up : 0.f;
    }
    if (v < s.nvec) store16(grad + s.head + (int64_t)v * N, pack(x, type));
  }
  if (has_ex) grad[s.extra(tid)] = (T)(of(ex) + (s.extra(tid) == token ? up : 0.f));
}

// Vectors of a chunk: 64 KB where lists of alternatives are made, else 32 KB; rows of up to
// 64 KB are whole.
constexpr int kWholeVecs = 256 * 16, kAltVecs = 256 * 16, kSumVecs = 256 * 8;
static_assert((int64_t)TKEF_ROWS_MAX_VOCAB / 4 <= 64 * (int64_t)kAltVecs, "a lane for each list");

int64_t row_vecs(int64_t V, int32_t dtype) { return V / (dtype == TKEF_DTYPE_F32 ? 4 : 8); }

int score_chunks(int64_t V, int64_t k, int32_t dtype) {
  const int64_t vecs = row_vecs(V, dtype);
  return vecs <= kWholeVecs ? 1 : (int)ceil_div(vecs, k > 0 ? kAltVecs : kSumVecs);
}

template <typename T, bool ALT>
void launch_whole(const ScoreArgs& a, hipStream_t s) {
  const int vecs = a.V / Span<T>::N;
  const dim3 grid((unsigned)a.rows);
  if (vecs <= 256 * 4)
    k_score_row<T, 256, 4, ALT, false><<<grid, 256, 0, s>>>(a, nullptr, nullptr);
  else if (vecs <= 256 * 8)
    k_score_row<T, 256, 8, ALT, false><<<grid, 256, 0, s>>>(a, nullptr, nullptr);
  else
    k_score_row<T, 256, 16, ALT, false><<<grid, 256, 0, s>>>(a, nullptr, nullptr);
}

}  // namespace

size_t score_workspace(int64_t rows, int64_t V, int64_t k, int32_t dtype) {
  const int chunks = score_chunks(V, 0, dtype);
  if (chunks == 1) return 0;
  const size_t sums = (size_t)rows * (size_t)chunks * sizeof(ScorePart);
  const size_t most = (size_t)rows * (size_t)score_chunks(V, k, dtype);
  const size_t alternatives = up256(most * sizeof(ScorePart)) + most * (size_t)k * 8;
  return sums > alternatives ? sums : alternatives;
}

hipError_t launch_score_forward(const ScoreArgs& a, void* ws, hipStream_t s) {
  const int chunks = score_chunks(a.V, a.k, a.dtype);
  const dim3 rows((unsigned)a.rows), split((unsigned)a.rows, (unsigned)chunks);
  return by_dtype(a.dtype, [&](auto* t) {
    using T = typename Pointee<decltype(t)>::type;
    ScorePart* parts = static_cast<ScorePart*>(ws);
    if (chunks == 1) {
      if (a.k > 0)
        launch_whole<T, true>(a, s);
      else
        launch_whole<T, false>(a, s);
    } else if (a.k > 0) {
      uint64_t* lists = reinterpret_cast<uint64_t*>(
          static_cast<char*>(ws) + up256((size_t)a.rows * (size_t)chunks * sizeof(ScorePart)));
      k_score_row<T, 256, 16, true, true><<<split, 256, 0, s>>>(a, parts, lists);
      k_score_join<T, true><<<rows, 64, 0, s>>>(a, parts, lists, chunks);
    } else {
      k_score_row<T, 256, 8, false, true><<<split, 256, 0, s>>>(a, parts, nullptr);
      k_score_join<T, false><<<rows, 64, 0, s>>>(a, parts, nullptr, chunks);
    }
  });
}

hipError_t launch_score_backward(const ScoreArgs& a, hipStream_t s) {
  return by_dtype(a.dtype, [&](auto* t) {
    using T = typename Pointee<decltype(t)>::type;
    const int64_t vecs = row_vecs(a.V, a.dtype);
    const dim3 grid((unsigned)a.rows, (unsigned)ceil_div(vecs, 256 * 8));
    k_score_grad<T, 256, 8><<<grid, 256, 0, s>>>(a);
  });
}

}  // namespace tkef

// gfx950 kernels for rows of logits over a vocabulary: a teacher's top logits,
// distillation on them (loss and gradient), verification of drafted tokens.
// Exponentials, sums and vectors of rows: tkef_rows_device.h.
#include <cmath>

#include <hip/hip_runtime.h>

#include "tkef.h"
#include "tkef_rows.h"
#include "tkef_rows_device.h"

#pragma clang fp contract(off)

namespace tkef {

namespace {

// ----------------------------------------------------------------------------
// top logits

constexpr uint32_t kNaNBits = 0x7FC00000u;

__device__ __forceinline__ void put_pair(const TopArgs& A, int64_t row, uint32_t pos,
                                         int32_t word, float x) {
  const int64_t o = row * A.k + pos;
  A.idx[o] = word;
  if (A.val_format == TKEF_VAL_F16)
    static_cast<_Float16*>(A.val)[o] = (_Float16)x;
  else
    static_cast<float*>(A.val)[o] = x;
}

// The rest of a selection, S * 2^(m a), by one thread.
__device__ __forceinline__ void put_rest(const TopArgs& A, int64_t row, float m, float S) {
  if (A.tail == nullptr) return;
  A.tail[row] = S != S ? __uint_as_float(kNaNBits)
                : m == kInf ? kInf
                : S > 0.f ? m * A.inv_t + kLn2 * log2_(S) : -kInf;
}

struct RadixLds {
  uint32_t hist[256];
  uint32_t red[16];
  float fred[16];
  uint32_t pick[2];
};

// Selection from a row of any values: radix select of the k-th largest order
// key over four 8-bit digits, then the ordered compaction and the rest's sum.
// Seven passes over the row, bound by them and by their LDS atomics (4.1 ms where all
// of 8,192 rows of 32,000 bfloat16 words come here, the ordinary way 0.1); the kernels
// below come here with rows that have NaN, that have more words in reach of the k first
// than LDS holds, and whose rest lies more than 2^-60 below their k-th word. The second
// kind is ordinary where k > 256 nears or passes the number of a part's vectors: their
// maxima then bound nothing, and up to all of its words are in reach (16-bit rows
// of 2,600 to 12,000 words from about k = V / 10 on, binary32 of 2,600 to 5,600 from V / 5).
template <typename T, int NT>
__device__ __forceinline__ void top_radix(const TopArgs& A, RadixLds& L, const T* p,
                                          int64_t row) {
  const int tid = threadIdx.x, V = A.V;
  uint32_t prefix = 0u, need = (uint32_t)A.k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) L.hist[tid] = 0u;
    __syncthreads();
    for (int i = tid; i < V; i += NT) {
      const uint32_t key = order_key(load1(p, i));
      if (shift == 24 || (key >> (shift + 8)) == prefix)
        atomicAdd(&L.hist[(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    // digit 255 - tid: the exclusive prefix counts the keys in higher digits
    const uint32_t mine = tid < 256 ? L.hist[255 - tid] : 0u;
    uint32_t total;
    const uint32_t above = block_scan<NT>(mine, L.red, &total);
    if (above < need && need <= above + mine) {
      L.pick[0] = 255u - (uint32_t)tid;
      L.pick[1] = need - above;
    }
    __syncthreads();
    prefix = (prefix << 8) | L.pick[0];
    need = L.pick[1];
  }
  // the k-th key, and how many of its class are taken (the lowest words)
  const uint32_t kth = prefix, quota = need;
  uint32_t done_gt = 0u, done_eq = 0u;
  float top = -kInf;
  int nan = 0;
  for (int base = 0; base < V; base += NT) {
    const int i = base + tid;
    const float x = i < V ? load1(p, i) : 0.f;
    const uint32_t key = i < V ? order_key(x) : 0u;
    const bool gt = i < V && key > kth, eq = i < V && key == kth;
    uint32_t total;
    // (both counts in one scan: at most 1,024 of each in a round)
    const uint32_t before =
        block_scan<NT>((gt ? 1u : 0u) | (eq ? 1u << 16 : 0u), L.red, &total);
    const uint32_t r_gt = done_gt + (before & 0xFFFFu), r_eq = done_eq + (before >> 16);
    if (gt || (eq && r_eq < quota))
      put_pair(A, row, r_gt + (r_eq < quota ? r_eq : quota), i, x);
    else if (i < V)
      top = x > top ? x : top;
    nan |= i < V && x != x;
    done_gt += total & 0xFFFFu;
    done_eq += total >> 16;
  }
  nan = __syncthreads_or(nan);
  if (nan && tid == 0) raise_status(A.status, TKEF_STATUS_NAN);
  top = block_reduce<NT>(top, L.fred, MaxOp());
  const float m = top == -kInf ? 0.f : top;
  float sum = 0.f;
  for (int i = tid; i < V; i += NT) {
    const float x = load1(p, i);
    if (order_key(x) < kth) sum += exp2_((x - m) * A.a);
  }
  sum = block_reduce<NT>(sum, L.fred, AddOp());
  if (tid == 0) {
    // the class of the k-th key that was not taken
    const float tie = key_value(kth);
    if (done_eq > quota && tie > -kInf)
      sum += (float)(done_eq - quota) * exp2_((tie - m) * A.a);
    if (top == kInf) sum = 1.f;
    put_rest(A, row, top, nan ? __uint_as_float(kNaNBits) : sum);
  }
}

// the least candidate at or above an order key
template <typename T>
__device__ __forceinline__ uint64_t floor_of(uint32_t key) {
  const T* type = nullptr;
  return (uint64_t)(key >> key_shift(type)) << kWordBits;
}

// Ranks by counting up to this many candidates (one a thread), by bisection above:
// counting costs a comparison for each pair, bisection some twelve rounds with a
// barrier each. 8,192 x 32,000 bfloat16: k = 128 (some 150 candidates) 132 us counted, 147
// bisected; k = 256 (some 290) 204 and 180.
constexpr int kRankLimit = 256;

template <int TPB, int KMAX>
struct FinishLds {
  // read as int4, wherever the struct lies; and fillers up to a multiple of 16
  alignas(16) int32_t chosen[KMAX + 16];
  uint64_t thr, top[TPB / 64];
  float others[kRankLimit];
  uint32_t count[2][TPB / 64];
  float red[TPB / 64];
  uint32_t ntaken;
};

// The k first of C candidates (LDS, all >= least, then eight zeros), their places in
// ascending order of words, and the rest: S * 2^(m a) and the candidates not taken. Up to kRankLimit
// candidates a thread counts the better ones of its own; beyond that the k-th
// candidate is bisected, a candidate's word being part of it, so that ties end
// at the lower words. A selected word's place is the number of selected lower
// words. False, with nothing written, where candidates below `lowest` would be
// needed or the rest, though it holds words with a probability, vanishes beside
// the last selected word. The same for all threads.
template <typename T, int TPB, int CAP, int KMAX>
__device__ __forceinline__ bool top_finish(const TopArgs& A, int64_t row, const T* p,
                                           const uint64_t* cand, int C, uint64_t least,
                                           uint64_t lowest, float m, float S,
                                           FinishLds<TPB, KMAX>& L) {
  constexpr int NW = TPB / 64, CPT = (CAP + TPB - 1) / TPB;
  static_assert(alignof(FinishLds<TPB, KMAX>) >= alignof(int4) && alignof(int4) == 16,
                "L.chosen is read as int4");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = A.k;
  if (C < k) return false;
  const bool more = k < A.V;
  uint64_t c[CPT];
  const bool counted = C <= kRankLimit;
  uint64_t thr;
  float left = 0.f;
  if (tid < 16) L.chosen[k + tid] = INT32_MAX;
  if (counted) {
    c[0] = tid < C ? cand[tid] : 0ull;
    int rank = 0;
    if (wave * 64 < C) {
      for (int j = 0; j < C; j += 8) {  // (zeros follow; all reads before the first use)
        ulonglong2 o[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          o[u] = *reinterpret_cast<const ulonglong2*>(&cand[j + 2 * u]);
#pragma unroll
        for (int u = 0; u < 4; ++u) rank += (o[u].x > c[0] ? 1 : 0) + (o[u].y > c[0] ? 1 : 0);
      }
    }
    if (tid < C) {
      if (rank < k)
        L.chosen[rank] = word_of(c[0]);
      else
        L.others[rank - k] = value_of<T>(c[0]);
      if (rank == k - 1) L.thr = c[0];
    }
    __syncthreads();
    thr = L.thr;
  } else {
    uint64_t hi = 0ull;
#pragma unroll
    for (int q = 0; q < CPT; ++q) {
      c[q] = 0ull;
      if (q * TPB < C) {
        c[q] = q * TPB + tid < C ? cand[q * TPB + tid] : 0ull;
        hi = c[q] > hi ? c[q] : hi;
      }
    }
    hi = wave_max64(hi);
    if (lane == 0) L.top[wave] = hi;
    if (tid == 0) L.ntaken = 0u;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) hi = L.top[w] > hi ? L.top[w] : hi;
    ++hi;
    // n_lo >= k candidates are >= lo, fewer than k are >= hi
    uint64_t lo = least;
    uint32_t n_lo = (uint32_t)C;
    for (int turn = 0; n_lo > (uint32_t)k && hi - lo > 1ull; turn ^= 1) {
      const uint64_t mid = lo + (hi - lo) / 2ull;
      uint32_t n = 0u;
#pragma unroll
      for (int q = 0; q < CPT; ++q)
        if (q * TPB < C) n += (uint32_t)__popcll(__ballot(c[q] >= mid));
      if (lane == 0) L.count[turn][wave] = n;
      __syncthreads();
      n = 0u;
#pragma unroll
      for (int w = 0; w < NW; ++w) n += L.count[turn][w];
      if (n >= (uint32_t)k) {
        lo = mid;
        n_lo = n;
      } else {
        hi = mid;
      }
    }
    thr = lo;
  }
  if (thr < lowest) return false;
  const float at_thr = value_of<T>(thr), base = at_thr == -kInf ? 0.f : at_thr;
  bool some = m != -kInf;  // unselected words that are not masked
  if (counted) {
    for (int j = lane; j < C - k; j += 64) left += exp2_((L.others[j] - base) * A.a);
    left = wave_sum(left);
    some |= C > k && L.others[0] != -kInf;
  } else {
    int mine = 0;
#pragma unroll
    for (int q = 0; q < CPT; ++q) {
      if (q * TPB >= C) continue;
      const bool take = c[q] >= thr;
      const uint64_t who = __ballot(take);
      if (who != 0ull) {
        uint32_t at = 0u;
        if (lane == 0) at = atomicAdd(&L.ntaken, (uint32_t)__popcll(who));
        at = __builtin_amdgcn_readfirstlane(at) +
             __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32),
                                       __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
        if (take) L.chosen[at] = word_of(c[q]);
      }
      if (!take && c[q] != 0ull) {
        const float x = value_of<T>(c[q]);
        left += exp2_((x - base) * A.a);
        mine |= x != -kInf;
      }
    }
    left = wave_sum(left);
    if (lane == 0) L.red[wave] = left;
    some |= __syncthreads_or(mine) != 0;
    left = wave_sum(lane < NW ? L.red[lane] : 0.f);
  }
  // the rest relative to the last selected word
  const float rest = S * rescale(m, base, A.a) + left;
  if (more && some && !(rest > 0x1p-60f)) return false;
  for (int j = tid; j < k; j += TPB) {
    const int32_t word = L.chosen[j];
    int place = 0;
    for (int i = 0; i < k; i += 16) {
      int4 o[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) o[u] = *reinterpret_cast<const int4*>(&L.chosen[i + 4 * u]);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        place += (o[u].x < word ? 1 : 0) + (o[u].y < word ? 1 : 0) + (o[u].z < word ? 1 : 0) +
                 (o[u].w < word ? 1 : 0);
    }
    put_pair(A, row, (uint32_t)place, word, load1(p, word));
  }
  if (tid == 0) put_rest(A, row, more && some ? base : -kInf, more && some ? rest : 0.f);
  return true;
}

// Parts of a row that is too long for one workgroup's registers. A part
// holds every `parts`-th piece of 1 KB of the row, so that words that lie
// together (frequent ones often do) spread over all parts, and hands on its
// words at or above a bound that about `want` of them reach: enough for
// its share of the k first. The words of the k first that it might hold back are
// below its bound, which the merge checks against the k-th.
struct PartHead {
  float bound, sum;    // the words below: sum * 2^(bound a)
  uint32_t key, count; // the bound's order key; candidates, kFullPart: too many, or NaN
};
constexpr int kPiece = 64;  // vectors
constexpr uint32_t kFullPart = 0xFFFFFFFFu;
struct TopParts {
  PartHead* heads;  // rows x parts
  uint64_t* lists;  // rows x parts x room
  int32_t parts, room, want;
};

// Workgroups of 256 a compute unit for which registers are allotted. Parts of 16
// vectors: 4 (64 us in five's 96 registers, which hold some in memory, 54 in four's;
// 509 x 131,071 binary32).
template <int TPB, int NV, int SUB, bool PART>
constexpr int top_workgroups() {
  return TPB != 256 ? 1 : PART ? 4 : SUB <= 2 && NV < 16 ? 8 - NV / 8 : 5;
}

// One workgroup takes a row, or a part of one, into registers, NV vectors a
// thread.
//   1. Each thread's maximum over each of its SUB shares. The k-th largest of
//      these TPB * SUB maxima (bisected on order keys by one wave) is at most the
//      k-th largest word: every selected word is at least that bound, and few
//      others are (for 64 of 256 shares of 125 words, about 74 in all).
//   2. One pass over the registers sums the exponentials of the words below
//      the bound; a vector with a word at or above it goes to its wave's part of
//      LDS instead, whose words the wave then sorts into candidates and others.
//   3. top_finish, or a part's list.
// Where more vectors or words reach the bound than LDS holds, they do so by ties
// (constant rows; rows with few words left unmasked; coarse values): the words above
// the least value at the bound are the candidates then, and the lowest words at
// that value fill up; so too where the bound lies beyond what Product takes. A NaN
// (in the sum), or too many words above the ties, send the row to top_radix.
// Bound by the reads for k <= 64 and rows of 32,000 words (8,192 of bfloat16: 100 to 110 us,
// 5 TB/s; as parts of 509 x 131,071 binary32, k = 256, 54 us, 4.9 TB/s), by the steps after
// them for short rows and larger k, which are a chain of barriers that five workgroups a
// compute unit hide in part (k = 256: 180 us; 8,000 words: k = 64 49, k = 256 155). Small
// workgroups for that reason: in 512 threads x 8 vectors k = 64 takes 132 us, in 1,024 x 4 343.
template <typename T, int TPB, int NV, int SUB, bool PART>
__global__ __launch_bounds__(TPB, (top_workgroups<TPB, NV, SUB, PART>())) void k_top_row(
    TopArgs A, TopParts P) {
  constexpr int N = Span<T>::N, NW = TPB / 64;
  constexpr int kKMax = PART ? 1 : TPB * SUB / 4;                 // words to select
  // (sorted rows bring whole vectors, an eighth more of them than words to select)
  constexpr int kCap = PART ? 1 : (kKMax + kKMax / 8 + 2) * 8;   // candidates
  constexpr int kVecs = PART && SUB > 1 ? 320 : 128;  // vectors of a wave
  constexpr int kGroups = TPB * SUB;
  struct Vecs {
    uint4 x[NW][kVecs];
    int32_t word[NW][kVecs];
  };
  union Shared {
    uint32_t group[kGroups];
    Vecs v;
    FinishLds<TPB, kKMax> finish;
    RadixLds radix;
  };
  __shared__ Shared S;
  __shared__ __align__(16) uint64_t cand[kCap + 8];
  __shared__ float red[NW];
  __shared__ uint32_t wave_count[NW], scan[NW];
  __shared__ uint32_t full, bound_key;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  const int part = PART ? (int)blockIdx.y : 0, parts = PART ? P.parts : 1;
  const T* type = nullptr;
  const Span<T> s(static_cast<const T*>(A.z) + row * A.ld, A.V);
  // vector t of slot i, ascending in (i, t): i * step + t, in a part the t / 64-th
  // of each `parts` pieces
  const int step = parts * TPB;
  const int v0 = PART ? (__builtin_amdgcn_readfirstlane(wave) * parts + part) * kPiece : 0;
  const int k = PART ? P.want : A.k;
  uint4 r[NV];
  const int own = PART ? lane : tid;
  load_slots<T, TPB, NV, true>(r, s, v0, step, own, PART ? kPiece : TPB);
  const int xi = s.extra(tid < s.extras ? tid : 0);
  const bool has_ex = part == 0 && tid < s.extras;
  const float ex = has_ex ? (float)s.p[xi] : -kInf;
  if (tid == 0) full = 0u;
  // 1. the bound
#pragma unroll
  for (int q = 0; q < SUB; ++q) {
    float m = q == 0 ? ex : -kInf;
#pragma unroll
    for (int i = q; i < NV; i += SUB) {
      m = max_packed(m, r[i], type);
    }
    S.group[q * TPB + tid] = order_key(m);
  }
  __syncthreads();
  if (wave == 0) {
    uint32_t g[kGroups / 64];
    uint32_t lo = 0xFFFFFFFFu, hi = 0u;
#pragma unroll
    for (int i = 0; i < kGroups / 64; ++i) {
      g[i] = S.group[i * 64 + lane];
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
    // at least k maxima have keys >= lo, fewer than k have keys >= hi
    const uint32_t least = 1u << key_shift(type), enough = (uint32_t)k + ((uint32_t)k >> 3) + 1u;
    while (hi - lo > least) {
      const uint32_t mid = lo + (hi - lo) / 2u;
      uint32_t c = 0u;
#pragma unroll
      for (int i = 0; i < kGroups / 64; ++i)
        c += (uint32_t)__popcll(__ballot(g[i] >= mid));
      if (c >= (uint32_t)k) {
        lo = mid;
        if (c <= enough) break;
      } else {
        hi = mid;
      }
    }
    if (lane == 0) bound_key = lo;
  }
  __syncthreads();
  uint32_t at_bound = bound_key;
  float bound = key_value(at_bound);
  bool ties = false;  // the candidates are the words above the bound
  // 2. candidates, and the sum of the others
  const Product ref(bound, A.a);
  float sum = 0.f;
  int held = 0;  // vectors in this wave's part
  const int tid2 = renew(own);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = v0 + i * step + tid2;
    float x[N];
    renew(r[i]);
    unpack(r[i], x, type);
    const bool above = max_of(-kInf, x) >= bound && v < s.nvec;
    const uint64_t who = __ballot(above);
    if (above) {
      const int at = held + (int)__builtin_amdgcn_mbcnt_hi(
                                (uint32_t)(who >> 32),
                                __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
      if (at < kVecs) {
        S.v.x[wave][at] = r[i];
        S.v.word[wave][at] = s.head + v * N;
      }
    }
    held += (int)__popcll(who);
    float e = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) e += exp2_(ref.exponent(x[n]));
    sum += above ? 0.f : e;
    asm volatile("" : "+v"(sum));  // (here, not after the last vector from kept registers)
  }
  sum *= ref.rest();
  if (held > kVecs) {
    held = 0;
    if (lane == 0) full = 1u;
  }
  // The wave's words that reach the bound are candidates: `each` gets them with
  // a number that counts them in a fixed order.
  const auto wave_words = [&](auto each) {
    int seen = 0;
    const auto one = [&](bool valid, float x, int32_t word) {
      const bool take = valid && (ties ? x > bound : x >= bound);
      const uint64_t who = __ballot(take);
      each(valid, take, x, word,
           seen + (int)__builtin_amdgcn_mbcnt_hi(
                      (uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u)));
      seen += (int)__popcll(who);
    };
    for (int i = 0; i < held * N; i += 64) {
      const int e = i + lane;
      const bool valid = e < held * N;
      const int at = valid ? e / N : 0;
      const float x = (float)reinterpret_cast<const T*>(&S.v.x[wave][at])[e % N];
      one(valid, x, S.v.word[wave][at] + e % N);
    }
    if (wave == 0) one(has_ex, ex, xi);
    return seen;
  };
  int C, mine;
  // candidates and sum of the workgroup, from each wave's
  const auto add_up = [&](int found) {
    sum = wave_sum(sum);
    if (lane == 0) {
      red[wave] = sum;
      wave_count[wave] = (uint32_t)found;
    }
    __syncthreads();
    C = mine = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      mine += w < wave ? (int)wave_count[w] : 0;
      C += (int)wave_count[w];
    }
    sum = wave_sum(lane < NW ? red[lane] : 0.f);
  };
  add_up(wave_words([&](bool valid, bool take, float x, int32_t, int) {
    if (valid && !take) sum += exp2_((x - ref.m) * A.a);
  }));
  // (the same for the whole workgroup, as all that is decided from here on)
  bool odd = sum != sum;
  const int room = PART ? P.room - A.k : kCap;
  bool many = full != 0u || C > room || !Product::fits(bound, A.a);
  int wanted = 0;  // of the words at the bound, with ties
  if (many && !odd) {
    // the least value that reaches the bound, and how many words do
    // (read again: registers held for this rare case would spill in all others)
    load_slots<T, TPB, NV, false>(r, s, v0, step, own, PART ? kPiece : TPB);
    float least = kInf;
    int reach = 0;
    const int tid3 = renew(own);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float x[N];
      renew(r[i]);
      unpack(r[i], x, type);
      const bool in = v0 + i * step + tid3 < s.nvec;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const bool at = in && x[n] >= bound;
        least = at ? fminf(least, x[n]) : least;
        reach += at ? 1 : 0;
      }
    }
    if (has_ex && ex >= bound) {
      least = fminf(least, ex);
      ++reach;
    }
    least = -wave_max(-least);
    for (int d = 32; d > 0; d >>= 1) reach += __shfl_xor(reach, d);
    __syncthreads();
    if (lane == 0) {
      red[wave] = least;
      wave_count[wave] = (uint32_t)reach;
    }
    if (tid == 0) full = 0u;
    __syncthreads();
    bound = kInf;
    reach = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      bound = fminf(bound, red[w]);
      reach += (int)wave_count[w];
    }
    at_bound = order_key(bound);
    ties = true;
    // the words above it, and the sum of those below
    sum = 0.f;
    held = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = v0 + i * step + tid3;
      float x[N];
      renew(r[i]);
      unpack(r[i], x, type);
      const bool above = max_of(-kInf, x) > bound;
      const uint64_t who = __ballot(above);
      if (above) {
        const int at = held + (int)__builtin_amdgcn_mbcnt_hi(
                                  (uint32_t)(who >> 32),
                                  __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
        if (at < kVecs) {
          S.v.x[wave][at] = r[i];
          S.v.word[wave][at] = s.head + v * N;
        }
      }
      held += (int)__popcll(who);
      float e = 0.f;
#pragma unroll
      for (int n = 0; n < N; ++n) e += x[n] >= bound ? 0.f : exp2_((x[n] - bound) * A.a);
      sum += above ? 0.f : e;
      asm volatile("" : "+v"(sum));
    }
    if (held > kVecs) {
      held = 0;
      if (lane == 0) full = 1u;
    }
    __syncthreads();  // (red and wave_count are read above)
    add_up(wave_words([&](bool valid, bool, float x, int32_t, int) {
      if (valid && !(x >= bound)) sum += exp2_((x - bound) * A.a);
    }));
    odd = sum != sum;  // (a NaN among vectors that were too many to look into before)
    many = full != 0u || C > room;
    // A row needs as many words at the bound as are missing of its k, a part
    // never more than k.
    const int at_it = reach - C, most = PART ? A.k : C < A.k ? A.k - C : 0;
    wanted = at_it < most ? at_it : most;
    if (bound != -kInf) sum += (float)(at_it - wanted);
  }
  // the lowest `wanted` words at the bound: `put` gets each with its number
  const auto fill = [&](auto put) {
    int done = 0;
    const auto round = [&](bool valid, int32_t word) {
      const bool tie = valid && load1(s.p, word) == bound;
      uint32_t total;
      const int at = done + (int)block_scan<TPB>(tie, scan, &total);
      if (tie && at < wanted) put(at, word);
      done += (int)total;
    };
    if (part == 0 && wanted > 0) round(tid < s.head, tid);
    for (int i = 0; i < NV && done < wanted; ++i)
      for (int e = tid; e < TPB * N + tid && done < wanted; e += TPB) {
        const int t = e / N;
        const int v = i * step + (PART ? (t / kPiece * parts + part) * kPiece + t % kPiece : t);
        round(v < s.nvec, s.head + v * N + e % N);
      }
    if (part == 0 && done < wanted) {
      const int32_t word = s.head + s.nvec * N + tid;
      round(word < A.V, word);
    }
  };
  if constexpr (PART) {
    const int64_t at = row * parts + part;
    const bool fits = !odd && !many;
    if (fits) {
      uint64_t* list = P.lists + at * P.room;
      wave_words([&](bool, bool take, float x, int32_t word, int n) {
        if (take) list[mine + n] = candidate<T>(order_key(x), word);
      });
      fill([&](int n, int32_t word) { list[C + n] = candidate<T>(at_bound, word); });
    }
    if (tid == 0) {
      PartHead h;
      h.bound = bound;
      h.sum = sum;
      h.key = at_bound;
      h.count = fits ? (uint32_t)(C + wanted) : kFullPart;
      P.heads[at] = h;
    }
  } else {
    bool done = false;
    if (!odd && !many) {
      wave_words([&](bool, bool take, float x, int32_t word, int n) {
        if (take) cand[mine + n] = candidate<T>(order_key(x), word);
      });
      fill([&](int n, int32_t word) { cand[C + n] = candidate<T>(at_bound, word); });
      C += wanted;
      if (tid < 8) cand[C + tid] = 0ull;
      __syncthreads();
      done = top_finish<T, TPB, kCap, kKMax>(A, row, s.p, cand, C, floor_of<T>(at_bound), 0ull,
                                             bound, sum, S.finish);
    }
    __syncthreads();
    if (!done) top_radix<T, TPB>(A, S.radix, s.p, row);
  }
}

// The k first of a row from its parts' lists. Bound by its chain of dependent steps: heads,
// candidates, some twelve rounds of bisection, places, values (509 rows of eight lists,
// k = 256, 540 candidates: 17 us, two workgroups a compute unit).
template <typename T, int TPB, int CAP>
__global__ __launch_bounds__(TPB) void k_top_merge(TopArgs A, TopParts P) {
  __shared__ __align__(16) uint64_t cand[CAP + 8];
  __shared__ uint32_t from[64];
  union Shared {
    FinishLds<TPB, TKEF_ROWS_MAX_K> finish;
    RadixLds radix;
  };
  __shared__ Shared S;
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t row = blockIdx.x;
  const T* p = static_cast<const T*>(A.z) + row * A.ld;
  // (every wave reads the heads; at most 64 of them)
  PartHead h = {-kInf, 0.f, 0u, 0u};
  if (lane < P.parts) h = P.heads[row * P.parts + lane];
  const bool odd = __ballot(h.count == kFullPart) != 0ull;
  bool done = false;
  if (!odd) {
    const uint32_t inc = wave_incl(h.count);
    if (tid < 64) from[lane] = inc - h.count;
    const int C = __builtin_amdgcn_readlane((int)inc, 63);
    const float m = wave_max(h.bound);
    const float sum = wave_sum(join_sum(h.bound, h.sum, m, A.a));
    // what a part held back lies below its bound; the least that does not
    const T* type = nullptr;
    const uint64_t lowest =
        wave_max64(lane < P.parts && h.key != 0u
                       ? (((uint64_t)((h.key - 1u) >> key_shift(type)) + 1ull) << kWordBits)
                       : 0ull);
    const uint64_t least = ~wave_max64(lane < P.parts ? ~floor_of<T>(h.key) : 0ull);
    __syncthreads();
    if (C <= CAP) {
      // Candidate i is in the last part that starts at or before it (one load a
      // candidate, four under way: 17 us against 21 over the lists' whole room)
      const uint64_t* lists = P.lists + row * P.parts * P.room;
      for (int i0 = tid; i0 < C; i0 += 4 * TPB) {
        uint64_t c[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t i = (uint32_t)(i0 + u * TPB);
          int part = 0;
#pragma unroll
          for (int d = 32; d > 0; d >>= 1)
            part += part + d < P.parts && from[part + d] <= i ? d : 0;
          if (i < (uint32_t)C) c[u] = lists[part * P.room + (int)(i - from[part])];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (i0 + u * TPB < C) cand[i0 + u * TPB] = c[u];
      }
      if (tid < 8) cand[C + tid] = 0ull;
      __syncthreads();
      done = top_finish<T, TPB, CAP, TKEF_ROWS_MAX_K>(A, row, p, cand, C, least, lowest,
                                                      m, sum, S.finish);
    }
  }
  __syncthreads();
  if (!done) top_radix<T, TPB>(A, S.radix, p, row);
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

// tau - m / temperature, with 1 / temperature in two parts so that the product's
// rounding does not enter
__device__ __forceinline__ float tail_over(float tau, float m, float inv_t, float inv_t_lo) {
  return __builtin_fmaf(-m, inv_t, tau) - m * inv_t_lo;
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
      t.tau == -kInf ? 0.f : exp2_(tail_over(t.tau, t.m, A.inv_t, A.inv_t_lo) * kLog2e);
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

// What a part of a row (a thread's share, a wave's, a chunk's) adds to its sums:
// the unlisted words' student sum (rm, rs), the listed words' student sum (zm,
// zs) and teacher sum (tm, ts), and
//   cross = sum_j 2^((t_j - tm) a) ((t_j - tm) - (z_j - zm)) / temperature
// over its listed words: both logits from their own maximum, so rows that lie
// far off zero (all words at a mask's value) lose nothing.
struct Part {
  float rm, rs, zm, zs, tm, ts, cross, pad;
};
static_assert(sizeof(Part) == kPartBytes, "workspace layout");

// cross of a part after its maxima move to (tm, zm)
__device__ __forceinline__ float moved_cross(const Part& p, float tm, float zm,
                                             const DistillArgs& A) {
  const float f = rescale(p.tm, tm, A.a), ts = p.ts * f;
  if (!(ts > 0.f)) return ts;  // (0, or NaN)
  const float dt = p.tm == tm ? 0.f : p.tm - tm, dz = p.zm == zm ? 0.f : p.zm - zm;
  return p.cross * f + ts * ((dt - dz) * A.inv_t);
}

__device__ __forceinline__ Part empty_part() {
  return Part{-kInf, 0.f, -kInf, 0.f, -kInf, 0.f, 0.f, 0.f};
}

__device__ __forceinline__ Part join(const Part& p, const Part& q, const DistillArgs& A) {
  Part r;
  r.rm = fmaxf(p.rm, q.rm);
  r.zm = fmaxf(p.zm, q.zm);
  r.tm = fmaxf(p.tm, q.tm);
  r.rs = join_sum(p.rm, p.rs, r.rm, A.a) + join_sum(q.rm, q.rs, r.rm, A.a);
  r.zs = join_sum(p.zm, p.zs, r.zm, A.a) + join_sum(q.zm, q.zs, r.zm, A.a);
  r.ts = join_sum(p.tm, p.ts, r.tm, A.a) + join_sum(q.tm, q.ts, r.tm, A.a);
  r.cross = moved_cross(p, r.tm, r.zm, A) + moved_cross(q, r.tm, r.zm, A);
  r.pad = 0.f;
  return r;
}

// one listed word (a sum of one term from its own maximum is 1, or NaN)
__device__ __forceinline__ Part entry_part(float t, float z) {
  Part p = empty_part();
  p.zm = z;
  p.zs = z == -kInf ? 0.f : exp2_(z - z);
  p.tm = t;
  p.ts = t == -kInf ? 0.f : exp2_(t - t);
  p.cross = p.ts > 0.f && z == -kInf ? kInf : 0.f;  // a wanted word that has no probability
  return p;
}

__device__ __forceinline__ Part wave_join(const Part& p, const DistillArgs& A) {
  Part r;
  r.rm = wave_max(p.rm);
  r.zm = wave_max(p.zm);
  r.tm = wave_max(p.tm);
  r.rs = wave_sum(join_sum(p.rm, p.rs, r.rm, A.a));
  r.zs = wave_sum(join_sum(p.zm, p.zs, r.zm, A.a));
  r.ts = wave_sum(join_sum(p.tm, p.ts, r.tm, A.a));
  r.cross = wave_sum(moved_cross(p, r.tm, r.zm, A));
  r.pad = 0.f;
  return r;
}

// what a row's gradient needs
struct RowSums {
  Teacher t;
  float rm, rs, zm, zs;  // student sums: unlisted, listed
  float loss;            // the divergence
};

__device__ __forceinline__ RowSums row_sums(const Part& p, const DistillArgs& A, int64_t row) {
  RowSums r;
  LogSum list;
  list.m = p.tm;
  list.S = p.ts;
  r.t = teacher_of(list, A, row);
  r.rm = p.rm;
  r.rs = p.rs;
  r.zm = p.zm;
  r.zs = p.zs;
  const float top = fmaxf(p.rm, p.zm);
  const float total = join_sum(p.rm, p.rs, top, A.a) + join_sum(p.zm, p.zs, top, A.a);
  // With logarithms from the maxima (t.m of the teacher, top of the student),
  //   sum_j p_j (log p_j - log q_j) + p_r (log p_r - log q_r)
  //     = cross / S + log total - log S + p_r ((tau - s t.m) - (s (rm - top) + log rs))
  float loss = moved_cross(p, r.t.m, top, A) * r.t.inv + kLn2 * (log2_(total) - log2_(r.t.S));
  if (r.t.p_rest > 0.f)
    loss += p.rs == 0.f ? kInf
                        : r.t.p_rest * (tail_over(r.t.tau, r.t.m, A.inv_t, A.inv_t_lo) -
                                        ((p.rm - top) * A.inv_t + kLn2 * log2_(p.rs)));
  if (!(total > 0.f) || !has_mass(r.t)) loss = __uint_as_float(0x7FC00000u);
  r.loss = loss;
  return r;
}

// the factors of a row's gradient: unlisted words get 2^((x - rm) a) * rest,
// listed ones 2^((z - zm) a) * list - p_j * up
struct GradScale {
  float rm, rest, zm, list, up;
};

__device__ __forceinline__ GradScale grad_scale(const RowSums& r, const DistillArgs& A, float up) {
  GradScale g;
  const float top = fmaxf(r.rm, r.zm);
  const float s_rest = rescale(r.rm, top, A.a), s_list = rescale(r.zm, top, A.a);
  const float total = r.rs * s_rest + r.zs * s_list;
  const float inv = 1.f / total;
  g.up = up;
  g.rm = r.rm == -kInf ? 0.f : r.rm;
  g.zm = r.zm == -kInf ? 0.f : r.zm;
  // q_i (1 - p_r / q_r) = 2^((x_i - rm) a) (s_rest / total - p_r / rs)
  g.rest = up * (s_rest * inv - (r.t.p_rest > 0.f && r.rs > 0.f ? r.t.p_rest / r.rs : 0.f));
  g.list = up * (s_list * inv);
  if (!(total > 0.f) || !has_mass(r.t)) g.rest = g.list = __uint_as_float(0x7FC00000u);
  return g;
}

// listed words of a row in LDS
struct ListLds {
  int32_t word[TKEF_ROWS_MAX_K];  // -1: left out
  float t[TKEF_ROWS_MAX_K], z[TKEF_ROWS_MAX_K];
};

__device__ __forceinline__ int used_entries(const DistillArgs& A, int64_t row) {
  if (A.count == nullptr) return A.k;
  const int c = A.count[row];
  return c < 0 ? 0 : c < A.k ? c : A.k;
}

enum { kLoss = 0, kStep = 1, kPart = 2 };

// One workgroup takes a row, or one of a row's chunks, and holds it in
// registers: NV vectors a thread, loaded once.
//   kLoss  whole row: loss and sums
//   kStep  whole row: loss and gradient, from the one read
//   kPart  chunk blockIdx.y of gridDim.y: its Part into `parts`
// Listed words are marked in LDS (a byte a vector) and struck from the
// registers before the maximum and the sum, so the unlisted sum is exact even
// where the list has nearly all the mass; the gradient's listed words are
// written over the vectors' stores after a barrier.
// One read and, in a step, one write of each word: bound by memory, the eight (loss)
// to twelve (step) operations a word, two of them exponentials, close behind. Step of
// 8,192 x 32,000 bfloat16 200 us, 5.2 TB/s read and written; of 1,021 x 131,071 binary16, one
// workgroup a compute unit, 127 us, 4.0 TB/s; loss of 4,096 x 32,000 bfloat16, an eighth
// of the rows without weight, 55 us, 4.2 TB/s: 14 us of a row's chain that nothing hides at
// the start and the end, and 10.6 ns a row, 6.1 TB/s (8,192 rows 101 us).
template <typename T, int TPB, int NV, int MODE>
__global__ __launch_bounds__(TPB) void k_distill_row(DistillArgs A, Part* parts) {
  constexpr int N = Span<T>::N, NW = TPB / 64;
  __shared__ __align__(16) uint8_t mark[TPB * NV];  // thread t's vectors at t * NV
  __shared__ uint32_t mark_extra;
  __shared__ ListLds list;
  __shared__ Part red[NW];
  __shared__ float fred[NW];
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t row = blockIdx.x;
  const int cnt = used_entries(A, row);
  const float w = A.weight != nullptr ? A.weight[row] : 1.f;
  if (cnt == 0 || w == 0.f) {
    if constexpr (MODE == kStep) zero_row<T, TPB>(static_cast<T*>(A.grad) + row * A.gld, A.V, 0, 1);
    if (MODE != kPart && tid == 0) {
      A.loss[row] = 0.f;
      if (MODE == kLoss && A.stats != nullptr) A.stats[row] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    return;
  }
  const Span<T> s(static_cast<const T*>(A.z) + row * A.ld, A.V);
  const int v0 = MODE == kPart ? (int)blockIdx.y * (TPB * NV) : 0;
  const bool edges = MODE != kPart || blockIdx.y == 0;
  const T* type = nullptr;
  uint4 r[NV];
  load_slots<T, TPB, NV, MODE != kPart>(r, s, v0);
  float ex = edges && tid < s.extras ? (float)s.p[s.extra(tid)] : -kInf;
  for (int i = tid; i < TPB * NV / 16; i += TPB)
    reinterpret_cast<uint4*>(mark)[i] = make_uint4(0u, 0u, 0u, 0u);
  if (tid == 0) mark_extra = 0u;
  __syncthreads();
  // the list: marks, and the sums over listed words
  Part part = empty_part();
  uint32_t bits = 0u;
  const int32_t* idx = A.idx + row * A.k;
  for (int j = tid; j < cnt; j += TPB) {
    bool mine = entry_ok(idx, j, A.V, &bits);
    if (mine) {
      const int e = idx[j] - s.head;
      const int v = e / N - v0;
      if (e < 0 || e >= s.nvec * N) {
        mine = edges;
        const int x = e < 0 ? idx[j] : idx[j] - s.nvec * N;
        if (mine) atomicOr(&mark_extra, 1u << x);
      } else if (v < 0 || v >= TPB * NV) {
        mine = false;
      } else {
        const int at = (v % TPB) * NV + v / TPB;
        atomicOr(reinterpret_cast<uint32_t*>(mark) + (at >> 2), (1u << (e % N)) << ((at & 3) * 8));
      }
    }
    float t = 0.f, z = 0.f;
    if (mine) {
      t = load_val(A.val, A.val_format, row * A.k + j);
      z = (float)s.p[idx[j]];
      part = join(part, entry_part(t, z), A);
    }
    list.word[j] = mine ? idx[j] : -1;
    list.t[j] = t;
    list.z[j] = z;
  }
  if (MODE != kPart || blockIdx.y == 0) raise_status(A.status, bits);
  __syncthreads();
  // strike the listed words, then the maximum and the sum of what is left
  if ((mark_extra >> (tid < 32 ? tid : 31)) & (tid < 32 ? 1u : 0u)) ex = -kInf;
  float m = ex;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const uint32_t b = mark[tid * NV + i];
    if (b != 0u) r[i] = strike(r[i], b, type);
    m = max_packed(m, r[i], type);
  }
  const Product ref(m, A.a);
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float x[N];
    renew(r[i]);
    unpack(r[i], x, type);
    float e = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) e += exp2_(ref.exponent(x[n]));
    sum += e;
  }
  part.rm = m;
  part.rs = sum * ref.rest() + exp2_((ex - ref.m) * A.a);
  part = wave_join(part, A);
  if (lane == 0) red[tid >> 6] = part;
  __syncthreads();
  {
    const int o = lane < NW ? lane : 0;
    part = red[o];
    if (lane >= NW) part.rs = part.zs = part.ts = part.cross = 0.f;
    part = wave_join(part, A);
  }
  const bool odd = !Product::fits(part.rm, A.a);  // (the same for the whole workgroup)
  if (odd) {
    float e = 0.f;
    for (int i = tid; i < s.nvec * N; i += TPB) {
      const int v = i / N - v0, at = (v % TPB) * NV + v / TPB;
      if (v >= 0 && v < TPB * NV && !((mark[at] >> (i % N)) & 1u))
        e += exp2_(((float)s.p[s.head + i] - part.rm) * A.a);
    }
    e += exp2_((ex - part.rm) * A.a);
    part.rs = block_reduce<TPB>(e, fred, AddOp());
  }
  if constexpr (MODE == kPart) {
    if (tid == 0) parts[row * gridDim.y + blockIdx.y] = part;
  } else {
    const RowSums sums = row_sums(part, A, row);
    if (tid == 0) {
      A.loss[row] = sums.loss * w * (A.temperature * A.temperature);
      if (MODE == kLoss && A.stats != nullptr)
        A.stats[row] = make_float4(sums.rm, sums.rs, sums.zm, sums.zs);
    }
    if constexpr (MODE == kStep) {
      const GradScale g = grad_scale(sums, A, w * A.temperature);
      T* grad = static_cast<T*>(A.grad) + row * A.gld;
      const int tid2 = renew(tid);
      const Product from(g.rm, A.a);
      const float scale = g.rest * from.rest();
      if (!odd) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int v = i * TPB + tid2;
          float x[N];
          renew(r[i]);
          unpack(r[i], x, type);
#pragma unroll
          for (int n = 0; n < N; ++n) x[n] = exp2_(from.exponent(x[n])) * scale;
          if (v < s.nvec) store16(grad + s.head + (int64_t)v * N, pack(x, type));
        }
      } else {
        for (int i = s.head + tid; i < s.head + s.nvec * N; i += TPB)
          grad[i] = (T)(exp2_(((float)s.p[i] - g.rm) * A.a) * g.rest);
      }
      if (tid < s.extras) grad[s.extra(tid)] = (T)(exp2_((ex - g.rm) * A.a) * g.rest);
      __syncthreads();
      for (int j = tid; j < cnt; j += TPB)
        if (list.word[j] >= 0)
          grad[list.word[j]] = (T)(exp2_((list.z[j] - g.zm) * A.a) * g.list -
                                   teacher_prob(list.t[j], A.a, sums.t) * g.up);
    }
  }
}

// Sum of a row's chunk parts, by every wave of a workgroup.
__device__ __forceinline__ Part join_parts(const Part* parts, int n, const DistillArgs& A) {
  Part p = empty_part();
  for (int i = (int)(threadIdx.x & 63); i < n; i += 64) p = join(p, parts[i], A);
  return wave_join(p, A);
}

// loss and sums of a row from its parts, one wave a row: bound by its launch and two
// rounds of loads (at most 128 parts of 32 bytes a row)
__global__ __launch_bounds__(64) void k_distill_join(DistillArgs A, const Part* parts, int chunks) {
  const int64_t row = blockIdx.x;
  const float w = A.weight != nullptr ? A.weight[row] : 1.f;
  float loss = 0.f;
  float4 stats = make_float4(0.f, 0.f, 0.f, 0.f);
  if (used_entries(A, row) != 0 && w != 0.f) {
    const RowSums s = row_sums(join_parts(parts + row * chunks, chunks, A), A, row);
    loss = s.loss * w * (A.temperature * A.temperature);
    stats = make_float4(s.rm, s.rs, s.zm, s.zs);
  }
  if (threadIdx.x == 0) {
    A.loss[row] = loss;
    if (A.stats != nullptr) A.stats[row] = stats;
  }
}

// Gradient of one chunk (blockIdx.y of gridDim.y) of a row, from the saved
// sums or (parts != nullptr) from the parts of the row, then with the loss.
// Chunks of 32 KB, each with its share of the list: no thread holds more than eight
// vectors, so many workgroups hide the loads. Bound by memory: backward of 4,096 x 32,000
// bfloat16, an eighth of the rows without weight, 95 us, 5.2 TB/s read and written
// (chunks of 16 KB 113 us against 106 without such rows, of 64 KB 105).
template <typename T, int TPB, int NV>
__global__ __launch_bounds__(TPB) void k_distill_grad(DistillArgs A, const Part* parts) {
  constexpr int N = Span<T>::N, NW = TPB / 64;
  __shared__ ListLds list;
  __shared__ float2 red[NW];
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t row = blockIdx.x;
  T* grad = static_cast<T*>(A.grad) + row * A.gld;
  const int cnt = used_entries(A, row);
  const float w = A.weight != nullptr ? A.weight[row] : 1.f;
  if (cnt == 0 || w == 0.f) {
    zero_row<T, TPB>(grad, A.V, (int)blockIdx.y, (int)gridDim.y);
    if (parts != nullptr && blockIdx.y == 0 && tid == 0) A.loss[row] = 0.f;
    return;
  }
  const Span<T> s(static_cast<const T*>(A.z) + row * A.ld, A.V);
  const int v0 = (int)blockIdx.y * (TPB * NV);
  const bool edges = blockIdx.y == 0;
  const T* type = nullptr;
  uint4 r[NV];
  load_slots<T, TPB, NV, true>(r, s, v0);
  const float ex = edges && tid < s.extras ? (float)s.p[s.extra(tid)] : -kInf;
  // the list: this chunk's words with their logits, and the teacher's sum
  LogSum teach;
  uint32_t bits = 0u;
  const int32_t* idx = A.idx + row * A.k;
  for (int j = tid; j < cnt; j += TPB) {
    const bool ok = entry_ok(idx, j, A.V, &bits);
    bool mine = false;
    float t = 0.f, z = 0.f;
    if (ok) {
      const int e = idx[j] - s.head;
      mine = e < 0 || e >= s.nvec * N ? edges : e / N >= v0 && e / N < v0 + TPB * NV;
      t = load_val(A.val, A.val_format, row * A.k + j);
      teach.add(t, A.a);
      if (mine) z = (float)s.p[idx[j]];
    }
    list.word[j] = mine ? idx[j] : -1;
    list.t[j] = t;
    list.z[j] = z;
  }
  if (blockIdx.y == 0 && parts == nullptr) raise_status(A.status, bits);
  RowSums sums;
  if (parts != nullptr) {
    sums = row_sums(join_parts(parts + row * gridDim.y, (int)gridDim.y, A), A, row);
    if (blockIdx.y == 0 && tid == 0) A.loss[row] = sums.loss * w * (A.temperature * A.temperature);
    __syncthreads();
  } else {
    const float tm = wave_max(teach.m);
    const float ts = wave_sum(join_sum(teach.m, teach.S, tm, A.a));
    if (lane == 0) red[tid >> 6] = make_float2(tm, ts);
    __syncthreads();
    const float2 o = red[lane < NW ? lane : 0];
    teach.m = wave_max(o.x);
    teach.S = wave_sum(lane < NW ? join_sum(o.x, o.y, teach.m, A.a) : 0.f);
    const float4 st = A.stats[row];
    sums.t = teacher_of(teach, A, row);
    sums.rm = st.x;
    sums.rs = st.y;
    sums.zm = st.z;
    sums.zs = st.w;
  }
  const float up = w * A.temperature * (A.dloss != nullptr ? A.dloss[row] : 1.f);
  const GradScale g = grad_scale(sums, A, up);
  const int tid2 = renew(tid);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = v0 + i * TPB + tid2;
    float x[N];
    unpack(r[i], x, type);
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = exp2_((x[n] - g.rm) * A.a) * g.rest;
    if (v < s.nvec) store16(grad + s.head + (int64_t)v * N, pack(x, type));
  }
  if (edges && tid < s.extras) grad[s.extra(tid)] = (T)(exp2_((ex - g.rm) * A.a) * g.rest);
  __syncthreads();
  for (int j = tid; j < cnt; j += TPB)
    if (list.word[j] >= 0)
      grad[list.word[j]] = (T)(exp2_((list.z[j] - g.zm) * A.a) * g.list -
                               teacher_prob(list.t[j], A.a, sums.t) * g.up);
}

// ----------------------------------------------------------------------------
// verification

__device__ __forceinline__ int draft_length(const VerifyArgs& A, int64_t b) {
  if (A.length == nullptr) return A.draft;
  const int n = A.length[b];
  return n < 0 ? 0 : n < A.draft ? n : A.draft;
}

// probability of logit x in a row whose sum is v (a row without words: 0)
__device__ __forceinline__ float prob(float x, float a, LogSum v) {
  return v.m == -kInf && v.S == 0.f ? 0.f : exp2_((x - v.m) * a) / v.S;
}

// (m, S) of a wave's words. Where m is beyond what Product takes, S may be anything.
template <typename T, int NV>
__device__ __forceinline__ LogSum regs_sum(const uint4 (&r)[NV], float ex, float a) {
  constexpr int N = Span<T>::N;
  const T* type = nullptr;
  LogSum v;
  v.m = ex;
#pragma unroll
  for (int i = 0; i < NV; ++i) v.m = max_packed(v.m, r[i], type);
  const Product ref(v.m, a);
  v.S = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float x[N];
    uint4 w = r[i];
    renew(w);
    unpack(w, x, type);
    float e = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) e += exp2_(ref.exponent(x[n]));
    v.S += e;
  }
  v.S = v.S * ref.rest() + exp2_((ex - ref.m) * a);
  const float m = wave_max(v.m);
  v.S = wave_sum(join_sum(v.m, v.S, m, a));
  v.m = m;
  return v;
}

// S of vectors [v0, v0 + n) of a row and, where `edges`, its extras, from their
// maximum m by differences, by one wave.
template <typename T>
__device__ __forceinline__ float far_sum(const Span<T>& s, int v0, int n, bool edges, float m,
                                         float a) {
  const T* type = nullptr;
  const int lane = threadIdx.x & 63, end = v0 + n < s.nvec ? v0 + n : s.nvec;
  float sum = edges && lane < s.extras ? exp2_(((float)s.p[s.extra(lane)] - m) * a) : 0.f;
  for (int v = v0 + lane; v < end; v += 64) {
    float x[Span<T>::N];
    unpack(load16<false>(s.vec(v)), x, type);
#pragma unroll
    for (int i = 0; i < Span<T>::N; ++i) sum += exp2_((x[i] - m) * a);
  }
  return wave_sum(sum);
}

// Sums of the rows at one place of a sequence, or of one chunk of them:
// workgroup (place, sequence, chunk), places outermost. The last chunk to end
// joins the place's sums and decides about its token; a rejection is posted, and
// workgroups of later places that start after it leave at once, so a large
// batch reads little beyond each sequence's first rejection. Nothing waits.
// Bound by memory with five operations a word close behind: 256 x 8 x 65,536 binary16 62 to
// 67 us for the 231 MB up to the rejections, 3.6 TB/s, and some tenth more read in vain;
// 37 x 7 x 131,071 binary32 29 to 32 us. One sequence: 5 us, a chain of three device round trips.
template <typename T, int TPB, int NV, bool CHECK>
__global__ __launch_bounds__(TPB) void k_verify_sums(VerifyArgs A, VerifyScratch W, int chunks) {
  constexpr int NW = TPB / 64;
  __shared__ float4 red[NW];
  __shared__ uint32_t posted;  // (CHECK)
  const int tid = threadIdx.x, lane = tid & 63;
  const uint32_t unit = blockIdx.x, chunk = unit % (uint32_t)chunks;
  const int64_t b = (unit / (uint32_t)chunks) % (uint32_t)A.batch;
  const int place = (int)(unit / (uint32_t)chunks / (uint32_t)A.batch);
  const int len = draft_length(A, b);
  if (place > len) return;
  if (CHECK && place > 0) {
    if (tid == 0) posted = agent_load(&W.rejected[b]);
    __syncthreads();
    if (posted > (uint32_t)(TKEF_VERIFY_MAX_DRAFT + 1 - place)) return;
  }
  const bool drafted = place < len;
  const T* tp = static_cast<const T*>(A.target) + b * A.tb + place * A.ti;
  const T* dp = static_cast<const T*>(A.drafts) + b * A.db + (drafted ? place : 0) * A.di;
  const Span<T> ts(tp, A.V), ds(dp, A.V);
  const int v0 = (int)chunk * (TPB * NV);
  uint4 r[NV], q[NV];
  load_slots<T, TPB, NV, false>(r, ts, v0);
  if (drafted) load_slots<T, TPB, NV, false>(q, ds, v0);
  const float rx = chunk == 0u && tid < ts.extras ? (float)tp[ts.extra(tid)] : -kInf;
  const float qx = drafted && chunk == 0u && tid < ds.extras ? (float)dp[ds.extra(tid)] : -kInf;
  LogSum p = regs_sum<T, NV>(r, rx, A.a), d;
  if (drafted) d = regs_sum<T, NV>(q, qx, A.a);
  if (lane == 0) red[tid >> 6] = make_float4(p.m, p.S, d.m, d.S);
  __syncthreads();
  if (tid >= 64) return;
  // the first wave alone from here on
  float4 s = red[lane < NW ? lane : 0];
  if (lane >= NW) s.y = s.w = 0.f;
  float m0 = wave_max(s.x), m1 = wave_max(s.z);
  if (!Product::fits(m0, A.a)) {
    const float S = far_sum(ts, v0, TPB * NV, chunk == 0u, m0, A.a);
    s.x = m0;
    s.y = lane == 0 ? S : 0.f;
  }
  if (drafted && !Product::fits(m1, A.a)) {
    const float S = far_sum(ds, v0, TPB * NV, chunk == 0u, m1, A.a);
    s.z = m1;
    s.w = lane == 0 ? S : 0.f;
  }
  const int64_t at = b * (A.draft + 1) + place;
  if (chunks > 1) {
    const float s0 = wave_sum(join_sum(s.x, s.y, m0, A.a));
    const float s1 = wave_sum(join_sum(s.z, s.w, m1, A.a));
    float2* mine = W.parts + 2 * (at * chunks + chunk);
    uint32_t last = 0u;
    if (lane == 0) {
      agent_put(mine, m0, s0);
      agent_put(mine + 1, m1, s1);
      last = arrive_last(&W.arrived[at], (uint32_t)chunks) ? 1u : 0u;
    }
    if (__builtin_amdgcn_readfirstlane(last) == 0u) return;
    s = make_float4(-kInf, 0.f, -kInf, 0.f);
    for (int c = lane; c < chunks; c += 64) {
      const float2 o = agent_get(W.parts + 2 * (at * chunks + c));
      const float2 e = agent_get(W.parts + 2 * (at * chunks + c) + 1);
      m0 = fmaxf(s.x, o.x);
      m1 = fmaxf(s.z, e.x);
      s.y = join_sum(s.x, s.y, m0, A.a) + join_sum(o.x, o.y, m0, A.a);
      s.w = join_sum(s.z, s.w, m1, A.a) + join_sum(e.x, e.y, m1, A.a);
      s.x = m0;
      s.z = m1;
    }
  }
  p.m = wave_max(s.x);
  p.S = wave_sum(join_sum(s.x, s.y, p.m, A.a));
  d.m = wave_max(s.z);
  d.S = wave_sum(join_sum(s.z, s.w, d.m, A.a));
  if (lane != 0) return;
  W.sums[at] = make_float4(p.m, p.S, d.m, d.S);
  if (!drafted) return;
  const int x = A.tokens[b * A.draft + place];
  bool ok = x >= 0 && x < A.V;
  if (ok)
    ok = A.uniform[b * A.draft + place] * prob((float)dp[x], A.a, d) < prob((float)tp[x], A.a, p);
  if (!ok)
    __hip_atomic_fetch_max(&W.rejected[b], (uint32_t)(TKEF_VERIFY_MAX_DRAFT + 1 - place),
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// a candidate of the race: larger score first, then the lower word
__device__ __forceinline__ uint64_t race_key(float score, int word) {
  return ((uint64_t)__float_as_uint(score) << 32) | (0xFFFFFFFFu - (uint32_t)word);
}

// The race over one chunk (blockIdx.x) of the row after the accepted tokens of
// sequence blockIdx.y: the best word of the residual and, in case that is empty,
// of the target's own probabilities. The noise does not depend on where the
// drafts ended and is asked for first. The last chunk to end writes the
// sequence's results and leaves its counters at zero.
// Bound by memory: 256 x 65,536 binary16 28 us, 4.8 TB/s of two rows and the noise; one
// sequence 5 us. Kept apart from the sums: what it reads is known when they have ended.
template <typename T, int TPB, int NV>
__global__ __launch_bounds__(TPB) void k_verify_race(VerifyArgs A, VerifyScratch W) {
  constexpr int N = Span<T>::N, NW = TPB / 64;
  __shared__ uint64_t red[2][NW];
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t b = blockIdx.y;
  const int places = A.draft + 1;
  // vectors of N words from the row's start (any alignment), the last of them cut
  const float* noise = A.noise + b * A.noise_ld;
  const int nvec = A.V / N, v0 = (int)blockIdx.x * (TPB * NV) + tid;
  uint4 e[NV][N / 4];
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (v0 + i * TPB < nvec) {
#pragma unroll
      for (int h = 0; h < N / 4; ++h)
        e[i][h] = load16_loose(noise + (int64_t)(v0 + i * TPB) * N + 4 * h);
    }
  const int len = draft_length(A, b);
  // (0: none posted, a place beyond every length. What the workspace holds chooses among
  // the call's rows, tokens and words and never leads outside them, also where it
  // was not readied or something else wrote it.)
  const uint32_t place = (uint32_t)(TKEF_VERIFY_MAX_DRAFT + 1) - W.rejected[b];
  const int n = place < (uint32_t)len ? (int)place : len;
  const bool drafted = n < len;
  const T* type = nullptr;
  const T* tp = static_cast<const T*>(A.target) + b * A.tb + n * A.ti;
  const T* dp = static_cast<const T*>(A.drafts) + b * A.db + (drafted ? n : 0) * A.di;
  uint4 r[NV], q[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (v0 + i * TPB < nvec) {
      r[i] = load16_loose(tp + (int64_t)(v0 + i * TPB) * N);
      if (drafted) q[i] = load16_loose(dp + (int64_t)(v0 + i * TPB) * N);
    }
  const float4 s = W.sums[b * places + n];
  // p = 2^((x - pm) a) * pi; nothing where the row has no words
  const float pm = s.x == -kInf ? 0.f : s.x, qm = s.z == -kInf ? 0.f : s.z;
  const float pi = s.y == 0.f ? 0.f : 1.f / s.y, qi = s.w == 0.f ? 0.f : 1.f / s.w;
  // Scores are quotients, not products with the hardware's reciprocal: that is off by a
  // unit, and infinite for noise below 2^-126. (256 x 65,536 binary16 28 us, products 27;
  // two quotients a word, for the residual and for the target's own, 34.) A thread
  // meets its words in ascending order: a tie keeps the first.
  struct Best {
    float score = 0.f;
    int word = 0;
    __device__ void meet(float mass, float noise_of, int w) {
      const float q = mass > 0.f ? mass / noise_of : 0.f;
      word = q > score ? w : word;
      score = q > score ? q : score;
    }
    __device__ uint64_t key() const { return score > 0.f ? race_key(score, word) : 0ull; }
  };
  Best residual, target;
  float most = 0.f;  // largest p met
  const auto prob_of = [&](float x) { return exp2_((x - pm) * A.a) * pi; };
  const auto offer = [&](float x, float y, float noise_of, int word) {
    const float p = prob_of(x);
    most = fmaxf(most, p);
    residual.meet(drafted ? p - exp2_((y - qm) * A.a) * qi : p, noise_of, word);
  };
  const auto word_of_vec = [](const uint4 (&u)[N / 4], int j) {
    const uint4 h = u[j / 4];
    return __uint_as_float(j % 4 == 0 ? h.x : j % 4 == 1 ? h.y : j % 4 == 2 ? h.z : h.w);
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = v0 + i * TPB;
    if (v < nvec) {
      float x[N], y[N];
      unpack(r[i], x, type);
      unpack(drafted ? q[i] : none_of(type), y, type);
#pragma unroll
      for (int j = 0; j < N; ++j) offer(x[j], y[j], word_of_vec(e[i], j), v * N + j);
    }
  }
  // a word after the vectors, by a thread that has met lower words alone
  const int w = nvec * N + tid;
  const bool more = blockIdx.x == 0 && w < A.V;
  if (more) offer((float)tp[w], drafted ? (float)dp[w] : -kInf, noise[w], w);
  // The target's own probabilities count where the whole row's residual is empty, so
  // they are raced for by waves that met no residual, from memory again.
  if (drafted && __ballot(residual.score > 0.f) == 0ull && __ballot(most > 0.f) != 0ull) {
    for (int i = 0; i < NV; ++i) {
      const int v = v0 + i * TPB;
      if (v >= nvec) break;
      float x[N];
      unpack(load16_loose(tp + (int64_t)v * N), x, type);
      uint4 u[N / 4];
#pragma unroll
      for (int h = 0; h < N / 4; ++h) u[h] = load16_loose(noise + (int64_t)v * N + 4 * h);
#pragma unroll
      for (int j = 0; j < N; ++j) target.meet(prob_of(x[j]), word_of_vec(u, j), v * N + j);
    }
    if (more) target.meet(prob_of((float)tp[w]), noise[w], w);
  }
  if (blockIdx.x == 0 && tid < n) {  // the accepted drafts
    const int token = A.tokens[b * A.draft + tid];
    A.tokens_out[b * places + tid] = token;
    if (A.logp != nullptr) {
      const float4 at = W.sums[b * places + tid];
      const float x =
          (uint32_t)token < (uint32_t)A.V
              ? (float)static_cast<const T*>(A.target)[b * A.tb + tid * A.ti + token]
              : -kInf;
      A.logp[b * places + tid] = (x - at.x) * A.inv_t - kLn2 * log2_(at.y);
    }
  }
  uint64_t over = wave_max64(residual.key()), own = wave_max64(target.key());
  if (lane == 0) {
    red[0][tid >> 6] = over;
    red[1][tid >> 6] = own;
  }
  __syncthreads();
  if (tid >= 64) return;
  over = wave_max64(red[0][lane < NW ? lane : 0]);
  own = wave_max64(red[1][lane < NW ? lane : 0]);
  if (gridDim.x > 1) {
    uint32_t last = 0u;
    if (lane == 0) {
      __hip_atomic_fetch_max(&W.best[2 * b], over, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_fetch_max(&W.best[2 * b + 1], own, __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_AGENT);
      last = arrive_last(&W.raced[b], gridDim.x) ? 1u : 0u;
    }
    if (__builtin_amdgcn_readfirstlane(last) == 0u) return;
    over = agent_load(&W.best[2 * b]);
    own = agent_load(&W.best[2 * b + 1]);
  }
  const uint64_t key = over != 0ull ? over : own;
  const uint32_t best = 0xFFFFFFFFu - (uint32_t)key;
  const int word = key != 0ull && best < (uint32_t)A.V ? (int)best : -1;
  if (lane < places) {  // (at most 64)
    if (lane >= n) {
      const int token = lane == n ? word : -1;
      A.tokens_out[b * places + lane] = token;
      if (A.logp != nullptr)
        A.logp[b * places + lane] =
            token < 0 ? 0.f : ((float)tp[token] - s.x) * A.inv_t - kLn2 * log2_(s.y);
    }
    agent_store(&W.arrived[b * places + lane], 0u);
  }
  if (lane == 0) {
    A.accepted[b] = n;
    uint32_t bits = s.y != s.y || (drafted && s.w != s.w) ? TKEF_STATUS_NAN : 0u;
    if (drafted) {
      const int x = A.tokens[b * A.draft + n];
      if (x < 0 || x >= A.V) bits |= TKEF_STATUS_INDEX_RANGE;
    }
    raise_status(A.status, bits);
    agent_store(&W.rejected[b], 0u);
    agent_store(&W.raced[b], 0u);
    agent_store(&W.best[2 * b], (uint64_t)0);
    agent_store(&W.best[2 * b + 1], (uint64_t)0);
  }
}

}  // namespace

// Registers hold a row of up to 16 vectors for each of 1,024 threads.
constexpr int kRowVecs = 1024 * 16;
constexpr int kChunkVecs = 256 * 8;
// The loss alone needs a row once, so it need not be held: beyond 64 KB, where
// whole rows leave few workgroups a compute unit, chunks of it read faster
// (128,000 bfloat16 words: 3.6 -> 5.5 TB/s; 64,000 binary32: 4.2 -> 5.6).
constexpr int kLossVecs = 256 * 16;
// The step holds a row from its loss to its gradient, in chunks it reads it twice (2,048 x
// 64,000 bfloat16: 107 us whole, 146; 1,021 x 131,064: 134, 147). In chunks all the same
// where a row beyond 128 KB would take a compute unit to itself and leave most
// without one (128,000 bfloat16: 64 rows 23 us whole, 14; 96 rows 23, 18; 128 rows 23, 23).
constexpr int64_t kFewRows = 96;

namespace {

// A row's selection: whole in one workgroup of 256 threads while they hold it (64 KB)
// and k is at most 256, else in parts of that size. Two exceptions:
//   k <= 128: whole up to 128 KB, in 512 threads (2,048 x 32,000 binary32, k = 64: 59 us
//   against 66 in two parts; 2,048 x 64,000 bfloat16, k = 128: 89 and 80; 16 rows of
//   64,000: 13 and 19);
//   k > 256: rows up to 64 KB in parts of 16 KB and a merge (8,192 x 32,000 bfloat16, k =
//   300: 318 us, whole in 1,024 threads 1,030; k = 512: 392, 1,139; k = 1,000: 1,304, 1,573).
constexpr int kPartVecs = 256 * 16, kSmallPartVecs = 256 * 4;
// candidates that a merge in 256 and in 1,024 threads has LDS for: 21 KB, which leaves
// room for other rows beside it, and 74 KB (rows of k = 1,000 and longer lists)
constexpr int kMergeSmall = 2560, kMergeLarge = 9216;

TopParts top_parts(int64_t V, int64_t k, int32_t dtype) {
  TopParts p{};
  const int64_t vecs = V / (dtype == TKEF_DTYPE_F32 ? 4 : 8);
  const bool small = k > 256 && vecs <= kPartVecs;
  p.parts = vecs <= 512 * 16 && k <= 128
                ? 1
                : (int32_t)ceil_div(vecs, small ? kSmallPartVecs : kPartVecs);
  if (p.parts == 1 && k <= 256) return p;
  // a part's share of the k first and four standard deviations of it
  const double share = (double)k / p.parts;
  int64_t want = (int64_t)(share + 4.0 * std::sqrt(share)) + 8;
  p.want = (int32_t)(want < k ? want : k);
  p.room = (int32_t)((p.want + p.want / 8 + 2) * 8 + k);
  return p;
}

}  // namespace

size_t top_workspace(int64_t rows, int64_t V, int64_t k, int32_t dtype) {
  const TopParts p = top_parts(V, k, dtype);
  if (p.room == 0) return 0;
  return up256((size_t)rows * (size_t)p.parts * sizeof(PartHead)) +
         (size_t)rows * (size_t)p.parts * (size_t)p.room * 8;
}

hipError_t launch_top(const TopArgs& a, void* ws, hipStream_t s) {
  TopParts p = top_parts(a.V, a.k, a.dtype);
  const dim3 rows((unsigned)a.rows), split((unsigned)a.rows, (unsigned)p.parts);
  return by_dtype(a.dtype, [&](auto* t) {
    using T = typename Pointee<decltype(t)>::type;
    const int vecs = a.V / Span<T>::N;
    if (p.room != 0) {
      p.heads = static_cast<PartHead*>(ws);
      p.lists = reinterpret_cast<uint64_t*>(
          static_cast<char*>(ws) + up256((size_t)a.rows * (size_t)p.parts * sizeof(PartHead)));
      if (a.k > 256 && vecs <= kPartVecs)
        k_top_row<T, 256, 4, 4, true><<<split, 256, 0, s>>>(a, p);
      else if (p.want <= 64)
        k_top_row<T, 256, 16, 1, true><<<split, 256, 0, s>>>(a, p);
      else
        k_top_row<T, 256, 16, 4, true><<<split, 256, 0, s>>>(a, p);
      // Twice what the parts want. Longer lists (by ties, or where k nears the number
      // of vectors) go by top_radix, which takes rows that short two to four times faster than
      // the larger merge: 8,192 bfloat16 rows of 4,096 words, k = 600, 333 us, 1,081 merged;
      // 9,700 words, k = 1,000, 764 and 1,379.
      if (p.parts * (2 * p.want + 64) <= kMergeSmall)
        k_top_merge<T, 256, kMergeSmall><<<rows, 256, 0, s>>>(a, p);
      else
        k_top_merge<T, 1024, kMergeLarge><<<rows, 1024, 0, s>>>(a, p);
    } else if (vecs > kPartVecs) {
      k_top_row<T, 512, 16, 1, false><<<rows, 512, 0, s>>>(a, p);
    } else if (a.k <= 64) {
      // Shares of whole threads, 256 of them: 8,192 x 8,000 bfloat16, k = 64, 52 us, 79
      // with four shares a thread; k = 16 of 32,000 91 and 95. Two shares for k <= 128 (8,000
      // words, k = 128: 70 us, 98 with four; 32,000 128 and 128, k = 65 114 and 119), four for
      // k <= 256: more of them are more keys to bisect and more LDS, fewer workgroups. The
      // fewest vectors a thread that hold the row, for the same reason.
      if (vecs <= 256 * 4)
        k_top_row<T, 256, 4, 1, false><<<rows, 256, 0, s>>>(a, p);
      else if (vecs <= 256 * 8)
        k_top_row<T, 256, 8, 1, false><<<rows, 256, 0, s>>>(a, p);
      else
        k_top_row<T, 256, 16, 1, false><<<rows, 256, 0, s>>>(a, p);
    } else if (a.k <= 128) {
      if (vecs <= 256 * 4)
        k_top_row<T, 256, 4, 2, false><<<rows, 256, 0, s>>>(a, p);
      else if (vecs <= 256 * 8)
        k_top_row<T, 256, 8, 2, false><<<rows, 256, 0, s>>>(a, p);
      else
        k_top_row<T, 256, 16, 2, false><<<rows, 256, 0, s>>>(a, p);
    } else {
      if (vecs <= 256 * 4)
        k_top_row<T, 256, 4, 4, false><<<rows, 256, 0, s>>>(a, p);
      else if (vecs <= 256 * 8)
        k_top_row<T, 256, 8, 4, false><<<rows, 256, 0, s>>>(a, p);
      else
        k_top_row<T, 256, 16, 4, false><<<rows, 256, 0, s>>>(a, p);
    }
  });
}

int distill_chunks(int64_t V, int32_t dtype, int64_t rows, bool gradient) {
  const int64_t vecs = V / (dtype == TKEF_DTYPE_F32 ? 4 : 8);
  const int most = !gradient ? kLossVecs : rows <= kFewRows ? kRowVecs / 2 : kRowVecs;
  return vecs <= most ? 1 : (int)ceil_div(vecs, kChunkVecs);
}

namespace {

// LDS that a step over rows of up to 64 KB asks for beyond its own, so that a
// compute unit takes three of them: with their stores beside the others' loads
// more in flight are slower (8,192 x 32,000 bfloat16: 206 us at three, 213 at four,
// 220 at five, 220 at two; the loss alone, which only reads, takes five).
constexpr unsigned kStepSpare = 34 << 10;

template <typename T, int MODE>
void launch_row(const DistillArgs& a, hipStream_t s) {
  const int vecs = a.V / Span<T>::N;
  const dim3 grid((unsigned)a.rows);
  if (vecs <= 256 * 4)
    k_distill_row<T, 256, 4, MODE><<<grid, 256, 0, s>>>(a, nullptr);
  else if (vecs <= 256 * 8)
    k_distill_row<T, 256, 8, MODE><<<grid, 256, 0, s>>>(a, nullptr);
  else if (vecs <= 256 * 16)
    k_distill_row<T, 256, 16, MODE><<<grid, 256, MODE == kStep ? kStepSpare : 0, s>>>(a, nullptr);
  else if constexpr (MODE == kStep) {
    if (vecs <= 512 * 16)
      k_distill_row<T, 512, 16, MODE><<<grid, 512, 0, s>>>(a, nullptr);
    else
      k_distill_row<T, 1024, 16, MODE><<<grid, 1024, 0, s>>>(a, nullptr);
  }
}

template <typename T>
void launch_parts(const DistillArgs& a, Part* parts, int chunks, hipStream_t s) {
  k_distill_row<T, 256, 8, kPart>
      <<<dim3((unsigned)a.rows, (unsigned)chunks), 256, 0, s>>>(a, parts);
}

template <typename T>
void launch_grad(const DistillArgs& a, const Part* parts, hipStream_t s) {
  const int vecs = a.V / Span<T>::N;
  const int chunks = vecs > kChunkVecs ? (vecs + kChunkVecs - 1) / kChunkVecs : 1;
  k_distill_grad<T, 256, 8><<<dim3((unsigned)a.rows, (unsigned)chunks), 256, 0, s>>>(a, parts);
}

}  // namespace

hipError_t launch_distill_forward(const DistillArgs& a, void* ws, hipStream_t s) {
  const int chunks = distill_chunks(a.V, a.dtype, a.rows, false);
  Part* parts = static_cast<Part*>(ws);
  return by_dtype(a.dtype, [&](auto* t) {
    using T = typename Pointee<decltype(t)>::type;
    if (chunks == 1) {
      launch_row<T, kLoss>(a, s);
    } else {
      launch_parts<T>(a, parts, chunks, s);
      k_distill_join<<<dim3((unsigned)a.rows), 64, 0, s>>>(a, parts, chunks);
    }
  });
}

hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t s) {
  return by_dtype(a.dtype, [&](auto* t) {
    using T = typename Pointee<decltype(t)>::type;
    launch_grad<T>(a, nullptr, s);
  });
}

hipError_t launch_distill_step(const DistillArgs& a, void* ws, hipStream_t s) {
  const int chunks = distill_chunks(a.V, a.dtype, a.rows, true);
  Part* parts = static_cast<Part*>(ws);
  return by_dtype(a.dtype, [&](auto* t) {
    using T = typename Pointee<decltype(t)>::type;
    if (chunks == 1) {
      launch_row<T, kStep>(a, s);
      return;
    }
    launch_parts<T>(a, parts, chunks, s);
    launch_grad<T>(a, parts, s);
  });
}

// Places are summed in units of 512 threads x 4 vectors of each row (256 x 8 x 65,536
// binary16 with its race: 89 us; 1,024 x 4 93, 256 x 4 95, 1,024 x 8 96), three of them
// a compute unit for their dynamic LDS: what starts before a rejection is posted
// is read in vain (37 x 7 x 131,071 binary32: 49 us, 51 with four). Where those would
// leave compute units idle, smaller units that look for no rejection: 256 x 4 (sums of 64 x 5
// x 32,000 bfloat16 14.2 us, 14.8 in 512 x 4, 17.8 in 256 x 1; 200 x 5 x 32,000 with the race 46 in
// 256 x 4, 44 in 512 x 4) or 256 x 1 (one sequence 6.0 us, 6.2 in 256 x 4, 7.2 in 512 x 4).
namespace {
constexpr int kUnitVecs = 512 * 4, kSmallVecs = 256 * 4;
constexpr int64_t kFewUnits = 1024, kTinyUnits = 64;
constexpr unsigned kUnitSpare = 50 << 10;
}  // namespace

bool verify_fits(int64_t batch, int64_t draft, int64_t V, int32_t dtype) {
  const int64_t vecs = V / (dtype == TKEF_DTYPE_F32 ? 4 : 8);
  return batch * (draft + 1) * ceil_div(vecs, kUnitVecs) <= (int64_t)1 << 22;
}

VerifyLayout verify_layout(int64_t batch, int64_t draft, int64_t V, int32_t dtype) {
  const int64_t vecs = V / (dtype == TKEF_DTYPE_F32 ? 4 : 8);
  const int64_t places = batch * (draft + 1), big = ceil_div(vecs, kUnitVecs);
  // small units serve batches with fewer than kFewUnits big ones
  const int64_t small = (places * big < kFewUnits ? places * big : kFewUnits) * 8;
  const int64_t parts = places * big > small ? places * big : small;
  VerifyLayout l;
  l.best = 0;
  l.rejected = up256((size_t)batch * 16);
  l.raced = l.rejected + up256((size_t)batch * 4);
  l.arrived = l.raced + up256((size_t)batch * 4);
  l.zeroed = l.arrived + up256((size_t)places * 4);
  l.sums = l.zeroed;
  l.parts = l.sums + up256((size_t)places * sizeof(float4));
  l.bytes = l.parts + up256((size_t)parts * 2 * sizeof(float2));
  return l;
}

hipError_t launch_verify(const VerifyArgs& a, const VerifyScratch& w, hipStream_t s) {
  return by_dtype(a.dtype, [&](auto* t) {
    using T = typename Pointee<decltype(t)>::type;
    const int64_t vecs = a.V / Span<T>::N, places = (int64_t)a.batch * (a.draft + 1);
    const int64_t big = ceil_div(vecs, kUnitVecs);
    if (places * big > kFewUnits) {
      k_verify_sums<T, 512, 4, true>
          <<<dim3((unsigned)(places * big)), 512, kUnitSpare, s>>>(a, w, (int)big);
    } else if (places * big > kTinyUnits) {
      const int64_t small = ceil_div(vecs, kSmallVecs);
      k_verify_sums<T, 256, 4, false>
          <<<dim3((unsigned)(places * small)), 256, 0, s>>>(a, w, (int)small);
    } else {
      const int64_t tiny = ceil_div(vecs, 256);
      k_verify_sums<T, 256, 1, false>
          <<<dim3((unsigned)(places * tiny)), 256, 0, s>>>(a, w, (int)tiny);
    }
    // (chunks of 4 KB of a row where those of 16 KB would leave compute units idle: one
    // sequence of 32,000 bfloat16 words 5.8 us, 6.4; 64 of them 11.2, 8.5 in the large ones)
    if (a.batch * ceil_div(vecs, 256 * 4) <= 128)
      k_verify_race<T, 256, 1>
          <<<dim3((unsigned)ceil_div(vecs, 256), (unsigned)a.batch), 256, 0, s>>>(a, w);
    else
      k_verify_race<T, 256, 4>
          <<<dim3((unsigned)ceil_div(vecs, 256 * 4), (unsigned)a.batch), 256, 0, s>>>(a, w);
  });
}

}  // namespace tkef

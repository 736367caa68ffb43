// gfx950 kernels for the embedding of tokens and its gradient. The gradient is a
// sum over each word's tokens: the tokens are sorted by word (stable, so a word's
// tokens stay in their order), the sorted ones are summed in tiles, and the sums of words
// that cross tiles are joined in their order. Nothing is added atomically: the same
// call gives the same bits.
#include <type_traits>

#include <hip/hip_runtime.h>

#include "tkef.h"
#include "tkef_embed.h"
#include "tkef_rows_device.h"

#pragma clang fp contract(off)

namespace tkef {

namespace {

// ----------------------------------------------------------------------------
// vectors of E elements from any address of the element's alignment

typedef uint32_t loose2_ __attribute__((ext_vector_type(2), aligned(2)));

// E elements of a type as they lie in memory: 16 or 8 bytes
template <typename T, int E>
using Packed = std::conditional_t<E * sizeof(T) == 16, loose4_, loose2_>;

template <typename T, int E>
__device__ __forceinline__ void unpack_vec(Packed<T, E> v, float (&x)[E], const T* type) {
  if constexpr (E * sizeof(T) == 16) {
    unpack(make_uint4(v.x, v.y, v.z, v.w), x, type);
  } else {
    static_assert(E == 4 && sizeof(T) == 2, "8 bytes of a 16-bit type");
    float y[8];
    unpack(make_uint4(v.x, v.y, 0u, 0u), y, type);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = y[i];
  }
}

template <typename T, int E>
__device__ __forceinline__ void load_vec(const T* p, float (&x)[E]) {
  if constexpr (E * sizeof(T) == 32) {
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const loose4_ v = *reinterpret_cast<const loose4_*>(p + i);
      x[i] = __uint_as_float(v.x);
      x[i + 1] = __uint_as_float(v.y);
      x[i + 2] = __uint_as_float(v.z);
      x[i + 3] = __uint_as_float(v.w);
    }
  } else {
    unpack_vec<T, E>(*reinterpret_cast<const Packed<T, E>*>(p), x, p);
  }
}

template <typename T, int E>
__device__ __forceinline__ void store_vec(T* p, const float (&x)[E]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const float y[4] = {x[i], x[i + 1], x[i + 2], x[i + 3]};
      store16(p + i, pack(y, static_cast<const float*>(nullptr)));
    }
  } else if constexpr (E == 8) {
    store16(p, pack(x, static_cast<const T*>(nullptr)));
  } else {
    const float y[8] = {x[0], x[1], x[2], x[3], 0.f, 0.f, 0.f, 0.f};
    const uint4 u = pack(y, static_cast<const T*>(nullptr));
    const loose2_ v = {u.x, u.y};
    __builtin_nontemporal_store(v, reinterpret_cast<loose2_*>(p));
  }
}

// Elements of a thread: 16 bytes of what is written, so that a wave writes whole lines (with
// 8 columns of binary32 a thread's two stores leave every other 16 bytes to each other:
// k_embed_sum of 65,536 bfloat16 rows of 1,000 into binary32 took 57 us in place of 51).
template <typename O>
constexpr int vector_of() {
  return sizeof(O) == 4 ? 4 : 8;
}
// the same of sums that are written as R, or in lists
template <typename O, typename R, bool LISTS>
constexpr int vector_of_sums() {
  return LISTS || sizeof(R) == 4 || sizeof(O) == 4 ? 4 : 8;
}

// A workgroup of 256 threads holds 256 >> lg groups of 1 << lg threads; a group has a row
// (or a tile), thread l of it the columns from (slice << lg + l) E on. The last vector of a row
// whose width is no multiple of E lies back over its neighbour's columns, so that it is whole;
// its thread writes the last `have` of its columns, from `skip` on. (Rows shorter than a
// vector: skip == 0, have < E.)
struct Columns {
  int group, c0, skip, have;
  template <int E>
  __device__ static Columns of(int lg, int width) {
    Columns c;
    const int tid = (int)threadIdx.x, l = tid & ((1 << lg) - 1);
    c.group = tid >> lg;
    c.c0 = (((int)blockIdx.y << lg) + l) * E;
    const int left = width - c.c0;
    c.skip = 0;
    c.have = left < 0 ? 0 : left < E ? left : E;
    if (left > 0 && left < E && width >= E) {
      c.skip = E - left;
      c.c0 = width - E;
    }
    return c;
  }
  __device__ bool none() const { return have == 0; }
};

template <typename T, int E>
__device__ __forceinline__ void load_row(const T* row, const Columns& c, float (&x)[E]) {
  if (c.skip + c.have == E) {
    load_vec<T, E>(row + c.c0, x);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = i < c.have ? (float)row[i] : 0.f;
  }
}
template <typename T, int E>
__device__ __forceinline__ void store_row(T* row, const Columns& c, const float (&x)[E]) {
  if (c.have == E) {
    store_vec<T, E>(row + c.c0, x);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (i >= c.skip && i < c.skip + c.have) row[c.c0 + i] = (T)x[i];
  }
}

// A row of partial sums: read again soon, so not streamed as results are.
template <int E>
__device__ __forceinline__ void keep_row(float* row, const Columns& c, const float (&x)[E]) {
  if (c.skip + c.have == E) {  // (a shared column's values are the same)
#pragma unroll
    for (int i = 0; i < E; i += 4)
      *reinterpret_cast<loose4_*>(row + c.c0 + i) =
          loose4_{__float_as_uint(x[i]), __float_as_uint(x[i + 1]), __float_as_uint(x[i + 2]),
                  __float_as_uint(x[i + 3])};
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (i < c.have) row[i] = x[i];
  }
}

// ----------------------------------------------------------------------------
// lookup

// Row i of out, by a group: 65,536 tokens of a 32,000 x 1,024 bfloat16 table take 27 us, 6.0 TB/s
// of the rows that occur and of what is written, which is streamed: 49 us with ordinary stores.
template <typename T, typename O>
__global__ __launch_bounds__(256) void k_embed_rows(EmbedArgs A, int lg) {
  constexpr int E = vector_of<O>();
  const Columns c = Columns::of<E>(lg, A.width);
  const int64_t i = (int64_t)blockIdx.x * (256 >> lg) + c.group;
  if (i >= A.n || c.none()) return;
  const int32_t word = A.tokens[i];
  const bool in = word >= 0 && word < A.V;
  float x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = 0.f;
  if (in) {
    load_row<T, E>(static_cast<const T*>(A.table) + word * A.table_ld, c, x);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] *= A.scale;
  }
  store_row<O, E>(static_cast<O*>(A.out) + i * A.out_ld, c, x);
  raise_status(A.status, !in && word != -1 && c.c0 == 0 ? TKEF_STATUS_INDEX_RANGE : 0u);
}

// ----------------------------------------------------------------------------
// rows of words without tokens

constexpr int kRestRows = 2;  // rows of a group under way
constexpr uint32_t kLine = 128;

// The rows w0 + (absent[0 .. count) << shift) of the gradient: zeros, or the added rows as they
// are (U: their bits). A group of 1 << lg threads has a row, the slices from `slice` on.
template <typename U>
__device__ __forceinline__ void put_rest(const EmbedArgs& A, const uint16_t* absent, int count,
                                         int64_t w0, int shift, int lg, int slice, int step) {
  constexpr int E = 16 / (int)sizeof(U);
  const int tid = (int)threadIdx.x, groups = (int)blockDim.x >> lg;
  U* grad = static_cast<U*>(A.grad);
  const U* add = static_cast<const U*>(A.add);
  if (A.width < E) {
    for (int r = tid; r < count; r += (int)blockDim.x)
      for (int e = 0; e < A.width; ++e) {
        const int64_t w = w0 + ((int64_t)absent[r] << shift);
        grad[w * A.grad_ld + e] = add != nullptr ? add[w * A.add_ld + e] : (U)0;
      }
    return;
  }
  const auto at = [&](int c) { return c + E < A.width ? c : A.width - E; };
  if (add == nullptr) {
    // A wave writes whole lines: first the vectors up to a line's beginning, then the rest.
    // (Overlapping vectors write the same. 131,071 x 1,000 binary32 but for 300 rows: 129 us
    // from the row's beginning, 107 us so.)
    lg = lg < 6 ? lg : 6;
    const int l = tid & ((1 << lg) - 1);
    for (int r = tid >> lg; r < count; r += (int)blockDim.x >> lg) {
      U* row = grad + (w0 + ((int64_t)absent[r] << shift)) * A.grad_ld;
      const uint32_t past = (uint32_t)(reinterpret_cast<uintptr_t>(row) & (kLine - 1));
      const int head = lg < 3 || past == 0u ? 0 : (int)((kLine - past) / sizeof(U));
      const auto zero = [&](int c) {
        __builtin_nontemporal_store(loose4_{0u, 0u, 0u, 0u},
                                    reinterpret_cast<loose4_*>(row + at(c)));
      };
      if (slice == 0 && l * E < head) zero(l * E);
      for (int c = head + ((slice << lg) + l) * E; c < A.width; c += (step << lg) * E) zero(c);
    }
    return;
  }
  for (;; slice += step) {
    int c0 = ((slice << lg) + (tid & ((1 << lg) - 1))) * E;
    if (c0 >= A.width) break;
    c0 = at(c0);
    for (int r = tid >> lg; r < count; r += groups * kRestRows) {
      loose4_ x[kRestRows];
      int64_t w[kRestRows];
#pragma unroll
      for (int j = 0; j < kRestRows; ++j) {
        const int k = r + j * groups;
        w[j] = w0 + ((int64_t)absent[k < count ? k : r] << shift);
        x[j] = __builtin_nontemporal_load(
            reinterpret_cast<const loose4_*>(add + w[j] * A.add_ld + c0));
      }
#pragma unroll
      for (int j = 0; j < kRestRows; ++j)
        if (r + j * groups < count)
          __builtin_nontemporal_store(x[j],
                                      reinterpret_cast<loose4_*>(grad + w[j] * A.grad_ld + c0));
    }
  }
}

__device__ __forceinline__ void put_rest(const EmbedArgs& A, const uint16_t* absent, int count,
                                         int64_t w0, int shift, int lg, int slice, int step) {
  if (A.grad_dtype == TKEF_DTYPE_F32)
    put_rest<uint32_t>(A, absent, count, w0, shift, lg, slice, step);
  else
    put_rest<uint16_t>(A, absent, count, w0, shift, lg, slice, step);
}

// ----------------------------------------------------------------------------
// tokens sorted by word

// Words are sorted bin by bin, 1 << lgw of them a bin, by an id that says both: id >> lgw is
// the bin. Lists want ascending words, so the id is the word. The dense gradient does
// not: there the words of a bin lie 1 << lgb apart (`spread`), since the frequent words of most
// vocabularies follow one another, and the bin that holds the most tokens decides how long the
// sort takes (65,536 tokens of 32,000 by rank: 38% lie in the first 64 words).
struct Bins {
  int lgw, lgb, count;
  bool spread;
  __host__ __device__ int ids() const { return count << lgw; }
  __device__ int32_t id(int32_t word) const {
    return spread ? (word & ((1 << lgb) - 1)) << lgw | word >> lgb : word;
  }
  __device__ int32_t word(int32_t id) const {
    return spread ? (id & ((1 << lgw) - 1)) << lgb | id >> lgw : id;
  }
};

struct Token {
  int32_t at, id;
};

struct EmbedScratch {
  Token* sorted;    // the batch's tokens that are words, by id, then by place
  int32_t* slots;   // of each of them: its word's number among its bin's words that occur
  int32_t* first;   // each id's first place in `sorted`, and how many these are
  int32_t* bins;    // per bin: words that occur
  int32_t* before;  // per bin: words that occur in the bins before it
  float* partial;   // per tile: sums of the word that began before it, of the one that goes on
  Token* part;      // large batches: pieces of kPiece tokens, each by bin
  int32_t* ends;    // bin x piece: places of a bin's tokens in a piece (and behind the last's)
};

constexpr int kSortThreads = 1024;
constexpr int kSortAhead = 8;  // tokens a lane reads at once
constexpr int kMaxBinBits = 9;

// Lanes of the wave whose word (lgw bits of it) is the lane's own, among the lanes of `who`.
template <int MOST>
__device__ __forceinline__ uint64_t same_word(uint32_t word, int lgw, uint64_t who) {
  uint64_t same = who;
#pragma unroll
  for (int b = 0; b < MOST; ++b)
    if (b < lgw) {
      const bool one = (word >> b) & 1u;
      const uint64_t with = __ballot(one);
      same &= one ? with : ~with;
    }
  return same;
}

__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                        __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

// Orders a wave's LDS accesses, which the hardware keeps in program order, for the compiler.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Large batches: each workgroup puts a piece of the batch in the order of its bins (stable,
// wave w has the w-th part of it), so that a bin's workgroup reads its own tokens alone.
// Latencies bound it: 65,536 tokens take 8 us and 13 in k_embed_sort, where they take 59 there
// alone; 16,384 take 8 + 12 against 20, which is where splitting begins.
constexpr int kPiece = 2048, kMaxPieces = TKEF_EMBED_MAX_ROWS / kPiece;
static_assert(kMaxPieces <= kSortThreads, "a thread for each piece");
constexpr int kSplitThreads = 256, kSplitWaves = kSplitThreads / 64;
constexpr int kSplitAhead = kPiece / kSplitThreads;
constexpr int kMaxBins = 1 << (20 - kMaxBinBits);
static_assert(TKEF_ROWS_MAX_VOCAB <= kMaxBins << kMaxBinBits, "bins of a vocabulary");

__global__ __launch_bounds__(kSplitThreads) void k_embed_split(EmbedArgs A, EmbedScratch W, Bins B,
                                                               int pieces) {
  extern __shared__ uint32_t hist[];  // wave x bin
  __shared__ uint32_t red[kSplitWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, bins = B.count;
  const int begin = (int)blockIdx.x * kPiece + wave * (64 * kSplitAhead);
  int32_t t[kSplitAhead];
#pragma unroll
  for (int j = 0; j < kSplitAhead; ++j) {
    const int i = begin + j * 64 + lane;
    t[j] = i < A.n ? A.tokens[i] : -1;
  }
  for (int i = tid; i < bins * kSplitWaves; i += kSplitThreads) hist[i] = 0u;
  __syncthreads();
  uint32_t* mine = hist + wave * bins;
  uint32_t bits = 0u;
#pragma unroll
  for (int j = 0; j < kSplitAhead; ++j) {
    const bool in = t[j] >= 0 && t[j] < A.V;
    if (!in && t[j] != -1) bits = TKEF_STATUS_INDEX_RANGE;
    t[j] = in ? B.id(t[j]) : -1;
    if (in) atomicAdd(&mine[t[j] >> B.lgw], 1u);
  }
  raise_status(A.status, bits);
  __syncthreads();
  // places of each bin, and of each wave's share of it: a thread has `each` bins
  const int each = (bins + kSplitThreads - 1) / kSplitThreads;
  const int b0 = tid * each, b1 = b0 + each < bins ? b0 + each : bins;
  uint32_t count = 0u, all;
  for (int b = b0; b < b1; ++b)
    for (int v = 0; v < kSplitWaves; ++v) count += hist[v * bins + b];
  uint32_t place = block_scan<kSplitThreads>(count, red, &all);
  for (int b = b0; b < b1; ++b) {
    W.ends[(int64_t)b * pieces + blockIdx.x] = (int32_t)place;
    for (int v = 0; v < kSplitWaves; ++v) {
      const uint32_t c = hist[v * bins + b];
      hist[v * bins + b] = place;
      place += c;
    }
  }
  if (tid == 0) W.ends[(int64_t)bins * pieces + blockIdx.x] = (int32_t)all;
  __syncthreads();
  const int lgb = 32 - __builtin_clz((uint32_t)bins);  // (bins at least 1)
  Token* out = W.part + (int64_t)blockIdx.x * kPiece;
#pragma unroll
  for (int j = 0; j < kSplitAhead; ++j) {
    const bool own = t[j] >= 0;
    const uint64_t who = __ballot(own);
    if (who == 0ull) continue;
    const uint32_t bin = own ? (uint32_t)t[j] >> B.lgw : 0u;
    const uint64_t same = same_word<20 - kMaxBinBits + 1>(bin, lgb, who);
    const int rank = lanes_below(same);
    const uint32_t at = mine[bin] + (uint32_t)rank;
    wave_fence();  // every lane has read before one writes, and before the next 64 read
    if (own) {
      out[at] = Token{begin + j * 64 + lane, t[j]};
      if (rank == 0) mine[bin] = at + (uint32_t)__popcll(same);
    }
    wave_fence();
  }
}

// Workgroup b sorts the tokens of bin b: it reads the tokens, counts its own word by word (and
// those of lower bins, which come before), and in a second reading puts its own in place; between
// them it writes the gradient's rows of words that do not occur (rest_lg >= 0). Wave w has the
// w-th share of the tokens, so a word's tokens are in the batch's order: waves in turn, and in a
// wave, lanes.
// PIECES: its tokens lie in the pieces that k_embed_split made; else all tokens are read.
// Without rows to write 1,000 tokens take 6 us, 8,192 11 us, a chain of barriers and LDS; the
// 66 MB of zeros of 32,000 x 512 hide behind it but for 5 us. The 131,071 x 1,000 rows beside
// 65,536 tokens are written at 4.9 TB/s, and copied at 4.8 TB/s read and written. (PIECES: 8 of its
// registers lie in scratch, 36 bytes a thread, so that two workgroups of 1,024 share a compute unit.)
// NT: 256 threads for up to 2,048 tokens (1,000: 6.4 us, 8.6 with 1,024 threads).
template <bool PIECES, int NT>
__global__ __launch_bounds__(NT, 8) void k_embed_sort(EmbedArgs A, EmbedScratch W, Bins B,
                                                     int rest_lg) {
  extern __shared__ uint32_t hist[];  // wave x word
  constexpr int NW = NT / 64;
  __shared__ uint32_t red[NW], below_of[NW];
  __shared__ uint32_t slot_of[1 << kMaxBinBits];
  __shared__ uint16_t absent[1 << kMaxBinBits];
  // of each piece: the bin's tokens before it, and where (less those) its own lie
  __shared__ int32_t piece_of[PIECES ? kMaxPieces : 1], part_of[PIECES ? kMaxPieces : 1];
  constexpr int kAhead = PIECES ? 4 : kSortAhead;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int words = 1 << B.lgw;
  const int32_t w0 = (int32_t)blockIdx.x << B.lgw;  // ids from here on
  const int pieces = (int)((A.n + kPiece - 1) / kPiece);
  int n = (int)A.n;
  uint32_t below = 0u, bits = 0u;
  if constexpr (PIECES) {
    uint32_t own = 0u, total;
    const int64_t at = (int64_t)blockIdx.x * pieces + tid;
    if (tid < pieces) {
      below = (uint32_t)W.ends[at];
      own = (uint32_t)W.ends[at + pieces] - below;
    }
    const uint32_t before = block_scan<NT>(own, red, &total);
    if (tid < pieces) {
      piece_of[tid] = (int32_t)before;
      part_of[tid] = tid * kPiece + (int32_t)(below - before);
    }
    n = (int)total;
    __syncthreads();
  }
  const int per = ((n + NT - 1) / NT) * 64;
  const int begin = wave * per, end = begin + per < n ? begin + per : n;
  int32_t t[kAhead], at_[PIECES ? kAhead : 1];
  const auto read = [&](int from) {
    if constexpr (PIECES) {
      int piece[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) piece[j] = 0;
      for (int step = 1 << (31 - __builtin_clz((uint32_t)pieces)); step > 0; step >>= 1)
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int p = piece[j] + step;
          if (p < pieces && piece_of[p] <= from + j * 64 + lane) piece[j] = p;
        }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = from + j * 64 + lane;
        const Token none = {0, -1};
        const Token k = i < end ? W.part[part_of[piece[j]] + i] : none;
        t[j] = k.id;
        at_[j] = k.at;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = from + j * 64 + lane;
        t[j] = i < end ? A.tokens[i] : -1;
      }
    }
  };
  // whether t is a word of the bin: its number there, else -1
  const auto own_of = [&](int32_t t_) {
    const int32_t number = (PIECES ? t_ : B.id(t_)) - w0;
    const bool in = PIECES ? t_ >= 0 : (uint32_t)t_ < (uint32_t)A.V;
    return in && (uint32_t)number < (uint32_t)words ? number : -1;
  };
  read(begin);
  for (int i = tid; i < words * NW; i += NT) hist[i] = 0u;
  __syncthreads();
  uint32_t* mine = hist + wave * words;
  for (int from = begin;;) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if constexpr (!PIECES) {
        const bool in = (uint32_t)t[j] < (uint32_t)A.V;
        if (!in && t[j] != -1) bits = TKEF_STATUS_INDEX_RANGE;
        below += in && B.id(t[j]) < w0 ? 1u : 0u;
      }
      t[j] = own_of(t[j]);
      if (t[j] >= 0) atomicAdd(&mine[t[j]], 1u);
    }
    from += kAhead * 64;
    if (from >= end) break;
    read(from);
  }
  if (blockIdx.x == 0) raise_status(A.status, bits);
  const bool again = per > kAhead * 64;
  if (again) read(begin);
  below = wave_incl(below);
  if (lane == 63) below_of[wave] = below;
  __syncthreads();
  uint32_t at = 0u;
#pragma unroll
  for (int w = 0; w < NW; ++w) at += below_of[w];
  // places of each word, and of each wave's share of it; both counts in one scan (at most
  // 2^20 tokens, 2^9 words)
  uint32_t count = 0u, all;
  if (tid < words)
    for (int v = 0; v < NW; ++v) count += hist[v * words + tid];
  const uint32_t ahead = block_scan<NT>(count | (count > 0u ? 1u << 21 : 0u), red, &all);
  if (tid < words) {
    uint32_t place = at + (ahead & ((1u << 21) - 1u));
    W.first[w0 + tid] = (int32_t)place;
    if (w0 + tid == B.ids() - 1) W.first[B.ids()] = (int32_t)(place + count);
    slot_of[tid] = ahead >> 21;
    if (count == 0u) absent[tid - (int)(ahead >> 21)] = (uint16_t)tid;
    for (int v = 0; v < NW; ++v) {
      const uint32_t c = hist[v * words + tid];
      hist[v * words + tid] = place;
      place += c;
    }
  }
  if (tid == 0) W.bins[blockIdx.x] = (int32_t)(all >> 21);
  __syncthreads();
  if (rest_lg >= 0) {
    // words of the bin (those that the vocabulary does not reach come last)
    const int b = (int)blockIdx.x, base = B.spread ? b : w0, shift = B.spread ? B.lgb : 0;
    const int reach = A.V > base ? ((A.V - 1 - base) >> shift) + 1 : 0;
    put_rest(A, absent, (reach < words ? reach : words) - (int)(all >> 21), base, shift, rest_lg, 0,
             1);
  }
  for (int from = begin;;) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (again) t[j] = own_of(t[j]);
      const bool own = t[j] >= 0;
      const uint64_t who = __ballot(own);
      if (who == 0ull) continue;
      const uint32_t word = own ? (uint32_t)t[j] : 0u;
      const uint64_t same = same_word<kMaxBinBits>(word, B.lgw, who);
      const int rank = lanes_below(same);
      const uint32_t place = mine[word] + (uint32_t)rank;
      wave_fence();  // every lane has read before one writes, and before the next 64 read
      if (own) {
        W.sorted[place] = Token{PIECES ? at_[PIECES ? j : 0] : from + j * 64 + lane, w0 + t[j]};
        if (A.nnz != nullptr) W.slots[place] = (int32_t)slot_of[word];
        if (rank == 0) mine[word] = place + (uint32_t)__popcll(same);
      }
      wave_fence();
    }
    from += kAhead * 64;
    if (from >= end) break;
    read(from);
  }
}

// ----------------------------------------------------------------------------
// sums

// Where a word's sum goes: a row of the gradient (R: its type), with another gradient's row
// added, or a piece of the lists (R: of their values), the number-th. Rounded once.
template <typename R, bool LISTS, int E>
__device__ __forceinline__ void put_sum(const EmbedArgs& A, int32_t word, int32_t number,
                                        const Columns& c, float (&x)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] *= A.scale;
  if constexpr (LISTS) {
    const int64_t o = (int64_t)number * A.width;
    const int32_t p = (int32_t)(A.offset + (int64_t)word * A.width + c.c0);
    if (c.have == E) {
#pragma unroll
      for (int e = 0; e < E; e += 4)
        store16(A.idx + o + c.c0 + e, make_uint4((uint32_t)(p + e), (uint32_t)(p + e + 1),
                                                 (uint32_t)(p + e + 2), (uint32_t)(p + e + 3)));
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e >= c.skip && e < c.skip + c.have) A.idx[o + c.c0 + e] = p + e;
    }
    store_row<R, E>(static_cast<R*>(A.val) + o, c, x);
  } else {
    if (A.add != nullptr) {
      float y[E];
      load_row<R, E>(static_cast<const R*>(A.add) + word * A.add_ld, c, y);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] += y[e];
    }
    store_row<R, E>(static_cast<R*>(A.grad) + word * A.grad_ld, c, x);
  }
}

// Rows of dout, K of them under way.
template <typename O, int E, int K>
__device__ __forceinline__ void load_rows(Packed<O, E> (&raw)[K], const O* dout, int64_t ld,
                                          const int32_t (&at)[K], const Columns& c) {
  if (c.skip + c.have == E) {
#pragma unroll
    for (int j = 0; j < K; ++j)
      raw[j] = *reinterpret_cast<const Packed<O, E>*>(dout + at[j] * ld + c.c0);
  } else {
#pragma unroll
    for (int j = 0; j < K; ++j) {
      O x[E];
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = i < c.have ? dout[at[j] * ld + i] : (O)0.f;
      raw[j] = __builtin_bit_cast(Packed<O, E>, x);
    }
  }
}

constexpr int kAhead = 8, kWaveAhead = 16;  // rows of a tile under way

// Group g sums the sorted tokens [g tile, (g + 1) tile). A word that lies within them is
// done; the sums of one that began before them, and of one that goes on behind them, are
// left for k_embed_join.
// WAVE: groups of whole waves. Lane l reads the tile's token l - 1, beside the number of tokens,
// and hands it on in a scalar register: one access and one address for a row, and a branch where
// the word changes.
// A tile is a chain of the tokens, their rows and the results, so it is short: 16 tokens up to
// 65,536 of them, whose rows are under way together (groups of whole waves; others 8 at a time),
// and 32 to 256 beyond, so that the joins have at most 4,096 tiles. 8,192 rows of 512 bfloat16 take
// 6.7 us. 57,344 of 1,000 with another gradient's rows added take 70 us, 4 TB/s of rows that lie
// apart.
template <typename O, typename R, bool LISTS, bool WAVE>
__global__ __launch_bounds__(256) void k_embed_sum(EmbedArgs A, EmbedScratch W, Bins B, int lg,
                                                   int tile) {
  constexpr int E = vector_of_sums<O, R, LISTS>();
  __shared__ int32_t number_of[LISTS ? kMaxBins : 1];
  __shared__ uint32_t red[4];
  Columns c = Columns::of<E>(lg, A.width);
  if constexpr (WAVE) c.group = __builtin_amdgcn_readfirstlane(c.group);
  const int64_t g = (int64_t)blockIdx.x * (256 >> lg) + c.group;
  const int lane = threadIdx.x & 63;
  // the token at p - 1 + lane (places behind the last lie in the workspace, but hold none)
  Token mine = {0, -1};
  int32_t my_slot = 0;
  const auto read = [&](int64_t p) {
    int64_t q = p - 1 + (lane < kWaveAhead + 2 ? lane : kWaveAhead + 1);
    q = q < 0 ? 0 : q < A.n ? q : A.n - 1;
    mine = W.sorted[q];
    if constexpr (LISTS) my_slot = W.slots[q];
  };
  if constexpr (WAVE) read(g * tile);
  const int total = W.first[B.ids()];
  if constexpr (LISTS) {
    // words that occur before each bin's: a thread has kEach bins
    constexpr int kEach = kMaxBins / 256;
    const int bins = B.count, b0 = (int)threadIdx.x * kEach;
    const bool writes = blockIdx.x == 0 && blockIdx.y == 0;
    uint32_t of[kEach], own = 0u, done;
#pragma unroll
    for (int i = 0; i < kEach; ++i) of[i] = b0 + i < bins ? (uint32_t)W.bins[b0 + i] : 0u;
#pragma unroll
    for (int i = 0; i < kEach; ++i) own += of[i];
    uint32_t before = block_scan<256>(own, red, &done);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      number_of[b0 + i] = (int32_t)before;
      if (writes && b0 + i < bins) W.before[b0 + i] = (int32_t)before;
      before += of[i];
    }
    if (writes && threadIdx.x == 0) *A.nnz = (int32_t)(done * (uint32_t)A.width);
    __syncthreads();
  }
  if (g * tile >= total || (!WAVE && c.none())) return;
  const int p0 = (int)g * tile, p1 = p0 + tile < total ? p0 + tile : total;
  const O* dout = static_cast<const O*>(A.dout);
  // the words before and behind the tile
  int32_t left = -1, right = -1;
  if constexpr (!WAVE) {
    if (p0 > 0) left = W.sorted[p0 - 1].id;
    if (p1 < total) right = W.sorted[p1].id;
  }
  float sum[E];
  int32_t id = -1, number = 0;
  const auto flush = [&]() {
    const bool before = id == left, behind = id == right;
    if (before || behind)
      keep_row<E>(W.partial + (2 * g + (before ? 0 : 1)) * A.width, c, sum);
    else
      put_sum<R, LISTS, E>(A, B.word(id), number, c, sum);
  };
  if constexpr (WAVE) {
    if (c.none()) {  // reads the last columns, writes nothing
      c.c0 = A.width - E;
      c.skip = E;
    }
    if (p0 > 0) left = __builtin_amdgcn_readlane(mine.id, 0);
    for (int p = p0;;) {
      const int count = p1 - p < kWaveAhead ? p1 - p : kWaveAhead;
      Packed<O, E> raw[kWaveAhead];
#pragma unroll
      for (int j = 0; j < kWaveAhead; ++j) {
        const int32_t at = __builtin_amdgcn_readlane(mine.at, 1 + (j < count ? j : count - 1));
        raw[j] = *reinterpret_cast<const Packed<O, E>*>(dout + at * A.out_ld + c.c0);
      }
      if (p + count == p1 && p1 < total) right = __builtin_amdgcn_readlane(mine.id, 1 + count);
#pragma unroll
      for (int j = 0; j < kWaveAhead; ++j)
        if (j < count) {
          float x[E];
          unpack_vec<O, E>(raw[j], x, dout);
          const int32_t next = __builtin_amdgcn_readlane(mine.id, 1 + j);
          if (next != id) {
            if (id >= 0) flush();
            id = next;
            if constexpr (LISTS)
              number = number_of[id >> B.lgw] + __builtin_amdgcn_readlane(my_slot, 1 + j);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] = x[e];
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += x[e];
          }
        }
      p += count;
      if (p >= p1) break;
      read(p);
    }
    flush();
    return;
  }
  for (int p = p0; p < p1; p += kAhead) {
    int32_t at[kAhead], of[kAhead], slot[LISTS ? kAhead : 1];
    Packed<O, E> raw[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int q = p + j < p1 ? p + j : p1 - 1;
      const Token t = W.sorted[q];
      at[j] = t.at;
      of[j] = t.id;
      if constexpr (LISTS) slot[j] = W.slots[q];
    }
    load_rows<O, E, kAhead>(raw, dout, A.out_ld, at, c);
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (p + j < p1) {
        float x[E];
        unpack_vec<O, E>(raw[j], x, dout);
        if (of[j] != id) {
          if (id >= 0) flush();
          id = of[j];
          if constexpr (LISTS) number = number_of[id >> B.lgw] + slot[j];
#pragma unroll
          for (int e = 0; e < E; ++e) sum[e] = x[e];
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) sum[e] += x[e];
        }
      }
  }
  flush();
}

// Partial sums [begin, end) of the word that goes on behind tile h0, in their order.
constexpr int kJoin = 8;  // under way
template <int E>
__device__ __forceinline__ void join_terms(const float* partial, int width, int h0, int begin,
                                           int end, const Columns& c, float (&sum)[E]) {
  for (int i = begin; i < end; i += kJoin) {
    float x[kJoin][E];
#pragma unroll
    for (int j = 0; j < kJoin; ++j)
      if (i + j < end) {
        const int64_t h = h0 + i + j;
        load_row<float, E>(partial + (2 * h + (i + j == 0 ? 1 : 0)) * width, c, x[j]);
      }
#pragma unroll
    for (int j = 0; j < kJoin; ++j)
      if (i + j < end) {
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = i + j == begin ? x[j][e] : sum[e] + x[j][e];
      }
  }
}

// The words that begin in a tile and go on behind it: their sums, tile after tile. The
// workgroups of a window (gridDim.z) look at its 64 tiles; each group takes one of the words of
// few tiles. Longer ones a workgroup takes together: its groups have equal parts of the
// tiles, which the first joins. A chain as well: 5 us for 8,192 tokens of 512 columns, 13 us for
// 57,344 of 1,000, whose most frequent word has 123 tiles. (NT: 256 threads where batches are not
// split, else 1,024: 65,536 tokens of 1,000 x 512 take 10 us with 1,024, 14 with 512, 24 with 256;
// the call of 8,192 tokens takes 27.8 us with 1,024, 26.9 with 256. There a word of three tiles is
// better shared by a workgroup's groups: 27.0 us, and 28.6 where a group takes up to eight.)
constexpr int kWindow = 64;
template <typename R, bool LISTS, int NT>
__global__ __launch_bounds__(NT) void k_embed_join(EmbedArgs A, EmbedScratch W, Bins B, int lg,
                                                    int tile, int tiles) {
  // tiles that a group takes alone, and of its part of more
  constexpr int E = 8, kAlone = NT == 256 ? 2 : kJoin, kLeast = NT == 256 ? 1 : kJoin;
  struct Word {
    int32_t h0, terms, id, number;
  };
  __shared__ float sums[NT][E];
  __shared__ Word few[kWindow], many[kWindow];
  __shared__ int found[2];
  const Columns c = Columns::of<E>(lg, A.width);
  const int tid = threadIdx.x, groups = NT >> lg;
  if (tid < kWindow) {
    const int g = (int)blockIdx.x * kWindow + tid;
    // (all read at once: places behind the last token hold no words, but lie in the workspace)
    const bool in = g + 1 < tiles;
    const int p0 = g * tile, p1 = p0 + tile, total = W.first[B.ids()];
    const int32_t left = in && p0 > 0 ? W.sorted[p0 - 1].id : -1;
    const int32_t id = in ? W.sorted[p1 - 1].id : -1, right = in ? W.sorted[p1].id : -1;
    const bool begins = in && p1 < total && id == right && id != left;
    Word w = {g, 0, id, 0};
    if (begins) {
      w.terms = (W.first[id + 1] - 1) / tile - g + 1;
      if constexpr (LISTS) w.number = W.before[id >> B.lgw] + W.slots[p1 - 1];
    }
    const uint64_t is_few = __ballot(begins && w.terms <= kAlone);
    const uint64_t is_many = __ballot(begins && w.terms > kAlone);
    if (begins) {
      if (w.terms <= kAlone)
        few[lanes_below(is_few)] = w;
      else
        many[lanes_below(is_many)] = w;
    }
    if (tid == 0) {
      found[0] = __popcll(is_few);
      found[1] = __popcll(is_many);
    }
  }
  __syncthreads();
  float sum[E];
  for (int k = (int)blockIdx.z * groups + c.group; k < found[0]; k += (int)gridDim.z * groups) {
    if (c.none()) break;
    const Word w = few[k];
    join_terms<E>(W.partial, A.width, w.h0, 0, w.terms, c, sum);
    put_sum<R, LISTS, E>(A, B.word(w.id), w.number, c, sum);
  }
  for (int k = (int)blockIdx.z; k < found[1]; k += (int)gridDim.z) {
    const Word w = many[k];
    const int share = (w.terms + groups - 1) / groups, per = share < kLeast ? kLeast : share;
    const int begin = c.group * per, end = begin + per < w.terms ? begin + per : w.terms;
    if (!c.none() && begin < end) {
      join_terms<E>(W.partial, A.width, w.h0, begin, end, c, sum);
#pragma unroll
      for (int e = 0; e < E; ++e) sums[tid][e] = sum[e];
    }
    __syncthreads();
    if (c.group == 0 && !c.none()) {
      for (int q = 1; q * per < w.terms; ++q)
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += sums[(q << lg) + tid][e];
      put_sum<R, LISTS, E>(A, B.word(w.id), w.number, c, sum);
    }
    __syncthreads();
  }
}

// ----------------------------------------------------------------------------
// few tokens: one launch, no workspace

constexpr int kFew = 256, kFewWords = 16, kFewAhead = 8;
// Tokens up to which a list is made so. Its search for earlier equal words goes through LDS token
// by token, 0.065 us each: of 32,000 x 515 binary32 10.7 us for 128 tokens, 14.9 for 192, 17.1 for
// 224 and 18.9 for 256, as sort, sums and join 15.9, 17.2, 17.0 and 17.6; of 512 bfloat16 ->
// binary16, 10.2, 14.5, 16.6 and 18.4 against 13.3, 14.2, 14.1 and 14.7. (The dense gradient, which
// has no such search: 13.9 us for 256 tokens, 23.2 as sort, sums and join for 257.)
constexpr int kFewList = 224;

// (a list of 37 tokens: 5.5 us, and 18 as sort, sums and join)
// Each workgroup reads all tokens. A group (of whole waves) has token i; if no earlier
// one is of its word, it sums the word's rows. Of the dense gradient, workgroups from
// `token_blocks` on write the rows of words that do not occur, kFewWords each.
template <typename O, typename R, bool LISTS>
__global__ __launch_bounds__(kFew) void k_embed_few(EmbedArgs A, int lg, int token_blocks,
                                                    int rest_lg) {
  constexpr int E = vector_of_sums<O, R, LISTS>(), kParts = kFew / 64;
  __shared__ int32_t word_at[kFew];
  __shared__ int32_t distinct[LISTS ? kFew : 1];
  __shared__ uint16_t absent[LISTS ? 1 : kFewWords];
  const int tid = threadIdx.x, lane = tid & 63, n = (int)A.n;
  int32_t mine = tid < n ? A.tokens[tid] : -1;
  if (mine < 0 || mine >= A.V) {
    if (mine != -1 && blockIdx.x == 0 && blockIdx.y == 0)
      raise_status(A.status, TKEF_STATUS_INDEX_RANGE);
    mine = -1;
  }
  word_at[tid] = mine;
  __syncthreads();
  int32_t tok[kParts];
#pragma unroll
  for (int i = 0; i < kParts; ++i) tok[i] = word_at[i * 64 + lane];
  if constexpr (!LISTS) {
    if ((int)blockIdx.x >= token_blocks) {
      const int64_t w0 = (int64_t)((int)blockIdx.x - token_blocks) * kFewWords;
      uint32_t gone = 0u;  // words that do not occur
      for (int w = 0; w < kFewWords; ++w) {
        bool hit = false;
#pragma unroll
        for (int i = 0; i < kParts; ++i) hit |= tok[i] == (int32_t)(w0 + w);
        if (__ballot(hit) == 0ull && w0 + w < A.V) gone |= 1u << w;
      }
      if (tid < kFewWords && ((gone >> tid) & 1u))
        absent[__popc(gone & ((1u << tid) - 1u))] = (uint16_t)tid;
      __syncthreads();
      put_rest(A, absent, __popc(gone), w0, 0, rest_lg, (int)blockIdx.y, (int)gridDim.y);
      return;
    }
  } else {
    bool again = mine < 0;
    for (int j = 0; j < tid && !again; ++j) again = word_at[j] == mine;
    distinct[tid] = again ? 0x7FFFFFFF : mine;
    __syncthreads();
  }
  const Columns c = Columns::of<E>(lg, A.width);
  const int i = (int)blockIdx.x * (kFew >> lg) + c.group;  // (the same for the whole wave)
  const int32_t word = __builtin_amdgcn_readfirstlane(i < n ? word_at[i] : -1);
  const auto below = [&](int32_t limit) {
    int count = 0;
    if constexpr (LISTS) {
#pragma unroll
      for (int p = 0; p < kParts; ++p) count += __popcll(__ballot(distinct[p * 64 + lane] < limit));
    }
    return count;
  };
  if constexpr (LISTS) {
    const int all = below(0x7FFFFFFF);
    if (blockIdx.x == 0 && blockIdx.y == 0 && tid == 0)
      *A.nnz = (int32_t)((uint32_t)all * (uint32_t)A.width);
  }
  if (word < 0) return;
  const int number = below(word);
  uint64_t same[kParts];
  bool earlier = false;
#pragma unroll
  for (int p = 0; p < kParts; ++p) {
    same[p] = __ballot(tok[p] == word);
    const int bits = i - p * 64;  // places of this part before i
    const uint64_t before = bits >= 64 ? ~0ull : bits > 0 ? (1ull << bits) - 1ull : 0ull;
    earlier |= (same[p] & before) != 0ull;
  }
  if (earlier || c.none()) return;
  const O* dout = static_cast<const O*>(A.dout);
  float sum[E];
  bool begun = false;
#pragma unroll
  for (int p = 0; p < kParts; ++p)
    while (same[p] != 0ull) {
      int32_t at[kFewAhead];
      Packed<O, E> raw[kFewAhead];
      int count = __popcll(same[p]);
#pragma unroll
      for (int j = 0; j < kFewAhead; ++j) {
        at[j] = j < count ? p * 64 + (int)__builtin_ctzll(same[p]) : at[0];
        same[p] &= same[p] - 1ull;
      }
      load_rows<O, E, kFewAhead>(raw, dout, A.out_ld, at, c);
#pragma unroll
      for (int j = 0; j < kFewAhead; ++j)
        if (j < count) {
          float x[E];
          unpack_vec<O, E>(raw[j], x, dout);
#pragma unroll
          for (int e = 0; e < E; ++e) sum[e] = begun ? sum[e] + x[e] : x[e];
          begun = true;
        }
    }
  put_sum<R, LISTS, E>(A, word, number, c, sum);
}

// threads of a group, as a power of two: a vector each, up to a workgroup
int lg_threads(int64_t width, int E) {
  const int64_t vecs = (width + E - 1) / E;
  int lg = 0;
  while (lg < 8 && ((int64_t)1 << lg) < vecs) ++lg;
  return lg;
}

unsigned slices(int64_t width, int E, int lg) {
  return (unsigned)ceil_div(width, (int64_t)E << lg);
}

// Tokens of a tile, in no more than 4,096 tiles.
constexpr int64_t kMostTiles = 4096;
constexpr int kTile = 16;
int tile_of(int64_t n) {
  int tile = kTile;
  while (tile * kMostTiles < n) tile *= 2;
  return tile;
}

// Batches from here on are split into pieces first.
constexpr int64_t kSplitFrom = 16384;

// 512 bins, more for vocabularies beyond 2^18
Bins bins_of(int64_t V, bool spread) {
  int lgv = 0;
  while (((int64_t)1 << lgv) < V) ++lgv;
  Bins b;
  b.lgw = lgv < 9 ? 0 : lgv - 9 < kMaxBinBits ? lgv - 9 : kMaxBinBits;
  b.lgb = lgv - b.lgw;
  b.spread = spread;
  b.count = spread ? 1 << b.lgb : (int)ceil_div(V, (int64_t)1 << b.lgw);
  return b;
}

template <typename F>
void by_types(int32_t a, int32_t b, F f) {
  for_dtype(a, [&](auto* x) { for_dtype(b, [&](auto* y) { f(x, y); }); });
}

}  // namespace

EmbedLayout embed_layout(int64_t rows, int64_t V, int64_t width) {
  const Bins b = bins_of(V, true);  // (no fewer than the lists')
  const size_t bins = up256((size_t)b.count * 4);
  EmbedLayout l;
  l.sorted = 0;
  l.slots = up256((size_t)rows * sizeof(Token));
  l.first = l.slots + up256((size_t)rows * 4);
  l.bins = l.first + up256((size_t)(b.ids() + 1) * 4);
  l.before = l.bins + bins;
  l.partial = l.before + bins;
  // (a call with fewer tokens than the plan's has no more tiles than this)
  const int64_t tiles = ceil_div(rows, kTile) < kMostTiles ? ceil_div(rows, kTile) : kMostTiles;
  l.part = l.partial + up256((size_t)tiles * 2 * (size_t)width * 4);
  const bool split = rows >= kSplitFrom;
  l.ends = l.part + (split ? up256((size_t)rows * sizeof(Token)) : 0);
  l.bytes = l.ends +
            (split ? up256((size_t)ceil_div(rows, kPiece) * (size_t)(b.count + 1) * 4) : 0);
  return l;
}

hipError_t launch_embed_forward(const EmbedArgs& a, hipStream_t s) {
  by_types(a.dtype, a.out_dtype, [&](auto* t, auto* o) {
    using T = typename Pointee<decltype(t)>::type;
    using O = typename Pointee<decltype(o)>::type;
    constexpr int E = vector_of<O>();
    const int lg = lg_threads(a.width, E);
    const dim3 one((unsigned)ceil_div(a.n, 256 >> lg), slices(a.width, E, lg));
    k_embed_rows<T, O><<<one, 256, 0, s>>>(a, lg);
  });
  return hipGetLastError();
}

namespace {

template <typename O, typename R, bool LISTS>
void launch_sums(const EmbedArgs& a, void* ws, int rest_lg, hipStream_t s) {
  constexpr int E = vector_of_sums<O, R, LISTS>();
  int lg = lg_threads(a.width, E);
  const unsigned cut = slices(a.width, E, lg);
  if (a.n <= (LISTS ? kFewList : kFew)) {
    lg = lg < 6 ? 6 : lg;  // whole waves
    const int64_t tokens = LISTS && a.n == 0 ? 1 : (a.n + (kFew >> lg) - 1) / (kFew >> lg);
    const int64_t rest = rest_lg < 0 ? 0 : ceil_div(a.V, kFewWords);
    if (tokens + rest > 0)
      k_embed_few<O, R, LISTS>
          <<<dim3((unsigned)(tokens + rest), cut), kFew, 0, s>>>(a, lg, (int)tokens, rest_lg);
    return;
  }
  const EmbedLayout l = embed_layout(a.n, a.V, a.width);
  char* base = static_cast<char*>(ws);
  EmbedScratch w;
  w.sorted = reinterpret_cast<Token*>(base + l.sorted);
  w.slots = reinterpret_cast<int32_t*>(base + l.slots);
  w.first = reinterpret_cast<int32_t*>(base + l.first);
  w.bins = reinterpret_cast<int32_t*>(base + l.bins);
  w.before = reinterpret_cast<int32_t*>(base + l.before);
  w.partial = reinterpret_cast<float*>(base + l.partial);
  w.part = reinterpret_cast<Token*>(base + l.part);
  w.ends = reinterpret_cast<int32_t*>(base + l.ends);
  const Bins b = bins_of(a.V, !LISTS);
  const int tile = tile_of(a.n);
  const int64_t tiles = ceil_div(a.n, tile);
  const auto sort = [&](auto kernel, int threads) {
    kernel<<<b.count, threads, ((size_t)(threads / 64) << b.lgw) * 4, s>>>(a, w, b, rest_lg);
  };
  if (a.n >= kSplitFrom) {
    const int pieces = (int)ceil_div(a.n, kPiece);
    k_embed_split<<<pieces, kSplitThreads, (size_t)kSplitWaves * (size_t)b.count * 4, s>>>(a, w, b,
                                                                                          pieces);
    sort(k_embed_sort<true, kSortThreads>, kSortThreads);
  } else if (a.n <= kSortAhead * 256 && b.lgw <= 8) {
    sort(k_embed_sort<false, 256>, 256);
  } else {
    sort(k_embed_sort<false, kSortThreads>, kSortThreads);
  }
  const dim3 sums((unsigned)ceil_div(tiles, 256 >> lg), cut);
  if (lg >= 6)
    k_embed_sum<O, R, LISTS, true><<<sums, 256, 0, s>>>(a, w, b, lg, tile);
  else
    k_embed_sum<O, R, LISTS, false><<<sums, 256, 0, s>>>(a, w, b, lg, tile);
  int jlg = lg_threads(a.width, 8);
  jlg = jlg < 6 ? jlg : 6;
  const auto join = [&](auto kernel, int threads, unsigned each) {
    kernel<<<dim3((unsigned)ceil_div(tiles, kWindow), slices(a.width, 8, jlg), each), threads, 0, s>>>(
        a, w, b, jlg, tile, (int)tiles);
  };
  if (a.n >= kSplitFrom)
    join(k_embed_join<R, LISTS, 1024>, 1024, 8u);
  else
    join(k_embed_join<R, LISTS, 256>, 256, 64u);
}

}  // namespace

hipError_t launch_embed_backward(const EmbedArgs& a, void* ws, hipStream_t s) {
  if (a.nnz != nullptr) {
    by_types(a.out_dtype, a.val_format == TKEF_VAL_F16 ? TKEF_DTYPE_F16 : TKEF_DTYPE_F32,
             [&](auto* o, auto* r) {
               using O = typename Pointee<decltype(o)>::type;
               using R = typename Pointee<decltype(r)>::type;
               if constexpr (!std::is_same_v<R, __bf16>) launch_sums<O, R, true>(a, ws, -1, s);
             });
    return hipGetLastError();
  }
  // rows of words without tokens: written, unless they are there
  const bool there = a.add == a.grad && a.add_ld == a.grad_ld;
  const int rest_lg =
      there ? -1 : lg_threads(a.width, a.grad_dtype == TKEF_DTYPE_F32 ? 4 : 8);
  by_types(a.out_dtype, a.grad_dtype, [&](auto* o, auto* r) {
    using O = typename Pointee<decltype(o)>::type;
    using R = typename Pointee<decltype(r)>::type;
    launch_sums<O, R, false>(a, ws, rest_lg, s);
  });
  return hipGetLastError();
}

}  // namespace tkef

// gfx950 kernels for the embedding of tokens and its gradient. The gradient is a
// sum over each word's tokens: the tokens are sorted by word (stable, so a word's
// tokens stay in their order), the sorted ones are summed in tiles, and the sums of words
// that cross tiles are joined in their order. Nothing is added atomically: the same
// call gives the same bits.
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

template <typename T, int E>
__device__ __forceinline__ void load_vec(const T* p, float (&x)[E]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const loose4_ v = *reinterpret_cast<const loose4_*>(p + i);
      x[i] = __uint_as_float(v.x);
      x[i + 1] = __uint_as_float(v.y);
      x[i + 2] = __uint_as_float(v.z);
      x[i + 3] = __uint_as_float(v.w);
    }
  } else if constexpr (E == 8) {
    const loose4_ v = *reinterpret_cast<const loose4_*>(p);
    unpack(make_uint4(v.x, v.y, v.z, v.w), x, p);
  } else {
    static_assert(E == 4, "8 bytes of a 16-bit type");
    const loose2_ v = *reinterpret_cast<const loose2_*>(p);
    float y[8];
    unpack(make_uint4(v.x, v.y, 0u, 0u), y, p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = y[i];
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
    *reinterpret_cast<loose2_*>(p) = v;
  }
}

// `ne` of E elements; whole vectors where they are all there
template <typename T, int E>
__device__ __forceinline__ void load_some(const T* p, int ne, float (&x)[E]) {
  if (ne == E) {
    load_vec<T, E>(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = i < ne ? (float)p[i] : 0.f;
  }
}
template <typename T, int E>
__device__ __forceinline__ void store_some(T* p, int ne, const float (&x)[E]) {
  if (ne == E) {
    store_vec<T, E>(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (i < ne) p[i] = (T)x[i];
  }
}

// elements of a vector of 16 bytes of the narrower type
template <typename A, typename B>
constexpr int vector_of() {
  return sizeof(A) == 4 && sizeof(B) == 4 ? 4 : 8;
}

// A workgroup of 256 threads holds 256 >> lg groups of 1 << lg threads; a group has a row
// (or a tile), thread l of it the columns (slice << lg + l) E ...
struct Columns {
  int group, c0, ne;
  template <int E>
  __device__ static Columns of(int lg, int width) {
    Columns c;
    const int tid = (int)threadIdx.x, l = tid & ((1 << lg) - 1);
    c.group = tid >> lg;
    c.c0 = (((int)blockIdx.y << lg) + l) * E;
    const int left = width - c.c0;
    c.ne = left < 0 ? 0 : left < E ? left : E;
    return c;
  }
};

// ----------------------------------------------------------------------------
// lookup

// R rows a group, all loads before the first store.
template <typename T, typename O, int R>
__global__ __launch_bounds__(256) void k_embed_rows(EmbedArgs A, int lg) {
  constexpr int E = vector_of<T, O>();
  const Columns c = Columns::of<E>(lg, A.width);
  const int groups = 256 >> lg;
  const int64_t i0 = ((int64_t)blockIdx.x * groups + c.group) * R;
  const T* table = static_cast<const T*>(A.table);
  O* out = static_cast<O*>(A.out);
  int32_t word[R];
#pragma unroll
  for (int r = 0; r < R; ++r) word[r] = i0 + r < A.n ? A.tokens[i0 + r] : -1;
  float x[R][E];
  uint32_t bits = 0u;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool in = word[r] >= 0 && word[r] < A.V;
    if (!in && word[r] != -1) bits = TKEF_STATUS_INDEX_RANGE;
#pragma unroll
    for (int e = 0; e < E; ++e) x[r][e] = 0.f;
    if (in && c.ne > 0) {
      load_some<T, E>(table + word[r] * A.table_ld + c.c0, c.ne, x[r]);
#pragma unroll
      for (int e = 0; e < E; ++e) x[r][e] *= A.scale;
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (i0 + r >= A.n || c.ne == 0) continue;
    store_some<O, E>(out + (i0 + r) * A.out_ld + c.c0, c.ne, x[r]);
  }
  raise_status(A.status, c.c0 == 0 ? bits : 0u);
}

// ----------------------------------------------------------------------------
// tokens sorted by word

struct Token {
  int32_t at, word;
};

struct EmbedScratch {
  Token* sorted;    // the batch's tokens that are words, by word, then by place
  int32_t* first;   // V + 1: each word's first place in `sorted`
  int32_t* slot;    // V: number of a word among its bin's words that occur
  int32_t* bins;    // per bin: words that occur; then of all bins before it
  float* partial;   // per tile: sums of the word that began before it, of the one that goes on
};

constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64;
constexpr int kMaxBinBits = 10;

// Lanes of the wave whose word (lgw bits) is the lane's own, among the lanes of `who`.
__device__ __forceinline__ uint64_t same_word(uint32_t word, int lgw, uint64_t who) {
  uint64_t same = who;
  for (int b = 0; b < lgw; ++b) {
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

// Workgroup b sorts the tokens of the words [b << lgw, (b + 1) << lgw): it reads all
// tokens, counts those of lower words (they come before) and its own word by word, and
// in a second reading puts its own in place. Wave w has the w-th share of the batch, so
// a word's tokens are in the batch's order: waves in turn, and in a wave, lanes.
__global__ __launch_bounds__(kSortThreads) void k_embed_sort(EmbedArgs A, EmbedScratch W, int lgw) {
  extern __shared__ uint32_t hist[];  // wave x word
  __shared__ uint32_t red[kSortWaves], below_of[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int words = 1 << lgw;
  const int32_t w0 = (int32_t)blockIdx.x << lgw;
  for (int i = tid; i < words * kSortWaves; i += kSortThreads) hist[i] = 0u;
  __syncthreads();
  const int n = (int)A.n;
  const int per = ((n + kSortWaves * 64 - 1) / (kSortWaves * 64)) * 64;
  const int begin = wave * per, end = begin + per < n ? begin + per : n;
  uint32_t* mine = hist + wave * words;
  uint32_t below = 0u, bits = 0u;
  for (int i = begin + lane; i < end; i += 64) {
    const int32_t t = A.tokens[i];
    const bool in = t >= 0 && t < A.V;
    if (!in && t != -1) bits = TKEF_STATUS_INDEX_RANGE;
    below += in && t < w0 ? 1u : 0u;
    if (in && t >= w0 && t - w0 < words) atomicAdd(&mine[t - w0], 1u);
  }
  if (blockIdx.x == 0) raise_status(A.status, bits);
  below = wave_incl(below);
  if (lane == 63) below_of[wave] = below;
  __syncthreads();
  uint32_t at = 0u;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) at += below_of[w];
  // places of each word, and of each wave's share of it
  uint32_t occur = 0u;
  for (int base = 0; base < words; base += kSortThreads) {
    const int w = base + tid;
    uint32_t count = 0u;
    if (w < words)
      for (int v = 0; v < kSortWaves; ++v) count += hist[v * words + w];
    uint32_t total, there;
    const uint32_t before = block_scan<kSortThreads>(count, red, &total);
    const uint32_t number = block_scan<kSortThreads>(count > 0u ? 1u : 0u, red, &there);
    if (w < words) {
      uint32_t place = at + before;
      if (w0 + w < A.V) {
        W.first[w0 + w] = (int32_t)place;
        W.slot[w0 + w] = (int32_t)(occur + number);
        if (w0 + w == A.V - 1) W.first[A.V] = (int32_t)(place + count);
      }
      for (int v = 0; v < kSortWaves; ++v) {
        const uint32_t c = hist[v * words + w];
        hist[v * words + w] = place;
        place += c;
      }
    }
    at += total;
    occur += there;
  }
  if (tid == 0) W.bins[blockIdx.x] = (int32_t)occur;
  __syncthreads();
  for (int i0 = begin; i0 < end; i0 += 64) {
    const int i = i0 + lane;
    const int32_t t = i < end ? A.tokens[i] : -1;
    const bool own = t >= w0 && t < A.V && t - w0 < words;
    const uint64_t who = __ballot(own);
    if (who == 0ull) continue;
    const uint32_t word = own ? (uint32_t)(t - w0) : 0u;
    const uint64_t same = same_word(word, lgw, who);
    const int rank = lanes_below(same);
    const uint32_t place = mine[word] + (uint32_t)rank;
    wave_fence();  // every lane has read before one writes, and before the next 64 read
    if (own) {
      W.sorted[place] = Token{i, t};
      if (rank == 0) mine[word] = place + (uint32_t)__popcll(same);
    }
    wave_fence();
  }
}

// Words that occur in the bins before each bin, and the lists' length.
__global__ __launch_bounds__(1024) void k_embed_bins(EmbedArgs A, EmbedScratch W, int bins) {
  __shared__ uint32_t red[16];
  uint32_t done = 0u;
  for (int base = 0; base < bins; base += 1024) {
    const int b = base + (int)threadIdx.x;
    uint32_t total;
    const uint32_t before = block_scan<1024>(b < bins ? (uint32_t)W.bins[b] : 0u, red, &total);
    if (b < bins) W.bins[b] = (int32_t)(done + before);
    done += total;
  }
  if (threadIdx.x == 0) *A.nnz = (int32_t)(done * (uint32_t)A.width);
}

// ----------------------------------------------------------------------------
// sums

// Where a word's sum goes: a row of the gradient (with another gradient's added), or a
// piece of the lists.
template <int E>
__device__ __forceinline__ void put_row(const EmbedArgs& A, const EmbedScratch& W, int lgw,
                                        int32_t word, const Columns& c, float (&x)[E]) {
  if (A.idx != nullptr) {
    const int64_t o = (int64_t)(W.bins[word >> lgw] + W.slot[word]) * A.width + c.c0;
    const int32_t p = (int32_t)(A.offset + (int64_t)word * A.width + c.c0);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e < c.ne) A.idx[o + e] = p + e;
    if (A.val_format == TKEF_VAL_F16)
      store_some<_Float16, E>(static_cast<_Float16*>(A.val) + o, c.ne, x);
    else
      store_some<float, E>(static_cast<float*>(A.val) + o, c.ne, x);
    return;
  }
  const auto row = [&](auto* g, const auto* add) {
    using G = typename Pointee<decltype(g)>::type;
    if (add != nullptr) {
      float y[E];
      load_some<G, E>(add + word * A.add_ld + c.c0, c.ne, y);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] += y[e];
    }
    store_some<G, E>(g + word * A.grad_ld + c.c0, c.ne, x);
  };
  if (A.grad_dtype == TKEF_DTYPE_F32)
    row(static_cast<float*>(A.grad), static_cast<const float*>(A.add));
  else if (A.grad_dtype == TKEF_DTYPE_F16)
    row(static_cast<_Float16*>(A.grad), static_cast<const _Float16*>(A.add));
  else
    row(static_cast<__bf16*>(A.grad), static_cast<const __bf16*>(A.add));
}

template <int E>
__device__ __forceinline__ void put_sum(const EmbedArgs& A, const EmbedScratch& W, int lgw,
                                        int32_t word, const Columns& c, float (&sum)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] *= A.scale;
  put_row<E>(A, W, lgw, word, c, sum);
}

constexpr int kAhead = 8;      // rows of a tile under way
constexpr int kWordsAGroup = 8;  // of words without tokens

// Group g sums the sorted tokens [g tile, (g + 1) tile). A word that lies within them is
// done; the sums of one that began before them, and of one that goes on behind them, are
// left for k_embed_join. Groups from `tiles` on write the rows of words without tokens,
// among the first `rest` words (0 or V).
template <typename O>
__global__ __launch_bounds__(256) void k_embed_sum(EmbedArgs A, EmbedScratch W, int lgw, int lg,
                                                   int tile, int64_t tiles, int64_t rest) {
  constexpr int E = sizeof(O) == 4 ? 4 : 8;
  const Columns c = Columns::of<E>(lg, A.width);
  const int64_t g = (int64_t)blockIdx.x * (256 >> lg) + c.group;
  if (c.ne == 0) return;
  if (g >= tiles) {
    const int64_t w0 = (g - tiles) * kWordsAGroup;
    for (int64_t w = w0; w < w0 + kWordsAGroup && w < rest; ++w)
      if (W.first[w] == W.first[w + 1]) {
        float x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = 0.f;
        put_row<E>(A, W, lgw, (int32_t)w, c, x);
      }
    return;
  }
  const int total = W.first[A.V];
  const int p0 = (int)(g * tile), p1 = p0 + tile < total ? p0 + tile : total;
  if (p0 >= p1) return;
  const O* dout = static_cast<const O*>(A.dout);
  float sum[E];
  int32_t word = W.sorted[p0].word;
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.f;
  const auto flush = [&]() {
    const bool before = W.first[word] < p0, behind = W.first[word + 1] > p1;
    if (before || behind) {
      float* to = W.partial + (2 * g + (before ? 0 : 1)) * A.width + c.c0;
      store_some<float, E>(to, c.ne, sum);
    } else {
      put_sum<E>(A, W, lgw, word, c, sum);
    }
  };
  for (int p = p0; p < p1; p += kAhead) {
    Token t[kAhead];
    float x[kAhead][E];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) t[j] = W.sorted[p + j < p1 ? p + j : p1 - 1];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      load_some<O, E>(dout + t[j].at * A.out_ld + c.c0, c.ne, x[j]);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (p + j >= p1) continue;
      if (t[j].word != word) {
        flush();
        word = t[j].word;
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] += x[j][e];
    }
  }
  flush();
}

// The word that begins in tile g and goes on behind it: its sums, tile after tile.
template <int E>
__global__ __launch_bounds__(256) void k_embed_join(EmbedArgs A, EmbedScratch W, int lgw, int lg,
                                                    int tile, int64_t tiles) {
  const Columns c = Columns::of<E>(lg, A.width);
  const int64_t g = (int64_t)blockIdx.x * (256 >> lg) + c.group;
  if (g >= tiles || c.ne == 0) return;
  const int total = W.first[A.V];
  const int64_t p0 = g * tile, p1 = p0 + tile;
  if (p1 >= total) return;
  const int32_t word = W.sorted[p1 - 1].word;
  const int end = W.first[word + 1];
  if (W.first[word] < p0 || end <= p1) return;
  float sum[E];
  load_some<float, E>(W.partial + (2 * g + 1) * A.width + c.c0, c.ne, sum);
  const int64_t last = (end - 1) / tile;
  for (int64_t h = g + 1; h <= last; h += 4) {
    float x[4][E];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      load_some<float, E>(W.partial + 2 * (h + j < last ? h + j : last) * A.width + c.c0, c.ne,
                          x[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (h + j <= last) {
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += x[j][e];
      }
  }
  put_sum<E>(A, W, lgw, word, c, sum);
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

constexpr int kLeastTile = 8;
int tile_of(int64_t n) {
  int tile = kLeastTile;
  while ((int64_t)tile * 4096 < n) tile *= 2;
  return tile;
}

// bits of a bin's words: about 512 bins
int bin_bits(int64_t V) {
  int lgw = 6;
  while (lgw < kMaxBinBits && (V >> lgw) > 512) ++lgw;
  return lgw;
}

template <typename F>
void by_types(int32_t a, int32_t b, F f) {
  (void)by_dtype(a, [&](auto* x) { (void)by_dtype(b, [&](auto* y) { f(x, y); }); });
}

}  // namespace

EmbedLayout embed_layout(int64_t rows, int64_t V, int64_t width) {
  EmbedLayout l;
  l.sorted = 0;
  l.first = up256((size_t)rows * sizeof(Token));
  l.slot = l.first + up256((size_t)(V + 1) * 4);
  l.bins = l.slot + up256((size_t)V * 4);
  l.partial = l.bins + up256((size_t)ceil_div(V, (int64_t)1 << bin_bits(V)) * 4);
  // (fewer tokens than the plan's have tiles no larger, and no more of them than this)
  const int64_t tiles = rows <= 4096 * kLeastTile ? ceil_div(rows, kLeastTile) : 4096;
  l.bytes = l.partial + up256((size_t)tiles * 2 * (size_t)width * 4);
  return l;
}

hipError_t launch_embed_forward(const EmbedArgs& a, hipStream_t s) {
  by_types(a.dtype, a.out_dtype, [&](auto* t, auto* o) {
    using T = typename Pointee<decltype(t)>::type;
    using O = typename Pointee<decltype(o)>::type;
    constexpr int E = vector_of<T, O>();
    const int lg = lg_threads(a.width, E);
    const dim3 one((unsigned)ceil_div(a.n, 256 >> lg), slices(a.width, E, lg));
    k_embed_rows<T, O, 1><<<one, 256, 0, s>>>(a, lg);
  });
  return hipGetLastError();
}

hipError_t launch_embed_backward(const EmbedArgs& a, void* ws, hipStream_t s) {
  const EmbedLayout l = embed_layout(a.n, a.V, a.width);
  char* base = static_cast<char*>(ws);
  EmbedScratch w;
  w.sorted = reinterpret_cast<Token*>(base + l.sorted);
  w.first = reinterpret_cast<int32_t*>(base + l.first);
  w.slot = reinterpret_cast<int32_t*>(base + l.slot);
  w.bins = reinterpret_cast<int32_t*>(base + l.bins);
  w.partial = reinterpret_cast<float*>(base + l.partial);
  const int lgw = bin_bits(a.V);
  const unsigned bins = (unsigned)ceil_div(a.V, (int64_t)1 << lgw);
  k_embed_sort<<<bins, kSortThreads, ((size_t)kSortWaves << lgw) * 4, s>>>(a, w, lgw);
  if (a.idx != nullptr) k_embed_bins<<<1, 1024, 0, s>>>(a, w, (int)bins);
  const int tile = tile_of(a.n);
  const int64_t tiles = a.n == 0 ? 0 : ceil_div(a.n, tile);
  // rows of words without tokens: written, unless they are there or lists have none
  const int64_t rest =
      a.idx != nullptr || (a.add == a.grad && a.add_ld == a.grad_ld) ? 0 : a.V;
  const int64_t groups = tiles + (rest > 0 ? ceil_div(rest, kWordsAGroup) : 0);
  return by_dtype(a.out_dtype, [&](auto* o) {
    using O = typename Pointee<decltype(o)>::type;
    constexpr int E = sizeof(O) == 4 ? 4 : 8;
    const int lg = lg_threads(a.width, E);
    const unsigned cut = slices(a.width, E, lg);
    if (groups > 0)
      k_embed_sum<O><<<dim3((unsigned)ceil_div(groups, 256 >> lg), cut), 256, 0, s>>>(
          a, w, lgw, lg, tile, tiles, rest);
    if (tiles > 1)
      k_embed_join<E><<<dim3((unsigned)ceil_div(tiles, 256 >> lg), cut), 256, 0, s>>>(
          a, w, lgw, lg, tile, tiles);
  });
}

}  // namespace tkef

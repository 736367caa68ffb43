// Device code that the operators on rows share: sums of exponentials, order
// keys, reductions, rows as 16-byte vectors, agent-scope hand-over.
//
// All exponentials are taken in base 2: exp(s x) = 2^(x a) with a = log2(e) / temperature.
// A sum of exponentials is held as a pair (m, S), meaning S * 2^(m a), with m
// its largest logit: each term is 2^((x - m) a). The difference is taken
// before the product, so logits at the lowest value of their type (a common
// mask) neither overflow nor lose their order.
#pragma once

#include <hip/hip_runtime.h>

#include "tkef.h"

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

// (x - m) a as one operation, fma(x, a, -c) with c = fl(m a): what c's rounding
// changes is the same factor for all x, 2^(c - m a), and rest() takes it out of
// their sum. m is held to where c's rounding is at most 2^5, so that neither that
// factor nor the terms leave the range: a sum whose own maximum lies below (masks
// at -1e10 or the type's lowest value, beside ordinary words) is 0 then, which is
// right beside them, and one whose row has no other words is taken again by the
// difference. One of eight operations a word: 145 ->
// 134 us for the step of 1,021 x 131,071 binary16, whose rows leave one workgroup
// a compute unit, 219 -> 206 for 8,192 x 32,000 bfloat16.
struct Product {
  float m, a, c;
  __device__ Product(float max, float a_) : a(a_) {
    const float limit = 0x1p30f / a;
    m = max == -kInf ? 0.f : fmaxf(fminf(max, limit), -limit);
    c = m * a;
  }
  __device__ float exponent(float x) const { return __builtin_fmaf(x, a, -c); }
  __device__ float rest() const { return exp2_(-__builtin_fmaf(m, a, -c)); }
  __device__ static bool fits(float max, float a) {
    return max == -kInf || __builtin_fabsf(max) < 0x1p30f / a;
  }
};

template <typename T>
__device__ __forceinline__ float load1(const T* p, int64_t i) {
  return (float)p[i];
}

// element i of rows of a type
__device__ __forceinline__ float load1_of(const void* p, int dtype, int64_t i) {
  return dtype == TKEF_DTYPE_F32   ? static_cast<const float*>(p)[i]
         : dtype == TKEF_DTYPE_F16 ? (float)static_cast<const _Float16*>(p)[i]
                                   : (float)static_cast<const __bf16*>(p)[i];
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

// ----------------------------------------------------------------------------
// rows in 16-byte vectors

// Elements before the first 16-byte boundary (the head) and those after the
// last whole vector are "extras", at most 14: every vector access is aligned
// whatever the row's address. Vector v holds elements head + v * N ...
template <typename T>
struct Span {
  static constexpr int N = 16 / (int)sizeof(T);
  const T* p;
  int head, nvec, extras;
  __device__ Span(const T* row, int V) : p(row) {
    head = (int)((16u - (uint32_t)(reinterpret_cast<uintptr_t>(row) & 15u)) & 15u) /
           (int)sizeof(T);
    head = head < V ? head : V;
    nvec = (V - head) / N;
    extras = V - nvec * N;
  }
  __device__ const T* vec(int v) const { return p + head + (int64_t)v * N; }
  // element index of extra i
  __device__ int extra(int i) const { return i < head ? i : i + nvec * N; }
};

__device__ __forceinline__ void unpack(uint4 r, float (&x)[4], const float*) {
  x[0] = __uint_as_float(r.x);
  x[1] = __uint_as_float(r.y);
  x[2] = __uint_as_float(r.z);
  x[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void unpack(uint4 r, float (&x)[8], const __bf16*) {
  const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}
typedef _Float16 half2_ __attribute__((ext_vector_type(2)));
typedef __bf16 bfloat2_ __attribute__((ext_vector_type(2)));
typedef float float2_ __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void unpack(uint4 r, float (&x)[8], const _Float16*) {
  const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const half2_ h = __builtin_bit_cast(half2_, u[i]);
    x[2 * i] = (float)h.x;
    x[2 * i + 1] = (float)h.y;
  }
}

__device__ __forceinline__ uint4 pack(const float (&x)[4], const float*) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                    __float_as_uint(x[3]));
}
template <typename H2>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const float2_ v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, H2));
}
__device__ __forceinline__ uint4 pack(const float (&x)[8], const __bf16*) {
  return make_uint4(pack2<bfloat2_>(x[0], x[1]), pack2<bfloat2_>(x[2], x[3]),
                    pack2<bfloat2_>(x[4], x[5]), pack2<bfloat2_>(x[6], x[7]));
}
__device__ __forceinline__ uint4 pack(const float (&x)[8], const _Float16*) {
  return make_uint4(pack2<half2_>(x[0], x[1]), pack2<half2_>(x[2], x[3]),
                    pack2<half2_>(x[4], x[5]), pack2<half2_>(x[6], x[7]));
}

// four -inf words of a type
__device__ __forceinline__ uint4 none_of(const float*) {
  return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u);
}
__device__ __forceinline__ uint4 none_of(const __bf16*) {
  return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u);
}
__device__ __forceinline__ uint4 none_of(const _Float16*) {
  return make_uint4(0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u);
}

// -inf in the places of a vector whose bit is set
__device__ __forceinline__ uint4 strike(uint4 r, uint32_t bits, const float*) {
  r.x = (bits & 1u) ? 0xFF800000u : r.x;
  r.y = (bits & 2u) ? 0xFF800000u : r.y;
  r.z = (bits & 4u) ? 0xFF800000u : r.z;
  r.w = (bits & 8u) ? 0xFF800000u : r.w;
  return r;
}
template <uint32_t kNone>
__device__ __forceinline__ uint32_t strike2(uint32_t w, uint32_t bits) {
  w = (bits & 1u) ? (w & 0xFFFF0000u) | kNone : w;
  return (bits & 2u) ? (w & 0x0000FFFFu) | (kNone << 16) : w;
}
__device__ __forceinline__ uint4 strike(uint4 r, uint32_t bits, const __bf16*) {
  return make_uint4(strike2<0xFF80u>(r.x, bits), strike2<0xFF80u>(r.y, bits >> 2),
                    strike2<0xFF80u>(r.z, bits >> 4), strike2<0xFF80u>(r.w, bits >> 6));
}
__device__ __forceinline__ uint4 strike(uint4 r, uint32_t bits, const _Float16*) {
  return make_uint4(strike2<0xFC00u>(r.x, bits), strike2<0xFC00u>(r.y, bits >> 2),
                    strike2<0xFC00u>(r.z, bits >> 4), strike2<0xFC00u>(r.w, bits >> 6));
}

// STREAM: what the call does not read again, past the caches' usual order.
typedef uint32_t uint4_ __attribute__((ext_vector_type(4)));
template <bool STREAM>
__device__ __forceinline__ uint4 load16(const void* p) {
  if constexpr (STREAM) {
    const uint4_ v = __builtin_nontemporal_load(static_cast<const uint4_*>(p));
    return make_uint4(v.x, v.y, v.z, v.w);
  } else {
    return *static_cast<const uint4*>(p);
  }
}
// 16 bytes at any address of the element's alignment; stores stream (backward of
// 4,096 x 32,000 bfloat16: 107 -> 95 us with streaming loads and stores, with
// either alone 107 to 109; the step of 8,192: 206 -> 200)
struct __attribute__((packed, aligned(2))) Loose16 {
  uint32_t x, y, z, w;
};
typedef uint32_t loose4_ __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void store16(void* p, uint4 r) {
  const uint4_ v = {r.x, r.y, r.z, r.w};
  __builtin_nontemporal_store(v, static_cast<loose4_*>(p));
}

// Makes the registers opaque: without it the compiler keeps the unpacked
// values of one pass for the next, in twice the registers.
__device__ __forceinline__ void renew(uint4& r) {
  asm("" : "+v"(r.x), "+v"(r.y), "+v"(r.z), "+v"(r.w));
}

__device__ __forceinline__ int renew(int i) {
  asm("" : "+v"(i));
  return i;
}

// Largest of three without the canonicalizing instructions that fmaxf brings
// for each operand. A quiet NaN is passed over, a signalling one may win: the
// sums over the same words carry either.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
template <int N>
__device__ __forceinline__ float max_of(float m, const float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 2) m = max3(m, x[i], x[i + 1]);
  return m;
}
// the same of a packed vector
template <typename T>
__device__ __forceinline__ float max_packed(float m, uint4 r, const T* type) {
  float x[Span<T>::N];
  unpack(r, x, type);
  return max_of(m, x);
}
__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("v_pk_max_f16 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ float max_packed(float m, uint4 r, const _Float16*) {
  const half2_ h = __builtin_bit_cast(half2_, pk_max(pk_max(r.x, r.y), pk_max(r.z, r.w)));
  return max3(m, (float)h.x, (float)h.y);
}

// Vectors v0 + i * step + t of a row, t < width across the threads that share v0;
// -inf in the places of those it has not.
// Every load is issued at an address inside the row, so the loads need no
// execution masks; only the slot that the row ends in is patched.
template <typename T, int TPB, int NV, bool STREAM>
__device__ __forceinline__ void load_slots(uint4 (&r)[NV], const Span<T>& s, int v0, int step,
                                           int t, int width) {
  const T* type = nullptr;
  const int last = s.nvec - 1;
  if (v0 > last) {
#pragma unroll
    for (int i = 0; i < NV; ++i) r[i] = none_of(type);
    return;
  }
  const char* base = reinterpret_cast<const char*>(s.p + s.head);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = v0 + i * step + t;
    r[i] = load16<STREAM>(base + (uint32_t)(v < last ? v : last) * 16u);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (v0 + i * step + width > s.nvec) {  // (the same for all threads of the width)
      const bool in = v0 + i * step + t < s.nvec;
      r[i].x = in ? r[i].x : none_of(type).x;
      r[i].y = in ? r[i].y : none_of(type).y;
      r[i].z = in ? r[i].z : none_of(type).z;
      r[i].w = in ? r[i].w : none_of(type).w;
    }
}
template <typename T, int TPB, int NV, bool STREAM>
__device__ __forceinline__ void load_slots(uint4 (&r)[NV], const Span<T>& s, int v0) {
  load_slots<T, TPB, NV, STREAM>(r, s, v0, TPB, (int)threadIdx.x, TPB);
}

// Wave reductions over DPP row shifts: lane 15 of each row of 16 lanes ends
// with its row's result; the four are then read and joined.
template <int CTRL>
__device__ __forceinline__ float dpp(float old, float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(x), CTRL,
                                                    0xF, 0xF, false));
}
__device__ __forceinline__ float lane_value(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, dpp<0x111>(x, x));
  x = fmaxf(x, dpp<0x112>(x, x));
  x = fmaxf(x, dpp<0x114>(x, x));
  return fmaxf(x, dpp<0x118>(x, x));
}
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<0x111>(0.f, x);
  x += dpp<0x112>(0.f, x);
  x += dpp<0x114>(0.f, x);
  return x + dpp<0x118>(0.f, x);
}
__device__ __forceinline__ float wave_max(float x) {
  x = row_max(x);
  return fmaxf(fmaxf(lane_value(x, 15), lane_value(x, 31)),
               fmaxf(lane_value(x, 47), lane_value(x, 63)));
}
__device__ __forceinline__ float wave_sum(float x) {
  x = row_sum(x);
  return (lane_value(x, 15) + lane_value(x, 31)) + (lane_value(x, 47) + lane_value(x, 63));
}

// fmaxf passes over a NaN; the sums carry it
__device__ __forceinline__ float join_sum(float m, float s, float top, float a) {
  return s * rescale(m, top, a);
}

__device__ __forceinline__ uint64_t wave_max64(uint64_t x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)x, d);
    x = o > x ? o : x;
  }
  return x;
}

// A candidate: the distinct upper bits of its order key, then the complement of
// its word, so that a larger candidate is selected first.
constexpr int kWordBits = 20;
static_assert(TKEF_ROWS_MAX_VOCAB <= 1 << kWordBits, "words of a candidate");
__device__ __forceinline__ constexpr int key_shift(const float*) { return 0; }
__device__ __forceinline__ constexpr int key_shift(const _Float16*) { return 13; }
__device__ __forceinline__ constexpr int key_shift(const __bf16*) { return 16; }

template <typename T>
__device__ __forceinline__ uint64_t candidate(uint32_t key, int32_t word) {
  const T* type = nullptr;
  return ((uint64_t)(key >> key_shift(type)) << kWordBits) |
         (uint32_t)((1 << kWordBits) - 1 - word);
}
__device__ __forceinline__ int32_t word_of(uint64_t c) {
  return (1 << kWordBits) - 1 - (int32_t)((uint32_t)c & ((1u << kWordBits) - 1u));
}
template <typename T>
__device__ __forceinline__ float value_of(uint64_t c) {
  const T* type = nullptr;
  uint32_t key = (uint32_t)(c >> kWordBits) << key_shift(type);
  if (!(key >> 31)) key |= (1u << key_shift(type)) - 1u;  // (a negative value's key is inverted)
  return key_value(key);
}

// Zeros over the vectors of chunk `chunk` of `chunks` of a row of grad (its own span: the
// gradient's address decides the vectors), the first chunk with the extras.
template <typename T, int TPB>
__device__ __forceinline__ void zero_row(T* g, int V, int chunk, int chunks) {
  const Span<T> s(g, V);
  const int per = (s.nvec + chunks - 1) / chunks;
  const int v0 = chunk * per, v1 = v0 + per < s.nvec ? v0 + per : s.nvec;
  for (int v = v0 + (int)threadIdx.x; v < v1; v += TPB)
    *reinterpret_cast<uint4*>(g + s.head + (int64_t)v * Span<T>::N) = make_uint4(0u, 0u, 0u, 0u);
  if (chunk == 0 && (int)threadIdx.x < s.extras) g[s.extra((int)threadIdx.x)] = (T)0.f;
}

// 16 bytes from any address of the element's alignment
__device__ __forceinline__ uint4 load16_loose(const void* p) {
  const Loose16 l = *static_cast<const Loose16*>(p);
  return make_uint4(l.x, l.y, l.z, l.w);
}

template <typename V>
__device__ __forceinline__ V agent_load(const V* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename V>
__device__ __forceinline__ void agent_store(V* p, V v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Counts an arrival at a counter of `of` workgroups; true for the last one.
// What the workgroups tell each other goes through agent-scope atomics alone,
// which act where all dies see them: the calling lane's own have ended there
// when its counter of outstanding accesses is zero, so the last arrival's
// atomic loads find all of them. (An acquire-release arrival would also write
// back and drop the die's L2, for every workgroup.)
__device__ __forceinline__ bool arrive_last(uint32_t* ticket, uint32_t of) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  const uint32_t before =
      __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  asm volatile("" ::: "memory");
  return before == of - 1u;
}

__device__ __forceinline__ void agent_put(float2* p, float a, float b) {
  (void)__hip_atomic_exchange(
      reinterpret_cast<unsigned long long*>(p),
      ((unsigned long long)__float_as_uint(b) << 32) | __float_as_uint(a), __ATOMIC_RELAXED,
      __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 agent_get(const float2* p) {
  const unsigned long long u = agent_load(reinterpret_cast<const unsigned long long*>(p));
  return make_float2(__uint_as_float((uint32_t)u), __uint_as_float((uint32_t)(u >> 32)));
}

// f(T*) for a type
template <typename F>
void for_dtype(int32_t dtype, F f) {
  switch (dtype) {
    case TKEF_DTYPE_F32: f(static_cast<float*>(nullptr)); break;
    case TKEF_DTYPE_F16: f(static_cast<_Float16*>(nullptr)); break;
    default: f(static_cast<__bf16*>(nullptr)); break;
  }
}

// the same with f's launches, and whether one failed (which can be asked once)
template <typename F>
hipError_t by_dtype(int32_t dtype, F f) {
  for_dtype(dtype, f);
  return hipGetLastError();
}

template <typename P>
struct Pointee;
template <typename T>
struct Pointee<T*> {
  using type = T;
};

inline int64_t ceil_div(int64_t a, int64_t b) { return a <= 0 ? 1 : (a + b - 1) / b; }
inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

}  // namespace tkef

// Rows of vocabulary logits: log probabilities of given tokens with entropy and the top alternatives, their gradient, the
// clipped PPO objective over tokens, and distillation from a teacher's top logits.  With z a row of V logits,
//   m = max z,  d_j = (z_j - m) / temperature,  e_j = exp d_j,  S = sum e_j,  log p_j = d_j - log S,
//   H = log S - (sum e_j d_j) / S                                     (terms of one sign: nothing cancels)
//
// The pass over a row: a thread takes up to TL_VECS vectors of 32 bytes at a time (a chunk of the group of threads that has the row), follows its own
// maximum and rescales its sums when that grows; warps, CTA and cluster join theirs in a fixed order.  A row has a warp, a CTA or the C CTAs of a
// cluster, by sizes (tl_plan).  A gradient goes over the row again, from the last chunk, which is still in registers, back to the first; what
// it reads then comes out of L2 for the most part (PPO of 4096 x 128000 bf16: 1.23 x the logits from memory).
//
// What bounds it: memory where a row is read once (4096 x 128000 bf16: 161..171 us, 5.5..5.9 TB/s; its gradient from statistics: 98 % of the rate of a
// copy).  An exponential and five to six other instructions fall on every element of a pass; at the rate of memory the special function unit has
// 11 of its 16 exponentials a cycle to do, and under the power limit (1.5 GHz) 14, so that the second pass of the objectives makes arithmetic and
// memory equals (PPO 4096 x 128000: 398..416 us, floor 309; distillation with 64 tokens and the tail 465..481).
//
// Exponents are base 2: x_j = z_j c - R with c = log2(e) / temperature and R = c m rounded, one fused multiply-add per element.  That R
// is rounded does not matter, as every x of a row has the same one; the results' scalars are made in 64 bits and add back the
// difference.  Rows of extreme logits, where c m is out of range or a -inf could not be told apart, subtract first (tl_plain).
#pragma once

#include <cuda_fp16.h>

#include <cfloat>

#include "common.cuh"
#include "ptx.cuh"

namespace bitrl {

constexpr int TL_ROW_WARPS = 8;       // of a CTA whose warps have a row each
constexpr int TL_MAX_WARPS = 16;      // of a CTA that has one row, or a share of it
constexpr int TL_VECS = 4;            // vectors that a thread holds
constexpr int TL_VEC_BYTES = 32;
constexpr int TL_MAX_CLUSTER = 16;
constexpr int TL_MAX_SMEM = 220 * 1024;
constexpr int TL_CANDIDATES = 2560;   // of a share for the top alternatives: all elements of a row that has a vector for fewer than 128 threads, and some
constexpr int TL_SEGMENTS = 1024;     // of which single elements are looked at
constexpr float TL_FAR = -1024.0f;    // an exponent that leaves nothing, and whose product with a gradient's factor stays finite
constexpr float TL_REST_ROUNDING = 0x1p-20f;  // what rounding its log probabilities may leave of a teacher's mass outside its tokens
constexpr double TL_LOG2E = 1.4426950408889634074, TL_LN2 = 0.69314718055994530942;

// The logits of a call: rows of V elements, ld apart.
template <class E>
struct TlRows {
  const E* z;
  long long ld;
  int T, V;
  int C;                  // CTAs of a row
  float c;                // log2(e) / temperature
  float ref_lo, ref_hi;   // maxima between these allow x = z c - R
  double it;              // 1 / temperature
};

template <class E>
struct TlGrad {
  E* dz;  // may be the logits
  long long ld;
};

__device__ __forceinline__ float tl_f32(float v) { return v; }
__device__ __forceinline__ float tl_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float tl_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ void tl_set(float* p, float v) { *p = v; }
__device__ __forceinline__ void tl_set(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void tl_set(__half* p, float v) { *p = __float2half_rn(v); }

// What differs by type: elements in a 32-bit word, -inf in all of them, the lowest number, conversions.
template <class E>
struct TlType;
template <>
struct TlType<float> {
  static constexpr int LOW_BITS = 0;  // of fp32 that the type does not have
  static constexpr int PER_WORD = 1;
  static constexpr uint32_t NEG_INF = 0xff800000u;
  static constexpr float LOWEST = -FLT_MAX;
};
template <>
struct TlType<__nv_bfloat16> {
  static constexpr int LOW_BITS = 16;
  static constexpr int PER_WORD = 2;
  static constexpr uint32_t NEG_INF = 0xff80ff80u;
  static constexpr float LOWEST = -0x1.fep127f;
};
template <>
struct TlType<__half> {
  static constexpr int LOW_BITS = 13;
  static constexpr int PER_WORD = 2;
  static constexpr uint32_t NEG_INF = 0xfc00fc00u;
  static constexpr float LOWEST = -65504.0f;
};

__device__ __forceinline__ float tl_max_nan(float a, float b) {  // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float tl_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t tl_word_max(uint32_t a, uint32_t b, const float*) {
  return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
}
__device__ __forceinline__ uint32_t tl_word_max(uint32_t a, uint32_t b, const __nv_bfloat16*) {
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t tl_word_max(uint32_t a, uint32_t b, const __half*) {
  uint32_t r;
  asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float tl_word_max1(uint32_t a, const float*) { return __uint_as_float(a); }
__device__ __forceinline__ float tl_word_max1(uint32_t a, const __nv_bfloat16*) {
  return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
}
__device__ __forceinline__ float tl_word_max1(uint32_t a, const __half*) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&a));
  return fmaxf(f.x, f.y);
}
// Elements 2 i and 2 i + 1 of a vector.
__device__ __forceinline__ float2 tl_pair(const uint32_t* w, int i, const float*) {
  return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
}
__device__ __forceinline__ float2 tl_pair(const uint32_t* w, int i, const __nv_bfloat16*) {
  return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ float2 tl_pair(const uint32_t* w, int i, const __half*) {
  return __half22float2(*reinterpret_cast<const __half2*>(w + i));
}
// The same with -inf raised to a number (NaN stays), where 0 * x must not be 0 * -inf.  Beside any maximum between ref_lo and ref_hi (at most
// 2^24 2^20 ln 2 from 0) the exponential of that number is 0; it is no further away than that needs, so that products of a gradient's factor with its x stay finite.
__device__ __forceinline__ float2 tl_pair_raised(const uint32_t* w, int i, const float* e) {
  const float2 f = tl_pair(w, i, e);
  return make_float2(tl_max_nan(f.x, -0x1p46f), tl_max_nan(f.y, -0x1p46f));
}
__device__ __forceinline__ float2 tl_pair_raised(const uint32_t* w, int i, const __nv_bfloat16* e) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w[i]), "r"(0xd680d680u));  // -2^46
  return tl_pair(&r, 0, e);
}
__device__ __forceinline__ float2 tl_pair_raised(const uint32_t* w, int i, const __half* e) {
  uint32_t r;
  asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(w[i]), "r"(0xfbfffbffu));  // -65504
  return tl_pair(&r, 0, e);
}
__device__ __forceinline__ void tl_put_pair(uint32_t* w, int i, float a, float b, const float*) {
  w[2 * i] = __float_as_uint(a);
  w[2 * i + 1] = __float_as_uint(b);
}
__device__ __forceinline__ void tl_put_pair(uint32_t* w, int i, float a, float b, const __nv_bfloat16*) {
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(b), "f"(a));
}
__device__ __forceinline__ void tl_put_pair(uint32_t* w, int i, float a, float b, const __half*) {
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(b), "f"(a));
}

// When a vector is read: once; for the first time, and again behind the statistics; for the last time.  What will be read again should outlive
// in L2 what is read once and what is written.
enum TlRead { TL_ONCE, TL_FIRST, TL_LAST };
template <TlRead WHEN>
__device__ __forceinline__ void tl_load_vec(const void* p, uint32_t* w) {
#define TL_LOAD(how)                                                                                                              \
  asm volatile("ld.global" how ".v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"                                                  \
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])                   \
               : "l"(p))
  if (WHEN == TL_ONCE)
    TL_LOAD("");
  else if (WHEN == TL_FIRST)
    TL_LOAD(".L2::evict_last");  // PPO 4096 x 128000: 409 us without, 402 with
  else
    TL_LOAD(".L1::evict_first.L2::evict_first");
#undef TL_LOAD
}
__device__ __forceinline__ void tl_store_vec(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.L1::no_allocate.L2::evict_first.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]),
               "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

__device__ __forceinline__ void tl_report_shape(int stage) {
  if (atomicCAS(&g_status[0], 0, BITRL_ERR_SHAPE) == 0) g_status[1] = stage;
}

// ---- a group of NT threads on a row (or a share of it): a CTA, or a warp --------------------------------------------
template <int NT>
__host__ __device__ constexpr int tl_threads() {  // of the CTA
  return NT == 32 ? 32 * TL_ROW_WARPS : NT;
}
template <int NT>
__device__ __forceinline__ void tl_sync() {
  if (NT == 32)
    __syncwarp();
  else
    __syncthreads();
}
template <int NT>
__device__ __forceinline__ int tl_tid() {
  return NT == 32 ? threadIdx.x & 31 : threadIdx.x;
}

// The part of a row that a group works on: vectors lo .. hi-1 of 32 bytes from the row's first 32-byte boundary on; rank 0 has the
// elements before it and behind the last whole vector too, at most 30 of them, one a lane of its first warp.
template <class E>
struct TlShare {
  static constexpr int A = TL_VEC_BYTES / sizeof(E);
  const E* z;
  int V, head, tail, lo, hi;
  bool edges;
  __device__ TlShare(const E* z_, int V_, int C, int rank) : z(z_), V(V_) {
    head = min(V, static_cast<int>((TL_VEC_BYTES - (reinterpret_cast<uintptr_t>(z) & (TL_VEC_BYTES - 1))) & (TL_VEC_BYTES - 1)) /
                      static_cast<int>(sizeof(E)));
    const int nvec = (V - head) / A, per = (nvec + C - 1) / C;
    tail = V - head - nvec * A;
    lo = min(nvec, rank * per);
    hi = min(nvec, lo + per);
    edges = rank == 0;
  }
  __device__ __forceinline__ const E* vec(int v) const { return z + head + static_cast<size_t>(v) * A; }
  // Element of an edge lane, or -1.
  __device__ __forceinline__ int edge(int i) const { return !edges ? -1 : i < head ? i : i < head + tail ? V - tail + (i - head) : -1; }
  __device__ __forceinline__ bool owns(int j) const {
    const int v = j - head;
    return v < 0 || j >= V - tail ? edges : v / A >= lo && v / A < hi;
  }
  // Bit of an element among the vectors', or -1: it is an edge (of lane edge_lane).
  __device__ __forceinline__ int bit(int j) const { return j < head || j >= V - tail ? -1 : j - head - lo * A; }
  __device__ __forceinline__ int edge_lane(int j) const { return j < head ? j : head + j - (V - tail); }
  // The elements of the share in ascending order.
  __device__ __forceinline__ int count() const { return (hi - lo) * A + (edges ? head + tail : 0); }
  __device__ __forceinline__ int at(int i) const {
    const int h = edges ? head : 0, n = (hi - lo) * A;
    return i < h ? i : i < h + n ? head + lo * A + (i - h) : V - tail + (i - h - n);
  }
};

// Loads slots 0 .. n_u-1 of a chunk that begins at vector v; what lies behind the share is -inf.
template <TlRead WHEN, class E, int NT>
__device__ __forceinline__ void tl_load_chunk(const TlShare<E>& s, int v, int n_u, uint32_t (&w)[TL_VECS][8]) {
#pragma unroll
  for (int u = 0; u < TL_VECS; ++u) {
    if (u < n_u) {
      const int at = v + u * NT + tl_tid<NT>();
      if (at < s.hi) {
        tl_load_vec<WHEN>(s.vec(at), w[u]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[u][i] = TlType<E>::NEG_INF;
      }
    }
  }
}
// The first pass of an objective, behind which a gradient reads again (but for the last chunk), or nothing does.
template <class E, int NT>
__device__ __forceinline__ void tl_load_first(const TlShare<E>& s, int v, int n_u, bool again, uint32_t (&w)[TL_VECS][8]) {
  if (again && v + NT * TL_VECS < s.hi)
    tl_load_chunk<TL_FIRST, E, NT>(s, v, n_u, w);
  else
    tl_load_chunk<TL_ONCE, E, NT>(s, v, n_u, w);
}
template <int NT>
__device__ __forceinline__ int tl_slots(int v, int hi) {
  return min(TL_VECS, (hi - v + NT - 1) / NT);
}

// ---- statistics ---------------------------------------------------------------------------------------------------
// S = sum of 2^x and W, both relative to ref, the largest logit met.  W is sum 2^x x (ENT: for the entropy), or another sum of
// exponentials.
struct TlAcc {
  float ref, S, W;
};

// May maxima like this one use x = z c - R?
template <class E>
__device__ __forceinline__ bool tl_fused(const TlRows<E>& a, float ref) {
  return ref >= a.ref_lo && ref <= a.ref_hi;
}
// x of one logit relative to ref, as the sums have it.
template <class E>
__device__ __forceinline__ float tl_x(const TlRows<E>& a, float v, float ref) {
  return tl_fused(a, ref) ? __fmaf_rn(v, a.c, -__fmul_rn(ref, a.c)) : __fmul_rn(v - ref, a.c);
}
// R - c ref, exactly: what sums relative to R lack of being relative to c ref.  0 where they subtract first.
template <class E>
__device__ __forceinline__ float tl_rounding(const TlRows<E>& a, float ref) {
  return tl_fused(a, ref) ? __fmaf_rn(-ref, a.c, __fmul_rn(ref, a.c)) : 0.0f;
}
// From sums relative to `ref` to sums relative to `to` >= ref.  R's rounding (up to a half at |R| = 2^24) is part of the step, as another
// reference has another, or none.
template <bool ENT, class E>
__device__ __forceinline__ void tl_rebase(const TlRows<E>& a, TlAcc& s, float to) {
  if (s.ref == to) return;
  const float sh = fmaxf(__fmaf_rn(s.ref - to, a.c, tl_rounding(a, s.ref) - tl_rounding(a, to)), TL_FAR);
  const float f = tl_exp2(sh);
  s.W = f * (ENT ? __fmaf_rn(s.S, sh, s.W) : s.W);
  s.S *= f;
  s.ref = to;
}
template <bool ENT, class E>
__device__ __forceinline__ void tl_merge(const TlRows<E>& a, TlAcc& s, TlAcc o) {
  const float m = fmaxf(s.ref, o.ref);
  tl_rebase<ENT>(a, s, m);
  tl_rebase<ENT>(a, o, m);
  s.S += o.S;
  s.W += o.W;
}
// One logit relative to itself: x is 0 but for the rounding of R.
template <class E>
__device__ __forceinline__ TlAcc tl_single(const TlRows<E>& a, float v) {
  if (v == -INFINITY) return {-INFINITY, 0.0f, 0.0f};
  if (!(v < INFINITY)) return {v == INFINITY ? v : -INFINITY, NAN, NAN};
  const float x = tl_x(a, v, v), e = tl_exp2(x);
  return {v, e, e * x};
}

// Rows that may not use x = z c - R: a chunk element by element, from memory.  Tokens whose bit in `mark` is set stay out.
// (By value: what has an address would live in memory on the way that everybody else takes.)
template <bool ENT, int NT, class E>
__device__ __noinline__ TlAcc tl_plain(const TlRows<E>& a, const E* first, int lo, int hi, int v, const uint32_t* mark, TlAcc acc) {
  constexpr int A = TlShare<E>::A;
  for (int u = 0; u < TL_VECS; ++u) {
    const int at = v + u * NT + tl_tid<NT>();
    if (at >= hi) break;
    for (int i = 0; i < A; ++i) {
      const int bit = (at - lo) * A + i;
      if (mark == nullptr || !(mark[bit >> 5] >> (bit & 31) & 1)) tl_merge<ENT>(a, acc, tl_single(a, tl_f32(first[static_cast<size_t>(at) * A + i])));
    }
  }
  return acc;
}

// Elements whose bits are set become -inf.
template <class E, int N>
__device__ __forceinline__ void tl_drop(uint32_t* w, uint32_t bits) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t b = bits >> (i * TlType<E>::PER_WORD);
    if (TlType<E>::PER_WORD == 1) {
      if (b & 1) w[i] = TlType<E>::NEG_INF;
    } else {
      if (b & 1) w[i] = (w[i] & 0xffff0000u) | (TlType<E>::NEG_INF & 0xffffu);
      if (b & 2) w[i] = (w[i] & 0xffffu) | (TlType<E>::NEG_INF & 0xffff0000u);
    }
  }
}

// Adds the chunk w (n_u slots from vector v on).
template <bool ENT, int NT, class E>
__device__ __forceinline__ void tl_accumulate(const TlRows<E>& a, const TlShare<E>& share, int v, int n_u, const uint32_t (&w)[TL_VECS][8],
                                              const uint32_t* mark, TlAcc& s, float& top) {
  const E* e = nullptr;
  uint32_t mw = TlType<E>::NEG_INF;
#pragma unroll
  for (int u = 0; u < TL_VECS; ++u)
    if (u < n_u) {
#pragma unroll
      for (int i = 0; i < 8; ++i) mw = tl_word_max(mw, w[u][i], e);
    }
  top = tl_word_max1(mw, e);
  const float m = fmaxf(s.ref, top);
  const bool empty = m == -INFINITY && a.ref_lo < 0.0f;  // nothing yet but -inf, or NaN: any reference will do
  if (!tl_fused(a, m) && !empty) {
    s = tl_plain<ENT, NT>(a, share.vec(0), share.lo, share.hi, v, mark, s);
    return;
  }
  tl_rebase<ENT>(a, s, m);
  const float R = empty ? 0.0f : __fmul_rn(m, a.c);
  const uint64_t c2 = ptx::pack_f32x2(__float_as_uint(a.c), __float_as_uint(a.c));
  const uint64_t r2 = ptx::pack_f32x2(__float_as_uint(-R), __float_as_uint(-R));
  uint64_t S2[2] = {0, 0}, W2[2] = {0, 0};
#pragma unroll
  for (int u = 0; u < TL_VECS; ++u)
    if (u < n_u) {
#pragma unroll
      for (int i = 0; i < TlShare<E>::A / 2; ++i) {
        const float2 z = ENT ? tl_pair_raised(w[u], i, e) : tl_pair(w[u], i, e);
        const uint64_t x2 = ptx::fma_f32x2(ptx::pack_f32x2(__float_as_uint(z.x), __float_as_uint(z.y)), c2, r2);
        float x, y;
        ptx::unpack_f32x2(x2, x, y);
        const uint64_t e2 = ptx::pack_f32x2(__float_as_uint(tl_exp2(x)), __float_as_uint(tl_exp2(y)));
        S2[i & 1] = ptx::add_f32x2(S2[i & 1], e2);
        if (ENT) W2[i & 1] = ptx::fma_f32x2(e2, x2, W2[i & 1]);
      }
    }
  float x, y;
  ptx::unpack_f32x2(ptx::add_f32x2(S2[0], S2[1]), x, y);
  s.S += x + y;
  if (ENT) {
    ptx::unpack_f32x2(ptx::add_f32x2(W2[0], W2[1]), x, y);
    s.W += x + y;
  }
}

// Joins lanes (xor distances below `span`): the same bits in all of them.
template <bool ENT, class E>
__device__ __forceinline__ void tl_join_lanes(const TlRows<E>& a, TlAcc& s, int span) {
  float m = s.ref;
  for (int o = span >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  tl_rebase<ENT>(a, s, m);
  for (int o = span >> 1; o > 0; o >>= 1) {
    s.S += __shfl_xor_sync(0xffffffffu, s.S, o);
    s.W += __shfl_xor_sync(0xffffffffu, s.W, o);
  }
}

// Before a CTA writes to another's shared memory that one has to run: all arrive at the start, and wait before their first word.
template <class E>
__device__ __forceinline__ void tl_begin(const TlRows<E>& a) {
  if (a.C > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void tl_wait_begun() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// What the warps of a CTA, and the CTAs of a cluster, tell one another.
struct TlXch {
  TlAcc red[TL_MAX_WARPS], acc[TL_MAX_CLUSTER];
};

// Joins the threads of a group, then the CTAs of a cluster, in a fixed order.  The result is in all lanes of the group's first warp.
// send() writes what else the CTAs tell one another.
template <int NT, bool ENT, class E, class Send>
__device__ __forceinline__ void tl_join(const TlRows<E>& a, TlAcc& s, TlXch* x, int rank, Send&& send) {
  tl_join_lanes<ENT>(a, s, 32);
  if (NT == 32) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int WARPS = NT / 32 > 0 ? NT / 32 : 1;
  if (lane == 0) x->red[warp] = s;
  __syncthreads();
  if (warp == 0) {
    s = x->red[lane & (WARPS - 1)];
    tl_join_lanes<ENT>(a, s, WARPS);
  }
  if (a.C == 1) return;
  tl_wait_begun();
  if (threadIdx.x < a.C) {
    const uint32_t to = ptx::mapa_u32(ptx::smem_u32(&x->acc[rank]), threadIdx.x);
    ptx::sts32_cluster(to, __float_as_uint(s.ref));
    ptx::sts32_cluster(to + 4, __float_as_uint(s.S));
    ptx::sts32_cluster(to + 8, __float_as_uint(s.W));
  }
  send();
  ptx::cluster_sync_all();
  if (warp == 0) {
    s = x->acc[lane & (a.C - 1)];
    tl_join_lanes<ENT>(a, s, a.C);
  }
}

// A row's scalars.  log S relative to the largest logit m itself, in 64 bits: the sums are relative to R instead of c m.
struct TlStat {
  float m, S;
  double log_rel, log_s, H;  // log S, log S relative to m, entropy
};
// (R - c ref) ln 2: what the logarithm of sums relative to R lacks.
template <class E>
__device__ __forceinline__ double tl_shift(const TlRows<E>& a, float ref) {
  return tl_fused(a, ref) ? (static_cast<double>(__fmul_rn(ref, a.c)) - static_cast<double>(ref) * static_cast<double>(a.c)) * TL_LN2 : 0.0;
}
template <bool ENT, class E>
__device__ __forceinline__ TlStat tl_stat(const TlRows<E>& a, const TlAcc& s) {
  TlStat r;
  r.m = s.ref;
  r.S = s.S;
  if (s.S == 0.0f) {
    r.log_s = r.log_rel = -INFINITY;
    r.H = 0.0;
    return r;
  }
  const double log_rel = log(static_cast<double>(s.S));
  r.log_rel = log_rel;
  r.log_s = log_rel + tl_shift(a, s.ref);
  r.H = ENT ? log_rel - TL_LN2 * (static_cast<double>(s.W) / static_cast<double>(s.S)) : 0.0;
  return r;
}
// log p of a logit: -inf for a logit of -inf, also in a row that has nothing else (S = 0), and NaN in a row without statistics.
template <class E>
__device__ __forceinline__ double tl_logp(const TlRows<E>& a, const TlStat& r, float v) {
  if (r.S == 0.0f) return -INFINITY;
  const float d = v - r.m;  // beyond fp32's range: -inf
  return (d == -INFINITY ? -INFINITY : (static_cast<double>(v) - static_cast<double>(r.m)) * a.it) - r.log_s;
}

// ---- gradients ------------------------------------------------------------------------------------------------------
// dz_j = 2^x_j (A + B x_j), element by element in one pass; B = 0 (LINEAR false) takes a factor alone.
struct TlCoef {
  float ref, A, B;
  bool zero;  // nothing but zeros
};
template <bool LINEAR, class E>
__device__ __forceinline__ float tl_coef_at(const TlRows<E>& a, const TlCoef& k, float v) {
  if (k.zero) return 0.0f;
  float x = tl_x(a, v, k.ref);
  if (LINEAR) {
    if (x < TL_FAR) x = TL_FAR;
    return tl_exp2(x) * __fmaf_rn(k.B, x, k.A);
  }
  return tl_exp2(x) * k.A;
}
template <bool LINEAR, int N, class E>
__device__ __forceinline__ void tl_coef_words(const TlRows<E>& a, const TlCoef& k, const uint32_t* w, uint32_t* out) {
  const E* e = nullptr;
  if (tl_fused(a, k.ref)) {
    const float R = __fmul_rn(k.ref, a.c);
    const uint64_t c2 = ptx::pack_f32x2(__float_as_uint(a.c), __float_as_uint(a.c));
    const uint64_t r2 = ptx::pack_f32x2(__float_as_uint(-R), __float_as_uint(-R));
    const uint64_t A2 = ptx::pack_f32x2(__float_as_uint(k.A), __float_as_uint(k.A));
    const uint64_t B2 = ptx::pack_f32x2(__float_as_uint(k.B), __float_as_uint(k.B));
#pragma unroll
    for (int i = 0; i < N * TlType<E>::PER_WORD / 2; ++i) {
      const float2 z = LINEAR ? tl_pair_raised(w, i, e) : tl_pair(w, i, e);
      const uint64_t x2 = ptx::fma_f32x2(ptx::pack_f32x2(__float_as_uint(z.x), __float_as_uint(z.y)), c2, r2);
      float x, y;
      ptx::unpack_f32x2(x2, x, y);
      float p = k.A, q = k.A;
      if (LINEAR) ptx::unpack_f32x2(ptx::fma_f32x2(B2, x2, A2), p, q);
      tl_put_pair(out, i, tl_exp2(x) * p, tl_exp2(y) * q, e);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N * TlType<E>::PER_WORD / 2; ++i) {
      const float2 z = tl_pair(w, i, e);
      tl_put_pair(out, i, tl_coef_at<LINEAR>(a, k, z.x), tl_coef_at<LINEAR>(a, k, z.y), e);
    }
  }
}

// First vector of a share's last chunk.
template <int NT, class E>
__device__ __forceinline__ int tl_last_chunk(const TlShare<E>& s) {
  return s.lo + (s.hi - s.lo - 1) / (NT * TL_VECS) * (NT * TL_VECS);
}

// Writes a share of the gradient, from its last chunk, which the threads still hold in w, back to the first: what was read last is the
// nearest.  Where the gradient's row has the logits' place within 32 bytes, a vector goes out as one; else the share goes element by
// element (a warp's stores side by side).
template <bool LINEAR, int NT, class E>
__device__ __forceinline__ void tl_write_gradient(const TlRows<E>& a, const TlShare<E>& s, const TlCoef& k, E* dz, uint32_t (&w)[TL_VECS][8]) {
  const int tid = tl_tid<NT>();
  if (((reinterpret_cast<uintptr_t>(dz) ^ reinterpret_cast<uintptr_t>(s.z)) & (TL_VEC_BYTES - 1)) == 0) {
    if (s.hi > s.lo) {
      const int last = tl_last_chunk<NT>(s);
      for (int v = last; v >= s.lo; v -= NT * TL_VECS) {
        const int n_u = tl_slots<NT>(v, s.hi);
        if (v != last && !k.zero) tl_load_chunk<TL_LAST, E, NT>(s, v, n_u, w);
#pragma unroll
        for (int u = 0; u < TL_VECS; ++u)
          if (u < n_u) {
            const int at = v + u * NT + tid;
            if (at < s.hi) {
              uint32_t out[8] = {0, 0, 0, 0, 0, 0, 0, 0};
              if (!k.zero) tl_coef_words<LINEAR, 8>(a, k, w[u], out);
              tl_store_vec(dz + s.head + static_cast<size_t>(at) * TlShare<E>::A, out);
            }
          }
      }
    }
    if (tid < 32) {
      const int j = s.edge(tid);
      if (j >= 0) tl_set(dz + j, k.zero ? 0.0f : tl_coef_at<LINEAR>(a, k, tl_f32(s.z[j])));
    }
  } else {
    const int n = s.count();
    for (int i = tid; i < n; i += NT) {
      const int j = s.at(i);
      tl_set(dz + j, k.zero ? 0.0f : tl_coef_at<LINEAR>(a, k, tl_f32(s.z[j])));
    }
  }
}

// d (G log p_a + E H) / dz_j = (G 1[j = a] - p_j (G + E (log p_j + H))) / temperature with p = 2^x / S, log p = x ln2 - log S (rel: S's).
template <class E>
__device__ __forceinline__ TlCoef tl_policy_coef(const TlRows<E>& a, float ref, double S, double log_rel, double H, double G, double ent) {
  TlCoef k;
  const double f = -a.it / S;
  k.ref = ref;
  k.A = static_cast<float>(f * (G + ent * (H - log_rel)));
  k.B = static_cast<float>(f * ent * TL_LN2);
  k.zero = S == 0.0 || (G == 0.0 && ent == 0.0);
  return k;
}

// The token's own element: what all elements have, and G, rounded once.
template <class E>
__device__ __forceinline__ void tl_write_token(const TlRows<E>& a, const TlCoef& k, float G, float picked, E* at) {
  tl_set(at, static_cast<float>(G * a.it + tl_coef_at<true>(a, k, picked)));
}

// ---- log probabilities, entropy, alternatives -------------------------------------------------------------------------
struct TlOut {
  const int* tokens;
  float *logp, *entropy, *stats;
  int* top_ids;
  float* top_logp;
  int k;
};

// Order of the alternatives: greater logit first, then the lower index.  -0 counts as 0; NaN and -inf are none (0).
__device__ __forceinline__ uint32_t tl_order(float v) {
  if (!(v > -INFINITY)) return 0;
  const uint32_t u = __float_as_uint(v + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float tl_order_value(uint32_t o) {
  return o == 0 ? -INFINITY : __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ unsigned long long tl_key(float v, int j) {
  const uint32_t o = tl_order(v);
  return o == 0 ? 0 : static_cast<unsigned long long>(o) << 32 | static_cast<uint32_t>(~j);
}
__device__ __forceinline__ int tl_key_token(unsigned long long key) { return static_cast<int>(~static_cast<uint32_t>(key)); }

template <int NT>
struct TlTop {
  unsigned long long cand[TL_CANDIDATES];
  unsigned long long best[BITRL_TOP_MAX];
  uint32_t seg[TL_SEGMENTS];  // chunk << 9 | thread
  uint32_t largest[NT], kth;
  uint32_t red[NT / 32];
  int n, n_best, n_seg;
};

template <int NT>
__device__ __forceinline__ int tl_cta_sum(int v, uint32_t* red) {
  v = __reduce_add_sync(0xffffffffu, v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  int s = 0;
#pragma unroll
  for (int i = 0; i < NT / 32; ++i) s += red[i];
  return s;
}

// The k greatest of t.cand[0 .. n-1] (distinct keys), in order, into t.best; t.n_best of them.
template <int NT>
__device__ __noinline__ void tl_rank(TlTop<NT>& t, int n, int k) {
  __syncthreads();
  unsigned long long least = 0;
  if (n > 2 * NT) {  // too many to compare each with each: find the k-th key bit by bit
    for (int b = 63; b >= 0; --b) {
      if (b < 32 && b >= 20) {  // indices are below 2^20: these bits are ones in every key
        least |= 1ull << b;
        continue;
      }
      const unsigned long long trial = least | 1ull << b;
      int c = 0;
      for (int i = threadIdx.x; i < n; i += NT) c += t.cand[i] >= trial;
      if (tl_cta_sum<NT>(c, t.red) >= k) least = trial;
    }
    // compact the k keys from `least` on into the front part: gathered in best first, then copied
    if (threadIdx.x == 0) t.n_best = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT)
      if (t.cand[i] >= least) t.best[atomicAdd(&t.n_best, 1)] = t.cand[i];
    __syncthreads();
    n = t.n_best;
    if (threadIdx.x < n) t.cand[threadIdx.x] = t.best[threadIdx.x];
    __syncthreads();
  }
  for (int i = threadIdx.x; i < n; i += NT) {
    const unsigned long long key = t.cand[i];
    int r = 0;
    for (int j = 0; j < n; ++j) r += t.cand[j] > key;
    if (r < k) t.best[r] = key;
  }
  if (threadIdx.x == 0) t.n_best = min(n, k);
  __syncthreads();
}

// The share's k greatest where more than TL_CANDIDATES elements are not below `floor_` (a value that at least k reach): values that
// many tokens share, or rows in an order that starves most threads.  Passes over the share, from memory.
template <int NT, class E>
__device__ __noinline__ void tl_top_exact(TlTop<NT>& t, const TlShare<E>& s, uint32_t floor_, int k) {
  const int n = s.count();
  auto above = [&](uint32_t o) {
    int c = 0;
    for (int i = threadIdx.x; i < n; i += NT) c += tl_order(tl_f32(s.z[s.at(i)])) > o;
    return tl_cta_sum<NT>(c, t.red);
  };
  uint32_t kth = floor_;  // the k-th greatest value: fewer than k lie above it
  if (above(kth) >= k) {
    uint32_t lo = kth, hi = 0xffffffffu;  // above(lo) >= k > above(hi)
    while (hi - lo > 1) {
      const uint32_t mid = lo + (hi - lo) / 2;
      if (above(mid) >= k)
        lo = mid;
      else
        hi = mid;
    }
    kth = hi;
  }
  __syncthreads();
  if (threadIdx.x == 0) t.n = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += NT) {
    const int j = s.at(i);
    const float v = tl_f32(s.z[j]);
    if (tl_order(v) > kth) t.cand[atomicAdd(&t.n, 1)] = tl_key(v, j);
  }
  __syncthreads();
  int have = t.n;
  __syncthreads();
  for (int base = 0; kth != 0 && base < n && have < k; base += NT) {  // of those equal to it, the first ones
    const int i = base + threadIdx.x;
    const int j = i < n ? s.at(i) : 0;
    const float v = i < n ? tl_f32(s.z[j]) : -INFINITY;
    const bool hit = tl_order(v) == kth;
    const uint32_t m = __ballot_sync(0xffffffffu, hit);
    if ((threadIdx.x & 31) == 0) t.red[threadIdx.x >> 5] = __popc(m);
    __syncthreads();
    int before = __popc(m & ((1u << (threadIdx.x & 31)) - 1)), all = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
      if (w < (threadIdx.x >> 5)) before += t.red[w];
      all += t.red[w];
    }
    if (hit && have + before < k) t.cand[have + before] = tl_key(v, j);
    have = min(k, have + all);
    __syncthreads();
  }
  tl_rank(t, have, k);
}

// The k-th greatest of the threads' largest logits is a value that at least k elements of the share reach, and seldom many more.  A
// segment is a thread's part of a chunk; `seg` has the largest logit of each.  Those that reach the value are listed, and a warp
// looks at the elements of a segment together, a word a lane.
template <int NT, class E>
__device__ __forceinline__ void tl_top(TlTop<NT>& t, const TlShare<E>& s, const float* seg, float mine, float edge_v, int edge_j, int k) {
  constexpr int STEP = NT * TL_VECS;
  const uint32_t order = tl_order(mine);
  t.largest[threadIdx.x] = order;
  __syncthreads();
  if (threadIdx.x < 32) {  // the k-th greatest, in one warp: no barrier in the loops
    uint32_t of[NT / 32], kth = 0;
#pragma unroll
    for (int i = 0; i < NT / 32; ++i) of[i] = t.largest[32 * i + threadIdx.x];
    if (k < 32 - TlType<E>::LOW_BITS) {  // few: one after the other is taken out
      for (int j = 0; j < k; ++j) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < NT / 32; ++i) m = max(m, of[i]);
        kth = __reduce_max_sync(0xffffffffu, m);
        const uint32_t have = __ballot_sync(0xffffffffu, m == kth);
        if (kth == 0) break;
        if (static_cast<int>(threadIdx.x) == __ffs(have) - 1) {
          bool taken = false;
#pragma unroll
          for (int i = 0; i < NT / 32; ++i)
            if (!taken && of[i] == kth) {
              of[i] = 0;
              taken = true;
            }
        }
      }
    } else {
      for (int b = 31; b >= TlType<E>::LOW_BITS; --b) {  // bit by bit; below, all values of the type have the same bits, or bits that decide nothing
        const uint32_t trial = kth | 1u << b;
        int c = 0;
#pragma unroll
        for (int i = 0; i < NT / 32; ++i) c += of[i] >= trial;
        c = __reduce_add_sync(0xffffffffu, c);
        if (c >= k) {
          kth = trial;
          if (c == k) break;
        }
      }
    }
    if (threadIdx.x == 0) {
      t.kth = kth;
      t.n = t.n_seg = 0;
    }
  }
  __syncthreads();
  const uint32_t kth = t.kth;
  const uint32_t bar = max(kth, 1u);
  auto offer = [&](float v, int j) {
    if (tl_order(v) >= bar) {
      const int at = atomicAdd(&t.n, 1);
      if (at < TL_CANDIDATES) t.cand[at] = tl_key(v, j);
    }
  };
  const int chunks = (s.hi - s.lo + STEP - 1) / STEP;
  if (order >= bar) {
    for (int c = 0; c < chunks; ++c)
      if (tl_order(seg[c * NT + threadIdx.x]) >= bar) {
        const int at = atomicAdd(&t.n_seg, 1);
        if (at < TL_SEGMENTS) t.seg[at] = c << 9 | threadIdx.x;
      }
    if (edge_j >= 0) offer(edge_v, edge_j);
  }
  __syncthreads();
  const int n_seg = t.n_seg, lane = threadIdx.x & 31;
  if (n_seg <= TL_SEGMENTS) {
    constexpr int BATCH = 8;  // segments of a warp on their way at once: memory is 1000 cycles and more away
    for (int i = threadIdx.x >> 5; i < n_seg; i += BATCH * (NT / 32)) {
      uint32_t word[BATCH];
      int at[BATCH];
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        const int q = i + b * (NT / 32);
        at[b] = -1;
        if (q < n_seg) {
          const uint32_t id = t.seg[q];
          const int v = s.lo + static_cast<int>(id >> 9) * STEP + (lane >> 3) * NT + static_cast<int>(id & 511);
          if (v < s.hi) {
            at[b] = s.head + v * TlShare<E>::A + (lane & 7) * TlType<E>::PER_WORD;
            word[b] = *reinterpret_cast<const uint32_t*>(s.z + at[b]);
          }
        }
      }
#pragma unroll
      for (int b = 0; b < BATCH; ++b)
        if (at[b] >= 0) {
          const uint32_t two[2] = {word[b], word[b]};
          const float2 f = tl_pair(two, 0, static_cast<const E*>(nullptr));
          offer(f.x, at[b]);
          if (TlType<E>::PER_WORD == 2) offer(f.y, at[b] + 1);
        }
    }
    __syncthreads();
  }
  const int n = t.n;
  if (n_seg > TL_SEGMENTS || n > TL_CANDIDATES)
    tl_top_exact(t, s, kth, k);
  else
    tl_rank(t, n, k);
}

template <class E>
__device__ __forceinline__ void tl_write_stat(const TlRows<E>& a, const TlOut& o, const TlStat& r, float picked, size_t t) {
  if (o.logp) o.logp[t] = static_cast<float>(tl_logp(a, r, picked));
  if (o.entropy) o.entropy[t] = static_cast<float>(r.H);
  if (o.stats) {
    o.stats[2 * t] = r.m;
    o.stats[2 * t + 1] = static_cast<float>(r.log_s);
  }
}

// One CTA (of a cluster) for a row; NT = 32: a warp, without alternatives.
template <class E, int NT, bool TOP>
__global__ void __launch_bounds__(tl_threads<NT>(), 1024 / tl_threads<NT>())
token_logprobs_kernel(const __grid_constant__ TlRows<E> a, const __grid_constant__ TlOut o) {
  extern __shared__ __align__(16) unsigned char tl_smem[];
  __shared__ TlXch xch;
  __shared__ TlStat stat;
  pdl_enter();
  const int row_of_cta = NT == 32 ? blockIdx.x * TL_ROW_WARPS + (threadIdx.x >> 5) : blockIdx.x / a.C;
  const int rank = NT == 32 ? 0 : blockIdx.x % a.C, tid = tl_tid<NT>();
  if (NT == 32 && row_of_cta >= a.T) return;
  const size_t t = row_of_cta;
  const int tok = o.tokens ? o.tokens[t] : 0;
  if (tok < 0 || tok >= a.V) {
    if (rank != 0) return;
    if (tid == 0) {
      if (tok >= a.V) tl_report_shape(60);
      if (o.logp) o.logp[t] = 0.0f;
      if (o.entropy) o.entropy[t] = 0.0f;
      if (o.stats) o.stats[2 * t] = o.stats[2 * t + 1] = 0.0f;
    }
    for (int i = tid; i < o.k; i += NT) {
      if (o.top_ids) o.top_ids[t * o.k + i] = -1;
      if (o.top_logp) o.top_logp[t * o.k + i] = -INFINITY;
    }
    return;
  }
  tl_begin(a);
  const TlShare<E> s(a.z + row_of_cta * a.ld, a.V, a.C, rank);
  const float picked = tl_f32(s.z[tok]);
  TlTop<NT>* top = reinterpret_cast<TlTop<NT>*>(tl_smem);
  unsigned long long* lists = reinterpret_cast<unsigned long long*>(tl_smem + sizeof(TlTop<NT>));  // [C][k], in rank 0
  float* seg = reinterpret_cast<float*>(lists + (a.C > 1 ? a.C * o.k : 0));
  uint32_t w[TL_VECS][8];
  TlAcc acc = {-INFINITY, 0.0f, 0.0f};
  const int edge_j = tid < 32 ? s.edge(tid) : -1;
  const float edge_v = edge_j >= 0 ? tl_f32(s.z[edge_j]) : -INFINITY;
  float mine = -INFINITY;
  for (int v = s.lo; v < s.hi; v += NT * TL_VECS) {
    const int n_u = tl_slots<NT>(v, s.hi);
    tl_load_chunk<TL_ONCE, E, NT>(s, v, n_u, w);
    float largest;
    tl_accumulate<true, NT>(a, s, v, n_u, w, nullptr, acc, largest);
    if (TOP) {
      mine = fmaxf(mine, largest);
      seg[(v - s.lo) / TL_VECS + tid] = largest;
    }
  }
  if (TOP) tl_top<NT>(*top, s, seg, fmaxf(mine, edge_v), edge_v, edge_j, o.k);
  if (edge_j >= 0) tl_merge<true>(a, acc, tl_single(a, edge_v));
  tl_join<NT, true>(a, acc, &xch, rank, [&] {  // with it the shares' alternatives, which meet in rank 0
    if (!TOP) return;
    const uint32_t to = ptx::mapa_u32(ptx::smem_u32(lists + rank * o.k), 0);
    for (int i = threadIdx.x; i < o.k; i += NT) {
      const unsigned long long key = i < top->n_best ? top->best[i] : 0;
      ptx::sts32_cluster(to + 8 * i, static_cast<uint32_t>(key));
      ptx::sts32_cluster(to + 8 * i + 4, static_cast<uint32_t>(key >> 32));
    }
  });
  if (rank != 0) return;
  if (tid == 0) {
    const TlStat r = tl_stat<true>(a, acc);
    if (TOP) stat = r;
    tl_write_stat(a, o, r, picked, t);
  }
  if (TOP) {
    if (a.C > 1) {
      // the greatest of the lists' last keys: k keys of its list reach it
      unsigned long long least = 0;
      for (int c = 0; c < a.C; ++c) least = max(least, lists[c * o.k + o.k - 1]);
      if (threadIdx.x == 0) top->n = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < a.C * o.k; i += NT)
        if (lists[i] != 0 && lists[i] >= least) top->cand[atomicAdd(&top->n, 1)] = lists[i];
      __syncthreads();
      tl_rank<NT>(*top, top->n, o.k);
    }
    __syncthreads();
    const TlStat r = stat;
    for (int i = threadIdx.x; i < o.k; i += NT) {
      const bool there = i < top->n_best;
      const unsigned long long key = there ? top->best[i] : 0;
      if (o.top_ids) o.top_ids[t * o.k + i] = there ? tl_key_token(key) : -1;
      if (o.top_logp) o.top_logp[t * o.k + i] = there ? static_cast<float>(tl_logp(a, r, tl_order_value(static_cast<uint32_t>(key >> 32)))) : -INFINITY;
    }
  }
}

// ---- the gradient of log probabilities and entropies --------------------------------------------------------------------
struct TlPolicy {
  const int* tokens;
  const float *stats, *entropy, *dlogp, *dentropy;
};

// The forward call gave log S relative to m; here the sums' reference is R.
template <class E>
__device__ __forceinline__ TlCoef tl_backward_coef(const TlRows<E>& a, const TlPolicy& o, size_t t, float G, float ent) {
  const float m = o.stats[2 * t];
  const double log_rel = static_cast<double>(o.stats[2 * t + 1]) - tl_shift(a, m);
  return tl_policy_coef(a, m, exp(log_rel), log_rel, o.entropy ? o.entropy[t] : 0.0, G, ent);
}

// A share of a row a CTA, without a word between them: everything that a row needs is in its statistics.
template <class E, int NT>
__global__ void __launch_bounds__(tl_threads<NT>(), 1024 / tl_threads<NT>())
token_logprobs_backward_kernel(const __grid_constant__ TlRows<E> a, const __grid_constant__ TlPolicy o, const __grid_constant__ TlGrad<E> g) {
  __shared__ TlCoef coef;
  pdl_enter();
  const int row = NT == 32 ? blockIdx.x * TL_ROW_WARPS + (threadIdx.x >> 5) : blockIdx.x / a.C;
  const int rank = NT == 32 ? 0 : blockIdx.x % a.C, tid = tl_tid<NT>();
  if (NT == 32 && row >= a.T) return;
  const size_t t = row;
  const TlShare<E> s(a.z + row * a.ld, a.V, a.C, rank);
  E* dz = g.dz + row * g.ld;
  const int tok = o.tokens ? o.tokens[t] : 0;
  const float G = o.dlogp ? o.dlogp[t] : 0.0f, ent = o.dentropy ? o.dentropy[t] : 0.0f;
  const bool live = tok >= 0 && tok < a.V && !(G == 0.0f && ent == 0.0f);
  if (tok >= a.V && tid == 0 && rank == 0) tl_report_shape(61);
  uint32_t w[TL_VECS][8];
  if (live && s.hi > s.lo) {
    const int v = tl_last_chunk<NT>(s);
    tl_load_chunk<TL_LAST, E, NT>(s, v, tl_slots<NT>(v, s.hi), w);
  }
  const bool hit = live && o.dlogp && s.owns(tok);
  const float picked = hit ? tl_f32(s.z[tok]) : 0.0f;
  TlCoef k = {0.0f, 0.0f, 0.0f, true};
  if (live) {
    if (tid == 0) k = tl_backward_coef(a, o, t, G, ent);
    if (NT == 32) {
      k.ref = __shfl_sync(0xffffffffu, k.ref, 0);
      k.A = __shfl_sync(0xffffffffu, k.A, 0);
      k.B = __shfl_sync(0xffffffffu, k.B, 0);
      k.zero = __shfl_sync(0xffffffffu, static_cast<int>(k.zero), 0);
    } else {
      if (tid == 0) coef = k;
      __syncthreads();
      k = coef;
    }
  }
  if (NT == 32) __syncwarp();  // the token's logit has been read
  tl_write_gradient<true, NT>(a, s, k, dz, w);
  if (hit && !k.zero) {
    tl_sync<NT>();
    if (tid == 0) tl_write_token(a, k, G, picked, dz + tok);
  }
}

// ---- the PPO objective over tokens ----------------------------------------------------------------------------------------
struct TlPpo {
  const int* tokens;
  const float *old_logp, *adv, *weight;
  float eps, beta;
  float* terms;
};

// What a row brings along beside its logits.
struct TlPpoRow {
  float picked, old_logp, adv, weight;
};
template <class E>
__device__ __forceinline__ TlPpoRow tl_ppo_row(const TlPpo& o, const E* z, size_t t, int tok) {
  return {tl_f32(z[tok]), o.old_logp[t], o.adv[t], o.weight ? o.weight[t] : 1.0f};
}
// The row's terms (written where `write`) and its gradient's coefficients; G: the token's own.
template <class E>
__device__ __forceinline__ TlCoef tl_ppo_finish(const TlRows<E>& a, const TlPpo& o, const TlPpoRow& p, const TlAcc& acc, size_t t, bool write, float& G) {
  const TlStat r = tl_stat<true>(a, acc);
  const double logp = tl_logp(a, r, p.picked);
  const float ratio = static_cast<float>(exp(logp - p.old_logp));
  const float s1 = ratio * p.adv, s2 = fminf(fmaxf(ratio, 1.0f - o.eps), 1.0f + o.eps) * p.adv;
  const float gain = s1 > s2 ? s2 : s1;  // a NaN stays
  if (write) *reinterpret_cast<float4*>(o.terms + 4 * t) = make_float4(ratio, gain, static_cast<float>(r.H), static_cast<float>(logp));
  G = 0.0f;
  if (p.weight == 0.0f) return {0.0f, 0.0f, 0.0f, true};
  if (s1 <= s2 || isnan(acc.S)) G = -p.weight * s1;  // a row with NaN or +inf shows it, also without entropy in the objective
  return tl_policy_coef(a, acc.ref, acc.S, r.log_rel, r.H, G, -p.weight * o.beta);
}

template <class E, int NT>
__global__ void __launch_bounds__(tl_threads<NT>(), 1024 / tl_threads<NT>())
ppo_token_kernel(const __grid_constant__ TlRows<E> a, const __grid_constant__ TlPpo o, const __grid_constant__ TlGrad<E> g) {
  __shared__ TlXch xch;
  __shared__ TlCoef coef;
  __shared__ float shared_G;
  pdl_enter();
  const int row = NT == 32 ? blockIdx.x * TL_ROW_WARPS + (threadIdx.x >> 5) : blockIdx.x / a.C;
  const int rank = NT == 32 ? 0 : blockIdx.x % a.C, tid = tl_tid<NT>();
  if (NT == 32 && row >= a.T) return;
  const size_t t = row;
  const TlShare<E> s(a.z + row * a.ld, a.V, a.C, rank);
  E* dz = g.dz ? g.dz + row * g.ld : nullptr;
  const int tok = o.tokens[t];
  uint32_t w[TL_VECS][8];
  TlCoef k = {0.0f, 0.0f, 0.0f, true};
  if (tok < 0 || tok >= a.V) {
    if (tid == 0 && rank == 0) {
      if (tok >= a.V) tl_report_shape(62);
      *reinterpret_cast<float4*>(o.terms + 4 * t) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    if (dz) tl_write_gradient<true, NT>(a, s, k, dz, w);
    return;
  }
  tl_begin(a);
  const TlPpoRow p = tl_ppo_row(o, s.z, t, tok);
  TlAcc acc = {-INFINITY, 0.0f, 0.0f};
  const int edge_j = tid < 32 ? s.edge(tid) : -1;
  const float edge_v = edge_j >= 0 ? tl_f32(s.z[edge_j]) : -INFINITY;
  for (int v = s.lo; v < s.hi; v += NT * TL_VECS) {
    const int n_u = tl_slots<NT>(v, s.hi);
    tl_load_first<E, NT>(s, v, n_u, dz != nullptr, w);
    float largest;
    tl_accumulate<true, NT>(a, s, v, n_u, w, nullptr, acc, largest);
  }
  if (edge_j >= 0) tl_merge<true>(a, acc, tl_single(a, edge_v));
  tl_join<NT, true>(a, acc, &xch, rank, [] {});  // everybody of the cluster has read its part of the row, and the token's logit
  float G = 0.0f;
  if (tid == 0) k = tl_ppo_finish(a, o, p, acc, t, rank == 0, G);
  if (!dz) return;
  if (NT == 32) {
    G = __shfl_sync(0xffffffffu, G, 0);
    k.ref = __shfl_sync(0xffffffffu, k.ref, 0);
    k.A = __shfl_sync(0xffffffffu, k.A, 0);
    k.B = __shfl_sync(0xffffffffu, k.B, 0);
    k.zero = __shfl_sync(0xffffffffu, static_cast<int>(k.zero), 0);
    __syncwarp();  // the token's logit has been read
  } else {
    if (tid == 0) {
      coef = k;
      shared_G = G;
    }
    __syncthreads();
    k = coef;
    G = shared_G;
  }
  tl_write_gradient<true, NT>(a, s, k, dz, w);
  if (!k.zero && s.owns(tok)) {
    tl_sync<NT>();
    if (tid == 0) tl_write_token(a, k, G, p.picked, dz + tok);
  }
}

// ---- distillation ---------------------------------------------------------------------------------------------------------
struct TlTeacher {
  const int* ids;
  const float *values, *weight;
  int K, tail;
  float* loss;
};

__device__ __forceinline__ double tl_warp_sum64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// loss = sum_k q_k (log q_k - log p_{id_k}) [+ q_r (log q_r - log p_r)], the teacher's q from its values, and
// dz_j = w ((sum q + q_r) p_j - sum_{id_k = j} q_k - [j outside the ids] q_r p_j / p_r) / temperature.
// p_r, the student's mass outside the ids, is summed over those tokens themselves: as a difference from 1 it would lose what
// decides a sure student's loss.  So the pass over the row leaves the named tokens out (their bits in a bitmap), and they are added
// one by one.  The loss is put together in 64 bits: its terms cancel where the student is near its teacher.  In the gradient every element is
// a multiple of 2^x; the named tokens' are written again, each with its q.

// A row's entries in shared memory.
struct TlTables {
  static constexpr int ARRAYS = 4;
  float *value, *zk, *qk;
  int* id;
  __device__ TlTables(void* p, int K) : value(static_cast<float*>(p)), zk(value + K), qk(zk + K), id(reinterpret_cast<int*>(qk + K)) {}
};

// What is found out about a row's teacher: sum q, sum q log q, sum q (z - base) / temperature (not normed without tail) and the named
// tokens' sum of exponentials.  dot and named over the tokens that the share owns.
struct TlLesson {
  float base;  // a named token's logit, so that what is summed stays small beside logits of any size
  double mass, own, dot;
  TlAcc named;
};

// Reads the entries tid, tid + n, ..., and with tail marks the named tokens: a bit for each element of the share's vectors, and for its
// edges; *twice, where a token is named again.  Is one of them a teacher's?  Their largest value and the first of them go to `largest` and `first`.
template <class Share>
__device__ __forceinline__ int tl_entries(const TlTeacher& o, const Share& s, size_t t, const TlTables& tab, uint32_t* mark, uint32_t* edge_marks, int* twice,
                                          bool report, int tid, int n, float& largest, int& first) {
  int any = 0;
  largest = -INFINITY;
  first = o.K;
  for (int k = tid; k < o.K; k += n) {
    int j = o.ids[t * o.K + k];
    if (j >= s.V) {
      if (report) tl_report_shape(63);
      j = -1;
    }
    const float v = o.values[t * o.K + k];
    tab.id[k] = j;
    tab.value[k] = v;
    if (j < 0) continue;
    any |= o.tail || v != -INFINITY;
    largest = fmaxf(largest, v);
    first = min(first, k);
    if (o.tail && s.owns(j)) {
      const int at = s.bit(j);
      const uint32_t bit = 1u << (at < 0 ? s.edge_lane(j) : at & 31);
      if (atomicOr(at < 0 ? edge_marks : &mark[at >> 5], bit) & bit) *twice = 1;
    }
  }
  return any;
}

// Entry k: its q, and its part in the sums; z: its token's logit, where the share owns it.
template <class E, class Share>
__device__ __forceinline__ void tl_study(const TlRows<E>& a, const TlTeacher& o, const Share& s, const TlTables& tab, bool twice, float largest, int k, float z,
                                         TlLesson& l) {
  const int j = tab.id[k];
  const bool here = j >= 0 && s.owns(j);
  const float v = tab.value[k];
  double p = 0.0;
  if (j >= 0 && v != -INFINITY) {
    const double lp = o.tail ? static_cast<double>(v) : (static_cast<double>(v) - largest) * a.it;
    p = exp(lp);
    l.mass += p;
    if (p != 0.0) {
      l.own += p * lp;
      if (here) l.dot += p * ((static_cast<double>(z) - l.base) * a.it);
    }
  }
  if (here && o.tail) {
    bool first = true;  // a token named twice has its mass once
    if (twice)
      for (int i = 0; i < k; ++i) first = first && tab.id[i] != j;
    if (first) tl_merge<false>(a, l.named, tl_single(a, z));
  }
  tab.zk[k] = z;
  tab.qk[k] = static_cast<float>(p);
}

// The row's scalars, of one warp.
struct TlMark {
  TlCoef coef;
  double f, total, log_s, norm;
  float m;
};
template <class E>
__device__ __forceinline__ TlMark tl_conclude(const TlRows<E>& a, const TlTeacher& o, const TlAcc& acc, const TlLesson& l, size_t t, bool write) {
  const int lane = threadIdx.x & 31;
  TlMark r;
  r.m = fmaxf(acc.ref, l.named.ref);
  const bool none = acc.S == 0.0f && l.named.S == 0.0f;
  // sums relative to m itself
  const float ref = lane & 1 ? l.named.ref : acc.ref, sum = lane & 1 ? l.named.S : acc.S;  // both at once: a lane each
  const double far = (static_cast<double>(ref) - r.m) * a.it + tl_shift(a, ref), part = sum == 0.0f ? 0.0 : static_cast<double>(sum) * exp(far);
  const double gap = __shfl_sync(0xffffffffu, far, 0), so = __shfl_sync(0xffffffffu, part, 0), sn = __shfl_sync(0xffffffffu, part, 1);
  double q_rest = o.tail && l.mass < 1.0 ? 1.0 - l.mass : 0.0;
  const bool below = so == 0.0;  // p_r, below what 64 bits hold; its logarithm need not be
  // Outside: no logit, none within fp32's reach, or a mask of the type's lowest value.
  const bool nothing = acc.S == 0.0f || (below && (acc.ref - r.m == -INFINITY || acc.ref == TlType<E>::LOWEST));
  if (o.tail && below && q_rest <= TL_REST_ROUNDING) q_rest = 0.0;
  const double lg = log(lane == 0 ? so + sn : lane == 1 ? static_cast<double>(acc.S) : lane == 2 ? q_rest : l.mass);  // all that are needed, at once
  r.log_s = __shfl_sync(0xffffffffu, lg, 0);
  const double log_out = nothing ? -INFINITY : gap + __shfl_sync(0xffffffffu, lg, 1);
  const double log_rest = __shfl_sync(0xffffffffu, lg, 2), log_mass = __shfl_sync(0xffffffffu, lg, 3);
  r.norm = o.tail ? 1.0 : 1.0 / l.mass;
  const double mass = o.tail ? l.mass : 1.0, own = o.tail ? l.own : l.own * r.norm - log_mass;
  r.total = mass + q_rest;
  if (write && lane == 0) {
    double loss = r.total * static_cast<double>(INFINITY);
    if (!none) {
      loss = own - l.dot * r.norm + mass * (r.log_s - (static_cast<double>(l.base) - r.m) * a.it);
      if (q_rest > 0.0) loss += q_rest * (log_rest - (log_out - r.log_s));
    }
    o.loss[t] = static_cast<float>(loss);
  }
  const float weight = o.weight ? o.weight[t] : 1.0f;
  r.f = static_cast<double>(weight) * a.it;
  r.coef.ref = nothing ? r.m : acc.ref;  // 2^x / S is p_j / p_r
  r.coef.A = nothing ? 0.0f : static_cast<float>(r.f * (r.total * (so / (so + sn)) - q_rest) / acc.S);
  r.coef.B = 0.0f;
  r.coef.zero = weight == 0.0f || none;
  return r;
}

// The named tokens' elements, each with its q; `at` of `n` threads.
template <class E, class Share>
__device__ __forceinline__ void tl_write_named(const TlRows<E>& a, const TlTeacher& o, const Share& s, const TlTables& tab, bool twice, const TlMark& r, E* dz, int at,
                                               int n) {
  for (int i = at; i < o.K; i += n) {
    const int j = tab.id[i];
    if (j < 0 || !s.owns(j)) continue;
    float sum = tab.qk[i];
    if (twice) {
      sum = 0.0f;
      for (int l = 0; l < o.K; ++l)
        if (tab.id[l] == j) sum += tab.qk[l];
    }
    const double p = exp((static_cast<double>(tab.zk[i]) - r.m) * a.it - r.log_s);
    tl_set(dz + j, static_cast<float>(r.f * (r.total * p - sum * r.norm)));
  }
}

// What the warps of a CTA, and the CTAs of a cluster, tell one another beside TlXch.
struct TlTaught {
  static constexpr int WARPS = BITRL_DISTILL_MAX / 32;  // that have entries
  float largest[WARPS];
  int first[WARPS];
  double mass[WARPS], own[WARPS], dot[WARPS];
  TlAcc named[WARPS];
  double dots[TL_MAX_CLUSTER];
  TlAcc nameds[TL_MAX_CLUSTER];
  TlMark mark;
};

template <class E, int NT>
__global__ void __launch_bounds__(tl_threads<NT>(), 1024 / tl_threads<NT>())
distill_topk_kernel(const __grid_constant__ TlRows<E> a, const __grid_constant__ TlTeacher o, const __grid_constant__ TlGrad<E> g, int mark_words) {
  constexpr int GROUPS = NT == 32 ? TL_ROW_WARPS : 1, A = TlShare<E>::A;
  extern __shared__ __align__(16) unsigned char tl_smem[];
  __shared__ TlXch xch;
  __shared__ TlTaught taught;
  __shared__ uint32_t edge_marks[GROUPS];
  __shared__ int twice_in[GROUPS];
  pdl_enter();
  const int row = NT == 32 ? blockIdx.x * GROUPS + (threadIdx.x >> 5) : blockIdx.x / a.C;
  const int rank = NT == 32 ? 0 : blockIdx.x % a.C, tid = tl_tid<NT>(), group = NT == 32 ? threadIdx.x >> 5 : 0;
  const int lane = threadIdx.x & 31, warp = NT == 32 ? 0 : threadIdx.x >> 5;
  if (NT == 32 && row >= a.T) return;
  const size_t t = row;
  const int words = TlTables::ARRAYS * o.K;
  const TlTables tab(reinterpret_cast<uint32_t*>(tl_smem) + group * words, o.K);
  uint32_t* mark = reinterpret_cast<uint32_t*>(tl_smem) + GROUPS * words + group * mark_words;
  const TlShare<E> s(a.z + row * a.ld, a.V, a.C, rank);
  E* dz = g.dz ? g.dz + row * g.ld : nullptr;
  uint32_t w[TL_VECS][8];

  tl_load_first<E, NT>(s, s.lo, tl_slots<NT>(s.lo, s.hi), dz != nullptr, w);  // on its way, though whether the row has a teacher is not known yet
  // The entries, as many threads as there are.
  const int nw = NT == 32 ? 1 : min(NT, o.K + 31) / 32;  // warps that have some
  if (o.tail)
    for (int i = tid; i < mark_words; i += NT) mark[i] = 0;
  if (tid == 0) {
    edge_marks[group] = 0;
    twice_in[group] = !o.tail;  // without marks nobody knows
  }
  tl_sync<NT>();
  float largest;
  int first;
  int any = tl_entries(o, s, t, tab, mark, &edge_marks[group], &twice_in[group], rank == 0, tid, NT, largest, first);
  if (warp < nw) {
    largest = warp_max(largest);
    first = __reduce_min_sync(0xffffffffu, first);
    if (NT != 32 && lane == 0) {
      taught.largest[warp] = largest;
      taught.first[warp] = first;
    }
  }
  if (NT == 32) {
    __syncwarp();
    any = __any_sync(0xffffffffu, any);
  } else {
    any = __syncthreads_or(any);
  }
  if (!any) {
    if (tid == 0 && rank == 0) o.loss[t] = 0.0f;
    const TlCoef none = {0.0f, 0.0f, 0.0f, true};
    if (dz) tl_write_gradient<false, NT>(a, s, none, dz, w);
    return;
  }
  tl_begin(a);
  const bool twice = twice_in[group];
  // What the entries need of the row is on its way while that streams by.
  TlLesson lesson = {0.0f, 0.0, 0.0, 0.0, {-INFINITY, 0.0f, 0.0f}};
  float zk = 0.0f;
  if (warp < nw) {
    if (NT != 32)
      for (int i = 0; i < nw; ++i) {
        largest = fmaxf(largest, taught.largest[i]);
        first = min(first, taught.first[i]);
      }
    lesson.base = tl_f32(s.z[tab.id[first]]);
    if (tid < o.K && tab.id[tid] >= 0 && s.owns(tab.id[tid])) zk = tl_f32(s.z[tab.id[tid]]);
  }
  const int edge_j = warp != 0 || (o.tail && edge_marks[group] >> lane & 1) ? -1 : s.edge(lane);
  const float edge_v = edge_j >= 0 ? tl_f32(s.z[edge_j]) : -INFINITY;

  TlAcc acc = {-INFINITY, 0.0f, 0.0f};  // outside the named tokens (tail), or everything
  for (int v = s.lo; v < s.hi; v += NT * TL_VECS) {
    const int n_u = tl_slots<NT>(v, s.hi);
    if (v != s.lo) tl_load_first<E, NT>(s, v, n_u, dz != nullptr, w);
    if (o.tail) {
#pragma unroll
      for (int u = 0; u < TL_VECS; ++u)
        if (u < n_u) {
          const int at = v + u * NT + tid - s.lo;
          const uint32_t m = at >= s.hi - s.lo ? 0 : A == 16 ? reinterpret_cast<const uint16_t*>(mark)[at] : reinterpret_cast<const uint8_t*>(mark)[at];
          if (m != 0) tl_drop<E, 8>(w[u], m);
        }
    }
    float l;
    tl_accumulate<false, NT>(a, s, v, n_u, w, o.tail ? mark : nullptr, acc, l);
  }
  if (edge_j >= 0) tl_merge<false>(a, acc, tl_single(a, edge_v));

  if (warp < nw) {
    if (!(fabsf(lesson.base) < INFINITY)) lesson.base = 0.0f;
    for (int k = tid; k < o.K; k += NT) {
      if (k != tid) zk = tab.id[k] >= 0 && s.owns(tab.id[k]) ? tl_f32(s.z[tab.id[k]]) : 0.0f;
      tl_study(a, o, s, tab, twice, largest, k, zk, lesson);
    }
    lesson.mass = tl_warp_sum64(lesson.mass);
    lesson.own = tl_warp_sum64(lesson.own);
    lesson.dot = tl_warp_sum64(lesson.dot);
    if (o.tail) tl_join_lanes<false>(a, lesson.named, 32);
    if (NT != 32 && lane == 0) {
      taught.mass[warp] = lesson.mass;
      taught.own[warp] = lesson.own;
      taught.dot[warp] = lesson.dot;
      taught.named[warp] = lesson.named;
    }
  }
  auto gather = [&](const double* dots, const TlAcc* nameds, int n) {  // in warp 0
    lesson.dot = tl_warp_sum64(lane < n ? dots[lane] : 0.0);
    lesson.named = lane < n ? nameds[lane] : TlAcc{-INFINITY, 0.0f, 0.0f};
    if (o.tail) tl_join_lanes<false>(a, lesson.named, 32);
  };
  if (a.C > 1) {  // the named tokens' sums travel with the shares'
    __syncthreads();
    if (warp == 0) gather(taught.dot, taught.named, nw);
  }
  tl_join<NT, false>(a, acc, &xch, rank, [&] {
    if (threadIdx.x >= a.C) return;
    const uint32_t to = ptx::mapa_u32(ptx::smem_u32(&taught.nameds[rank]), threadIdx.x);
    ptx::sts32_cluster(to, __float_as_uint(lesson.named.ref));
    ptx::sts32_cluster(to + 4, __float_as_uint(lesson.named.S));
    ptx::sts32_cluster(to + 8, 0u);
    const uint32_t td = ptx::mapa_u32(ptx::smem_u32(&taught.dots[rank]), threadIdx.x);
    ptx::sts32_cluster(td, static_cast<uint32_t>(__double2loint(lesson.dot)));
    ptx::sts32_cluster(td + 4, static_cast<uint32_t>(__double2hiint(lesson.dot)));
  });
  TlMark r;
  if (warp == 0) {
    if (NT != 32) {
      lesson.mass = tl_warp_sum64(lane < nw ? taught.mass[lane] : 0.0);
      lesson.own = tl_warp_sum64(lane < nw ? taught.own[lane] : 0.0);
      if (a.C > 1)
        gather(taught.dots, taught.nameds, a.C);
      else
        gather(taught.dot, taught.named, nw);
    }
    r = tl_conclude(a, o, acc, lesson, t, rank == 0);
    if (NT != 32 && lane == 0) taught.mark = r;
  }
  if (!dz) return;
  tl_sync<NT>();  // (a warp: the named tokens' logits have been read)
  if (NT != 32) r = taught.mark;
  tl_write_gradient<false, NT>(a, s, r.coef, dz, w);
  if (r.coef.zero) return;
  tl_sync<NT>();
  tl_write_named(a, o, s, tab, twice, r, dz, tid, NT);
}

// ---- host side: checks of arguments, launches --------------------------------------------------------------------
// What every call on rows of logits checks first.
inline bitrl_status tl_check(const void* logits, int32_t dtype, int32_t T, int32_t V, int64_t ld, double temperature) {
  if (dtype != BITRL_LOGITS_F32 && dtype != BITRL_LOGITS_BF16 && dtype != BITRL_LOGITS_F16) return BITRL_ERR_DTYPE;
  if (T < 0 || V < 1 || ld < V || ld > INT64_MAX / 8 / (T < 1 ? 1 : T) || !(temperature >= 0x1p-20 && temperature <= 0x1p20))
    return BITRL_ERR_SHAPE;
  if (V > BITRL_VOCAB_MAX) return BITRL_ERR_LIMIT;
  if (T > 0 && !logits) return BITRL_ERR_NULL;
  const uintptr_t size = dtype == BITRL_LOGITS_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(logits) % size != 0) return BITRL_ERR_ALIGN;
  return BITRL_OK;
}
// A gradient: rows of their own, or the logits themselves.
inline bitrl_status tl_check_out(const void* logits, int32_t dtype, int32_t T, int32_t V, int64_t ld, const void* dz, int64_t ld_out) {
  if (ld_out < V || ld_out > INT64_MAX / 8 / (T < 1 ? 1 : T)) return BITRL_ERR_SHAPE;
  const uintptr_t size = dtype == BITRL_LOGITS_F32 ? 4 : 2;
  const uintptr_t a = reinterpret_cast<uintptr_t>(logits), b = reinterpret_cast<uintptr_t>(dz);
  if (b % size != 0) return BITRL_ERR_ALIGN;
  if (T < 1 || (a == b && ld == ld_out)) return BITRL_OK;
  const uintptr_t na = size * ((T - 1) * static_cast<uintptr_t>(ld) + V), nb = size * ((T - 1) * static_cast<uintptr_t>(ld_out) + V);
  return a < b + nb && b < a + na ? BITRL_ERR_SHAPE : BITRL_OK;
}
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
// Calls f with a null pointer of the logits' type.
template <class F>
bitrl_status tl_dispatch(int32_t dtype, F&& f) {
  if (dtype == BITRL_LOGITS_F32) return f(static_cast<float*>(nullptr));
  if (dtype == BITRL_LOGITS_BF16) return f(static_cast<__nv_bfloat16*>(nullptr));
  return f(static_cast<__half*>(nullptr));
}

// The rows of a call.  Maxima may use x = z c - R as long as R is off by no more than 1 (|R| <= 2^24), so that the largest x is near 0.  That is
// also far above -2^46 (fp16: -65504, for maxima from -16384 on at temperatures up to 256), which a -inf counts as where a number is needed.
template <class E>
TlRows<E> tl_rows(const void* z, int T, int V, long long ld, double temperature) {
  TlRows<E> a;
  a.z = static_cast<const E*>(z);
  a.ld = ld;
  a.T = T;
  a.V = V;
  a.C = 1;
  a.it = 1.0 / temperature;
  a.c = static_cast<float>(TL_LOG2E / temperature);
  a.ref_hi = 0x1p24f / a.c;
  a.ref_lo = -a.ref_hi;
  if (std::is_same<E, __half>::value) a.ref_lo = temperature <= 256.0 ? fmaxf(a.ref_lo, -16384.0f) : INFINITY;
  return a;
}

template <auto Kernel, class... Args>
bitrl_status tl_launch(int threads, long long ctas, int C, size_t smem, cudaStream_t st, const Args&... args) {
  if (ctas > INT_MAX || smem > TL_MAX_SMEM) return BITRL_ERR_LIMIT;
  static std::atomic<uint64_t> known{0};  // devices on which the kernel may have that much shared memory, and clusters of 16
  int dev = 0;
  BITRL_CUDA(cudaGetDevice(&dev));
  const uint64_t bit = 1ull << (dev & 63);
  if (!(known.load(std::memory_order_relaxed) & bit)) {
    BITRL_CUDA(cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, TL_MAX_SMEM));
    BITRL_CUDA(cudaFuncSetAttribute(Kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    known.fetch_or(bit);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ctas));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(C);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = C > 1 ? 2 : 1;
  BITRL_CUDA(cudaLaunchKernelEx(&cfg, Kernel, args...));
  count_launch(1);
  return BITRL_OK;
}

// How rows are dealt out: NT threads on a row (32: a warp, TL_ROW_WARPS rows a CTA) or on one of its C shares.  Measured for bf16 and fp32, us a
// call, T x V:
//   * A CTA costs a few us however short its row: many short rows go to a warp each (log probabilities of 20000 x 2500: 32 by warps, 65 by 128
//     threads, 119 by 256), rows up to 16 KB x 2 to 128 threads (PPO 2000 x 8000: 14.5, by 256 20; 20 by a CTA of 512 and more).
//   * Long rows that are read once: 128 threads too, of which eight CTAs fit an SM, so that one's beginning and end fall into the
//     others' reading (distillation's loss, 1000 x 50021: 32, by 256 threads 35, by 512 44).
//   * Rows above 128 KB with a gradient: 512 threads.  They are read again behind their statistics, and the fewer rows are under way the more of
//     that comes out of L2 (PPO 4096 x 128000: 402 by 512, 423 by 256, 452 by 128).
//   * Few rows are cut into shares until three CTAs an SM have some, none below 256 vectors (PPO 20 x 128000: 22 whole, 8.0 in 8 shares, 7.9 in
//     16; 1 x 128000: 22, 6.2 and 5.6; 100 x 32000: 8.4 and 7.5 in 4).  Alternatives cost every share a selection: as many shares as SMs, none below
//     512 (16 x 32000: 8.8 whole, 14 in 16).
enum TlKind { TL_TOP, TL_SUMS, TL_GRADIENT };
struct TlPlan {
  int NT, C;
};
template <class E>
TlPlan tl_plan(const TlRows<E>& a, TlKind kind) {
  const int nvec = a.V / TlShare<E>::A, sms = sm_count();
  if (kind != TL_TOP && (nvec <= 128 ? a.T > 2 * sms : nvec <= 256 && a.T >= 16 * sms)) return {32, 1};
  TlPlan p = {nvec <= 1024 || (kind == TL_SUMS && a.T >= 6 * sms) ? 128 : kind == TL_GRADIENT && nvec > 4096 && a.T >= 2 * sms ? 512 : 256, 1};
  const int ctas = kind == TL_TOP ? sms : 3 * sms, least = kind == TL_TOP ? 512 : 256;
  while (p.C < TL_MAX_CLUSTER && static_cast<long long>(a.T) * 2 * p.C <= ctas && nvec / (2 * p.C) >= least) p.C *= 2;
  return p;
}
template <int First, int... Rest, class F>
bitrl_status tl_by_threads(int NT, F&& f) {
  if constexpr (sizeof...(Rest) > 0)
    if (NT != First) return tl_by_threads<Rest...>(NT, f);
  return f(std::integral_constant<int, First>());
}
template <class E>
long long tl_ctas(const TlRows<E>& a, int NT) {
  return NT == 32 ? (static_cast<long long>(a.T) + TL_ROW_WARPS - 1) / TL_ROW_WARPS : static_cast<long long>(a.T) * a.C;
}

template <class E>
bitrl_status launch_token_logprobs(TlRows<E> a, const TlOut& o, cudaStream_t st) {
  const TlPlan p = tl_plan(a, o.k > 0 ? TL_TOP : TL_SUMS);
  a.C = p.C;
  if (o.k == 0)
    return tl_by_threads<32, 128, 256>(p.NT, [&](auto nt) {
      constexpr int NT = decltype(nt)::value;
      return tl_launch<token_logprobs_kernel<E, NT, false>>(tl_threads<NT>(), tl_ctas(a, NT), a.C, 0, st, a, o);
    });
  return tl_by_threads<128, 256>(p.NT, [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    const int share = (a.V / TlShare<E>::A + a.C - 1) / a.C, chunks = (share + NT * TL_VECS - 1) / (NT * TL_VECS);
    const size_t smem = sizeof(TlTop<NT>) + (a.C > 1 ? sizeof(unsigned long long) * a.C * o.k : 0) + sizeof(float) * chunks * NT;
    return tl_launch<token_logprobs_kernel<E, NT, true>>(NT, tl_ctas(a, NT), a.C, smem, st, a, o);
  });
}

// Nothing joins a row's shares here, so there may be any number of them: one chunk of 128 threads each (2000 x 50021: 56 us, 61 by 512 threads).
template <class E>
bitrl_status launch_token_logprobs_backward(TlRows<E> a, const TlPolicy& o, const TlGrad<E>& g, cudaStream_t st) {
  const int NT_ = tl_plan(a, TL_GRADIENT).NT == 32 ? 32 : 128;
  a.C = NT_ == 32 ? 1 : (a.V / TlShare<E>::A + 128 * TL_VECS - 1) / (128 * TL_VECS);
  if (a.C < 1) a.C = 1;
  return tl_by_threads<32, 128>(NT_, [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    return tl_launch<token_logprobs_backward_kernel<E, NT>>(tl_threads<NT>(), tl_ctas(a, NT), 1, 0, st, a, o, g);
  });
}

template <class E>
bitrl_status launch_ppo_token(TlRows<E> a, const TlPpo& o, const TlGrad<E>& g, cudaStream_t st) {
  const TlPlan p = tl_plan(a, g.dz ? TL_GRADIENT : TL_SUMS);
  a.C = p.C;
  return tl_by_threads<32, 128, 256, 512>(p.NT, [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    return tl_launch<ppo_token_kernel<E, NT>>(tl_threads<NT>(), tl_ctas(a, NT), a.C, 0, st, a, o, g);
  });
}

template <class E>
bitrl_status launch_distill_topk(TlRows<E> a, const TlTeacher& o, const TlGrad<E>& g, cudaStream_t st) {
  const TlPlan p = tl_plan(a, g.dz ? TL_GRADIENT : TL_SUMS);
  a.C = p.C;
  const int share = (a.V / TlShare<E>::A + a.C - 1) / a.C;
  const int words = o.tail ? (share * TlShare<E>::A + 31) / 32 : 0;
  return tl_by_threads<32, 128, 256, 512>(p.NT, [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    const size_t smem = 4 * static_cast<size_t>(NT == 32 ? TL_ROW_WARPS : 1) * (TlTables::ARRAYS * o.K + words);
    return tl_launch<distill_topk_kernel<E, NT>>(tl_threads<NT>(), tl_ctas(a, NT), a.C, smem, st, a, o, g, words);
  });
}

}  // namespace bitrl

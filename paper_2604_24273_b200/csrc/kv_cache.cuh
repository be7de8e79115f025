// A paged key/value cache beside the encoder: appending new tokens (rotary embedding + paged write), planning an
// eviction by accumulated attention weight, moving rows, advancing the counters.  include/bitrl.h states the layout and the
// meaning of every argument; the attention that reads the cache is in attention_cached.cuh.
#pragma once

#include <climits>
#include <math.h>

#include <type_traits>

#include "attention.cuh"
#include "common.cuh"

namespace bitrl {

enum { KV_STAGE_BAD_SEQ = 121, KV_STAGE_BAD_TREE = 122, KV_STAGE_BAD_PAGE = 123, KV_STAGE_BAD_MOVE = 124 };

// One layer of a cache (or, for calls over all layers, its first layer) as the kernels see it.
struct KvView {
  unsigned short* k;  // bf16 [n_pages][n_kv][page][hd]
  unsigned short* v;
  float* mass;
  int* pos;
  const int* page_table;
  int* used;
  int* seen;
  int n_layers, n_pages, n_kv, page_shift, hd, n_seq, max_pages;
};

// The new tokens of a call.
struct KvBatch {
  const int* off;     // [n_seq + 1] or nullptr: max_new tokens each
  const int* parent;  // [T] or nullptr
  int max_new, T;
};

// Rows of a pool before row 0 of (page, kv head); 64-bit, a pool may hold more than 2^31 elements.
__device__ __forceinline__ long long kv_row(const KvView& c, int layer, int page, int head) {
  return ((static_cast<long long>(layer) * c.n_pages + page) * c.n_kv + head) << c.page_shift;
}

// Page of slot t of a sequence; -1 (and a status word) when the table names none.
__device__ __forceinline__ int kv_page(const KvView& c, int seq, int t) {
  const int p = c.page_table[static_cast<long long>(seq) * c.max_pages + (t >> c.page_shift)];
  if (p < 0 || p >= c.n_pages) {
    report_status(BITRL_ERR_SHAPE, KV_STAGE_BAD_PAGE);
    return -1;
  }
  return p;
}

struct KvSeq {
  int t0, m, used;  // first row of the batch, new tokens, slots in use before them
};

// Rows and slots of sequence s; false (and a status word) when they do not describe tokens that fit.
__device__ __forceinline__ bool kv_seq(const KvView& c, const KvBatch& b, int s, KvSeq& q) {
  if (b.off) {
    q.t0 = b.off[s];
    q.m = b.off[s + 1] - q.t0;
  } else {
    q.t0 = s * b.max_new;
    q.m = b.max_new;
  }
  q.used = c.used[s];
  const long long room = static_cast<long long>(c.max_pages) << c.page_shift;
  if (q.t0 < 0 || q.m < 0 || q.m > b.max_new || static_cast<long long>(q.t0) + q.m > b.T || q.used < 0 ||
      static_cast<long long>(q.used) + q.m > room || (b.parent && q.m > BITRL_TREE_MAX_TOKENS)) {
    report_status(BITRL_ERR_SHAPE, KV_STAGE_BAD_SEQ);
    return false;
  }
  return true;
}

// Copies the tree of a sequence into shared memory and checks it; all threads of the CTA call it, at least
// BITRL_TREE_MAX_TOKENS iterations of `n_threads` cover it.  On true, every walk p = par[p] from a token that is not
// padding strictly falls and ends at BITRL_PARENT_PAST.
__device__ __forceinline__ bool kv_load_tree(const KvBatch& b, const KvSeq& q, int* par, int n_threads) {
  for (int i = threadIdx.x; i < q.m; i += n_threads) par[i] = b.parent[q.t0 + i];
  __syncthreads();
  bool bad = false;
  for (int i = threadIdx.x; i < q.m; i += n_threads) {
    const int p = par[i];
    bad |= p < BITRL_PARENT_PAD || p >= i || (p >= 0 && par[p] == BITRL_PARENT_PAD);
  }
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) report_status(BITRL_ERR_SHAPE, KV_STAGE_BAD_TREE);
    return false;
  }
  return true;
}

// ---- append -------------------------------------------------------------------------------------------------------
// One pass over qkv: every element is read and written once (109 MB for 256 states of the 20/5-head backbone), so the
// copy rate bounds it (24.8 us, 4.4 TB/s; a plain copy of as much takes 16.7); single tokens are bound by the launch and one
// chain of dependent loads (7 us).  A CTA takes up to
// APP_TOKENS consecutive tokens of one sequence: its threads compute the (cos, sin) pairs, one each, then every thread
// rotates 8 dimensions and their 8 partners of each token with 16-byte loads and stores.
// Angles: position * theta^(-2f/hd) / (2 pi) in fp64 (turns), reduced to half a turn there, so that far positions lose
// nothing; the cosine and sine of the remainder are fp32.
constexpr int APP_THREADS = 256;
constexpr int APP_TOKENS = 4;

struct AppArgs {
  KvView c;
  KvBatch b;
  const unsigned short* qkv;
  unsigned short* q_out;
  int n_heads;
  int tiles;         // token tiles per sequence
  double turns[64];  // theta^(-2f/hd) / (2 pi), f < hd/2
};

template <int HD>
__global__ void __launch_bounds__(APP_THREADS) kv_append_kernel(const __grid_constant__ AppArgs a) {
  constexpr int HALF = HD / 2, CP = HD / 16;  // CP: pairs of 8-dimension chunks per head row
  __shared__ int par[BITRL_TREE_MAX_TOKENS];
  __shared__ __align__(16) float4 cs[APP_TOKENS][4][CP];  // (cos, sin) of dimensions 8 c + 2 w and the next
  __shared__ int depth_of[APP_TOKENS];                    // -1: padding
  pdl_enter();
  const KvView& c = a.c;
  const int s = blockIdx.x / a.tiles, first = (blockIdx.x - s * a.tiles) * APP_TOKENS;
  KvSeq q;
  if (!kv_seq(c, a.b, s, q)) return;
  if (first >= q.m) return;
  const int n = min(APP_TOKENS, q.m - first);
  const int seen = c.seen[s];
  if (seen < 0 || seen > INT_MAX - q.m) {
    if (threadIdx.x == 0) report_status(BITRL_ERR_SHAPE, KV_STAGE_BAD_SEQ);
    return;
  }
  const int heads = a.n_heads + 2 * c.n_kv, per_token = heads * CP;
  const long long width = static_cast<long long>(heads) * HD;
  // A thread keeps its place in the row (head, 8 dimensions and their partners) and takes the tokens of the tile together;
  // the first ones' loads are on their way while the angles are computed.
  uint4 x1[APP_TOKENS], x2[APP_TOKENS];
  auto load = [&](int r) {
    const unsigned short* src = a.qkv + (q.t0 + first) * width + (r / CP) * HD + 8 * (r % CP);
#pragma unroll
    for (int t = 0; t < APP_TOKENS; ++t)
      if (t < n) {
        x1[t] = *reinterpret_cast<const uint4*>(src + t * width);
        x2[t] = *reinterpret_cast<const uint4*>(src + t * width + HALF);
      }
  };
  if (static_cast<int>(threadIdx.x) < per_token) load(threadIdx.x);
  int page[APP_TOKENS];
#pragma unroll
  for (int t = 0; t < APP_TOKENS; ++t) page[t] = t < n ? kv_page(c, s, q.used + first + t) : -1;
  if (a.b.parent) {
    if (!kv_load_tree(a.b, q, par, APP_THREADS)) return;
    if (static_cast<int>(threadIdx.x) < n) {
      int d = -1;
      for (int i = par[first + threadIdx.x] == BITRL_PARENT_PAD ? -1 : static_cast<int>(first + threadIdx.x); i >= 0; i = par[i]) ++d;
      depth_of[threadIdx.x] = d;
    }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < n * HALF; i += APP_THREADS) {
    const int t = i / HALF, f = i - t * HALF;
    const int d = a.b.parent ? depth_of[t] : first + t;
    const double turn = static_cast<double>(seen + d) * a.turns[f];
    float sn, cn;
    sincospif(2.0f * static_cast<float>(turn - rint(turn)), &sn, &cn);
    reinterpret_cast<float2*>(&cs[t][(f & 7) >> 1][f >> 3])[f & 1] = make_float2(cn, sn);
  }
  __syncthreads();
  for (int r = threadIdx.x; r < per_token; r += APP_THREADS) {
    if (r >= APP_THREADS) load(r);
    const int head = r / CP, ch = r % CP, d0 = 8 * ch;
    const bool is_q = head < a.n_heads, is_k = !is_q && head < a.n_heads + c.n_kv;
    const int kvh = is_q ? 0 : head - a.n_heads - (is_k ? 0 : c.n_kv);
#pragma unroll
    for (int t = 0; t < APP_TOKENS; ++t) {
      if (t >= n || (a.b.parent && depth_of[t] < 0) || (!is_q && page[t] < 0)) continue;
      if (is_q || is_k) {
        uint32_t w1[4] = {x1[t].x, x1[t].y, x1[t].z, x1[t].w}, w2[4] = {x2[t].x, x2[t].y, x2[t].z, x2[t].w};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float4 e = cs[t][w][ch];
          const float x1a = __uint_as_float(w1[w] << 16), x1b = __uint_as_float(w1[w] & 0xffff0000u);
          const float x2a = __uint_as_float(w2[w] << 16), x2b = __uint_as_float(w2[w] & 0xffff0000u);
          const __nv_bfloat162 o1 = __floats2bfloat162_rn(fmaf(-x2a, e.y, __fmul_rn(x1a, e.x)), fmaf(-x2b, e.w, __fmul_rn(x1b, e.z)));
          const __nv_bfloat162 o2 = __floats2bfloat162_rn(fmaf(x1a, e.y, __fmul_rn(x2a, e.x)), fmaf(x1b, e.w, __fmul_rn(x2b, e.z)));
          w1[w] = *reinterpret_cast<const uint32_t*>(&o1);
          w2[w] = *reinterpret_cast<const uint32_t*>(&o2);
        }
        x1[t] = make_uint4(w1[0], w1[1], w1[2], w1[3]);
        x2[t] = make_uint4(w2[0], w2[1], w2[2], w2[3]);
      }
      unsigned short* dst;
      if (is_q) {
        dst = a.q_out + (static_cast<long long>(q.t0 + first + t) * a.n_heads + head) * HD + d0;
      } else {
        const int slot = q.used + first + t;
        const long long row = kv_row(c, 0, page[t], kvh) + (slot & ((1 << c.page_shift) - 1));
        dst = (is_k ? c.k : c.v) + row * HD + d0;
        if (is_k && ch == 0) {
          if (c.mass) c.mass[row] = 0.0f;
          c.pos[row] = seen + (a.b.parent ? depth_of[t] : first + t);
        }
      }
      *reinterpret_cast<uint4*>(dst) = x1[t];
      *reinterpret_cast<uint4*>(dst + HALF) = x2[t];
    }
  }
}

bitrl_status launch_kv_append(const KvView& c, const KvBatch& b, const void* qkv, int n_heads, double theta, void* q_out,
                              cudaStream_t st) {
  AppArgs a;
  a.c = c;
  a.b = b;
  a.qkv = static_cast<const unsigned short*>(qkv);
  a.q_out = static_cast<unsigned short*>(q_out);
  a.n_heads = n_heads;
  a.tiles = (b.max_new + APP_TOKENS - 1) / APP_TOKENS;
  // one power and 80-bit products (each off by 2^-64) in place of 64 powers
  const long double ratio = powl(static_cast<long double>(theta), -2.0L / c.hd);
  long double turn = 1.0L / (2.0L * 3.14159265358979323846264338327950288L);
  for (int f = 0; f < 64; ++f, turn *= ratio) a.turns[f] = f < c.hd / 2 ? static_cast<double>(turn) : 0.0;
  const dim3 grid(static_cast<unsigned>(c.n_seq) * a.tiles);
  BITRL_CUDA(c.hd == 128 ? launch_pdl(kv_append_kernel<128>, grid, dim3(APP_THREADS), 0, st, a)
                         : launch_pdl(kv_append_kernel<64>, grid, dim3(APP_THREADS), 0, st, a));
  count_launch(1);
  return BITRL_OK;
}

// ---- eviction plan --------------------------------------------------------------------------------------------------
// One CTA per (layer, sequence, kv head).  The weight of a slot becomes an unsigned key whose order is the numbers' order
// (NaN lowest, -0 = +0); 0 and the greatest key stand for slots that go and stay whatever their weight.  Protected slots come
// first, so the threshold lies in one group alone: as a rule the protected ones fit into the budget, stay, and the free ones
// compete; else (a second reading) the free ones go and the protected ones compete.  Selection: counts over up to 2048 equal
// steps of the key range that the group really spans (weights fill a few binades, so fixed digits would pile up in a few
// counters), then over the step that holds the threshold, until few keys are left in it (or one value), whose ranks are
// counted directly.  Two ordered passes over the keys count and write the ascending lists (ties: lower slots stay).
// Every slot is read from memory once, four by a lane, its key kept in shared memory.  Reading 8 bytes per slot would take 17 us
// for 2400 lists of up to 8192 slots; instructions bound it (65 us, 46 million warp instructions; with one slot per lane and bits
// per slot: 107 us).
constexpr int PLAN_BINS = 2048;
constexpr int PLAN_FEW = 128;  // keys whose ranks are counted directly

struct PlanArgs {
  KvView c;
  int budget, recent, sink, max_moves;
  int* moves;
  int* count;
  int smem_slots;  // keys that fit into shared memory; longer sequences read theirs again from global memory
};

__device__ __forceinline__ uint32_t plan_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.0f);
  const uint32_t k = u ^ (static_cast<uint32_t>(static_cast<int>(u) >> 31) | 0x80000000u);  // -inf is 0x007fffff: above NaN
  return (u & 0x7fffffffu) > 0x7f800000u ? 1u : k;
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) kv_evict_plan_kernel(const PlanArgs a) {
  constexpr int WARPS = THREADS / 32;
  extern __shared__ __align__(16) unsigned char plan_smem[];
  __shared__ int hist[PLAN_BINS];
  __shared__ int part[WARPS], part2[WARPS];
  __shared__ uint32_t few[PLAN_FEW];
  __shared__ uint32_t group_lo, group_hi, chosen;
  __shared__ int n_prot, wanted, n_few, inside;
  pdl_enter();
  const KvView& c = a.c;
  const int list = blockIdx.x;
  const int head = list % c.n_kv, s = (list / c.n_kv) % c.n_seq, layer = list / (c.n_kv * c.n_seq);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n = c.used[s], B = a.budget, seen = c.seen[s];
  const long long room = static_cast<long long>(c.max_pages) << c.page_shift;
  if (n < 0 || n > room) {
    if (threadIdx.x == 0) { report_status(BITRL_ERR_SHAPE, KV_STAGE_BAD_SEQ); a.count[list] = 0; }
    return;
  }
  if (n <= B) {
    if (threadIdx.x == 0) a.count[list] = 0;
    return;
  }
  const int slot_mask = (1 << c.page_shift) - 1, quads = (n + 3) >> 2;
  const bool cached = n <= a.smem_slots;
  uint4* key_s = reinterpret_cast<uint4*>(plan_smem);  // [quads]
  const int recent_from = seen > a.recent ? seen - a.recent : 0;
  const int* pages = c.page_table + static_cast<long long>(s) * c.max_pages;
  const long long base = kv_row(c, layer, 0, head);  // pool row of slot 0 of page 0
  const float* mass = c.mass + base;
  const int* pos = c.pos + base;
  const uint32_t page_rows = static_cast<uint32_t>(c.n_kv) << c.page_shift;  // rows of a layer are counted in 32 bits: memory ends before
  // pos < sink or >= recent_from, in one comparison
  const uint32_t sink = static_cast<uint32_t>(a.sink), span_free = recent_from > a.sink ? static_cast<uint32_t>(recent_from) - sink : 0u;
  // Keys of slots 4 i .. 4 i + 3 when protected slots stay (or, SWAP, compete while the free ones go); lo, hi: range of the
  // keys that compete; n_p: protected slots.
  auto keys_of = [&](auto swapped, int i, const float4& m, const int4& ps, uint32_t& lo, uint32_t& hi, int& n_p) {
    constexpr bool SWAP = decltype(swapped)::value;
    const float mv[4] = {m.x, m.y, m.z, m.w};
    const int pv[4] = {ps.x, ps.y, ps.z, ps.w};
    uint32_t k[4];
    const int have = n - 4 * i;  // slots of this quad, if it is the last
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t key = plan_key(mv[e]);
      const bool p = static_cast<uint32_t>(pv[e]) - sink >= span_free;
      k[e] = p == SWAP ? key : SWAP ? 0u : 0xffffffffu;
      if (have < 4 && e >= have) {
        k[e] = 0u;
        continue;
      }
      lo = min(lo, SWAP && !p ? 0xffffffffu : k[e]);
      hi = max(hi, !SWAP && p ? 0u : k[e]);
      n_p += p;
    }
    return make_uint4(k[0], k[1], k[2], k[3]);
  };
  auto at_quad = [&](int i, int page) { return static_cast<uint32_t>(page) * page_rows + static_cast<uint32_t>((4 * i) & slot_mask); };
  bool bad = false;
  uint32_t from = 0u, to = 0u;  // the threshold key lies in from .. to, which neither 0 nor the greatest key does; `want` slots of that range stay
  auto read = [&](auto swapped) {
    if (threadIdx.x == 0) {
      n_prot = 0;
      group_lo = 0xffffffffu;
      group_hi = 0u;
    }
    __syncthreads();
    int prot = 0;
    uint32_t lo = 0xffffffffu, hi = 0u;
    for (int i0 = threadIdx.x; i0 < quads; i0 += 2 * THREADS) {
      int page[2];
      float4 m[2];
      int4 ps[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = i0 + j * THREADS;
        page[j] = i < quads ? pages[(4 * i) >> c.page_shift] : 0;
        if (static_cast<uint32_t>(page[j]) >= static_cast<uint32_t>(c.n_pages)) {
          bad = true;
          page[j] = 0;
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t at = at_quad(i0 + j * THREADS, page[j]);
        m[j] = *reinterpret_cast<const float4*>(mass + at);
        ps[j] = *reinterpret_cast<const int4*>(pos + at);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = i0 + j * THREADS;
        if (i >= quads) break;
        const uint4 k = keys_of(swapped, i, m[j], ps[j], lo, hi, prot);
        if (cached) key_s[i] = k;
      }
    }
    prot = warp_sum_i(prot);
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) {
      atomicAdd(&n_prot, prot);
      atomicMin(&group_lo, lo);
      atomicMax(&group_hi, hi);
    }
    if (__syncthreads_or(bad)) return -1;
    from = group_lo;
    to = group_hi;
    return n_prot;
  };
  using Stay = std::integral_constant<bool, false>;
  using Compete = std::integral_constant<bool, true>;
  int P = read(Stay{});
  const bool swap = P >= B;
  if (swap) {
    __syncthreads();
    P = read(Compete{});
  }
  if (P < 0) {
    if (threadIdx.x == 0) { report_status(BITRL_ERR_SHAPE, KV_STAGE_BAD_PAGE); a.count[list] = 0; }
    return;
  }
  int want = swap ? B : B - P;
  auto keys_at = [&](int i) -> uint4 {  // i < quads
    if (cached) return key_s[i];
    const uint32_t at = at_quad(i, pages[(4 * i) >> c.page_shift]);
    const float4 m = *reinterpret_cast<const float4*>(mass + at);
    const int4 ps = *reinterpret_cast<const int4*>(pos + at);
    uint32_t lo = 0u, hi = 0u;
    int n_p = 0;
    return swap ? keys_of(Compete{}, i, m, ps, lo, hi, n_p) : keys_of(Stay{}, i, m, ps, lo, hi, n_p);
  };
  uint32_t thr = from;
  int at_thr = 0;  // slots whose key is the threshold
  auto each = [&](auto&& f) {
    for (int i = threadIdx.x; i < quads; i += THREADS) {
      const uint4 k = keys_at(i);
      f(k.x);
      f(k.y);
      f(k.z);
      f(k.w);
    }
  };
  // Each round takes 11 bits off the span, so three end it.  The bounds here and in the lists below hold even if weights change
  // meanwhile (a call on another stream, which is not allowed): then keys read twice contradict one another.
  if (threadIdx.x == 0) {
    chosen = 0u;
    wanted = inside = 0;
  }
#pragma unroll 1
  for (int round = 0; round < 4; ++round) {
    const uint32_t span = to - from;
    const int shift = span < PLAN_BINS ? 0 : 21 - __clz(span);  // span >> shift < PLAN_BINS
    for (int i = threadIdx.x; i < PLAN_BINS; i += THREADS) hist[i] = 0;
    if (threadIdx.x == 0) n_few = 0;
    __syncthreads();
    each([&](uint32_t key) {
      if (key - from <= span) atomicAdd(&hist[(key - from) >> shift], 1);
    });
    __syncthreads();
    // steps from the top: thread i owns PLAN_BINS / THREADS of them
    constexpr int PER = PLAN_BINS / THREADS;
    const int top = PLAN_BINS - 1 - PER * static_cast<int>(threadIdx.x);
    int mine = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) mine += hist[top - j];
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) part[warp] = incl;
    __syncthreads();
    int above = incl - mine;  // slots in higher steps than this thread's
    for (int w = 0; w < warp; ++w) above += part[w];
    if (above < want && above + mine >= want) {
      int j = 0;
      while (above + hist[top - j] < want) above += hist[top - j++];
      chosen = static_cast<uint32_t>(top - j);
      wanted = want - above;
      inside = hist[top - j];
    }
    __syncthreads();
    want = wanted;
    const int left = inside;
    from += chosen << shift;
    to = min(to, from + ((1u << shift) - 1u));
    if (shift == 0) {
      thr = from;
      at_thr = left;
      break;
    }
    if (left <= PLAN_FEW) {
      const uint32_t width = to - from;
      each([&](uint32_t key) {
        if (key - from <= width) {
          const int at = atomicAdd(&n_few, 1);
          if (at < PLAN_FEW) few[at] = key;  // more only if another stream changes the weights meanwhile
        }
      });
      __syncthreads();
      if (static_cast<int>(threadIdx.x) < left) {
        const uint32_t key = few[threadIdx.x];
        int greater = 0, equal = 0;
        for (int i = 0; i < left; ++i) {
          greater += few[i] > key;
          equal += few[i] == key;
        }
        if (greater < want && greater + equal >= want) {  // the same values from every thread that finds them
          chosen = key;
          wanted = want - greater;
          inside = equal;
        }
      }
      __syncthreads();
      thr = chosen;
      want = wanted;
      at_thr = inside;
      break;
    }
  }

  // ---- ordered passes: every warp owns a run of 128-slot blocks.  Of the at_thr slots that equal the threshold the `want`
  // lowest stay; as a rule that is all of them and no ranks are needed.
  const int blocks = (n + 127) >> 7, per_warp = (blocks + WARPS - 1) / WARPS, b0 = warp * per_warp, b1 = min(blocks, b0 + per_warp);
  const bool ranked = want < at_thr;
  auto equal_bits = [&](const uint4& k) {
    return (k.x == thr ? 1u : 0u) | (k.y == thr ? 2u : 0u) | (k.z == thr ? 4u : 0u) | (k.w == thr ? 8u : 0u);
  };
  auto inclusive = [&](int v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += u;
    }
    return v;
  };
  // Bits of this lane's four slots that stay; advances `ties`, the slots equal to the threshold so far.
  auto keep_bits = [&](int i, int& ties) -> uint32_t {
    const uint4 k = i < quads ? keys_at(i) : make_uint4(0u, 0u, 0u, 0u);
    uint32_t keep = (k.x >= thr ? 1u : 0u) | (k.y >= thr ? 2u : 0u) | (k.z >= thr ? 4u : 0u) | (k.w >= thr ? 8u : 0u);
    if (ranked) {
      const uint32_t eq = equal_bits(k);
      const int incl = inclusive(__popc(eq)), room_left = want - ties - (incl - __popc(eq));  // of this lane's ties so many stay
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (((eq >> e) & 1u) && __popc(eq & ((1u << e) - 1u)) >= room_left) keep &= ~(1u << e);
      ties += __shfl_sync(0xffffffffu, incl, 31);
    }
    return keep;
  };
  auto low_bits = [&](int i) { return 4 * i + 4 <= B ? 15u : 4 * i >= B ? 0u : (1u << (B - 4 * i)) - 1u; };  // slots < B
  int ties0 = 0;
  if (ranked) {
    int mine = 0;
    for (int b = b0; b < b1; ++b)
      if (32 * b + lane < quads) mine += __popc(equal_bits(keys_at(32 * b + lane)));
    mine = warp_sum_i(mine);
    __syncthreads();
    if (lane == 0) part[warp] = mine;
    __syncthreads();
    for (int w = 0; w < warp; ++w) ties0 += part[w];
  }
  int n_src = 0, n_dst = 0, ties = ties0;
  for (int b = b0; b < b1; ++b) {
    const uint32_t keep = keep_bits(32 * b + lane, ties), low = low_bits(32 * b + lane);
    n_src += __popc(keep & ~low);
    n_dst += __popc(~keep & low);
  }
  n_src = warp_sum_i(n_src);
  n_dst = warp_sum_i(n_dst);
  __syncthreads();
  if (lane == 0) { part[warp] = n_src; part2[warp] = n_dst; }
  __syncthreads();
  int at_src = 0, at_dst = 0;
  for (int w = 0; w < warp; ++w) { at_src += part[w]; at_dst += part2[w]; }
  if (threadIdx.x == 0) {
    int total = 0;
    for (int w = 0; w < WARPS; ++w) total += part[w];
    a.count[list] = min(total, a.max_moves);
  }
  int* out = a.moves + static_cast<long long>(list) * a.max_moves * 2;
  ties = ties0;
  for (int b = b0; b < b1; ++b) {
    const int i = 32 * b + lane;
    const uint32_t keep = keep_bits(i, ties), low = low_bits(i);
    const uint32_t src = keep & ~low, dst = ~keep & low;
    if (!__any_sync(0xffffffffu, (src | dst) != 0u)) continue;
    const int mine = __popc(src) | (__popc(dst) << 16);
    const int incl = inclusive(mine), before = incl - mine, all = __shfl_sync(0xffffffffu, incl, 31);
    int* to_src = out + 2 * (at_src + (before & 0xffff));
    int* to_dst = out + 2 * (at_dst + (before >> 16)) + 1;
    at_src += all & 0xffff;
    at_dst += all >> 16;
    if (max(at_src, at_dst) > a.max_moves) break;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if ((src >> e) & 1u) {
        *to_src = 4 * i + e;
        to_src += 2;
      }
      if ((dst >> e) & 1u) {
        *to_dst = 4 * i + e;
        to_dst += 2;
      }
    }
  }
}

template <int THREADS>
bitrl_status launch_kv_evict_plan_t(const PlanArgs& a, size_t smem, int limit, unsigned lists, cudaStream_t st) {
  static bool done[64] = {false};
  int dev = 0;
  BITRL_CUDA(cudaGetDevice(&dev));
  if (dev >= 0 && dev < 64 && !done[dev]) {
    BITRL_CUDA(cudaFuncSetAttribute(kv_evict_plan_kernel<THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, limit));
    done[dev] = true;
  }
  BITRL_CUDA(launch_pdl(kv_evict_plan_kernel<THREADS>, dim3(lists), dim3(THREADS), smem, st, a));
  count_launch(1);
  return BITRL_OK;
}

bitrl_status launch_kv_evict_plan(const KvView& c, int budget, int recent, int sink, int max_moves, int* moves, int* count,
                                  cudaStream_t st) {
  PlanArgs a{c, budget, recent, sink, max_moves, moves, count, 0};
  const int room = c.max_pages << c.page_shift;
  constexpr int LIMIT = 200 * 1024;
  a.smem_slots = room < LIMIT / 4 ? room : LIMIT / 4;
  const size_t smem = static_cast<size_t>(a.smem_slots) * 4;
  const long long lists = static_cast<long long>(c.n_layers) * c.n_seq * c.n_kv;
  // few lists: more threads on each
  return lists <= 2 * sm_count() ? launch_kv_evict_plan_t<512>(a, smem, LIMIT, static_cast<unsigned>(lists), st)
                                 : launch_kv_evict_plan_t<256>(a, smem, LIMIT, static_cast<unsigned>(lists), st);
}

// ---- moving rows ------------------------------------------------------------------------------------------------------
// A pure gather/scatter of head_dim rows, bound by the copy rate for long lists and by one chain of loads (count, move, page,
// row) for short ones.  A CTA takes the moves of one list THREADS at a time: a thread looks up the pool rows of one move and
// carries its mass and pos; then all threads move the rows of k and v, chunk by chunk, the next chunk's reads before this one's
// writes.  Sources and destinations ascend and no destination is above its source, so the source of a later move lies above
// every earlier destination: it is enough that a chunk is written after it and everything before it has been read.  Where a list's
// last destination lies below its first source (always so for an eviction) moves do not touch one another at all: no barrier,
// and the list may be spread over several CTAs.  1200 lists of up to 700 moves: 84 us, 5.2 TB/s, where rows of 256 bytes at
// scattered places read 0.79 of the rate of a plain copy; 12 rows per sequence, 30 layers: 5.6 us, the chain of loads.
constexpr int MOVE_ROWS = 4;  // rows of a chunk per lane group

struct MoveArgs {
  KvView c;
  const int* moves;
  const int* count;
  int max_moves, per_head, splits;
  int most;  // sources ascend: a list holds no more than max_moves, and no more than there are slots
};

template <int HD, int THREADS>
__global__ void __launch_bounds__(THREADS) kv_move_kernel(const MoveArgs a) {
  constexpr int LANES = HD / 8;                // lanes of 16 bytes per row
  constexpr int GROUPS = THREADS / (2 * LANES);  // moves side by side: one lane group for k, one for v
  constexpr int CHUNK = GROUPS * MOVE_ROWS;
  __shared__ long long from_s[THREADS], to_s[THREADS];  // pool rows; -1: skip
  pdl_enter();
  const KvView& c = a.c;
  const int list = blockIdx.x / a.splits, split = blockIdx.x - list * a.splits;
  const int head = list % c.n_kv, s = (list / c.n_kv) % c.n_seq, layer = list / (c.n_kv * c.n_seq);
  const int which = a.per_head ? list : s;
  const int n = a.count[which];
  const int2* mv = reinterpret_cast<const int2*>(a.moves) + static_cast<long long>(which) * a.max_moves;
  if (n < 0 || n > a.most) {
    if (threadIdx.x == 0) report_status(BITRL_ERR_SHAPE, KV_STAGE_BAD_MOVE);
    return;
  }
  if (n == 0) return;
  const bool apart = mv[n - 1].y < mv[0].x;
  int first = 0, step = THREADS;
  if (a.splits > 1) {
    if (apart) {
      first = split * THREADS;
      step = a.splits * THREADS;
    } else if (split > 0) {
      return;
    }
  }
  const int group = threadIdx.x / (2 * LANES), sub = threadIdx.x % (2 * LANES);
  uint4* pool = reinterpret_cast<uint4*>(sub >= LANES ? c.v : c.k) + sub % LANES;
  const int room = c.max_pages << c.page_shift, slot_mask = (1 << c.page_shift) - 1;
  const int* pages = c.page_table + static_cast<long long>(s) * c.max_pages;
  for (int base = first; base < n; base += step) {
    const int here = min(THREADS, n - base);
    long long fr = -1, to = -1;
    float w = 0.0f;
    int ps = 0;
    if (static_cast<int>(threadIdx.x) < here) {
      const int2 m = mv[base + threadIdx.x];
      const bool in = m.x >= 0 && m.x < room && m.y >= 0 && m.y < room;
      const int pf = in ? pages[m.x >> c.page_shift] : -1, pt = in ? pages[m.y >> c.page_shift] : -1;
      if (!in) {
        report_status(BITRL_ERR_SHAPE, KV_STAGE_BAD_MOVE);
      } else if (pf < 0 || pf >= c.n_pages || pt < 0 || pt >= c.n_pages) {
        report_status(BITRL_ERR_SHAPE, KV_STAGE_BAD_PAGE);
      } else {
        fr = kv_row(c, layer, pf, head) + (m.x & slot_mask);
        to = kv_row(c, layer, pt, head) + (m.y & slot_mask);
        if (c.mass) w = c.mass[fr];
        ps = c.pos[fr];
      }
    }
    from_s[threadIdx.x] = fr;
    to_s[threadIdx.x] = to;
    __syncthreads();  // the rows are known, and every mass and pos has been read
    if (to >= 0) {
      if (c.mass) c.mass[to] = w;
      c.pos[to] = ps;
    }
    uint4 row[2][MOVE_ROWS];
    auto read = [&](int chunk, uint4 (&r)[MOVE_ROWS]) {
#pragma unroll
      for (int u = 0; u < MOVE_ROWS; ++u) {
        const int i = chunk * CHUNK + u * GROUPS + group;
        if (i < here && from_s[i] >= 0) r[u] = pool[from_s[i] * LANES];
      }
    };
    auto write = [&](int chunk, const uint4 (&r)[MOVE_ROWS]) {
#pragma unroll
      for (int u = 0; u < MOVE_ROWS; ++u) {
        const int i = chunk * CHUNK + u * GROUPS + group;
        if (i < here && to_s[i] >= 0) pool[to_s[i] * LANES] = r[u];
      }
    };
    const int chunks = (here + CHUNK - 1) / CHUNK;
    read(0, row[0]);
    for (int k = 0; k < chunks; k += 2) {
      if (k + 1 < chunks) read(k + 1, row[1]);
      if (!apart) __syncthreads();  // everything up to chunk k (and k + 1) has been read
      write(k, row[0]);
      if (k + 1 < chunks) {
        if (k + 2 < chunks) read(k + 2, row[0]);
        if (!apart) __syncthreads();
        write(k + 1, row[1]);
      }
    }
    __syncthreads();  // from_s and to_s are free
  }
}

template <int HD>
bitrl_status launch_kv_move_hd(MoveArgs a, cudaStream_t st) {
  const long long lists = static_cast<long long>(a.c.n_layers) * a.c.n_seq * a.c.n_kv;
  const bool small = a.max_moves <= 64;  // short lists: small CTAs, so that all of them are resident together
  const int threads = small ? 64 : 256;
  long long splits = (4LL * sm_count() + lists - 1) / lists;
  const long long most = (a.max_moves + threads - 1) / threads;
  if (splits > most) splits = most;
  a.splits = static_cast<int>(splits);
  const dim3 grid(static_cast<unsigned>(lists * splits));
  BITRL_CUDA(small ? launch_pdl(kv_move_kernel<HD, 64>, grid, dim3(64), 0, st, a) : launch_pdl(kv_move_kernel<HD, 256>, grid, dim3(256), 0, st, a));
  count_launch(1);
  return BITRL_OK;
}

bitrl_status launch_kv_move(const KvView& c, const int* moves, const int* count, int max_moves, int per_head, cudaStream_t st) {
  const int room = c.max_pages << c.page_shift;
  const MoveArgs a{c, moves, count, max_moves, per_head, 1, max_moves < room ? max_moves : room};
  return c.hd == 128 ? launch_kv_move_hd<128>(a, st) : launch_kv_move_hd<64>(a, st);
}

// out[s, :] = row of the last new token of sequence s that is one (a tree may end in padding); sequences without such a token, and
// those whose tree is none, keep theirs.
__global__ void kv_pool_last_kernel(const KvView c, const KvBatch b, const uint4* h, int d8, uint4* out) {
  __shared__ int par[BITRL_TREE_MAX_TOKENS];
  __shared__ int last_s;
  pdl_enter();
  KvSeq q;
  if (!kv_seq(c, b, blockIdx.x, q)) return;
  int last = q.m - 1;
  if (b.parent) {
    if (threadIdx.x == 0) last_s = -1;
    if (!kv_load_tree(b, q, par, blockDim.x)) return;
    for (int i = threadIdx.x; i < q.m; i += blockDim.x)
      if (par[i] != BITRL_PARENT_PAD) atomicMax(&last_s, i);
    __syncthreads();
    last = last_s;
  }
  if (last < 0) return;
  const uint4* src = h + static_cast<long long>(q.t0 + last) * d8;
  uint4* dst = out + static_cast<long long>(blockIdx.x) * d8;
  for (int i = threadIdx.x; i < d8; i += blockDim.x) dst[i] = src[i];
}

bitrl_status launch_kv_pool_last(const KvView& c, const KvBatch& b, const void* h, int d, void* out, cudaStream_t st) {
  BITRL_CUDA(launch_pdl(kv_pool_last_kernel, dim3(c.n_seq), dim3(128), 0, st, c, b, static_cast<const uint4*>(h), d / 8,
                        static_cast<uint4*>(out)));
  count_launch(1);
  return BITRL_OK;
}

// ---- counters -----------------------------------------------------------------------------------------------------------
__global__ void kv_advance_kernel(const KvView c, const KvBatch b, const int* n_keep, int budget) {
  pdl_enter();
  const int s = blockIdx.x * blockDim.x + threadIdx.x;
  if (s >= c.n_seq) return;
  const int m = b.off ? b.off[s + 1] - b.off[s] : b.max_new;
  const int n = n_keep ? n_keep[s] : m;
  const long long used = static_cast<long long>(c.used[s]) + n, seen = static_cast<long long>(c.seen[s]) + n;
  if (m < 0 || m > b.max_new || n < 0 || n > m || c.used[s] < 0 || c.seen[s] < 0 || seen > INT_MAX || used > (static_cast<long long>(c.max_pages) << c.page_shift)) {
    report_status(BITRL_ERR_SHAPE, KV_STAGE_BAD_SEQ);
    return;
  }
  c.used[s] = static_cast<int>(budget > 0 && used > budget ? budget : used);
  c.seen[s] = static_cast<int>(seen);
}

bitrl_status launch_kv_advance(const KvView& c, const KvBatch& b, const int* n_keep, int budget, cudaStream_t st) {
  BITRL_CUDA(launch_pdl(kv_advance_kernel, dim3((c.n_seq + 127) / 128), dim3(128), 0, st, c, b, n_keep, budget));
  count_launch(1);
  return BITRL_OK;
}

}  // namespace bitrl

// A paged key/value cache beside the encoder: appending new tokens (rotary embedding + paged write), planning an
// eviction by accumulated attention weight, moving rows, advancing the counters.  include/bitrl.h states the layout and the
// meaning of every argument; the attention that reads the cache is in attention_cached.cuh.
#pragma once

#include <climits>
#include <math.h>

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
// copy rate bounds it; single tokens are bound by the launch and one chain of dependent loads.  A CTA takes up to
// APP_TOKENS consecutive tokens of one sequence: first its threads compute the (cos, sin) pairs, one each, then every
// thread rotates 8 dimensions and their 8 partners per step with 16-byte loads and stores.
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
  constexpr int HALF = HD / 2;
  __shared__ int par[BITRL_TREE_MAX_TOKENS];
  __shared__ float2 cs[APP_TOKENS][HALF];
  __shared__ int depth_of[APP_TOKENS];  // -1: padding
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
  if (a.b.parent) {
    if (!kv_load_tree(a.b, q, par, APP_THREADS)) return;
    if (threadIdx.x < n) {
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
    cs[t][f] = make_float2(cn, sn);
  }
  __syncthreads();
  constexpr int CP = HD / 16;  // pairs of 8-dimension chunks per head row
  const int heads = a.n_heads + 2 * c.n_kv;
  const long long width = static_cast<long long>(heads) * HD;
  const int per_token = heads * CP;
  for (int i = threadIdx.x; i < n * per_token; i += APP_THREADS) {
    const int t = i / per_token, r = i - t * per_token;
    const int head = r / CP, d0 = 8 * (r - head * CP);
    if (a.b.parent && depth_of[t] < 0) continue;
    const int tok = first + t;
    const unsigned short* src = a.qkv + (q.t0 + tok) * width + head * HD + d0;
    uint4 x1 = *reinterpret_cast<const uint4*>(src), x2 = *reinterpret_cast<const uint4*>(src + HALF);
    if (head < a.n_heads + c.n_kv) {
      uint32_t w1[4] = {x1.x, x1.y, x1.z, x1.w}, w2[4] = {x2.x, x2.y, x2.z, x2.w};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float2 e0 = cs[t][d0 + 2 * w], e1 = cs[t][d0 + 2 * w + 1];
        const float x1a = __uint_as_float(w1[w] << 16), x1b = __uint_as_float(w1[w] & 0xffff0000u);
        const float x2a = __uint_as_float(w2[w] << 16), x2b = __uint_as_float(w2[w] & 0xffff0000u);
        const __nv_bfloat162 o1 = __floats2bfloat162_rn(fmaf(-x2a, e0.y, __fmul_rn(x1a, e0.x)), fmaf(-x2b, e1.y, __fmul_rn(x1b, e1.x)));
        const __nv_bfloat162 o2 = __floats2bfloat162_rn(fmaf(x1a, e0.y, __fmul_rn(x2a, e0.x)), fmaf(x1b, e1.y, __fmul_rn(x2b, e1.x)));
        w1[w] = *reinterpret_cast<const uint32_t*>(&o1);
        w2[w] = *reinterpret_cast<const uint32_t*>(&o2);
      }
      x1 = make_uint4(w1[0], w1[1], w1[2], w1[3]);
      x2 = make_uint4(w2[0], w2[1], w2[2], w2[3]);
    }
    unsigned short* dst;
    if (head < a.n_heads) {
      dst = a.q_out + (static_cast<long long>(q.t0 + tok) * a.n_heads + head) * HD + d0;
    } else {
      const int kvh = (head - a.n_heads) % c.n_kv;
      const bool is_k = head < a.n_heads + c.n_kv;
      const int slot = q.used + tok, page = kv_page(c, s, slot);
      if (page < 0) continue;
      const long long row = kv_row(c, 0, page, kvh) + (slot & ((1 << c.page_shift) - 1));
      dst = (is_k ? c.k : c.v) + row * HD + d0;
      if (is_k && d0 == 0) {
        if (c.mass) c.mass[row] = 0.0f;
        c.pos[row] = seen + (a.b.parent ? depth_of[t] : tok);
      }
    }
    *reinterpret_cast<uint4*>(dst) = x1;
    *reinterpret_cast<uint4*>(dst + HALF) = x2;
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
// (NaN lowest, -0 = +0).  Protected slots come first, so the threshold lies in one group alone: the free slots when the
// protected ones fit into the budget, else the protected ones.  Selection: counts over up to 2048 equal steps of the key
// range that the group really spans (weights fill a few binades, so fixed digits would pile up in a few counters), then
// over the step that holds the threshold, until few keys are left in it (or one value), whose ranks are counted directly.
// One ordered pass then makes a bit per slot (ties: lower slots stay), another turns bits into the two ascending lists.
// Every slot is read from memory once, its key kept in shared memory.  8 bytes per slot would take 17 us for 2400 lists of up
// to 8192 slots; the passes over shared memory and the meeting points between them bound it.
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
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);  // -inf is 0x007fffff: above NaN
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
  const int words = (n + 31) >> 5;
  const bool cached = n <= a.smem_slots;
  uint32_t* key_s = reinterpret_cast<uint32_t*>(plan_smem);        // [min(n, smem_slots)]
  uint32_t* prot_s = key_s + a.smem_slots;                         // [words] bit per slot: protected
  uint32_t* keep_s = prot_s + (static_cast<int>(room) + 31) / 32;  // [words] bit per slot: stays
  const int recent_from = seen > a.recent ? seen - a.recent : 0, slot_mask = (1 << c.page_shift) - 1;
  const int* pages = c.page_table + static_cast<long long>(s) * c.max_pages;
  auto key_at = [&](int t) -> uint32_t {
    return cached ? key_s[t] : plan_key(c.mass[kv_row(c, layer, pages[t >> c.page_shift], head) + (t & slot_mask)]);
  };
  if (threadIdx.x == 0) {
    n_prot = 0;
    group_lo = 0xffffffffu;
    group_hi = 0u;
  }
  // ---- read every slot once: key, protected bit, range of the keys of either group
  int prot = 0;
  uint32_t lo[2] = {0xffffffffu, 0xffffffffu}, hi[2] = {0u, 0u};  // free, protected
  bool bad = false;
  for (int w = warp; w < words; w += 4 * WARPS) {
    int page[4], ps[4];
    float m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 32 * (w + i * WARPS) + lane;
      page[i] = t < n ? pages[t >> c.page_shift] : 0;
      if (page[i] < 0 || page[i] >= c.n_pages) {
        bad = true;
        page[i] = 0;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 32 * (w + i * WARPS) + lane;
      const long long r = kv_row(c, layer, page[i], head) + (t & slot_mask);
      ps[i] = t < n ? c.pos[r] : INT_MAX;
      m[i] = t < n ? c.mass[r] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = w + i * WARPS, t = 32 * at + lane;
      if (at >= words) break;
      const bool p = t < n && (ps[i] >= recent_from || ps[i] < a.sink);
      const uint32_t bits = __ballot_sync(0xffffffffu, p), key = plan_key(m[i]);
      if (t < n) {
        if (cached) key_s[t] = key;
        lo[0] = p ? lo[0] : min(lo[0], key);
        hi[0] = p ? hi[0] : max(hi[0], key);
        lo[1] = p ? min(lo[1], key) : lo[1];
        hi[1] = p ? max(hi[1], key) : hi[1];
      }
      if (lane == 0) prot_s[at] = bits;
      prot += __popc(bits);
    }
  }
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) { report_status(BITRL_ERR_SHAPE, KV_STAGE_BAD_PAGE); a.count[list] = 0; }
    return;
  }
  if (lane == 0 && prot) atomicAdd(&n_prot, prot);
  __syncthreads();
  const bool among_protected = n_prot >= B;  // which group the threshold lies in
  int want = among_protected ? B : B - n_prot;  // slots of that group that stay
  {
    const uint32_t l = __reduce_min_sync(0xffffffffu, lo[among_protected]), h = __reduce_max_sync(0xffffffffu, hi[among_protected]);
    if (lane == 0) {
      atomicMin(&group_lo, l);
      atomicMax(&group_hi, h);
    }
  }
  __syncthreads();
  uint32_t from = group_lo, to = group_hi;  // the threshold key lies in from .. to; `want` slots of that range stay
  uint32_t thr = from;
  int at_thr = 0;  // slots whose key is the threshold
  // words of this warp, as `in` flags with their keys
  auto each = [&](auto&& f) {
    for (int w = warp; w < words; w += WARPS) {
      const int t = 32 * w + lane;
      if (t < n && (((prot_s[w] >> lane) & 1u) != 0) == among_protected) f(key_at(t));
    }
  };
  while (true) {
    const uint32_t span = to - from;
    const int shift = span < PLAN_BINS ? 0 : 21 - __clz(span);  // span >> shift < PLAN_BINS
    for (int i = threadIdx.x; i < PLAN_BINS; i += THREADS) hist[i] = 0;
    if (threadIdx.x == 0) n_few = 0;
    __syncthreads();
    each([&](uint32_t key) {
      if (key >= from && key <= to) atomicAdd(&hist[(key - from) >> shift], 1);
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
      each([&](uint32_t key) {
        if (key >= from && key <= to) few[atomicAdd(&n_few, 1)] = key;
      });
      __syncthreads();
      if (threadIdx.x < left) {
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

  // ---- ordered decision: every warp owns a run of words.  Of the at_thr slots that equal the threshold the `want` lowest stay.
  const int per_warp = (words + WARPS - 1) / WARPS, w0 = warp * per_warp, w1 = min(words, w0 + per_warp);
  int tie_rank = 0;
  if (want < at_thr) {
    int ties = 0;
    for (int w = w0; w < w1; ++w) {
      const int t = 32 * w + lane;
      const bool in = t < n && (((prot_s[w] >> lane) & 1u) != 0) == among_protected;
      ties += __popc(__ballot_sync(0xffffffffu, in && key_at(t) == thr));
    }
    __syncthreads();
    if (lane == 0) part[warp] = ties;
    __syncthreads();
    for (int w = 0; w < warp; ++w) tie_rank += part[w];
  }
  int n_src = 0, n_dst = 0;
  for (int w = w0; w < w1; ++w) {
    const int t = 32 * w + lane;
    const bool p = ((prot_s[w] >> lane) & 1u) != 0, in = t < n && p == among_protected;
    const uint32_t key = in ? key_at(t) : 0u;
    bool keep = (p && !among_protected) || (in && key >= thr);
    if (want < at_thr) {
      const uint32_t tie = __ballot_sync(0xffffffffu, in && key == thr);
      if (in && key == thr) keep = tie_rank + __popc(tie & ((1u << lane) - 1u)) < want;
      tie_rank += __popc(tie);
    }
    const uint32_t kept = __ballot_sync(0xffffffffu, keep);
    if (lane == 0) keep_s[w] = kept;
    const uint32_t below = 32 * w + 32 <= B ? 0xffffffffu : 32 * w >= B ? 0u : (1u << (B - 32 * w)) - 1u;  // slots < B
    n_src += __popc(kept & ~below);
    n_dst += __popc(~kept & below);
  }
  __syncthreads();
  if (lane == 0) { part[warp] = n_src; part2[warp] = n_dst; }
  __syncthreads();
  int at_src = 0, at_dst = 0;
  for (int w = 0; w < warp; ++w) { at_src += part[w]; at_dst += part2[w]; }
  if (threadIdx.x == 0) {
    int total = 0;
    for (int w = 0; w < WARPS; ++w) total += part[w];
    a.count[list] = total;
  }
  int* out = a.moves + static_cast<long long>(list) * a.max_moves * 2;
  for (int w = w0; w < w1; ++w) {
    const uint32_t kept = keep_s[w], below = 32 * w + 32 <= B ? 0xffffffffu : 32 * w >= B ? 0u : (1u << (B - 32 * w)) - 1u;
    const uint32_t bs = kept & ~below, bd = ~kept & below, mine = 1u << lane;
    if (bs & mine) out[2 * (at_src + __popc(bs & (mine - 1u)))] = 32 * w + lane;
    if (bd & mine) out[2 * (at_dst + __popc(bd & (mine - 1u))) + 1] = 32 * w + lane;
    at_src += __popc(bs);
    at_dst += __popc(bd);
  }
}

template <int THREADS>
bitrl_status launch_kv_evict_plan_t(const PlanArgs& a, size_t smem, size_t limit, unsigned lists, cudaStream_t st) {
  static bool done[64] = {false};
  int dev = 0;
  BITRL_CUDA(cudaGetDevice(&dev));
  if (dev >= 0 && dev < 64 && !done[dev]) {
    BITRL_CUDA(cudaFuncSetAttribute(kv_evict_plan_kernel<THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(limit)));
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
  const size_t bits = static_cast<size_t>((room + 31) / 32) * 8;  // two bit arrays
  constexpr size_t LIMIT = 200 * 1024;
  if (bits > LIMIT) return BITRL_ERR_LIMIT;
  const size_t left = (LIMIT - bits) / 4;
  a.smem_slots = static_cast<int>(left < static_cast<size_t>(room) ? left : room);
  const size_t smem = static_cast<size_t>(a.smem_slots) * 4 + bits;
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
// and the list may be spread over several CTAs.
constexpr int MOVE_ROWS = 4;  // rows of a chunk per lane group

struct MoveArgs {
  KvView c;
  const int* moves;
  const int* count;
  int max_moves, per_head, splits;
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
  if (n < 0 || n > a.max_moves) {
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
  const MoveArgs a{c, moves, count, max_moves, per_head, 1};
  return c.hd == 128 ? launch_kv_move_hd<128>(a, st) : launch_kv_move_hd<64>(a, st);
}

// out[s, :] = row of the last new token of sequence s; sequences without new tokens keep theirs.
__global__ void kv_pool_last_kernel(const KvView c, const KvBatch b, const uint4* h, int d8, uint4* out) {
  pdl_enter();
  KvSeq q;
  if (!kv_seq(c, b, blockIdx.x, q) || q.m == 0) return;
  const uint4* src = h + static_cast<long long>(q.t0 + q.m - 1) * d8;
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
  if (m < 0 || m > b.max_new || n < 0 || n > m || seen > INT_MAX || used > (static_cast<long long>(c.max_pages) << c.page_shift)) {
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

// Attention of new tokens over a paged key/value cache (kv_cache.cuh), with the weight that every slot receives.
//
//   score(i, r) = q_i . k_r / sqrt(head_dim);  p = softmax over the slots r that token i sees;  att_i = sum_r p_r v_r
//   mass[r] += sum over the tokens i and the query heads of the kv head of p(i, r)
//
// The query heads of a kv head share its keys, so the rows of a sequence are the pairs (token, head of the group):
// row x = token * rep + j.  Everything works on logarithms to base two: t = score * log2(e), p = 2^(t - lse).
#pragma once

#include <cuda.h>

#include "attention.cuh"
#include "common.cuh"
#include "kv_cache.cuh"
#include "ptx.cuh"

namespace bitrl {

constexpr int AC_TREE_WORDS = BITRL_TREE_MAX_TOKENS / 32;

// Where a cut item of the tile kernels was left: two per CTA (0: the item began in an earlier CTA, 1: it begins here); s < 0: none.
struct AtCut {
  int s, x, h, ends;
};

struct AcArgs {
  KvView c;  // this layer
  KvBatch b;
  const unsigned short* q;  // bf16 [T][n_heads * HD]
  unsigned short* att;      // the same
  int n_heads, rep;
  float scale2;            // log2(e) / sqrt(head_dim)
  float* part_o;           // [parts][rows][HD] unnormalised results of cut items
  float2* part_ml;         // [parts][rows]: running maximum and sum
  float* lse;              // [T * n_heads]: maximum + log2(sum); +inf where a row sees nothing
  const uint32_t* anc;     // trees: [T][AC_TREE_WORDS], the tokens that a token sees
  const uint32_t* desc;    // trees: [T][AC_TREE_WORDS], the tokens that see a token
  const int* tree_ok;      // trees: [n_seq], else nullptr
  AtCut* cuts;             // tile kernels: [CTAs][2]
};

__device__ __forceinline__ float ac_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The maximum that a part of a row hands on.  Maxima pass over NaN: a part with nothing but NaN would look like one that sees
// nothing (-inf) and be left out, so a sum that is NaN takes its maximum along.
__device__ __forceinline__ float ac_part_max(float m, float l) { return l == l ? m : l; }
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Transposes an 8 x 8 matrix of 16-bit elements held as lane 4 i + j: row i, columns 2 j and 2 j + 1.
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// (x0, x1) -> bf16 pair (x0 in the low half)
__device__ __forceinline__ uint32_t pack_bf16x2(float x0, float x1) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(x0, x1);
  return *reinterpret_cast<const uint32_t*>(&p);
}
// Weights p0, p1 >= 0 as two bf16 halves each, p = hi + lo (p0 in the low half of a word): 16 significant bits, where one bf16 would
// move a result of few keys by up to 2^-8 of their magnitudes, as much as its own rounding.  hi is cut, not rounded, and 2^-20 of p
// keeps lo above zero wherever p is (down to 2^-100 and less): hi and lo then have one sign, and the two products with a value that is
// infinite are the same infinity.
__device__ __forceinline__ void ac_split(float p0, float p1, uint32_t& hi, uint32_t& lo) {
  const uint32_t b0 = __float_as_uint(p0), b1 = __float_as_uint(p1);
  hi = __byte_perm(b0, b1, 0x7632);
  constexpr float up = 1.0f + 0x1p-20f;
  float l0, l1;
  ptx::unpack_f32x2(ptx::fma_f32x2(ptx::pack_f32x2(b0, b1), ptx::pack_f32x2(__float_as_uint(up), __float_as_uint(up)),
                                   ptx::pack_f32x2((b0 & 0xffff0000u) | 0x80000000u, (b1 & 0xffff0000u) | 0x80000000u)), l0, l1);
  lo = pack_bf16x2(l0, l1);
}
// Ancestors of every new token as bits, anc[row][AC_TREE_WORDS]: bit j is set when token j of the sequence is the token
// itself or above it; padding has no bits.  desc is the transpose.  ok[s]: the sequence's tree is one.  One CTA per sequence.
__global__ void __launch_bounds__(BITRL_TREE_MAX_TOKENS)
attn_tree_kernel(const KvView c, const KvBatch b, uint32_t* anc, uint32_t* desc, int* ok) {
  __shared__ int par[BITRL_TREE_MAX_TOKENS];
  __shared__ uint32_t below[BITRL_TREE_MAX_TOKENS][AC_TREE_WORDS + 1];
  pdl_enter();
  const int s = blockIdx.x, i = threadIdx.x;
  KvSeq q;
  const bool good = kv_seq(c, b, s, q) && kv_load_tree(b, q, par, BITRL_TREE_MAX_TOKENS);
  if (i == 0) ok[s] = good;
  if (!good) return;
  uint32_t w[AC_TREE_WORDS];
#pragma unroll
  for (int k = 0; k < AC_TREE_WORDS; ++k) w[k] = below[i][k] = 0u;
  __syncthreads();
  if (i < q.m)
    for (int j = par[i] == BITRL_PARENT_PAD ? -1 : i; j >= 0; j = par[j]) {
#pragma unroll
      for (int k = 0; k < AC_TREE_WORDS; ++k) w[k] |= (j >> 5) == k ? 1u << (j & 31) : 0u;
      atomicOr(&below[j][i >> 5], 1u << (i & 31));
    }
  __syncthreads();
  if (i >= q.m) return;
  const long long at = (static_cast<long long>(q.t0) + i) * AC_TREE_WORDS;
  uint4* out = reinterpret_cast<uint4*>(anc + at);
  out[0] = make_uint4(w[0], w[1], w[2], w[3]);
  out[1] = make_uint4(w[4], w[5], w[6], w[7]);
  const uint32_t* d = below[i];
  out = reinterpret_cast<uint4*>(desc + at);
  out[0] = make_uint4(d[0], d[1], d[2], d[3]);
  out[1] = make_uint4(d[4], d[5], d[6], d[7]);
}
// Does token `tok` see the slot of new token j (j >= 0)?
__device__ __forceinline__ bool ac_sees_new(const uint32_t* anc, int tok, int j) {
  return anc ? ((anc[tok * AC_TREE_WORDS + (j >> 5)] >> (j & 31)) & 1u) != 0 : j <= tok;
}
__device__ __forceinline__ bool ac_is_pad(const uint32_t* anc, int tok) { return anc && !ac_sees_new(anc, tok, tok); }

// ---- few rows (at most 16 per sequence and kv head) ------------------------------------------------------------------
// Bound by the reading of keys and values.  Lengths are known on the device alone, so the work is cut there: the units (16
// slots of one sequence and kv head) of the whole batch form one list, sequence by sequence and head by head, and every
// warp of the grid takes an equal run of it, whatever the lengths are.  A warp needs nothing from the others: it brings its
// units in by TMA through a ring of its own, keeps a running maximum, sum and 16 x HD result, and leaves one result per
// (sequence, head) that it met.  Results of items that lie within one run are final; the others are joined by
// attn_few_join_kernel, which also turns the scores that this kernel leaves behind (fp32, 16 to 64 bytes per slot beside
// the 4 HD bytes of its key and value) into the weight of every slot, so that keys are read once.
// Scores come from mma.sync (eight rows fill its N; a tcgen05 tile has 128 rows).  The weights are split into two bf16
// halves (16 significant bits), which costs nothing where reading bounds the kernel.
// 128 sequences of up to 4096 slots, one token each, 20 heads over 5: 115 us for 633 MB, 5.5 TB/s (the join: 14 us); one
// sequence of 100k slots: 49 + 14 us; of 2000: 12.6 us together, a chain of two launches and their loads.
constexpr int AF_WARPS = 4;
constexpr int AF_CTAS = 2;  // per SM
constexpr int AF_THREADS = 32 * AF_WARPS;
constexpr int AJ_THREADS = 256, AJ_WARPS = AJ_THREADS / 32;
constexpr int AF_STAGES = 3;
constexpr int AF_ROWS = 16;
constexpr int AF_SLOTS = 16;   // slots of a unit
constexpr int AF_MIN_RUN = 2;  // units of a run at least (short lists use fewer warps)
enum { AF_WAIT_LOAD = 151 };

struct AfHead {
  int units, runs;  // of the whole list; runs in use
  int per, more;    // units of a run; the first `more` runs have one more
};

struct AfArgs {
  AcArgs a;
  int rows_cap;    // rows of a sequence and head at most: max_new * rep
  int score_rows;  // rows_cap rounded up to 4, 8 or 16
  int max_runs;
  int join_slots;  // slots of a CTA of the join
  float* scores;   // [pages][kv heads][page][score_rows] or nullptr: scores in base-two units, -inf where unseen
  AfHead* head;
  int* item_at;    // [n_seq * n_kv] place of an item's first unit in the list
};

// First unit of run r.
__device__ __forceinline__ int af_start(const AfHead& h, int r) { return r * h.per + min(r, h.more); }
// The run that holds unit g.
__device__ __forceinline__ int af_run_of(const AfHead& h, int g) {
  const int longer = h.more * (h.per + 1);
  return g < longer ? g / (h.per + 1) : h.more + (g - longer) / h.per;
}
// Units of one kv head of sequence s.
__device__ __forceinline__ int af_units(const AcArgs& a, int s, KvSeq& q) {
  if (!kv_seq(a.c, a.b, s, q) || q.m == 0 || (a.tree_ok && !a.tree_ok[s])) return 0;
  return (q.used + q.m + AF_SLOTS - 1) / AF_SLOTS;
}

template <int HD>
constexpr uint32_t af_smem_bytes() {
  return AF_WARPS * AF_STAGES * 2 * AF_SLOTS * HD * 2 + 1024;
}

// NG: groups of eight rows.
template <int HD, int NG>
__global__ void __launch_bounds__(AF_THREADS, AF_CTAS)
attn_few_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ AfArgs f) {
  constexpr int KS = HD / 16, MD = HD / 16, NH = HD / 64;
  constexpr uint32_t HALF = AF_SLOTS * 128, TILE = NH * HALF;  // a 64-dimension block of the keys (or values) of a unit
  extern __shared__ unsigned char af_smem_raw[];
  __shared__ __align__(8) unsigned long long bars[AF_WARPS * AF_STAGES];
  __shared__ int row_s[AF_WARPS * AF_STAGES];  // pool row of the unit in each place of the rings
  __shared__ int part[AF_WARPS], first_of[AF_THREADS + 1];
  const AcArgs& a = f.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, lm = lane >> 3, lr = lane & 7;
  const uint32_t bar = ptx::smem_u32(bars + warp * AF_STAGES);
  if (threadIdx.x < AF_WARPS * AF_STAGES) ptx::mbar_init(ptx::smem_u32(bars + threadIdx.x), 1);
  if (threadIdx.x == 0) {
    ptx::tma_prefetch_desc(&tmap_k);
    ptx::tma_prefetch_desc(&tmap_v);
  }
  ptx::mbar_init_fence();
  pdl_enter();

  // ---- this warp's run: units before every block of sequences, then a search
  KvSeq q;
  const int per = (a.c.n_seq + AF_THREADS - 1) / AF_THREADS, sb = min(a.c.n_seq, per * static_cast<int>(threadIdx.x));
  int sum = 0;
  for (int s = sb; s < min(a.c.n_seq, sb + per); ++s) sum += af_units(a, s, q);
  sum *= a.c.n_kv;
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) part[warp] = incl;
  __syncthreads();
  for (int w = 0; w < warp; ++w) incl += part[w];
  first_of[threadIdx.x + 1] = incl;
  if (threadIdx.x == 0) first_of[0] = 0;
  __syncthreads();
  AfHead head;
  head.units = static_cast<int>(first_of[AF_THREADS]);
  head.runs = min(f.max_runs, (head.units + AF_MIN_RUN - 1) / AF_MIN_RUN);
  head.per = head.runs > 0 ? head.units / head.runs : 0;
  head.more = head.units - head.per * head.runs;
  // neighbouring runs go to different CTAs, so that a short list spreads over all SMs
  const int r = warp * gridDim.x + blockIdx.x;
  if (blockIdx.x == 0 && threadIdx.x == 0) *f.head = head;
  if (r >= head.runs) return;
  const int w0 = af_start(head, r);
  int left = af_start(head, r + 1) - w0, s = 0, h = 0, u0 = 0;
  {
    int block = 0;  // the last block that begins at or before w0: blocks without units do not count
    for (int i = lane; i < AF_THREADS; i += 32)
      if (first_of[i] <= w0 && w0 < first_of[i + 1]) block = i;
    block = __reduce_max_sync(0xffffffffu, block);
    int rem = w0 - first_of[block];
    for (s = block * per;; ++s) {
      const int n = af_units(a, s, q) * a.c.n_kv;
      if (rem < n || s + 1 >= a.c.n_seq) break;
      rem -= n;
    }
    const int n = af_units(a, s, q);
    h = rem / n;
    u0 = rem % n;
  }

  // ---- loads, ahead of the arithmetic: a position of their own in the list; the page of the next unit is read one unit early
  const uint32_t raw = ptx::smem_u32(af_smem_raw), ring = ((raw + 1023u) & ~1023u) + warp * (AF_STAGES * 2 * TILE);
  const uint32_t rows_at = ptx::smem_u32(row_s + warp * AF_STAGES);
  const int slot_mask = (1 << a.c.page_shift) - 1;
  const int none_row = (a.c.n_pages * a.c.n_kv) << a.c.page_shift;  // behind the pool: such a copy fills with zeros
  int ls = s, lh = h, lu = u0, l_left = left;
  KvSeq lq = q;
  int l_units = af_units(a, ls, lq);
  const int* l_pages = a.c.page_table + static_cast<long long>(ls) * a.c.max_pages;
  int l_page = l_pages[(lu * AF_SLOTS) >> a.c.page_shift];
  auto load = [&](int stage) {
    if (l_left <= 0) return;
    if (lane == 0) {
      int row = none_row;
      if (l_page >= 0 && l_page < a.c.n_pages)
        row = ((l_page * a.c.n_kv + lh) << a.c.page_shift) + ((lu * AF_SLOTS) & slot_mask);
      else
        report_status(BITRL_ERR_SHAPE, KV_STAGE_BAD_PAGE);
      const uint32_t dst = ring + stage * 2 * TILE;
      ptx::sts32(rows_at + 4 * stage, row);
      ptx::mbar_arrive_expect_tx(bar + 8 * stage, 2 * TILE);
#pragma unroll
      for (int i = 0; i < NH; ++i) {
        ptx::tma_load_2d(dst + i * HALF, &tmap_k, 64 * i, row, bar + 8 * stage);
        ptx::tma_load_2d(dst + TILE + i * HALF, &tmap_v, 64 * i, row, bar + 8 * stage);
      }
    }
    if (--l_left <= 0) return;
    if (++lu == l_units) {
      lu = 0;
      if (++lh == a.c.n_kv) {
        lh = 0;
        do l_units = af_units(a, ++ls, lq);
        while (l_units == 0 && ls + 1 < a.c.n_seq);
        l_pages = a.c.page_table + static_cast<long long>(ls) * a.c.max_pages;
      }
    }
    l_page = l_pages[(lu * AF_SLOTS) >> a.c.page_shift];
  };
  for (int i = 0; i < AF_STAGES; ++i) load(i);
  uint32_t stage = 0, phase = 0;
  bool ok = true;

  while (ok && left > 0) {
    const int units = af_units(a, s, q);
    const int u1 = min(units, u0 + left), end = q.used + q.m, rows = q.m * a.rep;
    const uint32_t* anc = a.b.parent ? a.anc + static_cast<long long>(q.t0) * AC_TREE_WORDS : nullptr;
    if (u0 == 0 && lane == 0) f.item_at[s * a.c.n_kv + h] = af_start(head, r + 1) - left;
    // Products are transposed, slots (or dimensions) x rows: S^T = K Q^T, O^T = V^T P^T.  Eight rows fill the N of an
    // instruction, where they would fill half of its M.  This lane: rows 8 n + 2 t and the next; slots g and g + 8.
    uint32_t qb[NG][KS][2];
    int tok[NG][2];
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      const int x = 8 * n + g;  // B operand: the lane's row is g
      const bool live = x < rows;
      const int tk = live ? x / a.rep : 0;
      const unsigned short* row =
          a.q + (static_cast<long long>(q.t0 + tk) * a.n_heads + h * a.rep + (live ? x - tk * a.rep : 0)) * HD + 2 * t;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qb[n][ks][0] = live ? *reinterpret_cast<const uint32_t*>(row + 16 * ks) : 0u;
        qb[n][ks][1] = live ? *reinterpret_cast<const uint32_t*>(row + 16 * ks + 8) : 0u;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) tok[n][e] = min(8 * n + 2 * t + e, rows - 1) / a.rep;
    }
    float o[NG][MD][4];
    float m_run[NG][2], l_run[NG][2];
#pragma unroll
    for (int n = 0; n < NG; ++n) {
#pragma unroll
      for (int d = 0; d < MD; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][d][e] = 0.0f;
#pragma unroll
      for (int e = 0; e < 2; ++e) { m_run[n][e] = -INFINITY; l_run[n][e] = 0.0f; }
    }

    for (int u = u0; u < u1; ++u) {
      const int slot0 = u * AF_SLOTS;
      if (!__any_sync(0xffffffffu, ptx::mbar_wait(bar + 8 * stage, phase))) {
        ok = false;
        break;
      }
      const uint32_t ks_addr = ring + stage * 2 * TILE, vs_addr = ks_addr + TILE;
      float c[NG][4], c2[NG][4];  // two chains of products
#pragma unroll
      for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) c[n][e] = c2[n][e] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int key = 8 * (lm & 1) + lr, ch = 2 * ks + (lm >> 1);
        uint32_t ka[4];
        ldmatrix_x4(ks_addr + (ch >> 3) * HALF + key * 128 + (((ch ^ key) & 7) << 4), ka);
#pragma unroll
        for (int n = 0; n < NG; ++n) mma_bf16(ks & 1 ? c2[n] : c[n], ka, qb[n][ks][0], qb[n][ks][1]);
      }
      // ---- scale, mask; slots below used are seen by every row
      const bool masked = slot0 + AF_SLOTS > q.used;
#pragma unroll
      for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          c[n][e] = __fmul_rn(c[n][e] + c2[n][e], a.scale2);
          if (masked) {
            const int slot = slot0 + g + 8 * (e >> 1);
            const bool see = slot < end && (slot < q.used || ac_sees_new(anc, tok[n][e & 1], slot - q.used));
            c[n][e] = see ? c[n][e] : -INFINITY;
          }
        }
      if (f.scores) {
        const int row = static_cast<int>(ptx::lds32(rows_at + 4 * stage));
        if (row < none_row) {
          float* to = f.scores + static_cast<long long>(row + g) * f.score_rows + 2 * t;
#pragma unroll
          for (int n = 0; n < NG; ++n)
            if (8 * n + 2 * t < f.score_rows) {
              *reinterpret_cast<float2*>(to + 8 * n) = make_float2(c[n][0], c[n][1]);
              *reinterpret_cast<float2*>(to + 8 * f.score_rows + 8 * n) = make_float2(c[n][2], c[n][3]);
            }
        }
      }
      float alpha[NG][2];
      bool moved = false;
#pragma unroll
      for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float mx = fmaxf(c[n][e], c[n][2 + e]);
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          const float m_new = fmaxf(m_run[n][e], mx);
          alpha[n][e] = m_new == m_run[n][e] ? 1.0f : ac_exp2(m_run[n][e] - m_new);
          moved |= alpha[n][e] != 1.0f;
          m_run[n][e] = m_new;
        }
#pragma unroll
      for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) c[n][e] = c[n][e] == -INFINITY ? 0.0f : ac_exp2(c[n][e] - m_run[n][e & 1]);
#pragma unroll
      for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) l_run[n][e] = fmaf(l_run[n][e], alpha[n][e], c[n][e] + c[n][2 + e]);
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int n = 0; n < NG; ++n)
#pragma unroll
          for (int d = 0; d < MD; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][d][e] = __fmul_rn(o[n][d][e], alpha[n][e & 1]);
      }
      // A value that is not finite in a slot that some row does not see (or behind the last slot) must not reach that row as
      // 0 * inf: from the first new token's slot on such values become zero, and the rows that see them get them back below.
      bool odd = false;
      if (masked) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(TILE / 512); ++i) {
          const uint32_t at = vs_addr + (lane + 32 * i) * 16;
          const uint4 x = ptx::lds128(at);
          uint32_t w[4] = {x.x, x.y, x.z, x.w};
          bool hit = false;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const bool lo = (w[j] & 0x7f80u) == 0x7f80u, hi = (w[j] & 0x7f800000u) == 0x7f800000u;
            hit |= lo || hi;
            w[j] &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
          }
          if (hit && slot0 + (((lane + 32 * i) & 127) >> 3) >= q.used) {
            ptx::sts128(at, make_uint4(w[0], w[1], w[2], w[3]));
            odd = true;
          }
        }
        odd = __any_sync(0xffffffffu, odd);
        if (odd) ptx::fence_proxy_async_smem();  // the next copy into this place comes after these writes
        __syncwarp();
      }
      uint32_t ph[NG][2], pl[NG][2];  // B operand: row g, slots 2 t and the next (and + 8): blocks of 8 x 8 transposed
#pragma unroll
      for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t hi, lo;
          ac_split(c[n][2 * i], c[n][2 * i + 1], hi, lo);
          ph[n][i] = movmatrix_trans(hi);
          pl[n][i] = movmatrix_trans(lo);
        }
#pragma unroll
      for (int d = 0; d < MD; ++d) {
        const int key = 8 * (lm >> 1) + lr, ch = 2 * d + (lm & 1);
        uint32_t va[4];
        ldmatrix_x4_trans(vs_addr + (ch >> 3) * HALF + key * 128 + (((ch ^ key) & 7) << 4), va);
#pragma unroll
        for (int n = 0; n < NG; ++n) mma_bf16(o[n][d], va, ph[n][0], ph[n][1]);
#pragma unroll
        for (int n = 0; n < NG; ++n) mma_bf16(o[n][d], va, pl[n][0], pl[n][1]);
      }
      const int pool_row = odd ? static_cast<int>(ptx::lds32(rows_at + 4 * stage)) : none_row;
      if (pool_row < none_row) {  // rare
        const unsigned short* v = a.c.v + static_cast<long long>(pool_row) * HD;
#pragma unroll 1
        for (int key = max(q.used - slot0, 0); key < min(end - slot0, AF_SLOTS); ++key)
#pragma unroll
          for (int n = 0; n < NG; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (ac_sees_new(anc, tok[n][e], slot0 + key - q.used)) {
#pragma unroll
                for (int d = 0; d < MD; ++d)
#pragma unroll
                  for (int i = 0; i < 2; ++i) {
                    const unsigned short b = v[key * HD + 16 * d + 8 * i + g];
                    if ((b & 0x7f80u) == 0x7f80u) o[n][d][2 * i + e] += bf16_bits_to_float(b);
                  }
              }
      }
      __syncwarp();
      load(stage);  // the unit AF_STAGES ahead takes this one's place
      if (++stage == AF_STAGES) {
        stage = 0;
        phase ^= 1u;
      }
    }
    if (!ok) break;

    // ---- the item, or this run's part of it
    const bool whole = u0 == 0 && u1 == units;
    const int cut = 2 * r + (u0 == 0 ? 1 : 0);
#pragma unroll
    for (int n = 0; n < NG; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float l = l_run[n][e];
        l += __shfl_xor_sync(0xffffffffu, l, 4);
        l += __shfl_xor_sync(0xffffffffu, l, 8);
        l += __shfl_xor_sync(0xffffffffu, l, 16);
        const int x = 8 * n + 2 * t + e;
        if (x >= rows) continue;
        if (whole) {
          const bool none = l == 0.0f || ac_is_pad(anc, tok[n][e]);
          const float inv = none ? 0.0f : __fdiv_rn(1.0f, l);
          const long long row = static_cast<long long>(q.t0 + tok[n][e]) * a.n_heads + h * a.rep + x - tok[n][e] * a.rep;
#pragma unroll
          for (int d = 0; d < MD; ++d)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              a.att[row * HD + 16 * d + 8 * i + g] = none ? 0 : float_to_bf16_bits(__fmul_rn(o[n][d][2 * i + e], inv));
          if (g == 0) a.lse[row] = none ? INFINITY : m_run[n][e] + __log2f(l);
        } else {
          float* to = a.part_o + (static_cast<long long>(cut) * f.rows_cap + x) * HD + g;
#pragma unroll
          for (int d = 0; d < MD; ++d)
#pragma unroll
            for (int i = 0; i < 2; ++i) to[16 * d + 8 * i] = o[n][d][2 * i + e];
          if (g == 0) a.part_ml[static_cast<long long>(cut) * f.rows_cap + x] = make_float2(ac_part_max(m_run[n][e], l), l);
        }
      }
    left -= u1 - u0;
    u0 = 0;
    if (left > 0 && ++h == a.c.n_kv) {
      h = 0;
      while (++s + 1 < a.c.n_seq && af_units(a, s, q) == 0) {}
    }
  }
  if (!ok) {
    // failure path only: a copy that did not arrive in time may still be in flight
    if (lane == 0) report_timeout(AF_WAIT_LOAD);
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000LL) {}
  }
}

// Per item (sequence, kv head): joins the results of the runs that met it, in run order, and adds every slot's weights,
// p = 2^(score - lse), to mass.  The CTAs of an item share its slots, f.join_slots each, and the results, by threads (few parts)
// or by pieces of 8 dimensions (many parts: 4 parts side by side in a warp).  Short chains of loads bound it, so each thread
// keeps several under way.
template <int HD, int SR>
__global__ void __launch_bounds__(AJ_THREADS) attn_few_join_kernel(const __grid_constant__ AfArgs f) {
  pdl_enter();
  const AcArgs& a = f.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  __shared__ float lse_s[AF_ROWS], max_s[AF_ROWS], inv_s[AF_ROWS];
  const int h = blockIdx.x % a.c.n_kv, s = blockIdx.x / a.c.n_kv;
  KvSeq q;
  const int units = af_units(a, s, q), end = q.used + q.m, slot0 = blockIdx.y * f.join_slots;
  if (units == 0 || slot0 >= end) return;
  const int at = f.item_at[blockIdx.x], ctas = (end + f.join_slots - 1) / f.join_slots, rows = q.m * a.rep;
  const AfHead head = *f.head;
  const uint32_t* anc = a.b.parent ? a.anc + static_cast<long long>(q.t0) * AC_TREE_WORDS : nullptr;
  auto row_at = [&](int x) { return static_cast<long long>(q.t0 + x / a.rep) * a.n_heads + h * a.rep + x % a.rep; };
  const int ra = af_run_of(head, at), n = af_run_of(head, at + units - 1) - ra + 1;
  // The first slots' scores are on their way before the statistics are known.
  const int slot1 = min(end, slot0 + f.join_slots), slot_mask = (1 << a.c.page_shift) - 1;
  const int* pages = a.c.page_table + static_cast<long long>(s) * a.c.max_pages;
  long long row[4];  // pool row of each of this thread's slots; -1: none
  float4 sc[4][SR / 4];
  float old[4];
  auto fetch = [&](int base) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int slot = base + AJ_THREADS * i;
      row[i] = slot < slot1 ? pages[slot >> a.c.page_shift] : -1;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (row[i] < 0 || row[i] >= a.c.n_pages) {  // a bad page was reported by the kernel that read the keys
        row[i] = -1;
        continue;
      }
      row[i] = kv_row(a.c, 0, static_cast<int>(row[i]), h) + ((base + AJ_THREADS * i) & slot_mask);
      old[i] = a.c.mass[row[i]];
#pragma unroll
      for (int x = 0; x < SR / 4; ++x) sc[i][x] = reinterpret_cast<const float4*>(f.scores + row[i] * SR)[x];
    }
  };
  if (f.scores) fetch(slot0 + threadIdx.x);
  if (n == 1) {
    if (threadIdx.x < AF_ROWS) lse_s[threadIdx.x] = threadIdx.x < rows ? a.lse[row_at(threadIdx.x)] : INFINITY;
    __syncthreads();
  } else {
    auto part = [&](int k) { return static_cast<long long>(2 * (ra + k) + (k == 0 ? 1 : 0)) * f.rows_cap; };
    for (int x = warp; x < AF_ROWS; x += AJ_WARPS) {
      float m = -INFINITY, l = 0.0f;
      if (x < rows) {
        for (int kb = lane; kb - lane < n; kb += 32 * 8) {
          float2 ml[8];
          float top = -INFINITY, sum = 0.0f;
#pragma unroll
          for (int j = 0; j < 8; ++j) ml[j] = kb + 32 * j < n ? a.part_ml[part(kb + 32 * j) + x] : make_float2(-INFINITY, 0.0f);
#pragma unroll
          for (int j = 0; j < 8; ++j) top = fmaxf(top, ml[j].x);
          top = fmaxf(warp_max(top), m);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (ml[j].x != -INFINITY) sum = fmaf(ml[j].y, ac_exp2(ml[j].x - top), sum);
          l = fmaf(l, m == -INFINITY ? 0.0f : ac_exp2(m - top), warp_sum(sum));
          m = top;
        }
      }
      if (lane == 0) {
        const bool none = x >= rows || l == 0.0f || ac_is_pad(anc, x / a.rep);
        lse_s[x] = none ? INFINITY : m + __log2f(l);
        max_s[x] = m;
        inv_s[x] = none ? 0.0f : __fdiv_rn(1.0f, l);
      }
    }
    __syncthreads();
    if (n <= 16) {
      for (int i = blockIdx.y * AJ_THREADS + threadIdx.x; i < rows * (HD / 2); i += ctas * AJ_THREADS) {
        const int x = i / (HD / 2), d = 2 * (i - x * (HD / 2));
        const float m = max_s[x];
        float2 acc = make_float2(0.0f, 0.0f);
#pragma unroll 4
        for (int k = 0; k < n; ++k) {
          const float2 v = *reinterpret_cast<const float2*>(a.part_o + (part(k) + x) * HD + d);
          const float mk = a.part_ml[part(k) + x].x;
          const float w = mk == -INFINITY ? 0.0f : ac_exp2(mk - m);
          acc.x = fmaf(mk == -INFINITY ? 0.0f : v.x, w, acc.x);
          acc.y = fmaf(mk == -INFINITY ? 0.0f : v.y, w, acc.y);
        }
        const bool none = lse_s[x] == INFINITY;
        *reinterpret_cast<uint32_t*>(a.att + row_at(x) * HD + d) =
            none ? 0u : pack_bf16x2(__fmul_rn(acc.x, inv_s[x]), __fmul_rn(acc.y, inv_s[x]));
      }
    } else {
      const int k0 = lane >> 3, d = lane & 7;
      for (int i = blockIdx.y * AJ_WARPS + warp; i < rows * (HD / 8); i += ctas * AJ_WARPS) {
        const int x = i / (HD / 8), dim = (i - x * (HD / 8)) * 8 + d;
        const float m = max_s[x];
        float acc = 0.0f;
        for (int kb = k0; kb < n; kb += 64) {
          float v[16], mk[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int k = kb + 4 * j;
            v[j] = k < n ? a.part_o[(part(k) + x) * HD + dim] : 0.0f;
            mk[j] = k < n ? a.part_ml[part(k) + x].x : -INFINITY;
          }
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (mk[j] != -INFINITY) acc = fmaf(v[j], ac_exp2(mk[j] - m), acc);
        }
        acc += __shfl_xor_sync(0xffffffffu, acc, 8);
        acc += __shfl_xor_sync(0xffffffffu, acc, 16);
        const float v = lse_s[x] == INFINITY ? 0.0f : __fmul_rn(acc, inv_s[x]);
        const float w = __shfl_down_sync(0xffffffffu, v, 1);
        if (k0 == 0 && (d & 1) == 0) *reinterpret_cast<uint32_t*>(a.att + row_at(x) * HD + dim) = pack_bf16x2(v, w);
      }
    }
  }
  if (!f.scores) return;
  float lse[SR];
#pragma unroll
  for (int x = 0; x < SR; ++x) lse[x] = lse_s[x];
  for (int base = slot0 + threadIdx.x;;) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (row[i] < 0) continue;
      float got = 0.0f;
#pragma unroll
      for (int x = 0; x < SR / 4; ++x) {
        const float v[4] = {sc[i][x].x, sc[i][x].y, sc[i][x].z, sc[i][x].w};
#pragma unroll
        for (int e = 0; e < 4; ++e)  // -inf: not seen by the row, whatever the row's sum is (it can be NaN)
          got += lse[4 * x + e] == INFINITY || v[e] == -INFINITY ? 0.0f : ac_exp2(v[e] - lse[4 * x + e]);
      }
      a.c.mass[row[i]] = old[i] + got;
    }
    base += 4 * AJ_THREADS;
    if (base >= slot1) break;
    fetch(base);
  }
}

}  // namespace bitrl

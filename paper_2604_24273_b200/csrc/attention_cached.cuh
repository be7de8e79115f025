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
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// (x0, x1) -> bf16 pair (x0 in the low half)
__device__ __forceinline__ uint32_t pack_bf16x2(float x0, float x1) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(x0, x1);
  return *reinterpret_cast<const uint32_t*>(&p);
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
// attn_few_join_kernel, which also turns the scores that this kernel leaves behind (fp32, 4 to 64 bytes per slot beside
// the 4 HD bytes of its key and value) into the weight of every slot, so that keys are read once.
// Scores come from mma.sync (a 16-row tile fills its M; a tcgen05 tile has 128 rows).  The weights are split into two bf16
// halves (16 significant bits), which costs nothing where reading bounds the kernel.
constexpr int AF_WARPS = 8;
constexpr int AF_THREADS = 32 * AF_WARPS;
constexpr int AF_STAGES = 3;
constexpr int AF_ROWS = 16;
constexpr int AF_SLOTS = 16;   // slots of a unit
constexpr int AF_MIN_RUN = 4;  // units of a run at least (short lists use fewer warps)
enum { AF_WAIT_LOAD = 151 };

struct AfRun {
  int s, h, u, left;  // first unit (unit u of item (s, h)) and number of units
};
struct AfHead {
  int units, runs;  // of the whole list; runs in use
  int per, more;    // units of a run; the first `more` runs have one more
};

struct AfArgs {
  AcArgs a;
  int rows_cap;    // rows of a sequence and head at most: max_new * rep
  int score_rows;  // rows_cap rounded up to 4, 8 or 16
  int max_runs;
  float* scores;   // [pages][kv heads][page][score_rows] or nullptr: scores in base-two units, -inf where unseen
  AfHead* head;
  AfRun* run;      // [max_runs]
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

template <int HD>
__global__ void __launch_bounds__(AF_THREADS, 1)
attn_few_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ AfArgs f) {
  constexpr int KS = HD / 16, ND = HD / 8, NH = HD / 64;
  constexpr uint32_t HALF = AF_SLOTS * 128, TILE = NH * HALF;  // a 64-dimension block of the keys (or values) of a unit
  extern __shared__ unsigned char af_smem_raw[];
  __shared__ __align__(8) unsigned long long bars[AF_WARPS * AF_STAGES];
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
  if (r >= head.runs) {
    if (lane == 0) f.run[r].left = 0;
    return;
  }
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
  if (lane == 0) f.run[r] = AfRun{s, h, u0, left};

  // ---- loads, ahead of the arithmetic: a position of their own in the list
  const uint32_t raw = ptx::smem_u32(af_smem_raw), ring = ((raw + 1023u) & ~1023u) + warp * (AF_STAGES * 2 * TILE);
  const int slot_mask = (1 << a.c.page_shift) - 1;
  int ls = s, lh = h, lu = u0, l_left = left;
  KvSeq lq = q;
  int l_units = af_units(a, ls, lq);
  auto load = [&](int stage) {
    if (l_left <= 0) return;
    if (lane == 0) {
      const int slot0 = lu * AF_SLOTS;
      const int page = kv_page(a.c, ls, slot0);
      // a page that the table does not have: a row behind the pool, which fills with zeros
      const int row = page < 0 ? a.c.n_pages * a.c.n_kv << a.c.page_shift
                               : static_cast<int>(((page * a.c.n_kv + lh) << a.c.page_shift) + (slot0 & slot_mask));
      const uint32_t dst = ring + stage * 2 * TILE;
      ptx::mbar_arrive_expect_tx(bar + 8 * stage, 2 * TILE);
#pragma unroll
      for (int i = 0; i < NH; ++i) {
        ptx::tma_load_2d(dst + i * HALF, &tmap_k, 64 * i, row, bar + 8 * stage);
        ptx::tma_load_2d(dst + TILE + i * HALF, &tmap_v, 64 * i, row, bar + 8 * stage);
      }
    }
    --l_left;
    if (++lu == l_units && l_left > 0) {
      lu = 0;
      if (++lh == a.c.n_kv) {
        lh = 0;
        do l_units = af_units(a, ++ls, lq);
        while (l_units == 0 && ls + 1 < a.c.n_seq);
      }
    }
  };
  for (int i = 0; i < AF_STAGES; ++i) load(i);
  uint32_t stage = 0, phase = 0;
  bool ok = true;

  while (ok && left > 0) {
    const int units = af_units(a, s, q);
    const int u1 = min(units, u0 + left), end = q.used + q.m, rows = q.m * a.rep;
    const uint32_t* anc = a.b.parent ? a.anc + static_cast<long long>(q.t0) * AC_TREE_WORDS : nullptr;
    // queries of rows g and g + 8
    uint32_t qa[KS][4];
    int tok[2];
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      const int x = g + 8 * rr;
      const bool live = x < rows;
      tok[rr] = live ? x / a.rep : 0;
      const unsigned short* row =
          a.q + (static_cast<long long>(q.t0 + tok[rr]) * a.n_heads + h * a.rep + (live ? x - tok[rr] * a.rep : 0)) * HD + 2 * t;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qa[ks][rr] = live ? *reinterpret_cast<const uint32_t*>(row + 16 * ks) : 0u;
        qa[ks][2 + rr] = live ? *reinterpret_cast<const uint32_t*>(row + 16 * ks + 8) : 0u;
      }
    }
    float o[ND][4];
#pragma unroll
    for (int nd = 0; nd < ND; ++nd)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[nd][e] = 0.0f;
    float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.0f, 0.0f};

    for (int u = u0; u < u1; ++u) {
      const int slot0 = u * AF_SLOTS;
      if (!__any_sync(0xffffffffu, ptx::mbar_wait(bar + 8 * stage, phase))) {
        ok = false;
        break;
      }
      const uint32_t ks_addr = ring + stage * 2 * TILE, vs_addr = ks_addr + TILE;
      float c[2][4];
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) c[nt][e] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int key = 8 * (lm >> 1) + lr, ch = 2 * ks + (lm & 1);
        uint32_t kb[4];
        ldmatrix_x4(ks_addr + (ch >> 3) * HALF + key * 128 + (((ch ^ key) & 7) << 4), kb);
        mma_bf16(c[0], qa[ks], kb[0], kb[1]);
        mma_bf16(c[1], qa[ks], kb[2], kb[3]);
      }
      // ---- scale, mask; slots below used are seen by every row
      const bool masked = slot0 + AF_SLOTS > q.used;
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = __fmul_rn(c[nt][e], a.scale2);
          if (masked) {
            const int slot = slot0 + 8 * nt + 2 * t + (e & 1);
            const bool see = slot < end && (slot < q.used || ac_sees_new(anc, tok[e >> 1], slot - q.used));
            v = see ? v : -INFINITY;
          }
          c[nt][e] = v;
          mx[e >> 1] = fmaxf(mx[e >> 1], v);
        }
      if (f.scores) {
        const int page = kv_page(a.c, s, slot0);
        if (page >= 0) {
          float* at = f.scores + ((kv_row(a.c, 0, page, h) + (slot0 & slot_mask)) + 2 * t) * f.score_rows;
#pragma unroll
          for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int x = g + 8 * (e >> 1);
              if (x < f.score_rows) at[(8 * nt + (e & 1)) * f.score_rows + x] = c[nt][e];
            }
        }
      }
      float alpha[2];
#pragma unroll
      for (int rr = 0; rr < 2; ++rr) {
        mx[rr] = fmaxf(mx[rr], __shfl_xor_sync(0xffffffffu, mx[rr], 1));
        mx[rr] = fmaxf(mx[rr], __shfl_xor_sync(0xffffffffu, mx[rr], 2));
        const float m_new = fmaxf(m_run[rr], mx[rr]);
        alpha[rr] = m_new == m_run[rr] ? 1.0f : ac_exp2(m_run[rr] - m_new);
        m_run[rr] = m_new;
      }
      float add[2] = {0.0f, 0.0f};
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          c[nt][e] = c[nt][e] == -INFINITY ? 0.0f : ac_exp2(c[nt][e] - m_run[e >> 1]);
          add[e >> 1] += c[nt][e];
        }
      l_run[0] = fmaf(l_run[0], alpha[0], add[0]);
      l_run[1] = fmaf(l_run[1], alpha[1], add[1]);
      if (__any_sync(0xffffffffu, alpha[0] != 1.0f || alpha[1] != 1.0f)) {
#pragma unroll
        for (int nd = 0; nd < ND; ++nd) {
          o[nd][0] = __fmul_rn(o[nd][0], alpha[0]);
          o[nd][1] = __fmul_rn(o[nd][1], alpha[0]);
          o[nd][2] = __fmul_rn(o[nd][2], alpha[1]);
          o[nd][3] = __fmul_rn(o[nd][3], alpha[1]);
        }
      }
      // A value that is not finite in a slot that some row does not see (or behind the last slot) must not reach that row
      // as 0 * inf: such a unit goes through scalar sums over the seen slots.
      bool odd = false;
      if (masked) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(TILE / 512); ++i) {
          const uint4 x = ptx::lds128(vs_addr + (lane + 32 * i) * 16);
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) odd |= (w[j] & 0x7f80u) == 0x7f80u || (w[j] & 0x7f800000u) == 0x7f800000u;
        }
        odd = __any_sync(0xffffffffu, odd);
      }
      if (!odd) {
        uint32_t ph[4], pl[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p0 = c[i >> 1][2 * (i & 1)], p1 = c[i >> 1][2 * (i & 1) + 1];
          ph[i] = pack_bf16x2(p0, p1);
          pl[i] = pack_bf16x2(p0 - __uint_as_float(ph[i] << 16), p1 - __uint_as_float(ph[i] & 0xffff0000u));
        }
#pragma unroll
        for (int nd = 0; nd < ND; nd += 2) {
          const int key = 8 * (lm & 1) + lr, ch = nd + (lm >> 1);
          uint32_t vb[4];
          ldmatrix_x4_trans(vs_addr + (ch >> 3) * HALF + key * 128 + (((ch ^ key) & 7) << 4), vb);
          mma_bf16(o[nd], ph, vb[0], vb[1]);
          mma_bf16(o[nd + 1], ph, vb[2], vb[3]);
          mma_bf16(o[nd], pl, vb[0], vb[1]);
          mma_bf16(o[nd + 1], pl, vb[2], vb[3]);
        }
      } else {
        for (int key = 0; key < AF_SLOTS; ++key) {
          const int from = (lane & ~3) | ((key & 7) >> 1);  // the lane of this row group that holds the key's weight
          float p[2];
          bool see[2];
          const int slot = slot0 + key;
#pragma unroll
          for (int rr = 0; rr < 2; ++rr) {
            const float w00 = __shfl_sync(0xffffffffu, c[0][2 * rr], from), w01 = __shfl_sync(0xffffffffu, c[0][2 * rr + 1], from);
            const float w10 = __shfl_sync(0xffffffffu, c[1][2 * rr], from), w11 = __shfl_sync(0xffffffffu, c[1][2 * rr + 1], from);
            p[rr] = key < 8 ? ((key & 1) ? w01 : w00) : ((key & 1) ? w11 : w10);
            see[rr] = slot < end && (slot < q.used || ac_sees_new(anc, tok[rr], slot - q.used));
          }
#pragma unroll
          for (int nd = 0; nd < ND; ++nd) {
            const uint32_t w = ptx::lds32(vs_addr + (nd >> 3) * HALF + key * 128 + (((nd ^ key) & 7) << 4) + 4 * t);
            const float v0 = __uint_as_float(w << 16), v1 = __uint_as_float(w & 0xffff0000u);
            if (see[0]) { o[nd][0] = fmaf(p[0], v0, o[nd][0]); o[nd][1] = fmaf(p[0], v1, o[nd][1]); }
            if (see[1]) { o[nd][2] = fmaf(p[1], v0, o[nd][2]); o[nd][3] = fmaf(p[1], v1, o[nd][3]); }
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
    for (int rr = 0; rr < 2; ++rr) {
      l_run[rr] += __shfl_xor_sync(0xffffffffu, l_run[rr], 1);
      l_run[rr] += __shfl_xor_sync(0xffffffffu, l_run[rr], 2);
      const int x = g + 8 * rr;
      if (x >= rows) continue;
      if (whole) {
        const bool none = l_run[rr] == 0.0f || ac_is_pad(anc, tok[rr]);
        const float inv = none ? 0.0f : __fdiv_rn(1.0f, l_run[rr]);
        const long long row = static_cast<long long>(q.t0 + tok[rr]) * a.n_heads + h * a.rep + x - tok[rr] * a.rep;
#pragma unroll
        for (int nd = 0; nd < ND; ++nd)
          *reinterpret_cast<uint32_t*>(a.att + row * HD + 8 * nd + 2 * t) =
              none ? 0u : pack_bf16x2(__fmul_rn(o[nd][2 * rr], inv), __fmul_rn(o[nd][2 * rr + 1], inv));
        if (t == 0) a.lse[row] = none ? INFINITY : m_run[rr] + __log2f(l_run[rr]);
      } else {
        float* to = a.part_o + (static_cast<long long>(cut) * f.rows_cap + x) * HD;
#pragma unroll
        for (int nd = 0; nd < ND; ++nd) *reinterpret_cast<float2*>(to + 8 * nd + 2 * t) = make_float2(o[nd][2 * rr], o[nd][2 * rr + 1]);
        if (t == 0) a.part_ml[static_cast<long long>(cut) * f.rows_cap + x] = make_float2(m_run[rr], l_run[rr]);
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

// The runs again, without the keys: joins the items that were cut (in run order) and adds every slot's weights, p = 2^(score
// - lse), to mass.  The AJ_SPLIT warps of a run take its slots in turn, and of the results of a cut item each joins its share,
// 8 dimensions of a row at a time.  Everything here is short chains of loads, so several are kept in flight: four rows of
// statistics, four parts of a result, four slots per lane.
constexpr int AJ_SPLIT = 4;

// (maximum, sum) of two disjoint sets of keys.
__device__ __forceinline__ float2 aj_merge(float2 x, float2 y) {
  const float m = fmaxf(x.x, y.x);
  const float lx = x.x == -INFINITY ? 0.0f : __fmul_rn(x.y, ac_exp2(x.x - m)), ly = y.x == -INFINITY ? 0.0f : __fmul_rn(y.y, ac_exp2(y.x - m));
  return make_float2(m, lx + ly);
}

template <int HD, int SR>
__global__ void __launch_bounds__(AF_THREADS) attn_few_join_kernel(const __grid_constant__ AfArgs f) {
  pdl_enter();
  const AcArgs& a = f.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = blockIdx.y;
  __shared__ float lse_s[AF_WARPS][AF_ROWS], max_s[AF_WARPS][AF_ROWS], inv_s[AF_WARPS][AF_ROWS];
  const int r = warp * gridDim.x + blockIdx.x;
  const AfRun run = f.run[r];
  const AfHead head = *f.head;
  int left = run.left, s = run.s, h = run.h, u0 = run.u;
  int at = left > 0 ? af_start(head, r) : 0;  // place in the list
  const int slot_mask = (1 << a.c.page_shift) - 1;
  KvSeq q;
  while (left > 0) {
    const int units = af_units(a, s, q);
    const int u1 = min(units, u0 + left), end = q.used + q.m, rows = q.m * a.rep;
    const bool whole = u0 == 0 && u1 == units;
    const uint32_t* anc = a.b.parent ? a.anc + static_cast<long long>(q.t0) * AC_TREE_WORDS : nullptr;
    auto row_at = [&](int x) { return static_cast<long long>(q.t0 + x / a.rep) * a.n_heads + h * a.rep + x % a.rep; };
    if (whole) {
      if (lane < AF_ROWS) lse_s[warp][lane] = lane < rows ? a.lse[row_at(lane)] : INFINITY;
      __syncwarp();
    } else {
      const int ra = af_run_of(head, at - u0), rb = af_run_of(head, at - u0 + units - 1), n = rb - ra + 1, me = r - ra;
      auto part = [&](int k) { return static_cast<long long>(2 * (ra + k) + (k == 0 ? 1 : 0)) * f.rows_cap; };
      for (int x0 = 0; x0 < AF_ROWS; x0 += 4) {
        float2 ml[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) ml[i] = make_float2(-INFINITY, 0.0f);
        if (x0 < rows) {
          for (int k = lane; k < n; k += 32) {
            float2 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = x0 + i < rows ? a.part_ml[part(k) + x0 + i] : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i) ml[i] = aj_merge(ml[i], v[i]);
          }
#pragma unroll
          for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              ml[i] = aj_merge(ml[i], make_float2(__shfl_xor_sync(0xffffffffu, ml[i].x, o), __shfl_xor_sync(0xffffffffu, ml[i].y, o)));
        }
        if (lane < 4) {
          const float2 v = lane == 0 ? ml[0] : lane == 1 ? ml[1] : lane == 2 ? ml[2] : ml[3];
          const int x = x0 + lane;
          const bool none = x >= rows || v.y == 0.0f || ac_is_pad(anc, x / a.rep);
          lse_s[warp][x] = none ? INFINITY : v.x + __log2f(v.y);
          max_s[warp][x] = v.x;
          inv_s[warp][x] = none ? 0.0f : __fdiv_rn(1.0f, v.y);
        }
      }
      __syncwarp();
      // results: pieces of 8 dimensions, dealt to the warps of the item in turn; lanes: 4 parts side by side x 8 dimensions.
      // Eight loads of a lane are under way together: parts of one piece, or pieces where an item has few parts.
      const int k0 = lane >> 3, d = lane & 7, pieces = rows * (HD / 8), step = n * AJ_SPLIT;
      const int kn = n > 4 ? 8 : 1, pn = n > 4 ? 1 : 8;
      for (int i0 = me * AJ_SPLIT + sub; i0 < pieces; i0 += pn * step) {
        float acc[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = 0.0f;
        for (int kb = k0; kb < n; kb += 4 * kn) {
          float v[8], m[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int i = kn == 8 ? i0 : i0 + j * step, k = kn == 8 ? kb + 4 * j : kb, x = i / (HD / 8);
            const bool have = i < pieces && k < n;
            v[j] = have ? a.part_o[(part(k) + x) * HD + (i - x * (HD / 8)) * 8 + d] : 0.0f;
            m[j] = have ? a.part_ml[part(k) + x].x - max_s[warp][x] : -INFINITY;
          }
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (m[j] > -INFINITY || m[j] != m[j]) acc[j] = fmaf(v[j], ac_exp2(m[j]), acc[j]);
        }
        if (kn == 8) acc[0] = ((acc[0] + acc[1]) + (acc[2] + acc[3])) + ((acc[4] + acc[5]) + (acc[6] + acc[7]));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (j >= pn) break;
          acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], 8);
          acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], 16);
          const int i = i0 + j * step, x = i / (HD / 8);
          const bool none = i >= pieces || lse_s[warp][x & (AF_ROWS - 1)] == INFINITY;
          const float v = none ? 0.0f : __fmul_rn(acc[j], inv_s[warp][x]);
          const float w = __shfl_down_sync(0xffffffffu, v, 1);
          if (i < pieces && k0 == 0 && (d & 1) == 0)
            *reinterpret_cast<uint32_t*>(a.att + row_at(x) * HD + (i - x * (HD / 8)) * 8 + d) = pack_bf16x2(v, w);
        }
      }
    }
    if (f.scores) {
      float lse[SR];
#pragma unroll
      for (int x = 0; x < SR; ++x) lse[x] = lse_s[warp][x];
      const int slot1 = min(end, u1 * AF_SLOTS);
      const int* pages = a.c.page_table + static_cast<long long>(s) * a.c.max_pages;
      for (int base = u0 * AF_SLOTS + 128 * sub + lane; base < slot1; base += 128 * AJ_SPLIT) {
        int page[4];
        long long row[4];
        float4 sc[4][SR / 4];
        float old[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) page[i] = base + 32 * i < slot1 ? pages[(base + 32 * i) >> a.c.page_shift] : -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (page[i] >= a.c.n_pages) page[i] = -1;  // reported by the kernel that read the keys
          row[i] = page[i] < 0 ? 0 : kv_row(a.c, 0, page[i], h) + ((base + 32 * i) & slot_mask);
          if (page[i] >= 0) {
            old[i] = a.c.mass[row[i]];
#pragma unroll
            for (int x = 0; x < SR / 4; ++x) sc[i][x] = reinterpret_cast<const float4*>(f.scores + row[i] * SR)[x];
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (page[i] < 0) continue;
          float got = 0.0f;
#pragma unroll
          for (int x = 0; x < SR / 4; ++x) {
            const float v[4] = {sc[i][x].x, sc[i][x].y, sc[i][x].z, sc[i][x].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) got += lse[4 * x + e] == INFINITY ? 0.0f : ac_exp2(v[e] - lse[4 * x + e]);
          }
          a.c.mass[row[i]] = old[i] + got;
        }
      }
    }
    __syncwarp();
    left -= u1 - u0;
    at += u1 - u0;
    u0 = 0;
    if (left > 0 && ++h == a.c.n_kv) {
      h = 0;
      while (++s + 1 < a.c.n_seq && af_units(a, s, q) == 0) {}
    }
  }
}

}  // namespace bitrl

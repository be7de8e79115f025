// Attention of new tokens over a paged key/value cache (kv_cache.cuh), with the weight that every slot receives.
//
//   score(i, r) = q_i . k_r / sqrt(head_dim);  p = softmax over the slots r that token i sees;  att_i = sum_r p_r v_r
//   mass[r] += sum over the tokens i and the query heads of the kv head of p(i, r)
//
// The query heads of a kv head share its keys, so the rows of a sequence are the pairs (token, head of the group):
// row x = token * rep + j.  Everything works on logarithms to base two: t = score * log2(e), p = 2^(t - lse).
#pragma once

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
  int row_tiles;           // row tiles of the longest sequence
  int splits, split_keys;  // key ranges per row tile, slots per range (a multiple of 64)
  float* part_o;           // [splits][T * n_heads][HD] unnormalised partial results (splits > 1)
  float2* part_ml;         // [splits][T * n_heads]: running maximum and sum
  float* lse;              // [T * n_heads]: maximum + log2(sum); +inf where a row sees nothing
  const uint32_t* anc;     // trees: [T][AC_TREE_WORDS], the tokens that a token sees
  const uint32_t* desc;    // trees: [T][AC_TREE_WORDS], the tokens that see a token
  const int* tree_ok;      // trees: [n_seq], else nullptr
  AtCut* cuts;             // tiles: [CTAs][2]
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
// 16-byte asynchronous copy; bytes = 0 fills the destination with zeros and reads nothing.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
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

// First slot that no row of the tile of `rows` rows starting at row x0 sees.
__device__ __forceinline__ int ac_key_end(const KvSeq& q, int rep, bool tree, int x0, int rows) {
  return q.used + (tree ? q.m : min(q.m, (x0 + rows - 1) / rep + 1));
}

// ---- few rows: one 16-row tile per CTA -----------------------------------------------------------------------------
// Bound by the reading of keys and values.  The warps of a CTA share the rows and take different keys, 16 at a time, each
// through a ring of its own, so no barrier stands in the loop; every warp keeps its own running maximum, sum and 16 x HD
// result, and these are joined at the end.  Scores come from mma.sync (a 16-row tile fills its M; a tcgen05 tile has 128).
// The weights are split into two bf16 halves (16 significant bits), which costs nothing where reading bounds the kernel.
constexpr int AR_THREADS = 128;
constexpr int AR_WARPS = AR_THREADS / 32;
constexpr int AR_STAGES = 3;
constexpr int AR_ROWS = 16;
constexpr int AR_KEYS = 16;  // slots per step of a warp

template <int HD>
constexpr uint32_t ar_smem_bytes() {
  const uint32_t ring = AR_WARPS * AR_STAGES * 2 * AR_KEYS * HD * 2;
  const uint32_t join = AR_WARPS * AR_ROWS * (HD * 4 + 8);
  return ring > join ? ring : join;
}

template <int HD>
__global__ void __launch_bounds__(AR_THREADS) attn_rows_kernel(const __grid_constant__ AcArgs a) {
  constexpr int KS = HD / 16, ND = HD / 8, CH = HD / 8;
  constexpr uint32_t KV_BYTES = AR_KEYS * HD * 2;  // keys (or values) of one step
  extern __shared__ __align__(128) unsigned char ar_smem[];
  pdl_enter();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, lm = lane >> 3, lr = lane & 7;
  int idx = blockIdx.x;
  const int split = idx % a.splits;
  idx /= a.splits;
  const int rt = idx % a.row_tiles;
  idx /= a.row_tiles;
  const int head = idx % a.c.n_kv, s = idx / a.c.n_kv;
  KvSeq q;
  if (!kv_seq(a.c, a.b, s, q)) return;
  const int x0 = rt * AR_ROWS;
  if (x0 >= q.m * a.rep) return;
  const int end = ac_key_end(q, a.rep, a.b.parent != nullptr, x0, AR_ROWS);
  const int k0 = split * a.split_keys, k1 = min(end, k0 + a.split_keys);
  if (k0 >= end) return;
  if (a.tree_ok && !a.tree_ok[s]) return;
  const uint32_t* anc = a.b.parent ? a.anc + static_cast<long long>(q.t0) * AC_TREE_WORDS : nullptr;

  // ---- queries of rows g and g + 8 of the tile
  uint32_t qa[KS][4];
  int tok[2];
#pragma unroll
  for (int rr = 0; rr < 2; ++rr) {
    const int x = x0 + g + 8 * rr;
    const bool live = x < q.m * a.rep;
    tok[rr] = live ? x / a.rep : 0;
    const unsigned short* row =
        a.q + (static_cast<long long>(q.t0 + tok[rr]) * a.n_heads + head * a.rep + (live ? x - tok[rr] * a.rep : 0)) * HD + 2 * t;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qa[ks][rr] = live ? *reinterpret_cast<const uint32_t*>(row + 16 * ks) : 0u;
      qa[ks][2 + rr] = live ? *reinterpret_cast<const uint32_t*>(row + 16 * ks + 8) : 0u;
    }
  }

  const uint32_t ring = ptx::smem_u32(ar_smem) + warp * (AR_STAGES * 2 * KV_BYTES);
  const int slot_mask = (1 << a.c.page_shift) - 1;
  auto load = [&](int slot0, int stage) {  // slots [slot0, slot0 + 16) of one page
    const int page = kv_page(a.c, s, slot0);
    const long long row0 = kv_row(a.c, 0, page < 0 ? 0 : page, head) + (slot0 & slot_mask);
    const uint32_t dk = ring + stage * 2 * KV_BYTES;
#pragma unroll
    for (int u = 0; u < AR_KEYS * CH / 32; ++u) {
      const int i = lane + 32 * u, r = i / CH, ch = i % CH;
      const int slot = slot0 + r;
      const bool have = page >= 0 && slot < k1 && !(anc && slot >= q.used && ac_is_pad(anc, slot - q.used));
      const uint32_t off = r * (HD * 2) + ((ch ^ (r & 7)) << 4);
      const long long src = have ? (row0 + r) * HD + ch * 8 : 0;
      cp_async16(dk + off, a.c.k + src, have ? 16u : 0u);
      cp_async16(dk + KV_BYTES + off, a.c.v + src, have ? 16u : 0u);
    }
  };

  float o[ND][4];
#pragma unroll
  for (int nd = 0; nd < ND; ++nd)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[nd][e] = 0.0f;
  float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.0f, 0.0f};

  const int step = AR_WARPS * AR_KEYS;
  int slot0 = k0 + warp * AR_KEYS;
#pragma unroll
  for (int i = 0; i < AR_STAGES - 1; ++i) {
    if (slot0 + i * step < k1) load(slot0 + i * step, i);
    cp_async_commit();
  }
  int stage = 0;
  for (; slot0 < k1; slot0 += step) {
    cp_async_wait<AR_STAGES - 2>();
    __syncwarp();
    {
      const int ahead = slot0 + (AR_STAGES - 1) * step, st = stage == 0 ? AR_STAGES - 1 : stage - 1;
      if (ahead < k1) load(ahead, st);
      cp_async_commit();
    }
    const uint32_t ks_addr = ring + stage * 2 * KV_BYTES, vs_addr = ks_addr + KV_BYTES;
    float c[2][4];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) c[nt][e] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int key = 8 * (lm >> 1) + lr, ch = 2 * ks + (lm & 1);
      uint32_t kb[4];
      ldmatrix_x4(ks_addr + key * (HD * 2) + ((ch ^ (key & 7)) << 4), kb);
      mma_bf16(c[0], qa[ks], kb[0], kb[1]);
      mma_bf16(c[1], qa[ks], kb[2], kb[3]);
    }
    // ---- scale, mask; slots below used are seen by every row
    const bool masked = slot0 + AR_KEYS > q.used || slot0 + AR_KEYS > k1;
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float v = __fmul_rn(c[nt][e], a.scale2);
        if (masked) {
          const int slot = slot0 + 8 * nt + 2 * t + (e & 1);
          const bool see = slot < k1 && (slot < q.used || ac_sees_new(anc, tok[e >> 1], slot - q.used));
          v = see ? v : -INFINITY;
        }
        c[nt][e] = v;
        mx[e >> 1] = fmaxf(mx[e >> 1], v);
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
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float mm = m_run[e >> 1];
        c[nt][e] = c[nt][e] == -INFINITY ? 0.0f : ac_exp2(c[nt][e] - mm);
        sum[e >> 1] += c[nt][e];
      }
    l_run[0] = fmaf(l_run[0], alpha[0], sum[0]);
    l_run[1] = fmaf(l_run[1], alpha[1], sum[1]);
    if (__any_sync(0xffffffffu, alpha[0] != 1.0f || alpha[1] != 1.0f)) {
#pragma unroll
      for (int nd = 0; nd < ND; ++nd) {
        o[nd][0] = __fmul_rn(o[nd][0], alpha[0]);
        o[nd][1] = __fmul_rn(o[nd][1], alpha[0]);
        o[nd][2] = __fmul_rn(o[nd][2], alpha[1]);
        o[nd][3] = __fmul_rn(o[nd][3], alpha[1]);
      }
    }
    // A value that is not finite in a slot that some row does not see must not reach that row as 0 * inf: such a step
    // (new tokens only) goes through scalar sums over the seen slots.
    bool odd = false;
    if (masked) {
#pragma unroll
      for (int u = 0; u < AR_KEYS * CH / 32; ++u) {
        const uint4 x = ptx::lds128(vs_addr + (lane + 32 * u) * 16);
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
        ldmatrix_x4_trans(vs_addr + key * (HD * 2) + ((ch ^ (key & 7)) << 4), vb);
        mma_bf16(o[nd], ph, vb[0], vb[1]);
        mma_bf16(o[nd + 1], ph, vb[2], vb[3]);
        mma_bf16(o[nd], pl, vb[0], vb[1]);
        mma_bf16(o[nd + 1], pl, vb[2], vb[3]);
      }
    } else {
      for (int key = 0; key < AR_KEYS; ++key) {
        const int from = (lane & ~3) | ((key & 7) >> 1);  // the lane of this row group that holds the key's weight
        float p[2];
#pragma unroll
        for (int rr = 0; rr < 2; ++rr) {
          const float w00 = __shfl_sync(0xffffffffu, c[0][2 * rr], from), w01 = __shfl_sync(0xffffffffu, c[0][2 * rr + 1], from);
          const float w10 = __shfl_sync(0xffffffffu, c[1][2 * rr], from), w11 = __shfl_sync(0xffffffffu, c[1][2 * rr + 1], from);
          p[rr] = key < 8 ? ((key & 1) ? w01 : w00) : ((key & 1) ? w11 : w10);
        }
        const int slot = slot0 + key;
        bool see[2];
#pragma unroll
        for (int rr = 0; rr < 2; ++rr) see[rr] = slot < k1 && (slot < q.used || ac_sees_new(anc, tok[rr], slot - q.used));
#pragma unroll
        for (int nd = 0; nd < ND; ++nd) {
          const uint32_t w = ptx::lds32(vs_addr + key * (HD * 2) + ((nd ^ (key & 7)) << 4) + 4 * t);
          const float v0 = __uint_as_float(w << 16), v1 = __uint_as_float(w & 0xffff0000u);
          if (see[0]) { o[nd][0] = fmaf(p[0], v0, o[nd][0]); o[nd][1] = fmaf(p[0], v1, o[nd][1]); }
          if (see[1]) { o[nd][2] = fmaf(p[1], v0, o[nd][2]); o[nd][3] = fmaf(p[1], v1, o[nd][3]); }
        }
      }
    }
    __syncwarp();
    stage = stage == AR_STAGES - 1 ? 0 : stage + 1;
  }
  cp_async_wait<0>();

  // ---- join the warps
  __syncthreads();
  float* jo = reinterpret_cast<float*>(ar_smem);                                  // [warp][row][HD]
  float2* jml = reinterpret_cast<float2*>(jo + AR_WARPS * AR_ROWS * HD);          // [warp][row]
#pragma unroll
  for (int rr = 0; rr < 2; ++rr) {
    l_run[rr] += __shfl_xor_sync(0xffffffffu, l_run[rr], 1);
    l_run[rr] += __shfl_xor_sync(0xffffffffu, l_run[rr], 2);
    const int r = warp * AR_ROWS + g + 8 * rr;
    if (t == 0) jml[r] = make_float2(m_run[rr], l_run[rr]);
#pragma unroll
    for (int nd = 0; nd < ND; ++nd)
      *reinterpret_cast<float2*>(jo + r * HD + 8 * nd + 2 * t) = make_float2(o[nd][2 * rr], o[nd][2 * rr + 1]);
  }
  __syncthreads();
  constexpr int PER = AR_ROWS * HD / AR_THREADS;  // consecutive dimensions of one row per thread
  const int r = threadIdx.x / (HD / PER), d0 = (threadIdx.x % (HD / PER)) * PER;
  const int x = x0 + r;
  if (x >= q.m * a.rep) return;
  float m_all = -INFINITY, l_all = 0.0f, acc[PER];
#pragma unroll
  for (int w = 0; w < AR_WARPS; ++w) m_all = fmaxf(m_all, jml[w * AR_ROWS + r].x);
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.0f;
#pragma unroll
  for (int w = 0; w < AR_WARPS; ++w) {
    const float2 ml = jml[w * AR_ROWS + r];
    const float f = ml.x == -INFINITY ? 0.0f : ac_exp2(ml.x - m_all);
    if (ml.x == -INFINITY) continue;
    l_all = fmaf(ml.y, f, l_all);
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] = fmaf(jo[(w * AR_ROWS + r) * HD + d0 + i], f, acc[i]);
  }
  const int tk = x / a.rep;
  const long long row = static_cast<long long>(q.t0 + tk) * a.n_heads + head * a.rep + (x - tk * a.rep);
  if (a.splits > 1) {
    const long long at = static_cast<long long>(split) * a.b.T * a.n_heads + row;
#pragma unroll
    for (int i = 0; i < PER; i += 4)
      *reinterpret_cast<float4*>(a.part_o + at * HD + d0 + i) = make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
    if (d0 == 0) a.part_ml[at] = make_float2(m_all, l_all);
    return;
  }
  const bool none = l_all == 0.0f || ac_is_pad(anc, tk);
  const float inv = none ? 0.0f : __fdiv_rn(1.0f, l_all);
#pragma unroll
  for (int i = 0; i < PER; i += 2)
    *reinterpret_cast<uint32_t*>(a.att + row * HD + d0 + i) = none ? 0u : pack_bf16x2(__fmul_rn(acc[i], inv), __fmul_rn(acc[i + 1], inv));
  if (d0 == 0) a.lse[row] = none ? INFINITY : m_all + __log2f(l_all);
}

// Joins the key ranges of every row; one warp per row, ranges in ascending order.
template <int HD>
__global__ void __launch_bounds__(128) attn_join_kernel(const __grid_constant__ AcArgs a) {
  pdl_enter();
  const int lane = threadIdx.x & 31;
  // rows of a sequence: blockIdx = sequence * blocks per sequence + block, four rows each
  const int per_seq = (a.b.max_new * a.n_heads + 3) / 4;
  const int s = blockIdx.x / per_seq, i = (blockIdx.x - s * per_seq) * 4 + (threadIdx.x >> 5);
  KvSeq q;
  if (!kv_seq(a.c, a.b, s, q)) return;
  const int tok = i / a.n_heads, h = i - tok * a.n_heads;
  if (tok >= q.m) return;
  bool pad = false;
  if (a.b.parent) pad = a.b.parent[q.t0 + tok] == BITRL_PARENT_PAD;
  const int x = tok * a.rep + h % a.rep;
  const int end = ac_key_end(q, a.rep, a.b.parent != nullptr, x / AR_ROWS * AR_ROWS, AR_ROWS);
  const int n = (end + a.split_keys - 1) / a.split_keys;
  const long long row = static_cast<long long>(q.t0) * a.n_heads + i, stride = static_cast<long long>(a.b.T) * a.n_heads;
  float m_all = -INFINITY;
  for (int k = lane; k < n; k += 32) m_all = fmaxf(m_all, a.part_ml[k * stride + row].x);
  m_all = warp_max(m_all);
  constexpr int PER = HD / 32;
  float l_all = 0.0f, acc[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) acc[e] = 0.0f;
  for (int k = 0; k < n; ++k) {
    const float2 ml = a.part_ml[k * stride + row];
    if (ml.x == -INFINITY) continue;
    const float f = ac_exp2(ml.x - m_all);
    l_all = fmaf(ml.y, f, l_all);
    const float* po = a.part_o + (k * stride + row) * HD + lane * PER;
#pragma unroll
    for (int e = 0; e < PER; ++e) acc[e] = fmaf(po[e], f, acc[e]);
  }
  const bool none = pad || l_all == 0.0f;
  const float inv = none ? 0.0f : __fdiv_rn(1.0f, l_all);
#pragma unroll
  for (int e = 0; e < PER; e += 2)
    *reinterpret_cast<uint32_t*>(a.att + row * HD + lane * PER + e) = none ? 0u : pack_bf16x2(__fmul_rn(acc[e], inv), __fmul_rn(acc[e + 1], inv));
  if (lane == 0) a.lse[row] = none ? INFINITY : m_all + __log2f(l_all);
}

// ---- weight received by every slot ---------------------------------------------------------------------------------
// A second pass over the keys: with the final maximum and sum of every row known, a CTA owns 64 slots of one kv head, forms
// their scores with all rows of the sequence and adds up each slot's weights in registers; a slot belongs to one CTA, so
// nothing is added atomically.
constexpr int AS_THREADS = 128;
constexpr int AS_KEYS = 64;
constexpr int AS_ROWS = 64;  // rows per step

template <int HD>
constexpr uint32_t as_smem_bytes() {
  return AS_KEYS * HD * 2 + 2 * AS_ROWS * (HD * 2 + 4);
}

template <int HD>
__global__ void __launch_bounds__(AS_THREADS) attn_mass_few_kernel(const __grid_constant__ AcArgs a) {
  constexpr int KS = HD / 16, CH = HD / 8;
  constexpr uint32_t K_BYTES = AS_KEYS * HD * 2, Q_BYTES = AS_ROWS * HD * 2;
  extern __shared__ __align__(128) unsigned char am_smem[];
  pdl_enter();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, lm = lane >> 3, lr = lane & 7;
  const int tiles = (((a.c.max_pages << a.c.page_shift) + AS_KEYS - 1) / AS_KEYS);
  int idx = blockIdx.x;
  const int kt = idx % tiles;
  idx /= tiles;
  const int head = idx % a.c.n_kv, s = idx / a.c.n_kv;
  KvSeq q;
  if (!kv_seq(a.c, a.b, s, q)) return;
  const int slot0 = kt * AS_KEYS, end = q.used + q.m;
  if (slot0 >= end || q.m == 0) return;
  float* lse_s = reinterpret_cast<float*>(am_smem + K_BYTES + 2 * Q_BYTES);  // [2][AS_ROWS]
  if (a.tree_ok && !a.tree_ok[s]) return;
  const uint32_t* anc = a.b.parent ? a.anc + static_cast<long long>(q.t0) * AC_TREE_WORDS : nullptr;
  const uint32_t k_addr = ptx::smem_u32(am_smem), q_addr = k_addr + K_BYTES;
  const int slot_mask = (1 << a.c.page_shift) - 1;
  for (int i = threadIdx.x; i < AS_KEYS * CH; i += AS_THREADS) {
    const int r = i / CH, ch = i % CH, slot = slot0 + r;
    int page = -1;
    if (slot < end) page = kv_page(a.c, s, slot);
    const long long src = page < 0 ? 0 : (kv_row(a.c, 0, page, head) + (slot & slot_mask)) * HD + ch * 8;
    cp_async16(k_addr + r * (HD * 2) + ((ch ^ (r & 7)) << 4), a.c.k + src, page < 0 ? 0u : 16u);
  }
  const int rows = q.m * a.rep;
  // rows below the first that can see this tile's slots
  const int first = (!anc && slot0 > q.used ? min(q.m, slot0 - q.used) * a.rep : 0) / AS_ROWS * AS_ROWS;
  auto load_q = [&](int x0, int buf) {
    for (int i = threadIdx.x; i < AS_ROWS * CH; i += AS_THREADS) {
      const int r = i / CH, ch = i % CH, x = x0 + r;
      const int tk = x / a.rep;
      const long long row = static_cast<long long>(q.t0 + tk) * a.n_heads + head * a.rep + (x - tk * a.rep);
      cp_async16(q_addr + buf * Q_BYTES + r * (HD * 2) + ((ch ^ (r & 7)) << 4), a.q + (x < rows ? row * HD + ch * 8 : 0),
                 x < rows ? 16u : 0u);
    }
    if (threadIdx.x < AS_ROWS) {
      const int x = x0 + threadIdx.x, tk = x / a.rep;
      lse_s[buf * AS_ROWS + threadIdx.x] =
          x < rows ? a.lse[static_cast<long long>(q.t0 + tk) * a.n_heads + head * a.rep + (x - tk * a.rep)] : INFINITY;
    }
  };
  load_q(first, 0);
  cp_async_commit();
  uint32_t ka[KS][4];
  float got[2] = {0.0f, 0.0f};  // slots g and g + 8 of the warp's 16
  const int key_lo = slot0 + warp * 16 + g;
  const bool masked = slot0 + AS_KEYS > q.used;
  int buf = 0;
  for (int x0 = first; x0 < rows; x0 += AS_ROWS, buf ^= 1) {
    cp_async_wait<0>();
    __syncthreads();
    if (x0 + AS_ROWS < rows) load_q(x0 + AS_ROWS, buf ^ 1);
    cp_async_commit();
    if (x0 == first) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int key = warp * 16 + 8 * (lm & 1) + lr, ch = 2 * ks + (lm >> 1);
        ldmatrix_x4(k_addr + key * (HD * 2) + ((ch ^ (key & 7)) << 4), ka[ks]);
      }
    }
    for (int n0 = 0; n0 < AS_ROWS; n0 += 16) {
      if (x0 + n0 >= rows) break;
      float c[2][4];
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) c[nt][e] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int r = n0 + 8 * (lm >> 1) + lr, ch = 2 * ks + (lm & 1);
        uint32_t qb[4];
        ldmatrix_x4(q_addr + buf * Q_BYTES + r * (HD * 2) + ((ch ^ (r & 7)) << 4), qb);
        mma_bf16(c[0], ka[ks], qb[0], qb[1]);
        mma_bf16(c[1], ka[ks], qb[2], qb[3]);
      }
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = n0 + 8 * nt + 2 * t + (e & 1), x = x0 + r;
          const float lse = lse_s[buf * AS_ROWS + r];
          bool see = lse != INFINITY;
          if (masked) {
            const int slot = key_lo + 8 * (e >> 1);
            see = see && slot < end && (slot < q.used || ac_sees_new(anc, x / a.rep, slot - q.used));
          }
          if (see) got[e >> 1] += ac_exp2(fmaf(c[nt][e], a.scale2, -lse));
        }
    }
    __syncthreads();
  }
#pragma unroll
  for (int rr = 0; rr < 2; ++rr) {
    got[rr] += __shfl_xor_sync(0xffffffffu, got[rr], 1);
    got[rr] += __shfl_xor_sync(0xffffffffu, got[rr], 2);
    const int slot = key_lo + 8 * rr;
    if (t == 0 && slot < end) {
      const int page = kv_page(a.c, s, slot);
      if (page >= 0) {
        float* w = a.c.mass + kv_row(a.c, 0, page, head) + (slot & slot_mask);
        *w += got[rr];
      }
    }
  }
}

}  // namespace bitrl

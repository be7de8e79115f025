// Attention over the cache for more than 16 rows per sequence and kv head: tcgen05 tiles of 128 rows.
#pragma once

#include <cuda.h>

#include "attention_cached.cuh"
#include "gemm.cuh"
#include "ptx.cuh"

namespace bitrl {

// ---- work lists ------------------------------------------------------------------------------------------------------
// Lengths are known on the device alone, so the kernels cut their work there: pairs (sequence s, index x < nx), each
// holding n_kv items (kv heads) of cost(s, x) units, form one list, and CTA c of G takes its share [N c / G, N (c+1) / G) of it.
// Every CTA then has the same share whatever the lengths are; an item may be cut between neighbours.  What an item costs
// beside its units (loading queries, writing results) counts as AC_LEAD units in front of them: without, CTAs with many
// short items ended up to twice as late as the others.
constexpr int AC_LEAD = 1;
struct AcRun {
  int s, x, h, u;   // first place: item (s, x, h), place u of it (AC_LEAD places, then its units)
  long long left;   // places of this CTA
};

// All `n_threads` threads call it; `part` holds n_threads / 32 + 1 numbers of shared memory.  cost(s, x) >= 0.
template <class Cost>
__device__ __forceinline__ void ac_run_start(Cost cost, int n_seq, int nx, int n_kv, int n_threads, long long* part, AcRun* out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long pairs = static_cast<long long>(n_seq) * nx;
  const long long per = (pairs + n_threads - 1) / n_threads;
  const long long p0 = min(pairs, per * threadIdx.x), p1 = min(pairs, p0 + per);
  long long sum = 0;
  auto places = [&](long long p) {
    const int n = cost(static_cast<int>(p / nx), static_cast<int>(p % nx));
    return n > 0 ? n + AC_LEAD : 0;
  };
  for (long long p = p0; p < p1; ++p) sum += places(p);
  long long incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) part[warp] = incl;
  __syncthreads();
  long long before = 0, all = 0;
  for (int w = 0; w < n_threads / 32; ++w) {
    if (w < warp) before += part[w];
    all += part[w];
  }
  const long long excl = (before + incl - sum) * n_kv, N = all * n_kv;
  const long long w0 = N * blockIdx.x / gridDim.x, w1 = N * (blockIdx.x + 1) / gridDim.x;
  if (threadIdx.x == 0 && w0 >= w1) out->left = 0;
  if (w0 < w1 && w0 >= excl && w0 < excl + sum * n_kv) {
    long long rem = w0 - excl;
    for (long long p = p0; p < p1; ++p) {
      const int c = places(p);
      if (rem < static_cast<long long>(c) * n_kv) {
        *out = AcRun{static_cast<int>(p / nx), static_cast<int>(p % nx), static_cast<int>(rem / c), static_cast<int>(rem % c), w1 - w0};
        break;
      }
      rem -= static_cast<long long>(c) * n_kv;
    }
  }
  __syncthreads();
}

// Walks a run item by item: u0 .. u1 (not empty) are the units of item (s, x, h) that belong to the run, of `units` in all.
struct AcWalk {
  int s, x, h, u0, u1, units;
  int place;
  long long left;
  int nx, n_kv, n_seq;
  __device__ __forceinline__ AcWalk(const AcRun& r, int nx_, int n_kv_, int n_seq_)
      : s(r.s), x(r.x), h(r.h), u0(0), u1(0), units(0), place(r.u), left(r.left), nx(nx_), n_kv(n_kv_), n_seq(n_seq_) {}
  __device__ __forceinline__ bool take() {  // the part of the current item that lies in the run; false: it has no unit there
    const int end = static_cast<int>(min(static_cast<long long>(units + AC_LEAD), place + left));
    left -= end - place;
    u0 = max(0, place - AC_LEAD);
    u1 = max(0, end - AC_LEAD);
    return u1 > u0;
  }
  template <class Cost>
  __device__ __forceinline__ bool start(Cost cost) {
    if (left <= 0) return false;
    units = cost(s, x);
    return take() || next(cost);
  }
  template <class Cost>
  __device__ __forceinline__ bool next(Cost cost) {
    while (left > 0) {
      place = 0;
      if (++h == n_kv) {
        h = 0;
        do {
          if (++x == nx) {
            x = 0;
            if (++s >= n_seq) return false;
          }
          units = cost(s, x);
        } while (units == 0);
      }
      if (take()) return true;
    }
    return false;
  }
};

// ---- forward -----------------------------------------------------------------------------------------------------------
// An item is 256 rows (two tiles of 128, whole tokens each) of one kv head; a unit is 128 slots of its keys.  One CTA per SM:
//   warp 0      producer: queries of an item (3-D TMA: dims x heads of the group x tokens), then per unit the keys and the
//               values, page by page, 128-byte swizzled, through a ring of five tiles
//   warps 1, 2  MMA: S_a = Q_a K^T and O_a += (P_a hi + P_a lo) V for row tile a, 64 slots at a time (one issuer for both was what the
//               kernel waited for: 2400 cycles a step, of which 1360 issuing and 1000 in waits); each row tile has two score
//               buffers, so the scores of the next 64 slots are there when the softmax of the last 64 ends.  P replaces S in
//               tensor memory (A operand); V is the MN-major B operand.  512 columns: 2 x (2 x 64 of S, 128 of O).
//   warp 3      makes a unit's values harmless where some row must not see them: rows behind the last slot and of padding
//               become zero, and so do values that are not finite (rows that do see them get them back at the end)
//   warps 4-7, 8-11   softmax of row tile 0 / 1, one row per thread: no exchange between threads.  The running maximum is
//               followed only when it has grown by more than 2^8 (weights stay below 2^8, statistics and sums are fp32), so
//               the result is rescaled rarely.  Weights enter the product as two bf16 halves (ac_split), side by side in
//               the 64 columns that their scores leave; their sum is taken before.  (One bf16 each, half the value products,
//               added as much error as the rounding of the result: a chunk took 489 us with its weights pass in place of 561.)
// Bound: 1536 cycles of products and 1024 of exponentials per 128 x 128 tile for long chunks (scores take 3/4 of the rate
// with 64 columns, as both operands come from shared memory); the reading of keys and values for few rows.
// A chunk of 4096 tokens over 4100 slots (20 heads over 5 of 128): 298 us with the join behind it, tensor pipe busy for 69 % of the
// cycles, exponentials for 46 %; 64 states of 15 .. 40 tokens over 200 .. 2000 slots: 74 us; 16 trees of 48 over 1000 .. 8000: 77 us.
// Every wait is bounded; on expiry the CTA records a status word and leaves normally.
constexpr int AT_THREADS = 384;
constexpr int AT_KEYS = 128;
constexpr int AT_RING = 5;  // odd: a place holds keys and values in turn, so its V_READY barrier turns every second round
constexpr float AT_GROWTH = 8.0f;
enum { AT_WAIT_LOAD = 131, AT_WAIT_MMA = 132, AT_WAIT_SOFTMAX = 133, AT_WAIT_FIX = 134 };

template <int HD>
struct AtSmem {
  static constexpr uint32_t TILE = 128 * HD * 2, HALF = 128 * 128;  // HALF: one 64-dimension block of a tile
  static constexpr uint32_t Q = 0, RING = 2 * TILE, BAR = RING + AT_RING * TILE;
  static constexpr uint32_t KV_FULL = BAR, KV_EMPTY = KV_FULL + 8 * AT_RING, Q_FULL = KV_EMPTY + 8 * AT_RING, Q_EMPTY = Q_FULL + 8,
                            S_FULL = Q_EMPTY + 8, P_FULL = S_FULL + 32, O_DONE = P_FULL + 32, V_READY = O_DONE + 32, DRAIN = V_READY + 8 * AT_RING;
  static constexpr uint32_t MISC = DRAIN + 8;  // tensor-memory base, failed, odd
  static constexpr uint32_t RUN = MISC + 32, PART = RUN + 32;
  static constexpr uint32_t BYTES = PART + 8 * (AT_THREADS / 32 + 1) + 1024;  // + slack to align the base
  static_assert(AT_RING % 2 == 1 && BYTES <= 232448, "ring");
  // one CTA per SM: it takes all of tensor memory
  static constexpr uint32_t LAUNCH = BYTES > 120 * 1024 ? BYTES : 120 * 1024;
};

struct AtArgs {
  AcArgs a;
  int tok_tile;  // whole tokens of a 128-row tile
  int nx;        // items of the longest sequence
  int rows_cap;  // rows kept for each cut item: min(256, max_new * rep)
};

// Units (key tiles) of item (s, x).
__device__ __forceinline__ int at_units(const AtArgs& t, int s, int x, KvSeq& q) {
  if (!kv_seq(t.a.c, t.a.b, s, q)) return 0;
  const int tok0 = x * 2 * t.tok_tile;
  if (tok0 >= q.m || (t.a.tree_ok && !t.a.tree_ok[s])) return 0;
  const int end = q.used + (t.a.b.parent ? q.m : min(q.m, tok0 + 2 * t.tok_tile));
  return (end + AT_KEYS - 1) / AT_KEYS;
}
// 32 bits: which of the slots slot0 .. slot0 + 31 does token `tok` see?
__device__ __forceinline__ uint32_t at_seen(const AcArgs& a, const KvSeq& q, int tok, int slot0) {
  const int j0 = slot0 - q.used;  // place of the first slot among the new tokens
  if (j0 + 32 <= 0) return 0xffffffffu;
  if (!a.b.parent) {
    const int n = tok + 1 - j0;  // slots seen from slot0 on
    return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
  }
  const uint32_t* w = a.anc + static_cast<long long>(q.t0 + tok) * AC_TREE_WORDS;
  if (j0 >= BITRL_TREE_MAX_TOKENS) return 0u;
  if (j0 < 0) return ((w[0] << (-j0)) | ((1u << (-j0)) - 1u));
  const uint32_t lo = w[j0 >> 5], hi = (j0 >> 5) + 1 < AC_TREE_WORDS ? w[(j0 >> 5) + 1] : 0u;
  return __funnelshift_r(lo, hi, j0 & 31);
}

template <int HD>
__global__ void __launch_bounds__(AT_THREADS, 1)
attn_tiles_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                  const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ AtArgs t) {
  using M = AtSmem<HD>;
  constexpr int NH = HD / 64;
  extern __shared__ unsigned char at_smem_raw[];
  const uint32_t raw = ptx::smem_u32(at_smem_raw), base = (raw + 1023u) & ~1023u;
  unsigned char* sm = at_smem_raw + (base - raw);
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(sm + M::MISC);
  volatile uint32_t* failed = misc + 1;
  volatile uint32_t* odd = misc + 4;  // a value was made harmless
  const uint32_t failed_addr = base + M::MISC + 4;
  const AcArgs& a = t.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto wait = [&](uint32_t bar, uint32_t parity) { return ptx::mbar_wait_abortable(base + bar, parity, failed_addr); };
  auto give_up = [&](int stage) {
    report_timeout(stage);
    *failed = 1u;
  };

  if (threadIdx.x == 0) {
    *failed = 0u;
    *odd = 0u;
    for (int i = 0; i < AT_RING; ++i) {
      ptx::mbar_init(base + M::KV_FULL + 8 * i, 1);
      ptx::mbar_init(base + M::KV_EMPTY + 8 * i, 3);  // either issuer, and the warp that looks the values over
      ptx::mbar_init(base + M::V_READY + 8 * i, 1);
    }
    ptx::mbar_init(base + M::Q_FULL, 1);
    ptx::mbar_init(base + M::Q_EMPTY, 2);
    for (int i = 0; i < 4; ++i) {
      ptx::mbar_init(base + M::S_FULL + 8 * i, 1);
      ptx::mbar_init(base + M::P_FULL + 8 * i, 4);
      ptx::mbar_init(base + M::O_DONE + 8 * i, 1);
    }
    ptx::mbar_init(base + M::DRAIN, 2);
    ptx::mbar_init_fence();
    ptx::tma_prefetch_desc(&tmap_q);
    ptx::tma_prefetch_desc(&tmap_k);
    ptx::tma_prefetch_desc(&tmap_v);
  }
  if (warp == 1) {
    ptx::tmem_alloc(base + M::MISC, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = misc[0];
  // The kernels that follow may start only now: the weights pass reads the cache and the queries before it waits.
  pdl_wait_before();
  pdl_launch_next();
  AtCut* cuts = a.cuts + 2 * blockIdx.x;
  if (threadIdx.x < 2) cuts[threadIdx.x].s = -1;
  KvSeq q;
  auto cost = [&](int s, int x) { return at_units(t, s, x, q); };
  AcRun* run = reinterpret_cast<AcRun*>(sm + M::RUN);
  ac_run_start(cost, a.c.n_seq, t.nx, a.c.n_kv, AT_THREADS, reinterpret_cast<long long*>(sm + M::PART), run);

  AcWalk w(*run, t.nx, a.c.n_kv, a.c.n_seq);
  const int tok_tile = t.tok_tile, slots_mask = (1 << a.c.page_shift) - 1;
  // Has unit `u` a slot that some row of the item does not see?
  auto masked = [&](int u) {
    return (u + 1) * AT_KEYS > q.used + (a.b.parent ? 0 : w.x * 2 * tok_tile + 1);
  };
  // 64-slot steps of the run's part of the item; the last unit may have one
  auto steps_of = [&]() {
    const int end = q.used + (a.b.parent ? q.m : min(q.m, (w.x + 1) * 2 * tok_tile));
    return min(2 * (w.u1 - w.u0), (end - w.u0 * AT_KEYS + 63) / 64);
  };
  bool more = w.start(cost);
  if (warp < 4) {
  if (warp == 0) {
    // ------------------------------------------------------------------ producer
    uint32_t e = 0, qn = 0;  // tiles put into the ring; items
    bool ok = true;
    const int page = 1 << a.c.page_shift, pieces = AT_KEYS >> a.c.page_shift;
    const int piece = lane / NH, half = lane % NH;  // this lane's copy of a tile
    const int none = a.c.n_pages * a.c.n_kv * page;  // a row behind the pool: such a copy fills with zeros
    while (ok && more) {
      const int end = q.used + (a.b.parent ? q.m : min(q.m, (w.x + 1) * 2 * tok_tile));
      const int na = w.x * 2 * tok_tile + tok_tile < q.m ? 2 : 1;
      auto row_of = [&](int u) {  // first row of this lane's page of unit u
        const int slot = u * AT_KEYS + piece * page;
        if (piece >= pieces || slot >= end) return none;
        const int p = kv_page(a.c, w.s, slot);
        return p < 0 ? none : (p * a.c.n_kv + w.h) * page;
      };
      int row = row_of(w.u0);
      for (int u = w.u0; u < w.u1; ++u) {
        const int row_next = u + 1 < w.u1 ? row_of(u + 1) : 0;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv, ++e) {
          const uint32_t slot = e % AT_RING;
          if (!__any_sync(0xffffffffu, wait(M::KV_EMPTY + 8 * slot, ((e / AT_RING) & 1) ^ 1))) { ok = false; break; }
          if (lane == 0) ptx::mbar_arrive_expect_tx(base + M::KV_FULL + 8 * slot, M::TILE);
          __syncwarp();
          if (piece < pieces)
            ptx::tma_load_2d(base + M::RING + slot * M::TILE + half * M::HALF + piece * page * 128, kv ? &tmap_v : &tmap_k, 64 * half,
                             row, base + M::KV_FULL + 8 * slot);
          if (u == w.u0 && kv == 0) {  // the queries: the first keys need not wait for the place that the last item's leave
            if (!__any_sync(0xffffffffu, wait(M::Q_EMPTY, (qn & 1) ^ 1))) { ok = false; break; }
            if (lane == 0) ptx::mbar_arrive_expect_tx(base + M::Q_FULL, na * NH * 128 * a.rep * tok_tile);
            __syncwarp();
            if (lane < na * NH)
              ptx::tma_load_3d(base + M::Q + (lane / NH) * M::TILE + (lane % NH) * M::HALF, &tmap_q, 64 * (lane % NH), w.h * a.rep,
                               q.t0 + (w.x * 2 + lane / NH) * tok_tile, base + M::Q_FULL);
            ++qn;
          }
        }
        if (!ok) break;
        row = row_next;
      }
      more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AT_WAIT_LOAD);
  } else if (warp <= 2) {
    // ------------------------------------------------------------------ MMA issuers: row tile x
    constexpr uint32_t id_s = ptx::idesc_bf16(128, 64, false), id_o = ptx::idesc_bf16(128, HD, true);
    const int x = warp - 1;
    uint32_t e = 0, qn = 0, p_par = 0;  // p_par: phase of either P_FULL barrier, as bits
    bool ok = true;
    auto all_wait = [&](uint32_t bar, uint32_t parity) { return __any_sync(0xffffffffu, wait(bar, parity)); };
    auto full_wait = [&](uint32_t at) { return all_wait(M::KV_FULL + 8 * (at % AT_RING), (at / AT_RING) & 1); };
    auto commit = [&](uint32_t bar) {
      if (ptx::elect_one()) ptx::mma_commit(base + bar);
      __syncwarp();
    };
    auto scores = [&](uint32_t slot, int b) {  // half b of the keys in `slot`
      if (ptx::elect_one()) {
        const uint64_t qd = ptx::smem_desc_sw128(base + M::Q + x * M::TILE), kd = ptx::smem_desc_sw128(base + M::RING + slot * M::TILE + b * 8192);
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          const uint32_t off = ((k / 4) * M::HALF + (k % 4) * 32) >> 4;
          ptx::mma_bf16_ss(tmem + 128 * x + 64 * b, qd + off, kd + off, id_s, k != 0);
        }
        ptx::mma_commit(base + M::S_FULL + 8 * (2 * x + b));
      }
      __syncwarp();
    };
    while (ok && more) {
      const int steps = steps_of();
      if (!(ok = all_wait(M::Q_FULL, qn & 1))) break;
      ++qn;
      if (x == 1 && w.x * 2 * tok_tile + tok_tile >= q.m) {
        // no second row tile: this issuer only gives its leave for what it does not use
        if (lane == 0) ptx::mbar_arrive(base + M::Q_EMPTY);
        for (uint32_t i = 0; ok && i < 2u * (w.u1 - w.u0); ++i, ++e) {
          ok = full_wait(e);
          if (ok && lane == 0) ptx::mbar_arrive(base + M::KV_EMPTY + 8 * (e % AT_RING));
        }
        if (ok) more = w.next(cost);
        __syncwarp();
        continue;
      }
      if (!(ok = full_wait(e))) break;
      ptx::tc_fence_after_sync();
      for (int b = 0; b < min(steps, 2); ++b) scores(e % AT_RING, b);
      commit(M::KV_EMPTY + 8 * (e % AT_RING));
      if (steps <= 2) commit(M::Q_EMPTY);
      for (int i = 0; i < steps; ++i) {
        const int b = i & 1;
        const uint32_t ve = e + 2 * (i >> 1) + 1, ke = ve + 1;  // ring places of this unit's values and the next one's keys
        const bool next = i + 2 < steps;
        if (b == 0 && !(ok = all_wait(M::V_READY + 8 * (ve % AT_RING), (ve / (2 * AT_RING)) & 1))) break;
        if (!(ok = all_wait(M::P_FULL + 8 * (2 * x + b), (p_par >> b) & 1))) break;
        p_par ^= 1u << b;
        ptx::tc_fence_after_sync();
        if (ptx::elect_one()) {
          const uint64_t vd = ptx::smem_desc_mn_sw128(base + M::RING + (ve % AT_RING) * M::TILE + b * 8192, M::HALF);
#pragma unroll
          for (int k = 0; k < 8; ++k)  // the upper halves of the weights, then the lower ones
            ptx::mma_bf16_ts(tmem + 256 + 128 * x, tmem + 128 * x + 64 * b + 8 * k, vd + (k & 3) * (2048 >> 4), id_o, i != 0 || k != 0);
          ptx::mma_commit(base + M::O_DONE + 8 * (2 * x + b));
        }
        __syncwarp();
        if (b == 1 || i + 1 == steps) commit(M::KV_EMPTY + 8 * (ve % AT_RING));
        if (next) {
          if (b == 0 && !(ok = full_wait(ke))) break;
          scores(ke % AT_RING, b);
          if (b == 1 || i + 3 == steps) commit(M::KV_EMPTY + 8 * (ke % AT_RING));
        }
        if (i + 3 == steps) commit(M::Q_EMPTY);
      }
      e += 2 * (w.u1 - w.u0);
      if (ok) more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AT_WAIT_MMA);
  } else {
    // ------------------------------------------------------------------ values of masked units
    uint32_t e = 1;
    bool ok = true;
    while (ok && more) {
      const int end = q.used + q.m;
      for (int u = w.u0; u < w.u1; ++u, e += 2) {
        const uint32_t slot = e % AT_RING;
        // The keys' tile too: a place's barrier must be followed through every round, or a later one looks like this one.  And
        // the place goes on to the next round with this warp's leave alone: without it, this warp could come too late for a
        // round (one launch in 700 did), wait for the one after it, and nobody would say that its values are ready.
        if (!(ok = __any_sync(0xffffffffu, wait(M::KV_FULL + 8 * ((e - 1) % AT_RING), ((e - 1) / AT_RING) & 1)))) break;
        if (lane == 0) ptx::mbar_arrive(base + M::KV_EMPTY + 8 * ((e - 1) % AT_RING));
        if (!(ok = __any_sync(0xffffffffu, wait(M::KV_FULL + 8 * slot, (e / AT_RING) & 1)))) break;
        if (masked(u)) {
          // from the first slot that some row does not see; a lane takes 16 bytes of a row, four rows side by side (the swizzle
          // moves pieces inside a row, which does not matter here)
          const uint32_t tile = base + M::RING + slot * M::TILE + (lane & 7) * 16;
          const int r0 = max(0, q.used + (a.b.parent ? 0 : w.x * 2 * tok_tile + 1) - u * AT_KEYS), rl = min(AT_KEYS, end - u * AT_KEYS);
          const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
          for (int r = (rl & ~3) + (lane >> 3); r < AT_KEYS; r += 4)
            if (r >= rl) {
#pragma unroll
              for (int half = 0; half < NH; ++half) ptx::sts128(tile + half * M::HALF + r * 128, zero);
            }
          if (a.b.parent)
            for (int r = (r0 & ~3) + (lane >> 3); r < rl; r += 4)
              if (u * AT_KEYS + r >= q.used && a.b.parent[q.t0 + u * AT_KEYS + r - q.used] == BITRL_PARENT_PAD) {
#pragma unroll
                for (int half = 0; half < NH; ++half) ptx::sts128(tile + half * M::HALF + r * 128, zero);
              }
          __syncwarp();
          // is there an exponent of ones?  (two per word: a half of x that is zero)
          uint32_t hit = 0u;
#pragma unroll
          for (int half = 0; half < NH; ++half)
#pragma unroll 8
            for (int r = (r0 & ~3) + (lane >> 3); r < rl; r += 4) {
              const uint4 v = ptx::lds128(tile + half * M::HALF + r * 128);
              const uint32_t x0 = ~v.x & 0x7f807f80u, x1 = ~v.y & 0x7f807f80u, x2 = ~v.z & 0x7f807f80u, x3 = ~v.w & 0x7f807f80u;
              hit |= ((x0 - 0x00010001u) & ~x0) | ((x1 - 0x00010001u) & ~x1) | ((x2 - 0x00010001u) & ~x2) | ((x3 - 0x00010001u) & ~x3);
            }
          bool found = false;
          if (__any_sync(0xffffffffu, (hit & 0x80008000u) != 0u))
            for (int half = 0; half < NH; ++half)
              for (int r = (r0 & ~3) + (lane >> 3); r < rl; r += 4) {
                if (r < r0) continue;
                const uint32_t addr = tile + half * M::HALF + r * 128;
                const uint4 v = ptx::lds128(addr);
                uint32_t x[4] = {v.x, v.y, v.z, v.w};
                bool touch = false;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const bool lo = (x[j] & 0x7f80u) == 0x7f80u, hi = (x[j] & 0x7f800000u) == 0x7f800000u;
                  touch |= lo || hi;
                  if (lo) x[j] &= 0xffff0000u;
                  if (hi) x[j] &= 0x0000ffffu;
                }
                if (touch) ptx::sts128(addr, make_uint4(x[0], x[1], x[2], x[3]));
                found |= touch;
              }
          if (__any_sync(0xffffffffu, found) && lane == 0) *odd = 1u;  // for good: this warp runs ahead of the softmax by as many items as the ring allows
          ptx::fence_proxy_async_smem();
        }
        __syncwarp();
        if (lane == 0) {
          ptx::mbar_arrive(base + M::V_READY + 8 * slot);
          ptx::mbar_arrive(base + M::KV_EMPTY + 8 * slot);
        }
      }
      if (ok) more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AT_WAIT_FIX);
  }
  } else {
    // ------------------------------------------------------------------ softmax, one row per thread
    const int x = (warp - 4) >> 2;  // row tile
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const int r = (warp & 3) * 32 + lane, r_tok = r / a.rep, r_head = r - r_tok * a.rep;
    const uint32_t s_addr = tmem + 128 * x + lane_base, o_addr = tmem + 256 + 128 * x + lane_base;
    const bool wide = (reinterpret_cast<uintptr_t>(a.att) & 31u) == 0;  // att is 16-byte aligned at least
    uint32_t s_par = 0, o_par = 0;  // phases, as bits: of either score buffer, of the products from either buffer
    const uint64_t scale_x2 = ptx::pack_f32x2(__float_as_uint(a.scale2), __float_as_uint(a.scale2));
    bool ok = true;
    while (ok && more) {
      const int tok_first = (w.x * 2 + x) * tok_tile, tok = tok_first + r_tok;
      if (tok_first < q.m) {
        const bool exists = r_tok < tok_tile && tok < q.m;
        const int tk = min(tok, q.m - 1), steps = steps_of();
        float m_ref = -INFINITY, l = 0.0f;
        for (int i = 0; i < steps; ++i) {
          const int b = i & 1;
          if (!__any_sync(0xffffffffu, wait(M::S_FULL + 8 * (2 * x + b), (s_par >> b) & 1))) { ok = false; break; }
          s_par ^= 1u << b;
          ptx::tc_fence_after_sync();
          uint32_t s[2][32];
          ptx::tmem_ld_32x32b_x32(s_addr + 64 * b, s[0]);
          ptx::tmem_ld_32x32b_x32(s_addr + 64 * b + 32, s[1]);
          ptx::tmem_ld_wait();
          if (masked(w.u0 + (i >> 1))) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const uint32_t seen = at_seen(a, q, tk, w.u0 * AT_KEYS + 64 * i + 32 * c);
#pragma unroll
              for (int j = 0; j < 32; ++j) s[c][j] = (seen >> j) & 1u ? s[c][j] : 0xff800000u;
            }
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int j = 0; j < 32; j += 2)
              mx[(j >> 1) & 3] = fmaxf(mx[(j >> 1) & 3], fmaxf(__uint_as_float(s[c][j]), __uint_as_float(s[c][j + 1])));
          const float m2 = __fmul_rn(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), a.scale2);
          // every row goes by its own scores: which steps the warp walks through here does not change the others' bits (a tile
          // may hold rows of nobody, whatever shared memory held)
          const bool grown = m2 > m_ref + AT_GROWTH;
          if (i == 0) {
            m_ref = m2;
          } else if (__any_sync(0xffffffffu, grown && exists)) {
            // the product of the step before (the one before that is done: this step's scores came after it)
            if (!__any_sync(0xffffffffu, wait(M::O_DONE + 8 * (2 * x + (b ^ 1)), ((o_par >> (b ^ 1)) & 1) ^ 1))) { ok = false; break; }
            ptx::tc_fence_after_sync();
            const float f = grown ? ac_exp2(m_ref - m2) : 1.0f;
            if (grown) m_ref = m2;
            l = __fmul_rn(l, f);
#pragma unroll 1
            for (int c = 0; c < HD / 32; ++c) {
              uint32_t o[32];
              ptx::tmem_ld_32x32b_x32(o_addr + 32 * c, o);
              ptx::tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__fmul_rn(__uint_as_float(o[j]), f));
              ptx::tmem_st_32x32b_x32(o_addr + 32 * c, o);
            }
          }
          const float sub = m_ref == -INFINITY ? 0.0f : -m_ref;
          const uint64_t sub_x2 = ptx::pack_f32x2(__float_as_uint(sub), __float_as_uint(sub));
          uint64_t sum[2] = {0ull, 0ull};
          uint32_t p[2][32];  // upper and lower halves of the weights
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const int c = j >> 4, k = 2 * (j & 15);
            float p0, p1;
            ptx::unpack_f32x2(ptx::fma_f32x2(ptx::pack_f32x2(s[c][k], s[c][k + 1]), scale_x2, sub_x2), p0, p1);
            p0 = ac_exp2(p0);
            p1 = ac_exp2(p1);
            sum[j & 1] = ptx::add_f32x2(sum[j & 1], ptx::pack_f32x2(__float_as_uint(p0), __float_as_uint(p1)));
            ac_split(p0, p1, p[0][j], p[1][j]);
          }
          ptx::tmem_st_32x32b_x32(s_addr + 64 * b, p[0]);
          ptx::tmem_st_32x32b_x32(s_addr + 64 * b + 32, p[1]);
          float l0, l1;
          ptx::unpack_f32x2(ptx::add_f32x2(sum[0], sum[1]), l0, l1);
          l += l0 + l1;
          ptx::tmem_st_wait();
          ptx::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(base + M::P_FULL + 8 * (2 * x + b));
          o_par ^= 1u << b;
        }
        if (!ok) break;
        const int lb = (steps - 1) & 1;
        if (!__any_sync(0xffffffffu, wait(M::O_DONE + 8 * (2 * x + lb), ((o_par >> lb) & 1) ^ 1))) { ok = false; break; }
        ptx::tc_fence_after_sync();
        const bool whole = w.u0 == 0 && w.u1 == w.units;
        const bool fix = *odd != 0u;  // perhaps of another item: then there is nothing to give back below
        const bool pad = a.b.parent && exists && a.b.parent[q.t0 + tok] == BITRL_PARENT_PAD;
        const bool none = l == 0.0f || pad;
        const float inv = !whole ? 1.0f : none ? 0.0f : __fdiv_rn(1.0f, l);
        const long long row = static_cast<long long>(q.t0 + tok) * a.n_heads + w.h * a.rep + r_head;
        const int cut = 2 * blockIdx.x + (w.u0 == 0 ? 1 : 0);
        const int cut_row = x * tok_tile * a.rep + r;
        // parts lie dimension by dimension, so that the lanes' rows are neighbours (row by row, every store touched 32 lines
        // and writing a part took 20000 cycles)
        float* part = a.part_o + static_cast<long long>(cut) * HD * t.rows_cap + cut_row;
#pragma unroll 1
        for (int c = 0; c < HD / 32; ++c) {
          uint32_t o[32];
          ptx::tmem_ld_32x32b_x32(o_addr + 32 * c, o);
          ptx::tmem_ld_wait();
          if (fix && exists && !pad) {  // rare: values that are not finite, of masked units, for the rows that see them
            for (int at = max(q.used + (a.b.parent ? 0 : w.x * 2 * tok_tile + 1), w.u0 * AT_KEYS); at < min(q.used + q.m, w.u1 * AT_KEYS); ++at) {
              if (!(at_seen(a, q, tok, at) & 1u)) continue;
              const int pg = kv_page(a.c, w.s, at);
              if (pg < 0) continue;
              const unsigned short* v = a.c.v + (kv_row(a.c, 0, pg, w.h) + (at & slots_mask)) * HD + 32 * c;
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const unsigned short b = v[i];
                if ((b & 0x7f80u) == 0x7f80u) o[i] = __float_as_uint(__uint_as_float(o[i]) + bf16_bits_to_float(b));
              }
            }
          }
          if (!exists) continue;
          if (whole) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              uint32_t v[8];
#pragma unroll
              for (int j = 0; j < 8; ++j)
                v[j] = none ? 0u : pack_bf16x2(__fmul_rn(__uint_as_float(o[16 * i + 2 * j]), inv), __fmul_rn(__uint_as_float(o[16 * i + 2 * j + 1]), inv));
              if (wide) {
                ptx::stg256(a.att + row * HD + 32 * c + 16 * i, v);
              } else {
                uint4* dst = reinterpret_cast<uint4*>(a.att + row * HD + 32 * c + 16 * i);
                dst[0] = make_uint4(v[0], v[1], v[2], v[3]);
                dst[1] = make_uint4(v[4], v[5], v[6], v[7]);
              }
            }
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) part[static_cast<long long>(32 * c + i) * t.rows_cap] = __uint_as_float(o[i]);
          }
        }
        if (exists) {
          if (whole) a.lse[row] = none ? INFINITY : m_ref + __log2f(l);
          else a.part_ml[static_cast<long long>(cut) * t.rows_cap + cut_row] = make_float2(ac_part_max(m_ref, l), l);
        }
        if (!whole && threadIdx.x == 128) cuts[w.u0 == 0 ? 1 : 0] = AtCut{w.s, w.x, w.h, w.u1 == w.units};
        ptx::tc_fence_before_sync();
      }
      more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AT_WAIT_SOFTMAX);
  }

  // ---- teardown: every role leaves through here, also after a timeout ----
  __syncwarp();
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (*failed) {
    // Failure path only: copies and MMAs that nobody waited for may still be in flight.
    if (warp == 1 || warp == 2) {
      if (ptx::elect_one()) ptx::mma_commit(base + M::DRAIN);
      __syncwarp();
      ptx::mbar_wait(base + M::DRAIN, 0, 2000000LL);
    }
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000LL) {}
    __syncthreads();
  }
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

// Joins the cut items: the CTA in which an item begins and those after it each left a part.  Block (c, y) takes 32 rows of the
// item that begins in CTA c.
template <int HD>
__global__ void __launch_bounds__(256) attn_tiles_join_kernel(const __grid_constant__ AtArgs t, int n_ctas) {
  pdl_enter();
  const AcArgs& a = t.a;
  const int c0 = blockIdx.x;
  const AtCut head = a.cuts[2 * c0 + 1];
  if (head.s < 0) return;
  KvSeq q;
  if (!kv_seq(a.c, a.b, head.s, q)) return;
  constexpr int PER = HD / 8;  // dimensions of a thread
  const int cut_row = blockIdx.y * 32 + (threadIdx.x & 31), d0 = (threadIdx.x >> 5) * PER;
  const int tile_rows = t.tok_tile * a.rep;
  const int x = cut_row / tile_rows, r = cut_row - x * tile_rows;
  const int tok = (head.x * 2 + x) * t.tok_tile + r / a.rep;
  if (x > 1 || tok >= q.m) return;
  // the parts: slot 1 of this CTA, then slot 0 of the following ones up to the one in which the item ends (a CTA whose run is
  // empty has none)
  auto part_at = [&](int c) { return static_cast<long long>(c == c0 ? 2 * c0 + 1 : 2 * c) * t.rows_cap + cut_row; };
  float m_all = a.part_ml[part_at(c0)].x;
  int last = c0;
  while (last + 1 < n_ctas) {
    const AtCut cut = a.cuts[2 * ++last];
    if (cut.s < 0) continue;
    m_all = fmaxf(m_all, a.part_ml[part_at(last)].x);
    if (cut.ends) break;
  }
  float l = 0.0f, acc[PER], v[PER];
  auto fetch = [&](int c) {
    const float* p = a.part_o + (part_at(c) - cut_row) * HD + static_cast<long long>(d0) * t.rows_cap + cut_row;
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = p[static_cast<long long>(i) * t.rows_cap];
  };
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.0f;
  for (int c = c0; c <= last; ++c) {
    if (c != c0 && a.cuts[2 * c].s < 0) continue;
    fetch(c);
    const float2 ml = a.part_ml[part_at(c)];
    if (ml.x == -INFINITY) continue;
    const float f = ac_exp2(ml.x - m_all);
    l = fmaf(ml.y, f, l);
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] = fmaf(v[i], f, acc[i]);
  }
  const bool none = l == 0.0f || (a.b.parent && a.b.parent[q.t0 + tok] == BITRL_PARENT_PAD);
  const float inv = none ? 0.0f : __fdiv_rn(1.0f, l);
  const long long row = static_cast<long long>(q.t0 + tok) * a.n_heads + head.h * a.rep + r % a.rep;
#pragma unroll
  for (int i = 0; i < PER; i += 8) {
    uint32_t b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = none ? 0u : pack_bf16x2(__fmul_rn(acc[i + 2 * j], inv), __fmul_rn(acc[i + 2 * j + 1], inv));
    *reinterpret_cast<uint4*>(a.att + row * HD + d0 + i) = make_uint4(b[0], b[1], b[2], b[3]);
  }
  if (d0 == 0) a.lse[row] = none ? INFINITY : m_all + __log2f(l);
}

// ---- weight received by every slot ---------------------------------------------------------------------------------
// A second pass over the keys: the final maximum and sum of every row are known, so p = 2^(t - lse) directly.  The scores
// are formed transposed, S^T = K Q^T: a thread then owns one slot and adds up its weights over the rows in registers, in a
// fixed order and without a word to other threads.  An item is 256 slots (two tiles) of one kv head, a unit is one row tile;
// an item that is cut between CTAs leaves partial sums that attn_mass_join_kernel adds in order.
//   warp 0 producer (keys of an item, double-buffered; queries through a ring of two), warp 1 MMA (two accumulators per key
//   tile), warp 2 row statistics, warps 4-11 and 12-19 the sums of key tile 0 and 1, four warps for every other unit.
// Bound: 1024 cycles of exponentials per 128 x 128 tile (the products take 512) for long chunks; reading for short ones.
// A chunk of 4096 tokens over 4100 slots: 203 us, the exponentials' pipe busy for 59 % of the cycles.
constexpr int AM_THREADS = 640;
constexpr int AM_KEYS = 256;
enum { AM_WAIT_LOAD = 141, AM_WAIT_MMA = 142, AM_WAIT_LSE = 143, AM_WAIT_SUM = 144 };

template <int HD>
struct AmSmem {
  static constexpr uint32_t TILE = 128 * HD * 2, HALF = 128 * 128;
  static constexpr uint32_t K = 0, Q = 4 * TILE, LSE = Q + 2 * TILE;  // K [2][2 tiles], Q [2], LSE [4][128]
  static constexpr uint32_t LIVE = LSE + 4 * 512, SUM = LIVE + 64, BAR = SUM + 1024;  // LIVE [4][4] bits: columns that hold a row; SUM [2][128]
  static constexpr uint32_t K_FULL = BAR, K_EMPTY = K_FULL + 16, Q_FULL = K_EMPTY + 16, Q_EMPTY = Q_FULL + 16, S_FULL = Q_EMPTY + 16,
                            S_EMPTY = S_FULL + 32, L_FULL = S_EMPTY + 32, L_EMPTY = L_FULL + 32, SUM_FULL = L_EMPTY + 32, SUM_EMPTY = SUM_FULL + 16,
                            DRAIN = SUM_EMPTY + 16;
  static constexpr uint32_t MISC = DRAIN + 8, RUN = MISC + 8, PART = RUN + 32;
  static constexpr uint32_t BYTES = PART + 8 * (AM_THREADS / 32 + 1) + 1024;
  static constexpr uint32_t LAUNCH = BYTES > 120 * 1024 ? BYTES : 120 * 1024;  // one CTA per SM: it takes all of tensor memory
};

struct AmArgs {
  AcArgs a;
  int tok_tile;
  int nx;       // items of the longest sequence that the page table can hold
  float* part;  // [CTAs][2][256] sums of cut items
  AtCut* cuts;  // [CTAs][2], not those of the forward kernel, which are still read
};

// Row tiles that see some slot of item (s, x), from `first` on.
__device__ __forceinline__ int am_units(const AmArgs& t, int s, int x, KvSeq& q, int& first) {
  first = 0;
  if (!kv_seq(t.a.c, t.a.b, s, q) || (t.a.tree_ok && !t.a.tree_ok[s])) return 0;
  if (x * AM_KEYS >= q.used + q.m) return 0;
  if (!t.a.b.parent) first = max(0, x * AM_KEYS - q.used) / t.tok_tile;
  return (q.m + t.tok_tile - 1) / t.tok_tile - first;
}

// Columns c .. c + 31 of a row tile whose token sees the slot of new token j (j >= 0), as bits.
__device__ __forceinline__ uint32_t am_columns(const AcArgs& a, const KvSeq& q, int j, int tok0, int c) {
  if (!a.b.parent) {
    const int from = (j - tok0) * a.rep - c;  // rows from token j on
    return from >= 32 ? 0u : from <= 0 ? 0xffffffffu : 0xffffffffu << from;
  }
  if (j >= q.m) return 0u;
  // the (at most 32) tokens of the columns as bits, then each bit on the columns of its token
  const uint32_t* who = a.desc + static_cast<long long>(q.t0 + j) * AC_TREE_WORDS;
  const int t0 = tok0 + c / a.rep, at = t0 >> 5;
  if (at >= AC_TREE_WORDS) return 0u;
  uint32_t can = 0u, left = __funnelshift_r(who[at], at + 1 < AC_TREE_WORDS ? who[at + 1] : 0u, t0 & 31);
  for (int lo = (t0 - tok0) * a.rep - c; lo < 32; lo += a.rep, left >>= 1)  // lo: first column of the token
    if (left & 1u) {
      const int from = max(lo, 0), n = min(lo + a.rep, 32) - from;
      can |= (n >= 32 ? 0xffffffffu : (1u << n) - 1u) << from;
    }
  return can;
}

// Adds 2^(score + lse) over the 32 columns whose bit in `see` is set; lse: shared-memory address of -(maximum + log2 sum).
__device__ __forceinline__ void am_add(const uint32_t (&s)[32], uint32_t see, uint32_t lse, uint64_t scale_x2, float scale, float (&got)[4]) {
  if (__all_sync(0xffffffffu, see == 0xffffffffu)) {
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
      const uint4 e = ptx::lds128(lse + 4 * i);
      float p[4];
      ptx::unpack_f32x2(ptx::fma_f32x2(ptx::pack_f32x2(s[i], s[i + 1]), scale_x2, ptx::pack_f32x2(e.x, e.y)), p[0], p[1]);
      ptx::unpack_f32x2(ptx::fma_f32x2(ptx::pack_f32x2(s[i + 2], s[i + 3]), scale_x2, ptx::pack_f32x2(e.z, e.w)), p[2], p[3]);
#pragma unroll
      for (int k = 0; k < 4; ++k) got[k] += ac_exp2(p[k]);
    }
  } else if (__any_sync(0xffffffffu, see != 0u)) {
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
      const uint4 e = ptx::lds128(lse + 4 * i);
      const uint32_t ev[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if ((see >> (i + k)) & 1u) got[k] += ac_exp2(fmaf(__uint_as_float(s[i + k]), scale, __uint_as_float(ev[k])));
    }
  }
}

template <int HD>
__global__ void __launch_bounds__(AM_THREADS, 1)
attn_mass_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ AmArgs t) {
  using M = AmSmem<HD>;
  constexpr int NH = HD / 64;
  extern __shared__ unsigned char at_smem_raw[];
  const uint32_t raw = ptx::smem_u32(at_smem_raw), base = (raw + 1023u) & ~1023u;
  unsigned char* sm = at_smem_raw + (base - raw);
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(sm + M::MISC);
  volatile uint32_t* failed = misc + 1;
  const uint32_t failed_addr = base + M::MISC + 4;
  const AcArgs& a = t.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto wait = [&](uint32_t bar, uint32_t parity) {
    return __any_sync(0xffffffffu, ptx::mbar_wait_abortable(base + bar, parity, failed_addr));
  };
  auto give_up = [&](int stage) {
    report_timeout(stage);
    *failed = 1u;
  };
  if (threadIdx.x == 0) {
    *failed = 0u;
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(base + M::K_FULL + 8 * i, 1);
      ptx::mbar_init(base + M::K_EMPTY + 8 * i, 1);
      ptx::mbar_init(base + M::Q_FULL + 8 * i, 1);
      ptx::mbar_init(base + M::Q_EMPTY + 8 * i, 1);
      ptx::mbar_init(base + M::SUM_FULL + 8 * i, 4);
      ptx::mbar_init(base + M::SUM_EMPTY + 8 * i, 4);
    }
    for (int i = 0; i < 4; ++i) {
      ptx::mbar_init(base + M::S_FULL + 8 * i, 1);
      ptx::mbar_init(base + M::S_EMPTY + 8 * i, 4);
      ptx::mbar_init(base + M::L_FULL + 8 * i, 1);
      ptx::mbar_init(base + M::L_EMPTY + 8 * i, 16);
    }
    ptx::mbar_init(base + M::DRAIN, 1);
    ptx::mbar_init_fence();
    ptx::tma_prefetch_desc(&tmap_q);
    ptx::tma_prefetch_desc(&tmap_k);
  }
  if (warp == 1) {
    ptx::tmem_alloc(base + M::MISC, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = misc[0];
  // Of what the two kernels before it write, this one reads the rows' statistics alone (warp 2 waits for them); what comes
  // before the forward kernel is complete, since that lets its followers start only after its own wait.
  pdl_launch_next();
  AtCut* cuts = t.cuts + 2 * blockIdx.x;
  if (threadIdx.x < 2) cuts[threadIdx.x].s = -1;
  KvSeq q;
  int first;
  auto cost = [&](int s, int x) { return am_units(t, s, x, q, first); };
  AcRun* run = reinterpret_cast<AcRun*>(sm + M::RUN);
  ac_run_start(cost, a.c.n_seq, t.nx, a.c.n_kv, AM_THREADS, reinterpret_cast<long long*>(sm + M::PART), run);
  AcWalk w(*run, t.nx, a.c.n_kv, a.c.n_seq);
  const int tok_tile = t.tok_tile;
  auto key_tiles = [&]() { return w.x * AM_KEYS + 128 < q.used + q.m ? 2 : 1; };
  auto rows_of = [&](int u) { return min(tok_tile, q.m - (first + u) * tok_tile) * a.rep; };
  bool more = w.start(cost), ok = true;
  if (warp == 0) {
    // ------------------------------------------------------------------ producer
    uint32_t kn = 0, qn = 0;
    const int page = 1 << a.c.page_shift, pieces = 128 >> a.c.page_shift;
    const int tile = lane / (pieces * NH), piece = lane % (pieces * NH) / NH, half = lane % NH;
    const int none = a.c.n_pages * a.c.n_kv * page;  // a row behind the pool: such a copy fills with zeros
    while (ok && more) {
      const int na = key_tiles(), end = q.used + q.m;
      int row = none;
      if (tile < na) {
        const int slot = w.x * AM_KEYS + tile * 128 + piece * page;
        const int p = slot < end ? kv_page(a.c, w.s, slot) : -1;
        if (p >= 0) row = (p * a.c.n_kv + w.h) * page;
      }
      const uint32_t kb = kn & 1;
      if (!(ok = wait(M::K_EMPTY + 8 * kb, ((kn >> 1) & 1) ^ 1))) break;
      if (lane == 0) ptx::mbar_arrive_expect_tx(base + M::K_FULL + 8 * kb, na * M::TILE);
      __syncwarp();
      if (tile < na)
        ptx::tma_load_2d(base + M::K + (2 * kb + tile) * M::TILE + half * M::HALF + piece * page * 128, &tmap_k, 64 * half, row,
                         base + M::K_FULL + 8 * kb);
      ++kn;
      for (int u = w.u0; u < w.u1; ++u, ++qn) {
        const uint32_t qb = qn & 1;
        if (!(ok = wait(M::Q_EMPTY + 8 * qb, ((qn >> 1) & 1) ^ 1))) break;
        if (lane == 0) ptx::mbar_arrive_expect_tx(base + M::Q_FULL + 8 * qb, NH * 128 * a.rep * tok_tile);
        __syncwarp();
        if (lane < NH)
          ptx::tma_load_3d(base + M::Q + qb * M::TILE + lane * M::HALF, &tmap_q, 64 * lane, w.h * a.rep, q.t0 + (first + u) * tok_tile,
                           base + M::Q_FULL + 8 * qb);
      }
      if (ok) more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AM_WAIT_LOAD);
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    uint32_t kn = 0, qn = 0, un[2] = {0, 0};
    while (ok && more) {
      const int na = key_tiles();
      const uint32_t kb = kn & 1;
      if (!(ok = wait(M::K_FULL + 8 * kb, (kn >> 1) & 1))) break;
      ++kn;
      for (int u = w.u0; ok && u < w.u1; ++u, ++qn) {
        const uint32_t qb = qn & 1;
        if (!(ok = wait(M::Q_FULL + 8 * qb, (qn >> 1) & 1))) break;
        const uint32_t idesc = ptx::idesc_bf16(128, (rows_of(u) + 15) & ~15, false);
        for (int x = 0; x < na; ++x) {
          const uint32_t b = un[x] & 1;
          if (!(ok = wait(M::S_EMPTY + 8 * (2 * x + b), ((un[x] >> 1) & 1) ^ 1))) break;
          ++un[x];
          ptx::tc_fence_after_sync();
          if (ptx::elect_one()) {
            const uint64_t kd = ptx::smem_desc_sw128(base + M::K + (2 * kb + x) * M::TILE), qd = ptx::smem_desc_sw128(base + M::Q + qb * M::TILE);
#pragma unroll
            for (int k = 0; k < HD / 16; ++k) {
              const uint32_t off = ((k / 4) * M::HALF + (k % 4) * 32) >> 4;
              ptx::mma_bf16_ss(tmem + 256 * x + 128 * b, kd + off, qd + off, idesc, k != 0);
            }
            ptx::mma_commit(base + M::S_FULL + 8 * (2 * x + b));
          }
          __syncwarp();
        }
        if (!ok) break;
        if (ptx::elect_one()) {
          ptx::mma_commit(base + M::Q_EMPTY + 8 * qb);
          if (u + 1 == w.u1) ptx::mma_commit(base + M::K_EMPTY + 8 * kb);
        }
        __syncwarp();
      }
      if (ok) more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AM_WAIT_MMA);
  } else if (warp == 2) {
    // ------------------------------------------------------------------ row statistics
    pdl_wait_before();  // in every CTA, with work or without: what follows this kernel relies on it for what came before
    uint32_t n = 0;
    while (ok && more) {
      for (int u = w.u0; u < w.u1; ++u, ++n) {
        const uint32_t b = n & 3;
        const int rows = rows_of(u);
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = lane + 32 * i, tk = c / a.rep;
          v[i] = c < rows ? a.lse[static_cast<long long>(q.t0 + (first + u) * tok_tile + tk) * a.n_heads + w.h * a.rep + c - tk * a.rep] : INFINITY;
        }
        if (!(ok = wait(M::L_EMPTY + 8 * b, ((n >> 2) & 1) ^ 1))) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          reinterpret_cast<float*>(sm + M::LSE)[128 * b + lane + 32 * i] = -v[i];  // what the sums add
          const uint32_t live = __ballot_sync(0xffffffffu, v[i] != INFINITY);
          if (lane == 0) reinterpret_cast<uint32_t*>(sm + M::LIVE)[4 * b + i] = live;
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(base + M::L_FULL + 8 * b);
      }
      if (ok) more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AM_WAIT_LSE);
  } else if (warp >= 4) {
    // ------------------------------------------------------------------ sums, one slot per thread
    const int x = (warp - 4) >> 3, turn = ((warp - 4) >> 2) & 1;  // key tile; every other unit (its accumulator is `turn`)
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const int r = (warp & 3) * 32 + lane;
    const uint64_t scale_x2 = ptx::pack_f32x2(__float_as_uint(a.scale2), __float_as_uint(a.scale2));
    const uint32_t s_addr = tmem + 256 * x + 128 * turn + lane_base, s_bar = 8 * (2 * x + turn);
    float* other = reinterpret_cast<float*>(sm + M::SUM) + 128 * x + r;
    uint32_t un = 0, n = 0, mine = 0, items = 0;  // units of this key tile, of all items, of this warp's turn; items of this key tile
    while (ok && more) {
      const bool active = x < key_tiles();
      const int slot = w.x * AM_KEYS + 128 * x + r, j = slot - q.used, end = q.used + q.m;
      const bool whole = w.u0 == 0 && w.u1 == w.units;
      // where the sum goes, and what is there: read ahead of the sums
      long long row = -1;
      float before = 0.0f;
      if (active && turn == 0 && slot < end && whole) {
        const int page = kv_page(a.c, w.s, slot);
        if (page >= 0) {
          row = kv_row(a.c, 0, page, w.h) + (slot & ((1 << a.c.page_shift) - 1));
          before = a.c.mass[row];
        }
      }
      float got[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      for (int u = w.u0; u < w.u1; ++u, ++n) {
        const uint32_t b = n & 3;
        if (!(ok = wait(M::L_FULL + 8 * b, (n >> 2) & 1))) break;
        if (active && (un++ & 1) == static_cast<uint32_t>(turn)) {
          if (!(ok = wait(M::S_FULL + s_bar, mine & 1))) break;
          ++mine;
          ptx::tc_fence_after_sync();
          const int rows = rows_of(u);
          const int tok0 = (first + u) * tok_tile, last_slot = w.x * AM_KEYS + 128 * x + 127;
          const bool masked = last_slot >= q.used + (a.b.parent ? 0 : tok0 + 1);
          uint32_t s[2][32];
          ptx::tmem_ld_32x32b_x32(s_addr, s[0]);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            if (32 * c >= rows) break;
            ptx::tmem_ld_wait();
            if (32 * c + 32 < rows) {
              ptx::tmem_ld_32x32b_x32(s_addr + 32 * (c + 1), s[(c + 1) & 1]);
            } else {
              ptx::tc_fence_before_sync();
              __syncwarp();
              if (lane == 0) ptx::mbar_arrive(base + M::S_EMPTY + s_bar);
            }
            uint32_t see = ptx::lds32(base + M::LIVE + 16 * b + 4 * c);
            if (masked && j >= 0) see &= am_columns(a, q, j, tok0, 32 * c);
            am_add(s[c & 1], see, base + M::LSE + 512 * b + 128 * c, scale_x2, a.scale2, got);
          }
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(base + M::L_EMPTY + 8 * b);
      }
      if (!ok) break;
      float sum = (got[0] + got[1]) + (got[2] + got[3]);
      if (active) {
        // turn 1 hands its sum to turn 0
        if (turn == 1) {
          if (!(ok = wait(M::SUM_EMPTY + 8 * x, (items & 1) ^ 1))) break;
          *other = sum;
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(base + M::SUM_FULL + 8 * x);
        } else {
          if (!(ok = wait(M::SUM_FULL + 8 * x, items & 1))) break;
          sum += *other;
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(base + M::SUM_EMPTY + 8 * x);
          if (whole) {
            if (row >= 0) a.c.mass[row] = before + sum;
          } else {
            const int cut = w.u0 == 0 ? 1 : 0;
            t.part[(2 * static_cast<long long>(blockIdx.x) + cut) * AM_KEYS + 128 * x + r] = sum;
            if (threadIdx.x == 128) cuts[cut] = AtCut{w.s, w.x, w.h, w.u1 == w.units};
          }
        }
        ++items;
      }
      more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AM_WAIT_SUM);
  }

  // ---- teardown: every role leaves through here, also after a timeout ----
  __syncwarp();
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (*failed) {
    // Failure path only: copies and MMAs that nobody waited for may still be in flight.
    if (warp == 1) {
      if (ptx::elect_one()) ptx::mma_commit(base + M::DRAIN);
      __syncwarp();
      ptx::mbar_wait(base + M::DRAIN, 0, 2000000LL);
    }
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000LL) {}
    __syncthreads();
  }
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

// Adds the parts of the items that were cut, from the CTA in which an item begins onwards.
__global__ void __launch_bounds__(AM_KEYS) attn_mass_join_kernel(const __grid_constant__ AmArgs t, int n_ctas) {
  pdl_enter();
  const AcArgs& a = t.a;
  const int c0 = blockIdx.x;
  const AtCut head = t.cuts[2 * c0 + 1];
  if (head.s < 0) return;
  KvSeq q;
  if (!kv_seq(a.c, a.b, head.s, q)) return;
  const int slot = head.x * AM_KEYS + threadIdx.x;
  if (slot >= q.used + q.m) return;
  float sum = t.part[(2 * static_cast<long long>(c0) + 1) * AM_KEYS + threadIdx.x];
  for (int c = c0 + 1; c < n_ctas; ++c) {
    const AtCut cut = t.cuts[2 * c];
    if (cut.s < 0) continue;  // a CTA whose run is empty
    sum += t.part[2 * static_cast<long long>(c) * AM_KEYS + threadIdx.x];
    if (cut.ends) break;
  }
  const int page = kv_page(a.c, head.s, slot);
  if (page >= 0) a.c.mass[kv_row(a.c, 0, page, head.h) + (slot & ((1 << a.c.page_shift) - 1))] += sum;
}

// The same for at most two row tiles a sequence (trees, states), where reading the keys is what counts: the queries of a
// (sequence, kv head) stay in shared memory while its keys stream by.  An item is a (sequence, kv head), a unit 256 slots; a unit
// belongs to one CTA, so nothing is left to join.  Warps as above; with two row tiles four warps take each accumulator of a
// unit, with one they take every other unit of their key tile.  The sums go through shared memory to warp 3, which fetched
// the places that they are added to one unit earlier: page, weight and sum one after the other in the summing warps cost
// them 2 us a unit.  (In the form above, whose items reload their queries, trees of 48 tokens over 8000 slots took 84 us; here 48.)
template <int HD>
struct AnSmem {
  static constexpr uint32_t TILE = 128 * HD * 2, HALF = 128 * 128;
  static constexpr uint32_t K = 0, Q = 4 * TILE, LSE = Q + 2 * TILE;               // K [2][2 tiles], Q [2], LSE [2][128]
  static constexpr uint32_t LIVE = LSE + 1024, SUM = LIVE + 32, BAR = SUM + 4096;  // LIVE [2][4] bits, SUM [2][2 turns][256]
  static constexpr uint32_t K_FULL = BAR, K_EMPTY = K_FULL + 16, Q_FULL = K_EMPTY + 16, Q_EMPTY = Q_FULL + 8, S_FULL = Q_EMPTY + 8,
                            S_EMPTY = S_FULL + 32, L_FULL = S_EMPTY + 32, L_EMPTY = L_FULL + 8, SUM_FULL = L_EMPTY + 8, SUM_EMPTY = SUM_FULL + 16,
                            DRAIN = SUM_EMPTY + 16;
  static constexpr uint32_t MISC = DRAIN + 8, RUN = MISC + 8, PART = RUN + 32;
  static constexpr uint32_t BYTES = PART + 8 * (AM_THREADS / 32 + 1) + 1024;
  static constexpr uint32_t LAUNCH = BYTES > 120 * 1024 ? BYTES : 120 * 1024;  // one CTA per SM: it takes all of tensor memory
};

template <int HD>
__global__ void __launch_bounds__(AM_THREADS, 1)
attn_mass_near_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ AmArgs t) {
  using M = AnSmem<HD>;
  constexpr int NH = HD / 64;
  extern __shared__ unsigned char at_smem_raw[];
  const uint32_t raw = ptx::smem_u32(at_smem_raw), base = (raw + 1023u) & ~1023u;
  unsigned char* sm = at_smem_raw + (base - raw);
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(sm + M::MISC);
  volatile uint32_t* failed = misc + 1;
  const uint32_t failed_addr = base + M::MISC + 4;
  const AcArgs& a = t.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto wait = [&](uint32_t bar, uint32_t parity) {
    return __any_sync(0xffffffffu, ptx::mbar_wait_abortable(base + bar, parity, failed_addr));
  };
  auto give_up = [&](int stage) {
    report_timeout(stage);
    *failed = 1u;
  };
  if (threadIdx.x == 0) {
    *failed = 0u;
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(base + M::K_FULL + 8 * i, 1);
      ptx::mbar_init(base + M::K_EMPTY + 8 * i, 1);
      ptx::mbar_init(base + M::SUM_FULL + 8 * i, 16);
      ptx::mbar_init(base + M::SUM_EMPTY + 8 * i, 1);
    }
    ptx::mbar_init(base + M::Q_FULL, 1);
    ptx::mbar_init(base + M::Q_EMPTY, 1);
    ptx::mbar_init(base + M::L_FULL, 1);
    ptx::mbar_init(base + M::L_EMPTY, 16);
    for (int i = 0; i < 4; ++i) {
      ptx::mbar_init(base + M::S_FULL + 8 * i, 1);
      ptx::mbar_init(base + M::S_EMPTY + 8 * i, 4);
    }
    ptx::mbar_init(base + M::DRAIN, 1);
    ptx::mbar_init_fence();
    ptx::tma_prefetch_desc(&tmap_q);
    ptx::tma_prefetch_desc(&tmap_k);
  }
  if (warp == 1) {
    ptx::tmem_alloc(base + M::MISC, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = misc[0];
  pdl_launch_next();  // as in the form above: warp 2 waits
  KvSeq q;
  auto cost = [&](int s, int) {  // units of (sequence, head)
    if (!kv_seq(a.c, a.b, s, q) || q.m == 0 || (a.tree_ok && !a.tree_ok[s])) return 0;
    return (q.used + q.m + AM_KEYS - 1) / AM_KEYS;
  };
  AcRun* run = reinterpret_cast<AcRun*>(sm + M::RUN);
  ac_run_start(cost, a.c.n_seq, a.c.n_kv, 1, AM_THREADS, reinterpret_cast<long long*>(sm + M::PART), run);
  AcWalk w(*run, a.c.n_kv, 1, a.c.n_seq);  // w.x: the kv head
  const int tok_tile = t.tok_tile;
  auto key_tiles = [&](int u) { return u * AM_KEYS + 128 < q.used + q.m ? 2 : 1; };
  auto row_tiles = [&]() { return q.m > tok_tile ? 2 : 1; };
  auto rows_of = [&](int rt) { return min(tok_tile, q.m - rt * tok_tile) * a.rep; };
  bool more = w.start(cost), ok = true;
  if (warp == 0) {
    // ------------------------------------------------------------------ producer
    uint32_t kn = 0, qn = 0;
    const int page = 1 << a.c.page_shift, pieces = 128 >> a.c.page_shift;
    const int tile = lane / (pieces * NH), piece = lane % (pieces * NH) / NH, half = lane % NH;
    const int none = a.c.n_pages * a.c.n_kv * page;  // a row behind the pool: such a copy fills with zeros
    while (ok && more) {
      const int rts = row_tiles(), end = q.used + q.m;
      auto row_of = [&](int u) {
        const int slot = u * AM_KEYS + tile * 128 + piece * page;
        const int p = tile < 2 && slot < end ? kv_page(a.c, w.s, slot) : -1;
        return p < 0 ? none : (p * a.c.n_kv + w.x) * page;
      };
      int row = row_of(w.u0);
      for (int u = w.u0; u < w.u1; ++u, ++kn) {
        const int na = key_tiles(u), row_next = u + 1 < w.u1 ? row_of(u + 1) : none;
        const uint32_t kb = kn & 1;
        if (!(ok = wait(M::K_EMPTY + 8 * kb, ((kn >> 1) & 1) ^ 1))) break;
        if (lane == 0) ptx::mbar_arrive_expect_tx(base + M::K_FULL + 8 * kb, na * M::TILE);
        __syncwarp();
        if (tile < na)
          ptx::tma_load_2d(base + M::K + (2 * kb + tile) * M::TILE + half * M::HALF + piece * page * 128, &tmap_k, 64 * half, row,
                           base + M::K_FULL + 8 * kb);
        if (u == w.u0) {
          if (!(ok = wait(M::Q_EMPTY, (qn & 1) ^ 1))) break;
          ++qn;
          if (lane == 0) ptx::mbar_arrive_expect_tx(base + M::Q_FULL, rts * NH * 128 * a.rep * tok_tile);
          __syncwarp();
          if (lane < rts * NH)
            ptx::tma_load_3d(base + M::Q + (lane / NH) * M::TILE + (lane % NH) * M::HALF, &tmap_q, 64 * (lane % NH), w.x * a.rep,
                             q.t0 + (lane / NH) * tok_tile, base + M::Q_FULL);
        }
        row = row_next;
      }
      if (ok) more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AM_WAIT_LOAD);
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    uint32_t kn = 0, qn = 0, un[2] = {0, 0}, e_par = 0xf;  // products per key tile; phases of S_EMPTY, as bits
    while (ok && more) {
      const int rts = row_tiles();
      if (!(ok = wait(M::Q_FULL, qn & 1))) break;
      ++qn;
      for (int u = w.u0; ok && u < w.u1; ++u, ++kn) {
        const uint32_t kb = kn & 1;
        const int na = key_tiles(u);
        if (!(ok = wait(M::K_FULL + 8 * kb, (kn >> 1) & 1))) break;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if (x >= na || !ok) continue;
          for (int rt = 0; rt < rts; ++rt) {
            const uint32_t b = un[x]++ & 1, i = 2 * x + b;
            if (!(ok = wait(M::S_EMPTY + 8 * i, (e_par >> i) & 1))) break;
            e_par ^= 1u << i;
            ptx::tc_fence_after_sync();
            if (ptx::elect_one()) {
              const uint32_t idesc = ptx::idesc_bf16(128, (rows_of(rt) + 15) & ~15, false);
              const uint64_t kd = ptx::smem_desc_sw128(base + M::K + (2 * kb + x) * M::TILE), qd = ptx::smem_desc_sw128(base + M::Q + rt * M::TILE);
#pragma unroll
              for (int k = 0; k < HD / 16; ++k) {
                const uint32_t off = ((k / 4) * M::HALF + (k % 4) * 32) >> 4;
                ptx::mma_bf16_ss(tmem + 128 * i, kd + off, qd + off, idesc, k != 0);
              }
              ptx::mma_commit(base + M::S_FULL + 8 * i);
            }
            __syncwarp();
          }
        }
        if (!ok) break;
        if (ptx::elect_one()) {
          ptx::mma_commit(base + M::K_EMPTY + 8 * kb);
          if (u + 1 == w.u1) ptx::mma_commit(base + M::Q_EMPTY);
        }
        __syncwarp();
      }
      if (ok) more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AM_WAIT_MMA);
  } else if (warp == 2) {
    // ------------------------------------------------------------------ row statistics
    pdl_wait_before();
    uint32_t n = 0;
    while (ok && more) {
      const int rts = row_tiles();
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = lane + 32 * (i & 3), tk = c / a.rep, rt = i >> 2;
        v[i] = rt < rts && c < rows_of(rt)
                   ? a.lse[static_cast<long long>(q.t0 + rt * tok_tile + tk) * a.n_heads + w.x * a.rep + c - tk * a.rep]
                   : INFINITY;
      }
      if (!(ok = wait(M::L_EMPTY, (n & 1) ^ 1))) break;
      ++n;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        reinterpret_cast<float*>(sm + M::LSE)[lane + 32 * i] = -v[i];  // what the sums add
        const uint32_t live = __ballot_sync(0xffffffffu, v[i] != INFINITY);
        if (lane == 0) reinterpret_cast<uint32_t*>(sm + M::LIVE)[i] = live;
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(base + M::L_FULL);
      more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AM_WAIT_LSE);
  } else if (warp == 3) {
    // ------------------------------------------------------------------ sums into the cache, eight slots per lane
    uint32_t n = 0, un[2] = {0, 0};  // units; products of either key tile
    const int x = lane >> 4;         // key tile of this lane's slots
    const int slot_mask = (1 << a.c.page_shift) - 1;
    while (ok && more) {
      const int rts = row_tiles(), end = q.used + q.m;
      float* next_at = nullptr;
      float4 next[2];
      auto fetch = [&](int u) {
        const int slot = u * AM_KEYS + 8 * lane;
        next_at = nullptr;
        if (slot >= end) return;
        const int page = kv_page(a.c, w.s, slot);
        if (page < 0) return;
        next_at = a.c.mass + kv_row(a.c, 0, page, w.x) + (slot & slot_mask);
        next[0] = *reinterpret_cast<const float4*>(next_at);
        next[1] = *reinterpret_cast<const float4*>(next_at + 4);
      };
      fetch(w.u0);
      for (int u = w.u0; u < w.u1; ++u, ++n) {
        float* at = next_at;
        float m[8] = {next[0].x, next[0].y, next[0].z, next[0].w, next[1].x, next[1].y, next[1].z, next[1].w};
        if (u + 1 < w.u1) fetch(u + 1);
        const uint32_t buf = n & 1;
        if (!(ok = wait(M::SUM_FULL + 8 * buf, (n >> 1) & 1))) break;
        if (at) {
          const uint32_t first = rts == 2 ? 0 : (x ? un[1] : un[0]) & 1;
          const float* sums = reinterpret_cast<const float*>(sm + M::SUM) + (2 * buf + first) * AM_KEYS + 8 * lane;
#pragma unroll
          for (int i = 0; i < 8; ++i) m[i] += rts == 2 ? sums[i] + sums[AM_KEYS + i] : sums[i];
          const int slot = u * AM_KEYS + 8 * lane;
          if (slot + 8 <= end) {
            *reinterpret_cast<float4*>(at) = make_float4(m[0], m[1], m[2], m[3]);
            *reinterpret_cast<float4*>(at + 4) = make_float4(m[4], m[5], m[6], m[7]);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (slot + i < end) at[i] = m[i];
          }
        }
        un[0] += rts;
        if (key_tiles(u) == 2) un[1] += rts;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(base + M::SUM_EMPTY + 8 * buf);
      }
      if (ok) more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AM_WAIT_SUM);
  } else {
    // ------------------------------------------------------------------ sums, one slot per thread
    const int x = (warp - 4) >> 3, turn = ((warp - 4) >> 2) & 1;  // key tile; its accumulator
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const int r = (warp & 3) * 32 + lane;
    const uint64_t scale_x2 = ptx::pack_f32x2(__float_as_uint(a.scale2), __float_as_uint(a.scale2));
    const uint32_t s_addr = tmem + 256 * x + 128 * turn + lane_base, s_bar = 8 * (2 * x + turn);
    uint32_t un = 0, n = 0, units = 0, mine = 0;  // products of this key tile, items, units, products of this turn
    while (ok && more) {
      const int rts = row_tiles();
      if (!(ok = wait(M::L_FULL, n & 1))) break;
      ++n;
      for (int u = w.u0; u < w.u1; ++u, ++units) {
        const bool active = x < key_tiles(u);
        // the row tile in this turn's accumulator, if there is one
        const bool first = (un & 1) == static_cast<uint32_t>(turn);
        const bool take = active && (rts == 2 || first);
        const int rt = rts == 2 && !first ? 1 : 0;
        if (active) un += rts;
        float sum = 0.0f;
        if (take) {
          if (!(ok = wait(M::S_FULL + s_bar, mine & 1))) break;
          ++mine;
          ptx::tc_fence_after_sync();
          const int rows = rows_of(rt), tok0 = rt * tok_tile, j = u * AM_KEYS + 128 * x + r - q.used;
          const bool masked = u * AM_KEYS + 128 * x + 127 >= q.used + (a.b.parent ? 0 : tok0 + 1);
          float got[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          uint32_t s[2][32];
          ptx::tmem_ld_32x32b_x32(s_addr, s[0]);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            if (32 * c >= rows) break;
            ptx::tmem_ld_wait();
            if (32 * c + 32 < rows) {
              ptx::tmem_ld_32x32b_x32(s_addr + 32 * (c + 1), s[(c + 1) & 1]);
            } else {
              ptx::tc_fence_before_sync();
              __syncwarp();
              if (lane == 0) ptx::mbar_arrive(base + M::S_EMPTY + s_bar);
            }
            uint32_t see = ptx::lds32(base + M::LIVE + 16 * rt + 4 * c);
            if (masked && j >= 0) see &= am_columns(a, q, j, tok0, 32 * c);
            am_add(s[c & 1], see, base + M::LSE + 512 * rt + 128 * c, scale_x2, a.scale2, got);
          }
          sum = (got[0] + got[1]) + (got[2] + got[3]);
        }
        const uint32_t buf = units & 1;
        if (!(ok = wait(M::SUM_EMPTY + 8 * buf, ((units >> 1) & 1) ^ 1))) break;
        if (take) reinterpret_cast<float*>(sm + M::SUM)[(2 * buf + turn) * AM_KEYS + 128 * x + r] = sum;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(base + M::SUM_FULL + 8 * buf);
      }
      if (!ok) break;
      if (lane == 0) ptx::mbar_arrive(base + M::L_EMPTY);
      more = w.next(cost);
      __syncwarp();
    }
    if (!ok && lane == 0) give_up(AM_WAIT_SUM);
  }

  // ---- teardown: every role leaves through here, also after a timeout ----
  __syncwarp();
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (*failed) {
    // Failure path only: copies and MMAs that nobody waited for may still be in flight.
    if (warp == 1) {
      if (ptx::elect_one()) ptx::mma_commit(base + M::DRAIN);
      __syncwarp();
      ptx::mbar_wait(base + M::DRAIN, 0, 2000000LL);
    }
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000LL) {}
    __syncthreads();
  }
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------
struct AcPlan {
  bool few;                                    // few rows: attn_few_kernel; else tiles
  int rows_cap;                                // rows kept of a cut item
  int score_rows, runs, join_slots;            // few rows
  int tok_tile, nx, ctas;                      // tiles
  size_t lse_bytes, ml_bytes, o_bytes, cut_bytes, sum_bytes, score_bytes, anc_bytes, ok_bytes, run_bytes;
  size_t bytes() const { return lse_bytes + ml_bytes + o_bytes + cut_bytes + sum_bytes + score_bytes + 2 * anc_bytes + ok_bytes + run_bytes; }
  // Does every coordinate of the call fit?
  bool launchable(const KvView& c) const {
    return (static_cast<long long>(c.n_pages) * c.n_kv + 1) << c.page_shift <= INT_MAX &&
           static_cast<long long>(c.n_seq) * ((static_cast<long long>(c.max_pages) << c.page_shift) / AF_SLOTS + 1) * c.n_kv <= INT_MAX;
  }
};

inline size_t ac_up(size_t v) { return (v + 255) / 256 * 256; }

// Sizes alone decide: the lengths are known on the device only.
inline AcPlan ac_plan(const KvView& c, int T, int max_new, int n_heads) {
  AcPlan p = {};
  const int rep = n_heads / c.n_kv;
  const long long rows = static_cast<long long>(max_new) * rep;
  p.few = rows <= AF_ROWS;
  p.lse_bytes = ac_up(static_cast<size_t>(T) * n_heads * 4);
  p.anc_bytes = max_new <= BITRL_TREE_MAX_TOKENS ? ac_up(static_cast<size_t>(T) * AC_TREE_WORDS * 4) : 0;  // twice
  p.ok_bytes = ac_up(static_cast<size_t>(c.n_seq) * 4);
  if (p.few) {
    p.rows_cap = static_cast<int>(rows);
    p.score_rows = rows <= 4 ? 4 : rows <= 8 ? 8 : 16;
    // one run per resident warp: with two to four times as many, parts and their joining cost more than the evener end gives
    // (when tried, 100k slots of one sequence: 66 us against 82 .. 117; 128 sequences of up to 4096: 133 against 137 .. 139)
    p.runs = sm_count() * AF_WARPS * AF_CTAS;
    // slots of a CTA of the join: long stretches, unless they would leave SMs idle (2000 slots of one sequence: 13.3 us in
    // stretches of 2048, 9 us in stretches of 512, less in shorter ones; 128 sequences: no difference)
    const long long stretches = ((c.max_pages << c.page_shift) + 2047) / 2048;
    p.join_slots = stretches * c.n_seq * c.n_kv < 4LL * sm_count() ? (stretches * c.n_seq * c.n_kv < sm_count() / 8 ? 256 : 512) : 2048;
    p.ml_bytes = ac_up(static_cast<size_t>(2 * p.runs) * p.rows_cap * 8);
    p.o_bytes = ac_up(static_cast<size_t>(2 * p.runs) * p.rows_cap * c.hd * 4);
    p.run_bytes = 256 + ac_up(static_cast<size_t>(c.n_seq) * c.n_kv * 4);
    p.score_bytes = c.mass ? ac_up((static_cast<size_t>(c.n_pages) * c.n_kv << c.page_shift) * p.score_rows * 4) : 0;
  } else {
    p.tok_tile = 128 / rep;
    p.nx = (max_new + 2 * p.tok_tile - 1) / (2 * p.tok_tile);
    p.rows_cap = static_cast<int>(rows < 256 ? rows : 256);
    p.ctas = sm_count();
    p.ml_bytes = ac_up(static_cast<size_t>(2 * p.ctas) * p.rows_cap * 8);
    p.o_bytes = ac_up(static_cast<size_t>(2 * p.ctas) * p.rows_cap * c.hd * 4);
    p.cut_bytes = ac_up(static_cast<size_t>(4 * p.ctas) * sizeof(AtCut));  // of the forward and of the weights kernel
    p.sum_bytes = ac_up(static_cast<size_t>(2 * p.ctas) * AM_KEYS * 4);
  }
  return p;
}

template <class K>
bitrl_status ac_smem(K kernel, size_t bytes, bool (&done)[64]) {
  int dev = 0;
  BITRL_CUDA(cudaGetDevice(&dev));
  if (dev >= 0 && dev < 64 && !done[dev]) {
    BITRL_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)));
    done[dev] = true;
  }
  return BITRL_OK;
}

// Tensor map over bf16 data, 128-byte swizzle, boxes of 64 innermost elements.
inline bitrl_status ac_tensor_map(CUtensorMap* m, const void* p, int dims, const cuuint64_t* size, const cuuint64_t* stride,
                                  const cuuint32_t* box) {
  const encode_tiled_fn encode = get_encode_tiled();
  if (!encode) return cuda_fail(cudaErrorNotSupported);
  const cuuint32_t ones[3] = {1, 1, 1};
  const CUresult r = encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, dims, const_cast<void*>(p), size, stride, box, ones,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? BITRL_OK : cuda_fail(cudaErrorInvalidValue);
}

template <int HD>
bitrl_status launch_attention_cached_hd(const AcArgs& a, const AcPlan& p, bool mass, float* sums, const AfArgs& f, cudaStream_t st) {
  bitrl_status s;
  CUtensorMap mk, mv;
  const int page = 1 << a.c.page_shift;
  const cuuint64_t kv_size[2] = {HD, static_cast<cuuint64_t>(a.c.n_pages) * a.c.n_kv * page}, kv_stride[1] = {HD * 2};
  const cuuint32_t kv_box[2] = {64, static_cast<cuuint32_t>(p.few ? AF_SLOTS : page)};
  if ((s = ac_tensor_map(&mk, a.c.k, 2, kv_size, kv_stride, kv_box)) != BITRL_OK) return s;
  if ((s = ac_tensor_map(&mv, a.c.v, 2, kv_size, kv_stride, kv_box)) != BITRL_OK) return s;
  if (p.few) {
    static bool done[2][64] = {};
    const bool one = p.rows_cap <= 8;
    if ((s = one ? ac_smem(attn_few_kernel<HD, 1>, af_smem_bytes<HD>(), done[0])
                 : ac_smem(attn_few_kernel<HD, 2>, af_smem_bytes<HD>(), done[1])) != BITRL_OK) return s;
    const dim3 grid(p.runs / AF_WARPS);
    const dim3 join(static_cast<unsigned>(a.c.n_seq) * a.c.n_kv, ((a.c.max_pages << a.c.page_shift) + f.join_slots - 1) / f.join_slots);
    BITRL_CUDA(one ? launch_pdl(attn_few_kernel<HD, 1>, grid, dim3(AF_THREADS), af_smem_bytes<HD>(), st, mk, mv, f)
                   : launch_pdl(attn_few_kernel<HD, 2>, grid, dim3(AF_THREADS), af_smem_bytes<HD>(), st, mk, mv, f));
    BITRL_CUDA(p.score_rows == 4   ? launch_pdl(attn_few_join_kernel<HD, 4>, join, dim3(AJ_THREADS), 0, st, f)
               : p.score_rows == 8 ? launch_pdl(attn_few_join_kernel<HD, 8>, join, dim3(AJ_THREADS), 0, st, f)
                                   : launch_pdl(attn_few_join_kernel<HD, 16>, join, dim3(AJ_THREADS), 0, st, f));
    count_launch(2);
  } else {
    CUtensorMap mq;
    const cuuint64_t q_size[3] = {HD, static_cast<cuuint64_t>(a.n_heads), static_cast<cuuint64_t>(a.b.T)};
    const cuuint64_t q_stride[2] = {HD * 2, static_cast<cuuint64_t>(a.n_heads) * HD * 2};
    const cuuint32_t q_box[3] = {64, static_cast<cuuint32_t>(a.rep), static_cast<cuuint32_t>(p.tok_tile)};
    if ((s = ac_tensor_map(&mq, a.q, 3, q_size, q_stride, q_box)) != BITRL_OK) return s;
    static bool done[64] = {false};
    if ((s = ac_smem(attn_tiles_kernel<HD>, AtSmem<HD>::LAUNCH, done)) != BITRL_OK) return s;
    const AtArgs t{a, p.tok_tile, p.nx, p.rows_cap};
    BITRL_CUDA(launch_pdl(attn_tiles_kernel<HD>, dim3(p.ctas), dim3(AT_THREADS), AtSmem<HD>::LAUNCH, st, mq, mk, mv, t));
    BITRL_CUDA(launch_pdl(attn_tiles_join_kernel<HD>, dim3(p.ctas, (p.rows_cap + 31) / 32), dim3(256), 0, st, t, p.ctas));
    count_launch(2);
    if (mass) {
      const AmArgs m{a, p.tok_tile, ((a.c.max_pages << a.c.page_shift) + AM_KEYS - 1) / AM_KEYS, sums, a.cuts + 2 * p.ctas};
      if (p.nx == 1) {  // at most two row tiles a sequence
        static bool near_done[64] = {false};
        if ((s = ac_smem(attn_mass_near_kernel<HD>, AnSmem<HD>::LAUNCH, near_done)) != BITRL_OK) return s;
        BITRL_CUDA(launch_pdl(attn_mass_near_kernel<HD>, dim3(p.ctas), dim3(AM_THREADS), AnSmem<HD>::LAUNCH, st, mq, mk, m));
        count_launch(1);
        return BITRL_OK;
      }
      static bool mass_done[64] = {false};
      if ((s = ac_smem(attn_mass_kernel<HD>, AmSmem<HD>::LAUNCH, mass_done)) != BITRL_OK) return s;
      BITRL_CUDA(launch_pdl(attn_mass_kernel<HD>, dim3(p.ctas), dim3(AM_THREADS), AmSmem<HD>::LAUNCH, st, mq, mk, m));
      BITRL_CUDA(launch_pdl(attn_mass_join_kernel, dim3(p.ctas), dim3(AM_KEYS), 0, st, m, p.ctas));
      count_launch(2);
    }
  }
  return BITRL_OK;
}

bitrl_status launch_attention_cached(const KvView& c, const KvBatch& b, const void* q, int n_heads, bool mass, void* att,
                                     void* workspace, cudaStream_t st) {
  const AcPlan p = ac_plan(c, b.T, b.max_new, n_heads);
  unsigned char* w = static_cast<unsigned char*>(workspace);
  auto take = [&](size_t bytes) {
    unsigned char* at = w;
    w += bytes;
    return at;
  };
  AcArgs a;
  a.c = c;
  a.b = b;
  a.q = static_cast<const unsigned short*>(q);
  a.att = static_cast<unsigned short*>(att);
  a.n_heads = n_heads;
  a.rep = n_heads / c.n_kv;
  a.scale2 = static_cast<float>(1.4426950408889634 / sqrt(static_cast<double>(c.hd)));
  a.lse = reinterpret_cast<float*>(take(p.lse_bytes));
  a.part_ml = reinterpret_cast<float2*>(take(p.ml_bytes));
  a.part_o = reinterpret_cast<float*>(take(p.o_bytes));
  a.cuts = reinterpret_cast<AtCut*>(take(p.cut_bytes));
  float* sums = reinterpret_cast<float*>(take(p.sum_bytes));
  float* scores = reinterpret_cast<float*>(take(p.score_bytes));
  unsigned char* runs = take(p.run_bytes);
  uint32_t* anc = reinterpret_cast<uint32_t*>(take(p.anc_bytes));
  uint32_t* desc = reinterpret_cast<uint32_t*>(take(p.anc_bytes));
  int* ok = reinterpret_cast<int*>(take(p.ok_bytes));
  a.anc = b.parent ? anc : nullptr;
  a.desc = b.parent ? desc : nullptr;
  a.tree_ok = b.parent ? ok : nullptr;
  const AfArgs f{a, p.rows_cap, p.score_rows, p.runs, p.join_slots, mass ? scores : nullptr, reinterpret_cast<AfHead*>(runs),
                 reinterpret_cast<int*>(runs + 256)};
  if (b.parent) {
    BITRL_CUDA(launch_pdl(attn_tree_kernel, dim3(c.n_seq), dim3(BITRL_TREE_MAX_TOKENS), 0, st, c, b, anc, desc, ok));
    count_launch(1);
  }
  return c.hd == 128 ? launch_attention_cached_hd<128>(a, p, mass, sums, f, st) : launch_attention_cached_hd<64>(a, p, mass, sums, f, st);
}

}  // namespace bitrl

// Gradients of attention over whole sequences on the sm_100a tensor cores (bf16, head sizes up to 128).
//
//   S = Q K^T, dP = dO V^T, P = exp(scale S - lse), dS = P (dP - delta), delta = rowsum(dO * O);
//   dQ = scale dS K,  dV = P^T dO,  dK = scale dS^T Q.
// Two kernels, one per side: k_seq_dq_tc has 128 query rows of a head and goes over their keys (S, dP, dQ: three products per
// tile), k_seq_dkv_tc has 128 tokens of a KV head and goes over the queries of all heads of its group (S^T, dP^T, dV, dK: four).
// Seven products instead of the five that one kernel would need, but every sum stays in one CTA's tensor memory: no atomics on
// results, no fp32 copy of dQ in memory, the heads of a group added for free, and the same bits every time.
//
// Both have the forward kernel's roles: a TMA producer, an MMA issuer, two warps that pass the stages on (and patch tiles that some
// row does not see in full) and eight softmax warps, here two threads per row with half of the columns each.  P and dS are
// rounded to bf16 and are A operands in tensor memory, over the S and dP they came from; the tile that was K-major for the first
// products is read MN-major for the second.
//  * k_seq_dkv_tc, per tile of queries: dV and the next S^T run while dS is computed, dK and the next dP^T while the next P is.
//    At D = 128 tensor memory is full (S, dP, dV, dK: 4 x 128 columns) and nothing is buffered twice.  -lse and -delta of a tile's queries, which
//    run along a thread's columns, lie in shared memory.
//  * k_seq_dq_tc, per tile of keys: S is buffered twice and dS goes over the S it came from, so that softmax warps never wait.
// Bound by the chain of a step (scores, exponentials, dS, sums), of which tensor memory holds no second: the tensor pipe is busy 56 %
// (dQ) and 62 % (dK, dV) of the time.  Two sequences of 8192 tokens, 32 + 8 heads of 128, full attention: 1.32 ms (1.25 PFLOP/s of its
// three products) and 1.81 ms (1.22 PFLOP/s of its four).
// Non-finite values of tokens that a row does not see: they are taken out of the operands of the second products (0 * NaN), and
// the rows that do see them become NaN through lse, delta or a bit per key.
#include <cooperative_groups.h>

#include "ptenc_seq_tc.cuh"

namespace {

enum { B_KIND, B_START, B_LEN, B_PIN, B_CAP, B_E, B_HEAD, B_TILE, B_A, B_B, B_C, B_N, B_WORDS };

__device__ __forceinline__ SeqView bwd_view(volatile int* d) {
  SeqView s;
  s.start = d[B_START]; s.len = d[B_LEN]; s.pin = d[B_PIN]; s.cap = d[B_CAP]; s.e = d[B_E];
  return s;
}

template <int D>
struct BSmem {
  static constexpr int TILE = (D / 64) * HALF;
  // Two rings: of the tiles that two products use far apart (K, or Q) and of the others (V, or dO).
  static constexpr int RA = D == 128 ? 3 : 5, RB = D == 128 ? 2 : 5, STAGES = RA + RB;
  static constexpr int OFF_AB = STAGES * TILE;                       // the item's own two tiles
  static constexpr int OFF_STAT = OFF_AB + 2 * TILE;                 // float [2][2][128], see the kernels
  static constexpr int OFF_CLC = OFF_STAT + 4 * TM * 4;
  static constexpr int OFF_BAD = OFF_CLC + 16;                       // uint32 [2][2][4]: rows of patched tiles with non-finite values
  static constexpr int OFF_DESC = OFF_BAD + 64;
  static constexpr int OFF_BAR = (OFF_DESC + 2 * B_WORDS * 4 + 7) / 8 * 8;
  static constexpr int N_BAR = 3 * STAGES + 23;
  static constexpr int OFF_MISC = OFF_BAR + N_BAR * 8;
  static constexpr int TOTAL = OFF_MISC + 16;
  static_assert(TOTAL <= 232448, "shared memory of one CTA");
  // where the nt-th tile of a CTA lies, and its barriers' parity
  __device__ static __forceinline__ uint32_t stage_a(uint32_t nt) { return nt % RA; }
  __device__ static __forceinline__ uint32_t stage_b(uint32_t nt) { return RA + nt % RB; }
  __device__ static __forceinline__ uint32_t phase_a(uint32_t nt) { return (nt / RA) & 1; }
  __device__ static __forceinline__ uint32_t phase_b(uint32_t nt) { return (nt / RB) & 1; }
};

// Barriers after the stages' full, empty and ready ones.
enum { X_A_FULL, X_A_EMPTY, X_B_FULL, X_B_EMPTY, X_O_READ, X_SUMS, X_S_FULL, X_S_FULL1, X_DP_FULL, X_P_READY, X_DS_READY,
       X_ACC_FULL, X_ACC_EMPTY, X_STAT_FULL, X_STAT_FULL1, X_STAT_EMPTY, X_STAT_EMPTY1, X_ITEM_FULL, X_ITEM_FULL1, X_ITEM_EMPTY,
       X_ITEM_EMPTY1, X_CLC, X_DRAIN };

// What a CTA of either kernel does first; returns the TMEM base.  b_users: who frees the item's second tile; now: whether it waits for
// the kernel before.
template <int D>
__device__ __forceinline__ uint32_t bwd_begin(uint8_t* smem, uint32_t sb, int tid, int warp, int b_users, bool now) {
  using SM = BSmem<D>;
  constexpr int NS = SM::STAGES;
  volatile int* misc = reinterpret_cast<volatile int*>(smem + SM::OFF_MISC);
  const uint32_t full = sb + SM::OFF_BAR, empty = full + 8 * NS, ready = empty + 8 * NS, x = ready + 8 * NS;
  if (tid == 0) {
    for (int s = 0; s < NS; ++s) { bar_init(full + 8 * s, 1); bar_init(empty + 8 * s, 1); bar_init(ready + 8 * s, 1); }
    const int counts[] = {1, 1, 1, b_users, 8, 8, 1, 1, 1, 8, 8, 1, 8, 2, 2, 8, 8, 1, 1, 1 + 2 + 8, 1 + 2 + 8, 1, 1};
    for (int i = 0; i <= X_DRAIN; ++i) bar_init(x + 8 * i, counts[i]);
    misc[0] = misc[2] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sb + SM::OFF_MISC + 4), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (now) tree_after_previous();
  fence_before();
  __syncthreads();
  fence_after();
  return (uint32_t)misc[1];
}

// The producer of either kernel.  find(item, d) fills an item's words (all but the kind) and says whether it is one; own(d, which) and
// entry(d, tile, which) load the item's own two tiles and its ring entries.  EXTRA: one more entry of the second ring in front of an
// item's, entry(d, 0, 2).  ONCE: the CTA's own item and no other.  Everything is asked for as soon as its place is free, the next item's
// tiles under the end of the last one.
template <int D, bool EXTRA, bool ONCE, typename FIND, typename OWN, typename ENTRY>
__device__ __forceinline__ void bwd_produce(uint8_t* smem, uint32_t sb, FIND find, OWN own, ENTRY entry) {
  using SM = BSmem<D>;
  constexpr int NS = SM::STAGES, TILE = SM::TILE;
  volatile int* desc = reinterpret_cast<volatile int*>(smem + SM::OFF_DESC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + SM::OFF_MISC);
  const uint32_t full = sb + SM::OFF_BAR, empty = full + 8 * NS, x = empty + 16 * NS;
  uint32_t na = 0, nb = 0, seq = 0, asked = 0;           // ring entries, items and takeovers so far
  uint32_t got_a = 0, got_b = 0;                         // the items' own tiles
  bool okay = true;
  int item = (int)blockIdx.x;
  while (okay) {
    const uint32_t slot = seq & 1;
    if (item < 0) {
      if (bar_wait(x + 8 * (X_ITEM_EMPTY + slot), ((seq >> 1) & 1) ^ 1, abort_flag)) {
        desc[slot * B_WORDS + B_KIND] = 0;
        bar_arrive(x + 8 * (X_ITEM_FULL + slot));
      } else {
        okay = false;
      }
      break;
    }
    abort_flag[2] = abort_flag[2] + 1;                     // numbers looked at
    if (!ONCE) {
      bar_expect(x + 8 * X_CLC, 16);
      clc_ask(sb + SM::OFF_CLC, x + 8 * X_CLC);
    }
    int w[B_WORDS];
    if (find(item, w)) {
      if (!bar_wait(x + 8 * (X_ITEM_EMPTY + slot), ((seq >> 1) & 1) ^ 1, abort_flag)) { okay = false; break; }
      volatile int* d = desc + slot * B_WORDS;
      for (int i = B_START; i < B_WORDS; ++i) d[i] = w[i];
      d[B_KIND] = 1;
      bar_arrive(x + 8 * (X_ITEM_FULL + slot));
      if (!bar_wait(x + 8 * X_A_EMPTY, (seq & 1) ^ 1, abort_flag)) { okay = false; break; }
      bar_expect(x + 8 * X_A_FULL, TILE);
      own(w, 0, sb + SM::OFF_AB, x + 8 * X_A_FULL);
      ++got_a;
      auto ring_a = [&](int t) -> bool {
        const uint32_t s = SM::stage_a(na);
        if (!bar_wait(empty + 8 * s, SM::phase_a(na) ^ 1, abort_flag)) return false;
        bar_expect(full + 8 * s, (uint32_t)TILE);
        entry(w, t, 0, sb + s * TILE, full + 8 * s);
        ++na;
        return true;
      };
      auto ring_b = [&](int t, int which) -> bool {
        const uint32_t s = SM::stage_b(nb);
        if (!bar_wait(empty + 8 * s, SM::phase_b(nb) ^ 1, abort_flag)) return false;
        bar_expect(full + 8 * s, (uint32_t)TILE);
        entry(w, t, which, sb + s * TILE, full + 8 * s);
        ++nb;
        return true;
      };
      if (!ring_a(0) || !bar_wait(x + 8 * X_B_EMPTY, (seq & 1) ^ 1, abort_flag)) { okay = false; break; }
      bar_expect(x + 8 * X_B_FULL, TILE);
      own(w, 1, sb + SM::OFF_AB + TILE, x + 8 * X_B_FULL);
      ++got_b;
      ++seq;
      if (EXTRA) okay = ring_b(0, 2);
      okay = okay && ring_b(0, 1);
      for (int t = 1; t < w[B_N] && okay; ++t) okay = ring_a(t) && ring_b(t, 1);
    }
    if (ONCE) {
      item = -1;
    } else if (okay) {
      if (!bar_wait(x + 8 * X_CLC, asked & 1, abort_flag)) { okay = false; break; }
      item = clc_answer(sb + SM::OFF_CLC);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      ++asked;
    }
  }
  if (!okay) {
    *abort_flag = 1;
    if (!ONCE) bar_drain(x + 8 * X_CLC, asked & 1);
  }
  // whatever the other roles did, copies in flight land before the shared memory goes away
  for (uint32_t i = 1; i <= (uint32_t)SM::RA && i <= na; ++i) bar_drain(full + 8 * SM::stage_a(na - i), SM::phase_a(na - i));
  for (uint32_t i = 1; i <= (uint32_t)SM::RB && i <= nb; ++i) bar_drain(full + 8 * SM::stage_b(nb - i), SM::phase_b(nb - i));
  if (!okay && got_a > 0) bar_drain(x + 8 * X_A_FULL, (got_a - 1) & 1);
  if (!okay && got_b > 0) bar_drain(x + 8 * X_B_FULL, (got_b - 1) & 1);
}

template <int D>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int h, int row, uint32_t bar) {
#pragma unroll
  for (int hf = 0; hf < D / 64; ++hf) tma_3d(dst + hf * HALF, map, hf * 64, h, row, bar);
}

// D (fp32, 128 x 128) = A B^T, both K-major tiles in shared memory.
template <int D>
__device__ __forceinline__ void mma_scores(uint32_t d, uint32_t a, uint32_t b) {
  const uint64_t da = desc_k(a), db = desc_k(b);
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    const uint64_t off = ((k >> 2) * HALF + (k & 3) * 32) >> 4;
    mma_ss(d, da + off, db + off, tt_idesc(SN, 0), k > 0);
  }
}
// D (fp32, 128 x D) += A B, A bf16 in tensor memory (64 columns of it at the start of each half of `a`), B 128 rows as they lie.
template <int D>
__device__ __forceinline__ void mma_sums(uint32_t d, uint32_t a, uint32_t b, bool replace) {
  const uint64_t db = desc_mn(b);
#pragma unroll
  for (int k = 0; k < 8; ++k) mma_ts(d, a + (k >> 2) * 64 + (k & 3) * 8, db + (k * 2048 >> 4), tt_idesc(D, 1), k > 0 ? 1u : (replace ? 0u : 1u));
}

// One row of a gradient, columns [c0, c1), from tensor memory.
template <int D>
__device__ __forceinline__ void store_row(uint32_t t, int c0, int c1, float f, __nv_bfloat16* to, int Dr, bool real, bool wide) {
#pragma unroll 1
  for (int c = c0; c < c1; c += 16) {
    float o[16];
    ld16(t + c, o);
    wait_ld();
    uint32_t pk[8];
#pragma unroll
    for (int y = 0; y < 16; y += 2) pk[y >> 1] = tt_pack(o[y] * f, o[y + 1] * f);
    if (!real) continue;
    if (c + 16 <= Dr) tt_store(to + c, pk, wide);
    else if (c < Dr) *reinterpret_cast<uint4*>(to + c) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
  }
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

__device__ __forceinline__ void bwd_end(uint32_t tmem, int warp) {
  fence_before();
  __syncthreads();
  if (warp == 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------ dq
// Also leaves -lse (base 2) and -delta of every row for the other kernel, [Hq][n] each.
//
// delta = rowsum(dO * O) is off by the rounding of O to bf16.  Where a row sees many tokens that is little beside the products it
// is taken from; where it sees few, O has the size of V and dQ comes out at up to 2.5 times the error of its other roundings.  So delta
// is corrected by what is left of sum_j p_ij (dP_ij - delta), which is zero for the right delta: items of few tiles (DQ_FIRST) go over
// their tiles twice, the first time for that sum alone; the others form it beside dS, and the other kernel gets the corrected delta.
// (Error of dQ in the 2-norm, sequences of 8192 tokens / rollouts under a window of 1024: 2.7e-3 without, 2.5e-3 with up to 4 tiles, 2.4e-3
// with up to 6 or 8, both passes of the rollouts 1.77, 1.82, 1.85 and 2.00 ms then.)
constexpr int DQ_FIRST = 6;
template <int D>
__global__ void __launch_bounds__(ST_THREADS, 1)
k_seq_dq_tc(const __grid_constant__ SeqArgs a, const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
            const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmO) {
  using SM = BSmem<D>;
  constexpr int NS = SM::STAGES, TILE = SM::TILE;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sb = tt_u32(smem);
  volatile int* desc = reinterpret_cast<volatile int*>(smem + SM::OFF_DESC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + SM::OFF_MISC);
  uint32_t* s_bad = reinterpret_cast<uint32_t*>(smem + SM::OFF_BAD);           // [tile & 1][4]: keys with non-finite values
  const uint32_t full = sb + SM::OFF_BAR, empty = full + 8 * NS, ready = empty + 8 * NS, X = ready + 8 * NS;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t tmem = bwd_begin<D>(smem, sb, tid, warp, 2, true);
  const uint32_t tS = tmem, tP = tmem + 2 * SN, tA = tmem + 3 * SN;            // S [2], dP, dQ
  auto range_of = [](volatile int* d) { SeqRange r; r.np = d[B_A]; r.s0 = d[B_B]; r.s1 = d[B_C]; return r; };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(ST_REGS_LOW));
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, bar_wait(bar, parity, abort_flag)); };
    auto next = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, item_wait(bar, parity, abort_flag, abort_flag + 2)); };
    if (warp == 0) {
      if (lane == 0)
        bwd_produce<D, true, false>(smem, sb,
          [&](int item, int* w) -> bool {
            const int at = (int)gridDim.x - 1 - item, number = at / a.Hq;
            SeqView s;
            int tile;
            if (!seq_find(a, number, TM, &s, &tile)) return false;
            const int i0 = tile * TM;
            const SeqRange r = seq_keys(s, i0, min(i0 + TM, s.len) - 1, SN);
            w[B_START] = s.start; w[B_LEN] = s.len; w[B_PIN] = s.pin; w[B_CAP] = s.cap; w[B_E] = s.e; w[B_HEAD] = at - number * a.Hq;
            const int n = seq_count(r);
            w[B_TILE] = tile; w[B_A] = r.np; w[B_B] = r.s0; w[B_C] = r.s1;
            w[B_N] = n <= DQ_FIRST ? 2 * n : n;
            return true;
          },
          [&](const int* w, int t, uint32_t dst, uint32_t bar) {
            load_tile<D>(dst, t == 0 ? &tmQ : &tmG, w[B_HEAD], w[B_START] + w[B_TILE] * TM, bar);
          },
          [&](const int* w, int t, int which, uint32_t dst, uint32_t bar) {
            SeqRange r;
            if (which == 2) { load_tile<D>(dst, &tmO, w[B_HEAD], w[B_START] + w[B_TILE] * TM, bar); return; }
            r.np = w[B_A]; r.s0 = w[B_B]; r.s1 = w[B_C];
            load_tile<D>(dst, which ? &tmV : &tmK, w[B_HEAD] / a.g, w[B_START] + seq_at(r, t < seq_count(r) ? t : t - seq_count(r)) * SN, bar);
          });
    } else if (warp == 1) {
      // ================================================================ MMA issuer
      const bool leader = tt_elect();
      uint32_t seq = 0, nt = 0;                            // items, tiles
      bool okay = true;
      auto send = [&](uint32_t bar) { if (leader) commit(bar); __syncwarp(); };
      while (okay) {
        const uint32_t slot = seq & 1;
        if (!next(X + 8 * (X_ITEM_FULL + slot), (seq >> 1) & 1)) { okay = false; break; }
        volatile int* d = desc + slot * B_WORDS;
        const int kind = __shfl_sync(0xffffffffu, d[B_KIND], 0), n = __shfl_sync(0xffffffffu, d[B_N], 0);
        const int pre = __shfl_sync(0xffffffffu, seq_count(range_of(d)) < d[B_N] ? d[B_N] / 2 : 0, 0);      // steps without dQ
        if (kind == 0) break;
        __syncwarp();
        if (leader) bar_arrive(X + 8 * (X_ITEM_EMPTY + slot));
        if (!wait(X + 8 * X_A_FULL, seq & 1)) { okay = false; break; }
        auto scores = [&](int t) -> bool {                 // S of tile t
          const uint32_t s = SM::stage_a(nt + t), buf = (nt + t) & 1;
          if (!wait(ready + 8 * s, SM::phase_a(nt + t))) return false;
          if (leader) {
            mma_scores<D>(tS + buf * SN, sb + SM::OFF_AB, sb + s * TILE);
            commit(X + 8 * (X_S_FULL + buf));
            if (t == n - 1) commit(X + 8 * X_A_EMPTY);     // the next item's Q may come
          }
          __syncwarp();
          return true;
        };
        auto values = [&](int t) -> bool {                 // dP of tile t
          const uint32_t at = nt + t + seq + 1, s = SM::stage_b(at);             // an O tile per item is in that ring too
          if (t == 0 && !wait(X + 8 * X_B_FULL, seq & 1)) return false;
          if (!wait(ready + 8 * s, SM::phase_b(at))) return false;
          if (leader) {
            mma_scores<D>(tP, sb + SM::OFF_AB + TILE, sb + s * TILE);
            commit(X + 8 * X_DP_FULL);
            commit(empty + 8 * s);
            if (t == n - 1) commit(X + 8 * X_B_EMPTY);
          }
          __syncwarp();
          return true;
        };
        okay = scores(0) && values(0) && (n == 1 || scores(1));
        for (int t = 0; t < n && okay; ++t) {
          if (!wait(X + 8 * X_DS_READY, (nt + t) & 1)) { okay = false; break; }
          fence_after();
          if (t + 1 < n && !values(t + 1)) { okay = false; break; }
          if (t == pre && !wait(X + 8 * X_ACC_EMPTY, (seq & 1) ^ 1)) { okay = false; break; }
          const uint32_t s = SM::stage_a(nt + t);
          if (leader) {
            if (t >= pre) mma_sums<D>(tA, tS + ((nt + t) & 1) * SN, sb + s * TILE, t == pre);
            commit(empty + 8 * s);
          }
          __syncwarp();
          if (t + 2 < n && !scores(t + 2)) { okay = false; break; }
        }
        if (!okay) break;
        send(X + 8 * X_ACC_FULL);
        nt += n;
        ++seq;
      }
      if (leader) {
        if (!okay) *abort_flag = 1;
        commit(X + 8 * X_DRAIN);
        bar_drain(X + 8 * X_DRAIN, 0);
      }
      __syncwarp();
    } else {
      // ================================================================ passes the stages on: warp 2 the K tiles, warp 3 the V tiles
      const int me = warp - 2;
      uint32_t seq = 0, nt = 0;
      bool okay = true;
      while (okay) {
        const uint32_t slot = seq & 1;
        if (!next(X + 8 * (X_ITEM_FULL + slot), (seq >> 1) & 1)) { okay = false; break; }
        volatile int* d = desc + slot * B_WORDS;
        if (d[B_KIND] == 0) break;
        const SeqView s = bwd_view(d);
        const SeqRange r = range_of(d);
        const int n = d[B_N], tiles = seq_count(r), i0 = d[B_TILE] * TM, low1 = s.low(i0 + TM - 1);
        if (me == 1) {
          // the O tile is the softmax warps' alone: when they have read it and dO, this warp frees both
          const uint32_t at = nt + seq, sg = SM::stage_b(at);
          if (!wait(full + 8 * sg, SM::phase_b(at)) || !wait(X + 8 * X_O_READ, seq & 1)) { okay = false; break; }
          if (lane == 0) {
            bar_arrive(ready + 8 * sg);                    // nobody waits for it, but the stage's phases go on
            bar_arrive(empty + 8 * sg);
            bar_arrive(X + 8 * X_B_EMPTY);
          }
          __syncwarp();
        }
        for (int t = 0; t < n; ++t) {
          // Each ring has its own warp, which waits for each of its tiles in turn and without which none is used: a wait tells a
          // stage's phase from the one two rounds before or after.
          const uint32_t at = me == 0 ? nt + t : nt + t + seq + 1, sg = me == 0 ? SM::stage_a(at) : SM::stage_b(at);
          if (!wait(full + 8 * sg, me == 0 ? SM::phase_a(at) : SM::phase_b(at))) { okay = false; break; }
          if (me == 0) {
            const int tile = seq_at(r, t < tiles ? t : t - tiles);
            uint32_t* bad = s_bad + 4 * ((nt + t) & 1);    // read with the tile two before
            if (!wait(X + 8 * (X_STAT_EMPTY + ((nt + t) & 1)), (((nt + t) >> 1) & 1) ^ 1)) { okay = false; break; }
            if (!seq_all(s, i0, low1, tile * SN, tile * SN + SN - 1)) {
              if (lane < 4) bad[lane] = 0;
              __syncwarp();
              patch_tile(smem + sg * TILE, D / 64, tile * SN, s.len, 0, 1, bad);
            }
          }
          __syncwarp();
          if (lane == 0) bar_arrive(ready + 8 * sg);
        }
        if (!okay) break;
        __syncwarp();
        if (lane == 0) bar_arrive(X + 8 * (X_ITEM_EMPTY + slot));
        ++seq;
        nt += n;
      }
      if (!okay && lane == 0) *abort_flag = 1;
    }
  } else {
    // ================================================================ softmax: two threads per row, half of a tile's keys each
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(ST_REGS_HIGH));
    const int half = (warp - 4) >> 2, quarter = warp & 3, lrow = 32 * quarter + lane;
    const uint32_t lane_off = (uint32_t)(32 * quarter) << 16;
    const float sl2 = a.scale * ST_LOG2E;
    float* s_sums = reinterpret_cast<float*>(smem + SM::OFF_STAT);             // [item & 1][half][row]
    uint32_t seq = 0, nt = 0;
    bool fine = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
      if (fine && !bar_wait(bar, parity, abort_flag)) { fine = false; *abort_flag = 1; }
    };
    while (true) {
      const uint32_t slot = seq & 1;
      if (fine && !item_wait(X + 8 * (X_ITEM_FULL + slot), (seq >> 1) & 1, abort_flag, abort_flag + 2)) { fine = false; *abort_flag = 1; }
      if (!__all_sync(0xffffffffu, fine)) break;
      volatile int* d = desc + slot * B_WORDS;
      if (d[B_KIND] == 0) break;
      const SeqView s = bwd_view(d);
      const SeqRange r = range_of(d);
      const int n = d[B_N], tiles = seq_count(r), pre = n - tiles, i0 = d[B_TILE] * TM, h = d[B_HEAD], row = i0 + lrow,
                low = s.low(row), low1 = s.low(i0 + TM - 1);
      const bool real = row < s.len;
      // delta from the O and dO tiles in shared memory: both threads of a row form it, so that no barrier stands between the warps.
      // (Read from memory, rows far apart, it cost 8000 cycles an item; so 1000.)
      const long long orow = (long long)(s.start + row) * a.Hq + h;
      const float nlse = real ? -a.lse[orow] * ST_LOG2E : 0.f;
      const uint32_t oat = nt + seq;
      wait(X + 8 * X_B_FULL, seq & 1);
      wait(full + 8 * SM::stage_b(oat), SM::phase_b(oat));
      float sum = 0.f;
      {
        const uint8_t* to = smem + SM::stage_b(oat) * TILE + lrow * 128;
        const uint8_t* tg = smem + SM::OFF_AB + TILE + lrow * 128;
        float part[2] = {0.f, 0.f};
#pragma unroll 4
        for (int c = 0; c < D / 8; ++c) {
          const int at = (c >> 3) * HALF + (((c & 7) ^ (lrow & 7)) << 4);
          const uint4 u = *reinterpret_cast<const uint4*>(to + at), v = *reinterpret_cast<const uint4*>(tg + at);
          const __nv_bfloat162* x = reinterpret_cast<const __nv_bfloat162*>(&u);
          const __nv_bfloat162* y = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 p = __bfloat1622float2(x[k]), q = __bfloat1622float2(y[k]);
            part[k & 1] = fmaf(p.x, q.x, fmaf(p.y, q.y, part[k & 1]));
          }
        }
        sum = part[0] + part[1];
      }
      __syncwarp();
      if (lane == 0) bar_arrive(X + 8 * X_O_READ);
      float ndelta = -sum;
      const bool alone = s.alone(row);
      const uint64_t scl2 = tt_two(sl2, sl2), nlse2 = tt_two(nlse, nlse);
      uint64_t nd2 = tt_two(ndelta, ndelta), rest = 0ull;
      // adds both halves' rests to delta and leaves it for the other kernel
      auto correct = [&]() {
        float* sums = s_sums + (seq & 1) * 2 * TM;       // of the item before last, which everybody has read
        float lo, hi;
        tt_both(rest, lo, hi);
        sums[half * TM + lrow] = lo + hi;
        __syncwarp();
        if (lane == 0) bar_arrive(X + 8 * X_SUMS);
        wait(X + 8 * X_SUMS, seq & 1);
        ndelta -= sums[lrow] + sums[TM + lrow];
        nd2 = tt_two(ndelta, ndelta);
        if (real && half == 0) {
          const long long at = (long long)h * a.n + s.start + row;
          a.delta[at] = ndelta;
          a.delta[(long long)a.Hq * a.n + at] = nlse;
        }
      };
#pragma unroll 1
      for (int t = 0; t < n; ++t, ++nt) {
        const uint32_t buf = nt & 1, ts = tS + buf * SN + 64 * half + lane_off, tp = tP + 64 * half + lane_off;
        const int j0 = seq_at(r, t < tiles ? t : t - tiles) * SN;
        if (pre > 0 && t == pre) correct();
        wait(X + 8 * (X_S_FULL + buf), (nt >> 1) & 1);
        fence_after();
        float p[64];
        ld32(ts, p);
        ld32(ts + 32, p + 32);
        wait_ld();
        const bool all = seq_all(s, i0, low1, j0, j0 + SN - 1);
#pragma unroll
        for (int y = 0; y < 64; y += 2) {
          tt_both(tt_fma2(tt_two(p[y], p[y + 1]), scl2, nlse2), p[y], p[y + 1]);
          p[y] = tt_ex2(p[y]);
          p[y + 1] = tt_ex2(p[y + 1]);
        }
        if (!all) {
          const uint32_t* bad = s_bad + 4 * buf + 2 * half;
          const uint32_t b0 = bad[0], b1 = bad[1];
          if ((b0 | b1) != 0) {                          // rare: keys with non-finite values
#pragma unroll
            for (int y = 0; y < 64; ++y)
              if (((y < 32 ? b0 : b1) >> (y & 31)) & 1u) p[y] = __int_as_float(0x7fffffff);
          }
        }
        wait(X + 8 * X_DP_FULL, nt & 1);
        fence_after();
        const int jh = j0 + 64 * half;
#pragma unroll
        for (int c = 0; c < 64; c += 32) {
          float x[32];
          uint32_t pk[16];
          ld32(tp + c, x);
          wait_ld();
#pragma unroll
          for (int y = 0; y < 32; y += 2)
            tt_both(tt_mul2(tt_add2(tt_two(x[y], x[y + 1]), nd2), tt_two(p[c + y], p[c + y + 1])), x[y], x[y + 1]);
          if (!all) {
            const uint32_t keep = alone ? 0u : st_run(0, row + 1, jh + c) & ~st_run(s.pin, low, jh + c);
#pragma unroll
            for (int y = 0; y < 32; ++y)
              if (!(keep & (1u << y))) x[y] = 0.f;
          }
#pragma unroll
          for (int y = 0; y < 32; y += 2) rest = tt_add2(rest, tt_two(x[y], x[y + 1]));
          if (t < pre) continue;
          // dS in bf16, half a step of 2^-8: the product's operands are of one type
#pragma unroll
          for (int y = 0; y < 32; y += 2) pk[y >> 1] = tt_pack(x[y], x[y + 1]);
          st16(ts + c / 2, pk);
        }
        wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) { bar_arrive(X + 8 * X_DS_READY); bar_arrive(X + 8 * (X_STAT_EMPTY + buf)); }
      }
      if (pre == 0) correct();
      wait(X + 8 * X_ACC_FULL, seq & 1);
      fence_after();
      const bool wide = (reinterpret_cast<uintptr_t>(a.dq) & 31) == 0 && a.D % 16 == 0 && a.dqs % 16 == 0;
      store_row<D>(tA + lane_off, half * (D / 2), (half + 1) * (D / 2), fine ? a.scale : __int_as_float(0x7fffffff),
                   static_cast<__nv_bfloat16*>(a.dq) + (s.start + row) * a.dqs + (long long)h * a.D, a.D, real, wide);
      fence_before();
      __syncwarp();
      if (lane == 0) { bar_arrive(X + 8 * X_ACC_EMPTY); bar_arrive(X + 8 * (X_ITEM_EMPTY + slot)); }
      ++seq;
    }
  }
  bwd_end(tmem, warp);
}

// ------------------------------------------------------------------------------------------------ dk, dv
// A pinned token is seen by all that follow, however long the sequence, where any other is seen by the W after it: an item of pinned
// tokens can take longer than all the rest of the call (19 rollouts of up to 6774 tokens, window 1024: 371 steps, the average per SM
// 226).  So items with more than twice the steps of the longest of the others are dealt to clusters of SPLIT_CTAS CTAs, a share of
// the steps each, in a launch of their own; the sums are joined through distributed shared memory, in order.  The other launch runs
// beside it: it starts when the last of the clusters have, and waits for them at its end.  Both passes of that call: 1620 us; 1853 in
// one launch with the pinned tiles first, 1654 with items of once the others' steps dealt out too.
constexpr int SPLIT_CTAS = 4;
// The steps of the item of a tile of tokens: tiles of queries from its own to the last that sees one of them, of every head.
__device__ __forceinline__ int dkv_tiles(const SeqView& s, int tile) {
  const int j0 = tile * TM, last = j0 < s.pin ? s.len - 1 : s.last(min(j0 + TM, s.len) - 1);
  return last / TM - tile + 1;
}
__device__ __forceinline__ bool dkv_long(const SeqArgs& a, const SeqView& s, int tile, int tiles) {
  return a.pins > 0 && tile * TM < s.pin && tiles * a.g > max(2 * ((a.window + TM - 1) / TM + 1) * a.g, SPLIT_CTAS);
}
// The long items' numbers: a.pins tiles of every sequence.
__device__ __forceinline__ bool dkv_find_long(const SeqArgs& a, int number, SeqView* s, int* tile) {
  const int b = number / a.pins;
  *tile = number - b * a.pins;
  return seq_at_start(a, b, s) && *tile * TM < min(s->pin, s->len) && dkv_long(a, *s, *tile, dkv_tiles(*s, *tile));
}

template <int D, bool SPLIT>
__global__ void __launch_bounds__(ST_THREADS, 1)
k_seq_dkv_tc(const __grid_constant__ SeqArgs a, const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
             const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmG) {
  using SM = BSmem<D>;
  constexpr int NS = SM::STAGES, TILE = SM::TILE;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sb = tt_u32(smem);
  volatile int* desc = reinterpret_cast<volatile int*>(smem + SM::OFF_DESC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + SM::OFF_MISC);
  uint32_t* s_bad = reinterpret_cast<uint32_t*>(smem + SM::OFF_BAD);           // [Q or dO][4], of the warp that patches
  volatile uint32_t* s_odd = s_bad + 8;                                        // [buffer]: rows of dO were patched
  float* s_stat = reinterpret_cast<float*>(smem + SM::OFF_STAT);               // [buffer][-lse or -delta][128]
  const uint32_t full = sb + SM::OFF_BAR, empty = full + 8 * NS, ready = empty + 8 * NS, X = ready + 8 * NS;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int part = SPLIT ? (int)blockIdx.x % SPLIT_CTAS : 0, own = (int)blockIdx.x / SPLIT_CTAS;      // a cluster's item
  SeqView sv;
  int sv_tile = 0;
  if (SPLIT) {
    tree_after_previous();
    __threadfence();
    tree_let_next_start();
    if (!dkv_find_long(a, own / a.Hkv, &sv, &sv_tile)) return;                 // the whole cluster agrees
  }
  // Without long items this launch waits for the gradients of the queries itself.  Beside them it does not: each of their CTAs has waited before it
  // let this launch start, so that kernel and all before it are over and what they wrote is in L2.  It is not promised to a reader that has
  // not waited itself, and L1 may hold lines of an earlier call: hence the fences on both sides, and delta and lse are read past L1.  (With a wait
  // of its own, that is behind the long items: both passes of 19 rollouts 1651 -> 1720 us, the gradients of one of 32768 tokens 1470 -> 1990.)
  if (!SPLIT && a.pins > 0) __threadfence();
  const uint32_t tmem = bwd_begin<D>(smem, sb, tid, warp, 1, !SPLIT && a.pins == 0);
  // S^T, dP^T, dV, dK.  Narrow heads leave tensor memory for a second S^T, which is formed while P is: dK and dV of two sequences of 8192
  // tokens, 32 + 8 heads of 64, 1.22 ms, 1.40 with one.  At D = 128 there is none; with P in shared memory in its stead, so that
  // S^T could be overwritten as soon as it had been read, and a Q tile less in its ring, 1.96 ms instead of 1.80.
  constexpr int BUFS = D == 128 ? 1 : 2;
  const uint32_t tS = tmem, tP = tmem + BUFS * SN, tV = tP + SN, tK = tV + D;
  static_assert((BUFS + 1) * SN + 2 * D <= 512, "tensor memory");
  // An item's steps: head by head, tiles B_TILE .. B_TILE + B_A - 1 of each; of them the B_N from B_B on.

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(ST_REGS_LOW));
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, bar_wait(bar, parity, abort_flag)); };
    auto next = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, item_wait(bar, parity, abort_flag, abort_flag + 2)); };
    if (warp == 0) {
      if (lane == 0)
        bwd_produce<D, false, SPLIT>(smem, sb,
          [&](int item, int* w) -> bool {
            SeqView s;
            int tile;
            if (SPLIT) { s = sv; tile = sv_tile; item = own; }
            else if (!seq_find(a, item / a.Hkv, TM, &s, &tile)) return false;
            const int tiles = dkv_tiles(s, tile), n = tiles * a.g;
            if (!SPLIT && dkv_long(a, s, tile, tiles)) return false;
            const int first = SPLIT ? (int)((long long)n * part / SPLIT_CTAS) : 0;
            w[B_START] = s.start; w[B_LEN] = s.len; w[B_PIN] = s.pin; w[B_CAP] = s.cap; w[B_E] = s.e; w[B_HEAD] = item % a.Hkv;
            w[B_TILE] = tile; w[B_A] = tiles; w[B_B] = first; w[B_C] = 0;
            w[B_N] = (SPLIT ? (int)((long long)n * (part + 1) / SPLIT_CTAS) : n) - first;
            return true;
          },
          [&](const int* w, int t, uint32_t dst, uint32_t bar) {
            load_tile<D>(dst, t == 0 ? &tmK : &tmV, w[B_HEAD], w[B_START] + w[B_TILE] * TM, bar);
          },
          [&](const int* w, int t, int which, uint32_t dst, uint32_t bar) {
            const int u = w[B_B] + t, hh = u / w[B_A];
            load_tile<D>(dst, which ? &tmG : &tmQ, w[B_HEAD] * a.g + hh, w[B_START] + (w[B_TILE] + u - hh * w[B_A]) * TM, bar);
          });
    } else if (warp == 1) {
      // ================================================================ MMA issuer
      const bool leader = tt_elect();
      uint32_t seq = 0, nt = 0;
      bool okay = true;
      auto send = [&](uint32_t bar) { if (leader) commit(bar); __syncwarp(); };
      while (okay) {
        const uint32_t slot = seq & 1;
        if (!next(X + 8 * (X_ITEM_FULL + slot), (seq >> 1) & 1)) { okay = false; break; }
        volatile int* d = desc + slot * B_WORDS;
        const int kind = __shfl_sync(0xffffffffu, d[B_KIND], 0), n = __shfl_sync(0xffffffffu, d[B_N], 0);
        if (kind == 0) break;
        __syncwarp();
        if (leader) bar_arrive(X + 8 * (X_ITEM_EMPTY + slot));
        if (!wait(X + 8 * X_A_FULL, seq & 1)) { okay = false; break; }
        // S^T (which 0) or dP^T (1) of tile t
        auto product = [&](int t, int which) -> bool {
          const uint32_t s = which ? SM::stage_b(nt + t) : SM::stage_a(nt + t);
          if (which && t == 0 && !wait(X + 8 * X_B_FULL, seq & 1)) return false;
          if (!wait(ready + 8 * s, which ? SM::phase_b(nt + t) : SM::phase_a(nt + t))) return false;
          if (leader) {
            mma_scores<D>(which ? tP : tS + (BUFS - 1) * ((nt + t) & 1) * SN, sb + SM::OFF_AB + which * TILE, sb + s * TILE);
            commit(X + 8 * (which ? X_DP_FULL : X_S_FULL + (BUFS - 1) * ((nt + t) & 1)));
            if (t == n - 1) commit(X + 8 * (which ? X_B_EMPTY : X_A_EMPTY));     // the next item's V or K may come
          }
          __syncwarp();
          return true;
        };
        okay = product(0, 0) && product(0, 1);
        if (okay && !wait(X + 8 * X_ACC_EMPTY, (seq & 1) ^ 1)) okay = false;
        for (int t = 0; t < n && okay; ++t) {
          const uint32_t sq = SM::stage_a(nt + t), sg = SM::stage_b(nt + t);
          if (BUFS == 2 && t + 1 < n && !product(t + 1, 0)) { okay = false; break; }
          if (!wait(X + 8 * X_P_READY, (nt + t) & 1)) { okay = false; break; }
          fence_after();
          if (leader) { mma_sums<D>(tV, tS + (BUFS - 1) * ((nt + t) & 1) * SN, sb + sg * TILE, t == 0); commit(empty + 8 * sg); }
          __syncwarp();
          if (BUFS == 1 && t + 1 < n && !product(t + 1, 0)) { okay = false; break; }
          if (!wait(X + 8 * X_DS_READY, (nt + t) & 1)) { okay = false; break; }
          fence_after();
          if (leader) { mma_sums<D>(tK, tP, sb + sq * TILE, t == 0); commit(empty + 8 * sq); }
          __syncwarp();
          if (t + 1 < n && !product(t + 1, 1)) { okay = false; break; }
        }
        if (!okay) break;
        send(X + 8 * X_ACC_FULL);
        nt += n;
        ++seq;
      }
      if (leader) {
        if (!okay) *abort_flag = 1;
        commit(X + 8 * X_DRAIN);
        bar_drain(X + 8 * X_DRAIN, 0);
      }
      __syncwarp();
    } else {
      // ================================================================ warp 2: Q tiles and -lse; warp 3: dO tiles and -delta
      const int me = warp - 2;
      uint32_t seq = 0, nt = 0;
      uint32_t* bad = s_bad + 4 * me;
      bool okay = true;
      while (okay) {
        const uint32_t slot = seq & 1;
        if (!next(X + 8 * (X_ITEM_FULL + slot), (seq >> 1) & 1)) { okay = false; break; }
        volatile int* d = desc + slot * B_WORDS;
        if (d[B_KIND] == 0) break;
        const SeqView s = bwd_view(d);
        const int n = d[B_N], tile0 = d[B_TILE], tiles = d[B_A], j0 = tile0 * TM, until = seq_seen_until(s, j0, j0 + TM - 1);
        int at = d[B_B] % tiles;                           // the tile within its head
        const float* stat = a.delta + (me == 0 ? (long long)a.Hq * a.n : 0) + ((long long)d[B_HEAD] * a.g + d[B_B] / tiles) * a.n + s.start;
        for (int t = 0; t < n; ++t) {
          const uint32_t sg = me == 0 ? SM::stage_a(nt + t) : SM::stage_b(nt + t), buf = (nt + t) & 1;
          const int i0 = (tile0 + at) * TM;
          // asked for early: rows past the end are not seen by anybody
          float v[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int i = i0 + lane + 32 * y;
            v[y] = i < s.len ? __ldcg(stat + i) : 0.f;     // past L1: see the launch of the others
          }
          if (!wait(full + 8 * sg, me == 0 ? SM::phase_a(nt + t) : SM::phase_b(nt + t))) { okay = false; break; }
          bool odd = false;
          if (!(i0 + TM <= s.len && j0 + TM - 1 <= i0 && i0 + TM - 1 <= until)) {
            if (lane < 4) bad[lane] = 0;
            __syncwarp();
            odd = patch_tile(smem + sg * TILE, D / 64, i0, s.len, 0, 1, bad);
            if (odd) {
              __syncwarp();
#pragma unroll
              for (int y = 0; y < 4; ++y)
                if ((bad[y] >> lane) & 1u) v[y] = __int_as_float(0x7fffffff);    // whoever sees the row becomes NaN
            }
          }
          __syncwarp();
          if (lane == 0) bar_arrive(ready + 8 * sg);
          if (!wait(X + 8 * (X_STAT_EMPTY + buf), (((nt + t) >> 1) & 1) ^ 1)) { okay = false; break; }
#pragma unroll
          for (int y = 0; y < 4; ++y) s_stat[buf * 2 * TM + me * TM + lane + 32 * y] = v[y];
          if (me == 1 && lane == 0) s_odd[buf] = odd;
          __syncwarp();
          if (lane == 0) bar_arrive(X + 8 * (X_STAT_FULL + buf));
          if (++at == tiles) { at = 0; stat += a.n; }
        }
        if (!okay) break;
        __syncwarp();
        if (lane == 0) bar_arrive(X + 8 * (X_ITEM_EMPTY + slot));
        ++seq;
        nt += n;
      }
      if (!okay && lane == 0) *abort_flag = 1;
    }
    __syncwarp();
    if (SPLIT) { cluster_sync(); cluster_sync(); }         // the softmax warps' two
  } else {
    // ================================================================ softmax: two threads per token, half of a tile's queries each
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(ST_REGS_HIGH));
    const int half = (warp - 4) >> 2, quarter = warp & 3, lrow = 32 * quarter + lane;
    const uint32_t lane_off = (uint32_t)(32 * quarter) << 16;
    const uint32_t tp = tP + 64 * half + lane_off;
    const float sl2 = a.scale * ST_LOG2E;
    const uint64_t scl2 = tt_two(sl2, sl2);
    uint32_t seq = 0, nt = 0;
    bool fine = true, done = false;
    auto wait = [&](uint32_t bar, uint32_t parity) {
      if (fine && !bar_wait(bar, parity, abort_flag)) { fine = false; *abort_flag = 1; }
    };
    while (true) {
      const uint32_t slot = seq & 1;
      if (fine && !item_wait(X + 8 * (X_ITEM_FULL + slot), (seq >> 1) & 1, abort_flag, abort_flag + 2)) { fine = false; *abort_flag = 1; }
      if (!__all_sync(0xffffffffu, fine)) break;
      volatile int* d = desc + slot * B_WORDS;
      if (d[B_KIND] == 0) break;
      const SeqView s = bwd_view(d);
      const int n = d[B_N], tile0 = d[B_TILE], tiles = d[B_A], j0 = tile0 * TM, col = j0 + lrow, last = s.last(col),
                until = seq_seen_until(s, j0, j0 + TM - 1);
      const bool alone = s.alone(col);
      const int skip = d[B_B] % tiles;
      int i0 = j0 + skip * TM, left = tiles - skip;
#pragma unroll 1
      for (int t = 0; t < n; ++t, ++nt) {
        const uint32_t buf = nt & 1, ts = tS + (BUFS - 1) * buf * SN + 64 * half + lane_off;
        const float* st = s_stat + buf * 2 * TM + 64 * half;
        const bool all = i0 + TM <= s.len && j0 + TM - 1 <= i0 && i0 + TM - 1 <= until;
        const int lo = col - i0 - 64 * half, hi = last - i0 - 64 * half;       // columns [lo, hi] see this token
        wait(X + 8 * (X_STAT_FULL + buf), (nt >> 1) & 1);
        wait(X + 8 * (X_S_FULL + (BUFS - 1) * buf), BUFS == 1 ? nt & 1 : (nt >> 1) & 1);
        fence_after();
        float p[64];
        ld32(ts, p);
        ld32(ts + 32, p + 32);
        wait_ld();
#pragma unroll
        for (int c = 0; c < 64; c += 32) {
          uint32_t pk[16];
#pragma unroll
          for (int y = c; y < c + 32; y += 4) {
            const float4 v = *reinterpret_cast<const float4*>(st + y);
            tt_both(tt_fma2(tt_two(p[y], p[y + 1]), scl2, tt_two(v.x, v.y)), p[y], p[y + 1]);
            tt_both(tt_fma2(tt_two(p[y + 2], p[y + 3]), scl2, tt_two(v.z, v.w)), p[y + 2], p[y + 3]);
#pragma unroll
            for (int z = 0; z < 4; ++z) p[y + z] = tt_ex2(p[y + z]);
          }
          if (!all) {
            if (s_odd[buf] != 0) {                       // rare: a non-finite row of dO, whose delta is NaN, reaches dV too
#pragma unroll
              for (int y = c; y < c + 32; ++y) p[y] = fmaf(0.f, st[TM + y], p[y]);
            }
            const uint32_t keep = st_run(lo, hi + 1, c);
#pragma unroll
            for (int y = 0; y < 32; ++y)
              if (!(keep & (1u << y))) p[c + y] = 0.f;
          }
          // P in bf16, half a step of 2^-8 per weight, as in the forward pass
#pragma unroll
          for (int y = 0; y < 32; y += 2) pk[y >> 1] = tt_pack(p[c + y], p[c + y + 1]);
          st16(ts + c / 2, pk);
        }
        wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(X + 8 * X_P_READY);
        wait(X + 8 * X_DP_FULL, nt & 1);
        fence_after();
        float x[64];
        ld32(tp, x);
        ld32(tp + 32, x + 32);
        wait_ld();
#pragma unroll
        for (int c = 0; c < 64; c += 32) {
          uint32_t pk[16];
#pragma unroll
          for (int y = c; y < c + 32; y += 4) {
            const float4 v = *reinterpret_cast<const float4*>(st + TM + y);
            tt_both(tt_mul2(tt_add2(tt_two(x[y], x[y + 1]), tt_two(v.x, v.y)), tt_two(p[y], p[y + 1])), x[y], x[y + 1]);
            tt_both(tt_mul2(tt_add2(tt_two(x[y + 2], x[y + 3]), tt_two(v.z, v.w)), tt_two(p[y + 2], p[y + 3])), x[y + 2], x[y + 3]);
          }
          if (!all) {
            const uint32_t keep = st_run(alone && i0 == j0 ? lo + 1 : lo, hi + 1, c);          // this token's own query is at lo
#pragma unroll
            for (int y = 0; y < 32; ++y)
              if (!(keep & (1u << y))) x[c + y] = 0.f;
          }
#pragma unroll
          for (int y = 0; y < 32; y += 2) pk[y >> 1] = tt_pack(x[c + y], x[c + y + 1]);
          st16(tp + c / 2, pk);
        }
        wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) { bar_arrive(X + 8 * X_DS_READY); bar_arrive(X + 8 * (X_STAT_EMPTY + buf)); }
        i0 += TM;
        if (--left == 0) { left = tiles; i0 = j0; }
      }
      wait(X + 8 * X_ACC_FULL, seq & 1);
      fence_after();
      if (SPLIT) {
        done = true;
        break;
      }
      const bool real = col < s.len;
      const float f = !fine ? __int_as_float(0x7fffffff) : half == 0 ? 1.f : a.scale;
      void* base = half == 0 ? a.dv : a.dk;
      const long long stride = half == 0 ? a.dvs : a.dks;
      const bool wide = (reinterpret_cast<uintptr_t>(base) & 31) == 0 && a.D % 16 == 0 && stride % 16 == 0;
      store_row<D>((half == 0 ? tV : tK) + lane_off, 0, D, f,
                   static_cast<__nv_bfloat16*>(base) + (s.start + col) * stride + (long long)d[B_HEAD] * a.D, a.D, real, wide);
      fence_before();
      __syncwarp();
      if (lane == 0) { bar_arrive(X + 8 * X_ACC_EMPTY); bar_arrive(X + 8 * (X_ITEM_EMPTY + slot)); }
      ++seq;
    }
    if (SPLIT) {
      // This CTA's sums to its shared memory, over the rings, which nothing writes to any more; then a share of the rows of all.
      constexpr int LD = D + 4;
      static_assert(2 * TM * LD * 4 <= NS * TILE, "sums lie over the rings");
      float* sums = reinterpret_cast<float*>(smem);      // [dV, dK][token][LD]
      float* mine = sums + (half * TM + lrow) * LD;
#pragma unroll 1
      for (int c = 0; c < D; c += 16) {
        float o[16];
        ld16((half == 0 ? tV : tK) + lane_off + c, o);
        wait_ld();
#pragma unroll
        for (int y = 0; y < 16; y += 4) {
          if (!fine || !done) o[y] = __int_as_float(0x7fffffff);
          *reinterpret_cast<float4*>(mine + c + y) = make_float4(o[y], o[y + 1], o[y + 2], o[y + 3]);
        }
      }
      __syncwarp();
      cluster_sync();
      const int j0 = sv_tile * TM, hk = own % a.Hkv;
#pragma unroll 1
      for (int x = part * 256 + tid - 128; x < 2 * TM * (D / 8); x += 256 * SPLIT_CTAS) {
        const int which = x / (TM * (D / 8)), row = x / (D / 8) % TM, c = 8 * (x % (D / 8));
        float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int q = 0; q < SPLIT_CTAS; ++q) {
          const float* from = cooperative_groups::this_cluster().map_shared_rank(sums + (which * TM + row) * LD + c, q);
          const float4 u = *reinterpret_cast<const float4*>(from), v = *reinterpret_cast<const float4*>(from + 4);
          o[0] += u.x; o[1] += u.y; o[2] += u.z; o[3] += u.w;
          o[4] += v.x; o[5] += v.y; o[6] += v.z; o[7] += v.w;
        }
        if (j0 + row >= sv.len || c >= a.D) continue;    // D is a multiple of 8
        const float f = which == 0 ? 1.f : a.scale;
        const long long at = (sv.start + j0 + row) * (which == 0 ? a.dvs : a.dks) + (long long)hk * a.D + c;
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(which == 0 ? a.dv : a.dk) + at) =
            make_uint4(tt_pack(o[0] * f, o[1] * f), tt_pack(o[2] * f, o[3] * f), tt_pack(o[4] * f, o[5] * f), tt_pack(o[6] * f, o[7] * f));
      }
      __syncwarp();
      cluster_sync();                                    // nobody leaves while its sums may be read
    }
  }
  if (!SPLIT && a.pins > 0) tree_after_previous();       // the long items: whoever waits for this launch waits for them too
  bwd_end(tmem, warp);
}

template <int D>
cudaError_t bwd_launch(const SeqArgs& a, int dev, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const CUtensorMap& g,
                       const CUtensorMap& o, unsigned numbers, cudaStream_t st) {
  static PtencOnce once;
  cudaError_t e = ptenc_first_use(once, dev, [] {
    cudaError_t x = ptenc_allow_smem(k_seq_dq_tc<D>, BSmem<D>::TOTAL);
    if (x == cudaSuccess) x = ptenc_allow_smem(k_seq_dkv_tc<D, true>, BSmem<D>::TOTAL);
    return x != cudaSuccess ? x : ptenc_allow_smem(k_seq_dkv_tc<D, false>, BSmem<D>::TOTAL);
  });
  if (e != cudaSuccess) return e;
  e = tree_launch(k_seq_dq_tc<D>, dim3(numbers * a.Hq), ST_THREADS, BSmem<D>::TOTAL, 0, st, a, q, k, v, g, o);
  if (e != cudaSuccess) return e;
  if (a.pins > 0)
    e = tree_launch(k_seq_dkv_tc<D, true>, dim3((unsigned)(a.pins * a.B) * a.Hkv * SPLIT_CTAS), ST_THREADS, BSmem<D>::TOTAL, SPLIT_CTAS, st,
                    a, q, k, v, g);
  if (e != cudaSuccess) return e;
  return tree_launch(k_seq_dkv_tc<D, false>, dim3(numbers * a.Hkv), ST_THREADS, BSmem<D>::TOTAL, 0, st, a, q, k, v, g);
}

}  // namespace

bool seq_backward_tc(const SeqArgs& args, int dtype, int dev, cudaStream_t st, cudaError_t* e) {
  SeqArgs a = args;
  const long long numbers = seq_numbers(a.n, a.B, TM);
  // Most tiles of a sequence that may be pinned; where there would be more numbers for them than for all the others, so that most
  // sequences are shorter than the window and the items of pinned tokens hardly longer than others, none is set apart.
  const long long pins = a.window > 0 && a.pinned != nullptr ? (a.window - 1 + TM - 1ll) / TM : 0;
  a.pins = pins * a.B <= numbers ? (int)pins : 0;
  if (dtype != PTENC_DTYPE_BF16 || a.D > 128 || SPLIT_CTAS * numbers * a.Hq >= (1ll << 31)) return false;
  CUtensorMap q, k, v, g, o;
  if (!seq_map(&q, a.q, a.D, a.Hq, a.n, a.qs) || !seq_map(&k, a.k, a.D, a.Hkv, a.n, a.ks) || !seq_map(&v, a.v, a.D, a.Hkv, a.n, a.vs) ||
      !seq_map(&g, a.dout, a.D, a.Hq, a.n, (long long)a.Hq * a.D) || !seq_map(&o, a.out, a.D, a.Hq, a.n, (long long)a.Hq * a.D))
    return false;
  *e = a.D <= 64 ? bwd_launch<64>(a, dev, q, k, v, g, o, (unsigned)numbers, st) : bwd_launch<128>(a, dev, q, k, v, g, o, (unsigned)numbers, st);
  return true;
}

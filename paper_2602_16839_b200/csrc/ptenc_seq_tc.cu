// Attention over whole sequences on the sm_100a tensor cores (bf16, head sizes up to 128).
//
// Forward.  A work item is 256 query rows of a (sequence, head): two row tiles of 128, each a stream with its own S, P and O in
// tensor memory (2 x (128 + D) columns), over the K/V tiles of 128 tokens that either sees.  Per CTA (one per SM; the grid is one CTA
// per item, late tiles first, and a running CTA takes over the next one that has not been launched, clusterlaunchcontrol):
//  * warp 0, one lane: producer.  Finds the item, TMA-loads its Q tiles and the K and V tiles (128-byte swizzle; plain loads) into a
//    ring of stages.  Heads narrower than the tile's 64 or 128 columns are filled up with zeros by the TMA unit.
//  * warp 1: issues the MMAs (one elected lane): S = Q K^T (both K-major in shared memory), O += P V (P bf16 in tensor memory over the
//    S it came from, V as it lies, MN-major).  One stream's products run under the other's softmax.
//  * warps 2 and 3: patches.  In V tiles that some row does not see in full they clear the rows past the sequence's end and take
//    non-finite values out of the others, since 0 * NaN would carry them into rows that do not see them; rows that do get them back
//    at the end.
//  * warps 4..11: softmax, four warps per stream, a row per thread with its 128 scores in registers: mask, maximum, running sum in
//    fp32 (base 2), P rounded to bf16.  O is rescaled only when the maximum has grown by more than 2^8.
//  * Bound by the chain from a tile's scores to its P, two streams deep: the tensor pipe and the exponentials' unit are each busy half of
//    the time; at D = 64 the exponentials' unit is busy 60 % of it, the tensor pipe 30 %.  16384 tokens, 28 + 4 heads of 128, causal: 1.61 ms
//    after a rest, 1.20 PFLOP/s, 1.77 ms for seconds on end.
//  * Every wait is bounded, by 8 ms in which the CTA does not get on at all (fwd_wait): one that runs out raises an abort flag, every role leaves, copies and products in flight are drained and
//    tensor memory is freed; the item's rows become NaN, those of items that the CTA had not begun may be left as they were.
#include "ptenc_seq_tc.cuh"

namespace {

constexpr int ST_ROWS = 2 * TM;                // query rows of an item

// ------------------------------------------------------------------------------------------------ layout
// Item description words in shared memory.  J_ODD .. J_ODD_END - 1: its tiles between the first and the last that values were taken out of.
enum { J_KIND, J_START, J_LEN, J_PIN, J_CAP, J_E, J_HEAD, J_ROW0, J_NP, J_S0, J_S1, J_N, J_ODD, J_ODD_END, J_WORDS };

template <int D>
struct FSmem {
  static constexpr int TILE = (D / 64) * HALF;                       // bytes of a 128-row tile
  static constexpr int RK = D == 128 ? 2 : 5, RV = D == 128 ? 3 : 5, STAGES = RK + RV;       // rings of K and V tiles
  static constexpr int OFF_Q = STAGES * TILE;                        // two Q tiles
  static constexpr int OFF_CLC = OFF_Q + 2 * TILE;                   // 16 bytes of answer
  static constexpr int OFF_DESC = OFF_CLC + 16;                      // int [2][J_WORDS]
  static constexpr int OFF_BAR = (OFF_DESC + 2 * J_WORDS * 4 + 7) / 8 * 8;
  static constexpr int N_BAR = 3 * STAGES + 20;
  static constexpr int OFF_MISC = OFF_BAR + N_BAR * 8;               // int [4]
  static constexpr int TOTAL = OFF_MISC + 16;
  static_assert(TOTAL <= 232448, "shared memory of one CTA");
  // where the nt-th tile of a CTA lies, and its barriers' parity
  __device__ static __forceinline__ uint32_t stage_k(uint32_t nt) { return nt % RK; }
  __device__ static __forceinline__ uint32_t stage_v(uint32_t nt) { return RK + nt % RV; }
  __device__ static __forceinline__ uint32_t phase_k(uint32_t nt) { return (nt / RK) & 1; }
  __device__ static __forceinline__ uint32_t phase_v(uint32_t nt) { return (nt / RV) & 1; }
};

// What a stream's 128 rows see of an item's tiles.
struct Stream {
  SeqRange r;
  __device__ __forceinline__ Stream(const SeqView& s, int row0, int st) {
    const int i0 = row0 + TM * st;
    if (i0 >= s.len) { r.np = 0; r.s0 = 1; r.s1 = 0; return; }
    r = seq_keys(s, i0, min(i0 + TM, s.len) - 1, SN);
  }
  __device__ __forceinline__ bool uses(int tile) const { return tile < r.np || (tile >= r.s0 && tile <= r.s1); }
  __device__ __forceinline__ int last() const { return r.s1 >= r.s0 ? r.s1 : r.np - 1; }      // -1: none
};

__device__ __forceinline__ SeqView view_of(volatile int* d) {
  SeqView s;
  s.start = d[J_START]; s.len = d[J_LEN]; s.pin = d[J_PIN]; s.cap = d[J_CAP]; s.e = d[J_E];
  return s;
}
// Bounded wait of the forward kernel: it lasts for as long as the CTA gets on, and 8 ms more.  The word counts the numbers that the producer has
// looked at, the tiles that it has asked for, and the tiles that the epilogue has searched; below zero the CTA has given up.  Numbers that
// belong to no tile (one per empty sequence and head), the tiles that only the other stream sees (a whole chunk, where one leaves inside an
// item) and a search through a chunk's tiles can each take longer than 8 ms.
constexpr int F_ABORT = -0x7fffffff - 1;
__device__ __forceinline__ bool fwd_wait(uint32_t bar, uint32_t parity, volatile int* progress) {
  if (bar_try(bar, parity)) return true;
  int seen = -1;
  for (uint32_t tries = 0; tries < TT_POLLS; ++tries) {
    if (bar_try(bar, parity)) return true;
    const int now = *progress;
    if (now < 0) return false;
    if (now != seen) tries = 0;
    seen = now;
  }
  return false;
}
// Adds the non-finite values that were taken out of V tiles u0 .. u1 - 1 of an item to 16 columns, c < D, of a row that sees them.  The whole
// warp calls it, each lane with its row: a lane looks at a token's 16 values, what is found goes round.  After an eviction inside an item the tiles that
// some row does not see are a whole chunk, so the search is counted as getting on, tile by tile, while the other roles wait.
__device__ __noinline__ void add_odd(float* o, const __nv_bfloat16* v, long long vs, int c, int D, const SeqView s, int row, int row0,
                                     SeqRange r, int u0, int u1, int* progress) {
  const int lane = threadIdx.x & 31, lo = s.low(row), low1 = s.low(row0 + ST_ROWS - 1);
  for (int u = u0; u < u1; ++u) {
    const int j0 = seq_at(r, u) * SN;
    if (seq_all(s, row0, low1, j0, j0 + SN - 1)) continue;
    uint4 w[SN / 32][2];
#pragma unroll
    for (int k = 0; k < SN / 32; ++k) {
      const int j = j0 + 32 * k + lane;
      const uint4* from = reinterpret_cast<const uint4*>(v + (long long)j * vs + c);
      w[k][0] = w[k][1] = make_uint4(0u, 0u, 0u, 0u);
      if (j < s.len) {
        w[k][0] = from[0];
        if (c + 8 < D) w[k][1] = from[1];
      }
    }
#pragma unroll
    for (int k = 0; k < SN / 32; ++k) {
      const uint32_t e[8] = {w[k][0].x, w[k][0].y, w[k][0].z, w[k][0].w, w[k][1].x, w[k][1].y, w[k][1].z, w[k][1].w};
      bool hit = false;
#pragma unroll
      for (int y = 0; y < 8; ++y) hit |= (e[y] & 0x7f80u) == 0x7f80u || (e[y] & 0x7f800000u) == 0x7f800000u;
      for (uint32_t hits = __ballot_sync(0xffffffffu, hit); hits != 0; hits &= hits - 1) {
        const int from = __ffs((int)hits) - 1, j = j0 + 32 * k + from;
        const bool sees = row < s.len && j <= row && (j < s.pin || j >= lo);
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const uint32_t x = __shfl_sync(0xffffffffu, e[y], from);
          const float x0 = __uint_as_float(x << 16), x1 = __uint_as_float(x & 0xffff0000u);
          if (sees && !isfinite(x0)) o[2 * y] += x0;
          if (sees && !isfinite(x1)) o[2 * y + 1] += x1;
        }
      }
    }
    if (lane == 0) atomicAdd(progress, 1);
  }
}

// ------------------------------------------------------------------------------------------------ forward
template <int D>
__global__ void __launch_bounds__(ST_THREADS, 1)
k_seq_fwd_tc(const __grid_constant__ SeqArgs a, const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
             const __grid_constant__ CUtensorMap tmV) {
  using SM = FSmem<D>;
  constexpr int NS = SM::STAGES, TILE = SM::TILE, DH = D / 64;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sb = tt_u32(smem);
  volatile int* desc = reinterpret_cast<volatile int*>(smem + SM::OFF_DESC);
  volatile int* misc = reinterpret_cast<volatile int*>(smem + SM::OFF_MISC);    // [0] how far the CTA is, [1] TMEM base
  int* progress = reinterpret_cast<int*>(smem + SM::OFF_MISC);
  auto st_wait = [&](uint32_t bar, uint32_t parity) -> bool { return fwd_wait(bar, parity, misc); };
  const uint32_t full = sb + SM::OFF_BAR, empty = full + 8 * NS, ready = empty + 8 * NS;
  const uint32_t s_full = ready + 8 * NS, p_full = s_full + 16, o_full = p_full + 16, o_empty = o_full + 16,
                 q_full = o_empty + 16, q_empty = q_full + 8, item_full = q_empty + 8, item_empty = item_full + 16,
                 clc = item_empty + 16, drain = clc + 8, s_read = drain + 8, p_empty = s_read + 16;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    for (int s = 0; s < NS; ++s) { bar_init(full + 8 * s, 1); bar_init(empty + 8 * s, 1); bar_init(ready + 8 * s, 2); }
    for (int s = 0; s < 2; ++s) {
      bar_init(s_full + 8 * s, 1);
      bar_init(p_full + 8 * s, 4);
      bar_init(o_full + 8 * s, 1);
      bar_init(o_empty + 8 * s, 4);
      bar_init(s_read + 8 * s, 4);
      bar_init(p_empty + 8 * s, 1);
      bar_init(item_full + 8 * s, 1);
      bar_init(item_empty + 8 * s, 1 + 2 + 8);           // MMA, patch and softmax warps
    }
    bar_init(q_full, 1);
    bar_init(q_empty, 1);
    bar_init(clc, 1);
    bar_init(drain, 1);
    misc[0] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sb + SM::OFF_MISC + 4), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tree_after_previous();
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = (uint32_t)misc[1];
  const uint32_t tS = tmem, tO = tmem + 2 * SN;          // S [stream] of 128 columns, O [stream] of D columns
  // Narrow heads leave tensor memory for P beside S: the next S is formed as soon as S has been read, under the same tile's weights
  // (two sequences of 8192 tokens, 32 + 8 heads of 64: 799 us, 837 with P over S, where the next S waits for the product with P).
  constexpr bool AHEAD = D == 64;
  const uint32_t tP = AHEAD ? tmem + 2 * SN + 2 * D : tS, P_STEP = AHEAD ? SN / 2 : SN;         // P [stream]

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(ST_REGS_LOW));
    if (warp == 0) {
      // ================================================================ producer
      if (lane == 0) {
        uint32_t nt = 0, seq = 0, asked = 0;               // tiles, items and takeovers so far
        bool half = false;                                 // the last tile's K alone has been asked for
        bool okay = true;
        int item = (int)blockIdx.x;
        while (okay) {
          if (item < 0) {
            if (st_wait(item_empty + 8 * (seq & 1), ((seq >> 1) & 1) ^ 1)) {
              desc[(seq & 1) * J_WORDS + J_KIND] = 0;
              bar_arrive(item_full + 8 * (seq & 1));
            } else {
              okay = false;
            }
            break;
          }
          atomicAdd(progress, 1);
          bar_expect(clc, 16);
          clc_ask(sb + SM::OFF_CLC, clc);
          const int number = (int)(gridDim.x - 1 - item) / a.Hq, h = (int)(gridDim.x - 1 - item) - number * a.Hq;
          SeqView s;
          int tile;
          if (seq_find(a, number, ST_ROWS, &s, &tile)) {
            const uint32_t slot = seq & 1;
            const int row0 = tile * ST_ROWS;
            const SeqRange r = seq_keys(s, row0, min(row0 + ST_ROWS, s.len) - 1, SN);
            const int n = seq_count(r);
            if (!st_wait(item_empty + 8 * slot, ((seq >> 1) & 1) ^ 1)) { okay = false; break; }
            volatile int* d = desc + slot * J_WORDS;
            d[J_START] = s.start; d[J_LEN] = s.len; d[J_PIN] = s.pin; d[J_CAP] = s.cap; d[J_E] = s.e; d[J_HEAD] = h;
            d[J_ROW0] = row0; d[J_NP] = r.np; d[J_S0] = r.s0; d[J_S1] = r.s1; d[J_N] = n; d[J_ODD] = n; d[J_ODD_END] = 0;
            d[J_KIND] = 1;
            bar_arrive(item_full + 8 * slot);
            const bool two = row0 + TM < s.len;
            if (!st_wait(q_empty, (seq & 1) ^ 1)) { okay = false; break; }
            bar_expect(q_full, (uint32_t)((two ? 2 : 1) * TILE));
            for (int t = 0; t < (two ? 2 : 1); ++t)
              for (int hf = 0; hf < DH; ++hf)
                tma_3d(sb + SM::OFF_Q + t * TILE + hf * HALF, &tmQ, hf * 64, h, s.start + row0 + t * TM, q_full);
            ++seq;
            const int hk = h / a.g;
            for (int i = 0; i < n; ++i, ++nt) {
              atomicAdd(progress, 1);
              const int j = s.start + seq_at(r, i) * SN;
              uint32_t sg = SM::stage_k(nt);
              if (!st_wait(empty + 8 * sg, SM::phase_k(nt) ^ 1)) { okay = false; break; }
              bar_expect(full + 8 * sg, (uint32_t)TILE);
              for (int hf = 0; hf < DH; ++hf) tma_3d(sb + sg * TILE + hf * HALF, &tmK, hf * 64, hk, j, full + 8 * sg);
              sg = SM::stage_v(nt);
              if (!st_wait(empty + 8 * sg, SM::phase_v(nt) ^ 1)) { okay = false; half = true; break; }
              bar_expect(full + 8 * sg, (uint32_t)TILE);
              for (int hf = 0; hf < DH; ++hf) tma_3d(sb + sg * TILE + hf * HALF, &tmV, hf * 64, hk, j, full + 8 * sg);
            }
          }
          // the answer is waited for whatever happened: it is a copy in flight
          if (okay) {
            if (!st_wait(clc, asked & 1)) { okay = false; break; }
            item = clc_answer(sb + SM::OFF_CLC);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            ++asked;
          }
        }
        if (!okay) { misc[0] = F_ABORT; bar_drain(clc, asked & 1); }
        // whatever the other roles did, copies in flight land before the shared memory goes away
        const uint32_t nk = nt + (half ? 1 : 0);
        for (uint32_t i = 1; i <= (uint32_t)SM::RK && i <= nk; ++i) bar_drain(full + 8 * SM::stage_k(nk - i), SM::phase_k(nk - i));
        for (uint32_t i = 1; i <= (uint32_t)SM::RV && i <= nt; ++i) bar_drain(full + 8 * SM::stage_v(nt - i), SM::phase_v(nt - i));
        if (seq > 0 && !okay) bar_drain(q_full, (seq - 1) & 1);
      }
    } else if (warp == 1) {
      // ================================================================ MMA issuer: the whole warp takes every step, one lane issues
      const bool leader = tt_elect();
      auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
        return __all_sync(0xffffffffu, st_wait(bar, parity));
      };
      auto get = [&](int x) -> int { return __shfl_sync(0xffffffffu, x, 0); };
      constexpr uint32_t ID_QK = tt_idesc(SN, 0), ID_PV = tt_idesc(D, 1);
      uint32_t nt = 0, seq = 0;                            // tiles and items
      uint32_t np0 = 0, np1 = 0, ni0 = 0, ni1 = 0;         // tiles and items of the streams
      uint32_t ns0 = 0, ns1 = 0;                           // their scores so far
      bool okay = true;
      while (okay) {
        if (!__all_sync(0xffffffffu, st_wait(item_full + 8 * (seq & 1), (seq >> 1) & 1))) { okay = false; break; }
        volatile int* d = desc + (seq & 1) * J_WORDS;
        const int kind = get(d[J_KIND]);
        if (kind == 0) break;
        const SeqView s = view_of(d);
        const int row0 = get(d[J_ROW0]), n = get(d[J_N]);
        SeqRange r;
        r.np = get(d[J_NP]); r.s0 = get(d[J_S0]); r.s1 = get(d[J_S1]);
        __syncwarp();
        if (leader) bar_arrive(item_empty + 8 * (seq & 1));
        const Stream u0(s, row0, 0), u1(s, row0, 1);
        const int last0 = u0.last(), last1 = u1.last();
        if (!wait(q_full, seq & 1)) { okay = false; break; }
        ++seq;
        auto issue_s = [&](int st, int i) -> bool {
          if (AHEAD) {                                     // the scores before have been read
            uint32_t& ns = st ? ns1 : ns0;
            if (ns > 0 && !wait(s_read + 8 * st, (ns - 1) & 1)) return false;
            ++ns;
            fence_after();
          }
          const uint32_t sg = SM::stage_k(nt + i);
          const uint64_t dq = desc_k(sb + SM::OFF_Q + st * TILE), dk = desc_k(sb + sg * TILE);
          if (leader) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              const uint64_t off = ((k >> 2) * HALF + (k & 3) * 32) >> 4;        // the address field counts 16 bytes
              mma_ss(tS + st * SN, dq + off, dk + off, ID_QK, k > 0);
            }
            commit(s_full + 8 * st);
          }
          __syncwarp();
          return true;
        };
        auto wait_k = [&](int i) -> bool { return wait(full + 8 * SM::stage_k(nt + i), SM::phase_k(nt + i)); };
        auto release = [&](uint32_t stage) {               // free once what has been issued is done
          if (leader) commit(empty + 8 * stage);
          __syncwarp();
        };
        auto step = [&](int st, int i, int tile, bool& v_there, bool first, uint32_t& np, uint32_t& ni, bool last) -> bool {
          const uint32_t sg = SM::stage_v(nt + i);
          if (!v_there && !wait(ready + 8 * sg, SM::phase_v(nt + i))) return false;
          v_there = true;
          if (first && !wait(o_empty + 8 * st, (ni & 1) ^ 1)) return false;      // O of the item before is out
          const uint64_t dv = desc_mn(sb + sg * TILE);
          if (!wait(p_full + 8 * st, np & 1)) return false;
          fence_after();
          if (leader) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              mma_ts(tO + st * D, tP + st * P_STEP + k * 8, dv + (k * 2048 >> 4), ID_PV, k > 0 ? 1u : (first ? 0u : 1u));
            if (AHEAD) commit(p_empty + 8 * st);
          }
          __syncwarp();
          ++np;
          if (last) {
            if (leader) commit(o_full + 8 * st);
            __syncwarp();
            ++ni;
          }
          return true;
        };
        okay = wait_k(0);
        fence_after();
        const int t0 = seq_at(r, 0);
        if (okay && u0.uses(t0)) okay = issue_s(0, 0);
        if (okay && u1.uses(t0)) okay = issue_s(1, 0);
        auto q_done = [&]() {                              // all scores of the item have been issued: the next item's Q may come
          if (leader) commit(q_empty);
          __syncwarp();
        };
        if (okay) release(SM::stage_k(nt));
        if (okay && n == 1) q_done();
        bool first0 = true, first1 = true;
        for (int i = 0; i < n && okay; ++i) {
          const int tile = seq_at(r, i), next = i + 1 < n ? seq_at(r, i + 1) : -1;
          bool v_there = false;
          const bool k0 = next >= 0 && u0.uses(next), k1 = next >= 0 && u1.uses(next);
          if (AHEAD && next >= 0) {
            okay = wait_k(i + 1);
            fence_after();
            if (okay && k0) okay = issue_s(0, i + 1);
            if (okay && k1) okay = issue_s(1, i + 1);
            if (!okay) break;
            release(SM::stage_k(nt + i + 1));
            if (i + 2 == n) q_done();
          }
          if (u0.uses(tile)) {
            okay = step(0, i, tile, v_there, first0, np0, ni0, tile == last0);
            first0 = false;
          }
          if (!AHEAD && okay && next >= 0) { okay = wait_k(i + 1); fence_after(); }
          if (!AHEAD && okay && k0) okay = issue_s(0, i + 1);
          if (okay && u1.uses(tile)) {
            okay = step(1, i, tile, v_there, first1, np1, ni1, tile == last1);
            first1 = false;
          }
          if (!okay) break;
          release(SM::stage_v(nt + i));
          if (AHEAD) continue;
          if (k1) okay = issue_s(1, i + 1);
          if (next >= 0) release(SM::stage_k(nt + i + 1));
          if (i + 2 == n) q_done();
        }
        nt += n;
      }
      if (leader) {
        if (!okay) misc[0] = F_ABORT;
        commit(drain);                                     // MMAs still in flight finish before tensor memory is freed
        bar_drain(drain, 0);
      }
      __syncwarp();
    } else {
      // ================================================================ patch warps
      uint32_t nt = 0, seq = 0;
      bool okay = true;
      auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
        return __all_sync(0xffffffffu, st_wait(bar, parity));
      };
      while (okay) {
        if (!__all_sync(0xffffffffu, st_wait(item_full + 8 * (seq & 1), (seq >> 1) & 1))) { okay = false; break; }
        volatile int* d = desc + (seq & 1) * J_WORDS;
        if (d[J_KIND] == 0) break;
        const SeqView s = view_of(d);
        const int row0 = d[J_ROW0], n = d[J_N], low1 = s.low(row0 + ST_ROWS - 1);
        SeqRange r;
        r.np = d[J_NP]; r.s0 = d[J_S0]; r.s1 = d[J_S1];
        for (int i = 0; i < n; ++i) {
          const int tile = seq_at(r, i);
          // These warps wait for each V tile in turn, and none is used without them: a wait tells a stage's phase from the one two
          // rounds before or after.
          const uint32_t sg = SM::stage_v(nt + i);
          if (!wait(full + 8 * sg, SM::phase_v(nt + i))) { okay = false; break; }
          if (!seq_all(s, row0, low1, tile * SN, tile * SN + SN - 1) &&
              patch_tile(smem + sg * TILE, DH, tile * SN, s.len, warp - 2, 2, nullptr) && lane == 0) {
            atomicMin(const_cast<int*>(d) + J_ODD, i);
            atomicMax(const_cast<int*>(d) + J_ODD_END, i + 1);
          }
          __syncwarp();
          if (lane == 0) bar_arrive(ready + 8 * sg);
        }
        if (!okay) break;
        __syncwarp();
        if (lane == 0) bar_arrive(item_empty + 8 * (seq & 1));
        ++seq;
        nt += n;
      }
      if (!okay && lane == 0) misc[0] = F_ABORT;
    }
  } else {
    // ================================================================ softmax: stream st, a row per thread
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(ST_REGS_HIGH));
    const int st = (warp - 4) >> 2, quarter = warp & 3;
    const uint32_t lane_off = (uint32_t)(32 * quarter) << 16;
    const uint32_t ts = tS + st * SN + lane_off, to = tO + st * D + lane_off, tp = tP + st * P_STEP + lane_off;
    const float sl2 = a.scale * ST_LOG2E, slack = 8.f / sl2;
    uint32_t seq = 0, ntile = 0, nitem = 0;
    bool fine = true;                                    // false: a wait ran out; go through the motions, never wait again
    auto wait = [&](uint32_t bar, uint32_t parity) {
      if (fine && !st_wait(bar, parity)) { fine = false; misc[0] = F_ABORT; }
    };
    while (true) {
      if (fine && !st_wait(item_full + 8 * (seq & 1), (seq >> 1) & 1)) { fine = false; misc[0] = F_ABORT; }
      if (!__all_sync(0xffffffffu, fine)) break;
      volatile int* d = desc + (seq & 1) * J_WORDS;
      if (d[J_KIND] == 0) break;
      const SeqView s = view_of(d);
      const int row0 = d[J_ROW0], n = d[J_N], h = d[J_HEAD];
      SeqRange r;
      r.np = d[J_NP]; r.s0 = d[J_S0]; r.s1 = d[J_S1];
      const Stream us(s, row0, st);
      const int i0 = row0 + TM * st, row = i0 + 32 * quarter + lane, low = s.low(row), low1 = s.low(i0 + TM - 1);
      const int last = us.last();
      float m = -INFINITY, l = 0.f;                      // running maximum (of the raw scores) and sum
      bool first = true;
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        const int tile = seq_at(r, i);
        if (!us.uses(tile)) continue;
        wait(s_full + 8 * st, ntile & 1);
        ++ntile;
        fence_after();
        float x[SN];
#pragma unroll
        for (int c = 0; c < SN; c += 32) ld32(ts + c, x + c);
        wait_ld();
        if (AHEAD) {
          fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(s_read + 8 * st);
        }
        if (!seq_all(s, i0, low1, tile * SN, tile * SN + SN - 1)) {
          const int j0 = tile * SN;
#pragma unroll
          for (int c = 0; c < SN; c += 32) {
            const uint32_t keep = st_run(0, row + 1, j0 + c) & ~st_run(s.pin, low, j0 + c);
#pragma unroll
            for (int y = 0; y < 32; ++y)
              if (!(keep & (1u << y))) x[c + y] = -INFINITY;
          }
        }
        float mx[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
        for (int y = 4; y < SN - 4; y += 8)
#pragma unroll
          for (int z = 0; z < 4; ++z) mx[z] = tt_max3(mx[z], x[y + 2 * z], x[y + 2 * z + 1]);
        const float mine = tt_max3(tt_max3(mx[0], mx[1], mx[2]), tt_max3(mx[3], x[SN - 4], x[SN - 3]), fmaxf(x[SN - 2], x[SN - 1]));
        const float mnew = tt_max3(m, mine, mine);
        if (AHEAD) {                                     // the product with the last P is done: O is at rest, and P may be written
          wait(p_empty + 8 * st, ntile & 1);
          fence_after();
        }
        if (first) {
          m = mnew;
          first = false;
        } else {
          const bool grown = !(mnew <= m + slack);       // NaN counts; nothing seen yet and nothing now (-inf) does not
          if (__any_sync(0xffffffffu, grown)) {
            // between the references as they were rounded, which for large scores is not their distance
            const float corr = grown ? tt_ex2(__fmul_rn(m, sl2) - __fmul_rn(mnew, sl2)) : 1.f;
            if (grown) m = mnew;
            l *= corr;
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {            // O is at rest: without AHEAD S of this tile came after the products before it
              float o[16];
              ld16(to + c, o);
              wait_ld();
#pragma unroll
              for (int y = 0; y < 16; ++y) o[y] *= corr;
              st16(to + c, reinterpret_cast<uint32_t*>(o));
            }
          }
        }
        // an infinite maximum makes the row NaN, as inf - inf does
        const float neg = m == -INFINITY ? 0.f : m == INFINITY ? __int_as_float(0x7fffffff) : -__fmul_rn(m, sl2);
        const uint64_t neg2 = tt_two(neg, neg), scl2 = tt_two(sl2, sl2);
        uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
        for (int c = 0; c < SN; c += 32) {
          uint32_t pk[16];
#pragma unroll
          for (int y = 0; y < 32; y += 2) {
            float e0, e1;
            tt_both(tt_fma2(tt_two(x[c + y], x[c + y + 1]), scl2, neg2), e0, e1);
            e0 = tt_ex2(e0);
            e1 = tt_ex2(e1);
            sum[(y >> 1) & 1] = tt_add2(sum[(y >> 1) & 1], tt_two(e0, e1));
            pk[y >> 1] = tt_pack(e0, e1);                // P in bf16, half a step of 2^-8 per weight; the sum is of the weights as they were
          }
          st16(tp + c / 2, pk);
        }
        // P is handed over in one piece: in halves or quarters its product would start earlier, but each hand-over costs the warp more
        // (16384 tokens, 28 heads of 128: 1535 us, in halves 1555, in quarters 1760)
        wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(p_full + 8 * st);
        float s0, s1;
        tt_both(tt_add2(sum[0], sum[1]), s0, s1);
        l += s0 + s1;
      }
      // ---- the item's rows ------------------------------------------------------------------------------------------------
      if (last >= 0) {
        wait(o_full + 8 * st, nitem & 1);
        ++nitem;
        fence_after();
        // one lane's: tiles that only the other stream sees may still be added
        const int odd0 = __shfl_sync(0xffffffffu, d[J_ODD], 0), odd1 = __shfl_sync(0xffffffffu, d[J_ODD_END], 0);
        const float inv = !fine || m == -INFINITY ? __int_as_float(0x7fffffff) : 1.f / l;     // every score -inf: NaN
        const long long orow = (long long)(s.start + row) * a.Hq + h;
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + orow * a.D;
        const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(a.v) + s.start * a.vs + (long long)(h / a.g) * a.D;
        const bool real = row < s.len, wide = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0 && a.D % 16 == 0;
#pragma unroll 1
        for (int c = 0; c < D; c += 16) {
          float o[16];
          ld16(to + c, o);
          wait_ld();
          if (odd0 < odd1 && c < a.D) {                  // rare
            float x[16];
#pragma unroll
            for (int y = 0; y < 16; ++y) x[y] = o[y];
            add_odd(x, v, a.vs, c, a.D, s, row, row0, r, odd0, odd1, progress);
#pragma unroll
            for (int y = 0; y < 16; ++y) o[y] = x[y];
          }
          uint32_t pk[8];
#pragma unroll
          for (int y = 0; y < 16; y += 2) pk[y >> 1] = tt_pack(o[y] * inv, o[y + 1] * inv);
          if (!real) continue;
          if (c + 16 <= a.D) tt_store(out + c, pk, wide);
          else if (c < a.D) *reinterpret_cast<uint4*>(out + c) = make_uint4(pk[0], pk[1], pk[2], pk[3]);   // D is a multiple of 8
        }
        if (real && a.lse != nullptr) a.lse[orow] = (__fmul_rn(m, sl2) + log2f(l)) * ST_LN2 + (fine ? 0.f : inv);
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(o_empty + 8 * st);
      }
      __syncwarp();
      if (lane == 0) bar_arrive(item_empty + 8 * (seq & 1));
      ++seq;
    }
  }

  fence_before();
  __syncthreads();
  if (warp == 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------ host
template <int D>
cudaError_t fwd_launch(const SeqArgs& a, int dev, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, unsigned grid,
                       cudaStream_t st) {
  static PtencOnce once;
  const cudaError_t e = ptenc_first_use(once, dev, [] { return ptenc_allow_smem(k_seq_fwd_tc<D>, FSmem<D>::TOTAL); });
  if (e != cudaSuccess) return e;
  return tree_launch(k_seq_fwd_tc<D>, dim3(grid), ST_THREADS, FSmem<D>::TOTAL, 0, st, a, q, k, v);
}

}  // namespace

bool seq_forward_tc(const SeqArgs& a, int dtype, int dev, cudaStream_t st, cudaError_t* e) {
  const long long grid = seq_numbers(a.n, a.B, ST_ROWS) * a.Hq;
  if (dtype != PTENC_DTYPE_BF16 || a.D > 128 || grid >= (1ll << 31)) return false;
  CUtensorMap q, k, v;
  if (!seq_map(&q, a.q, a.D, a.Hq, a.n, a.qs) || !seq_map(&k, a.k, a.D, a.Hkv, a.n, a.ks) || !seq_map(&v, a.v, a.D, a.Hkv, a.n, a.vs))
    return false;
  *e = a.D <= 64 ? fwd_launch<64>(a, dev, q, k, v, (unsigned)grid, st) : fwd_launch<128>(a, dev, q, k, v, (unsigned)grid, st);
  return true;
}

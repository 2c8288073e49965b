// Attention of a draft tree over the cache on the sm_100a tensor cores (bf16, head_dim 64 or 128).
//
// The T nodes of a tree times the g heads that share a KV head are R = T g query rows over the same K and V: R flop per
// byte read.  Up to about 250 rows HBM is the bound (6.5 TB/s against 1.65 PFLOP/s), above it the tensor cores, so both
// products run on tcgen05 with accumulators in tensor memory and every K/V byte is read once per 2 x 128 rows.
//
// A row tile is the nodes that fit 128 rows (128 / g nodes, row = node * g + head).  A work item is a block of one or two
// row tiles of a (layer, sequence, KV head) against a stretch of its K/V tiles of 128 slots; the draft's own K/V rows are
// one more tile at the end.  Per CTA (one per SM, persistent, items handed out by a counter):
//  * warp 0, one lane: producer.  Describes the item, then TMA-loads its Q tiles and the K and V tiles (128-byte swizzle;
//    plain loads of this GPU's own memory) into a ring of stages.
//  * warp 1: issues the MMAs (one elected lane).  Two streams, each with its own S, P and O in tensor memory: with two row
//    tiles a stream per row tile; with one, the K/V tiles alternate between the streams and the two results are merged at
//    the end.  One stream's products run under the other's softmax.  S = Q K^T (both K-major in shared memory), O += P V (P
//    bf16 in tensor memory over the S it came from, V as it lies: tokens x head_dim, MN-major).
//  * warps 2 and 3: patches.  Warp 2 works out what each node sees (ptenc_tree.cuh); both pass every stage on, and in the
//    tiles where some slot is not seen by some node they clear the V rows that nobody sees and take non-finite values out of
//    the V rows that only some nodes see, since 0 * NaN would carry them into the other nodes' rows.
//  * warps 4..19: softmax, eight warps per stream, a row per thread and half of a tile's tokens: S from tensor memory, mask,
//    maximum (the two halves exchange theirs through shared memory), running sum in fp32 (base 2), P rounded to bf16 back to
//    tensor memory.  A warp alone is bound by its own latencies, so four warps share a scheduler.  O is rescaled only when
//    the maximum has grown by more than 2^8, which for most rows is never after the first tiles.  Non-finite values that
//    were taken out of V are added to the rows that see them.
//  * Items that are a part of a block's tiles leave fp32 partials.  When the call has so few blocks that clusters of two, four
//    or eight CTAs can hold all their parts, a block's parts are a cluster: they stay in shared memory and every CTA joins
//    some of the rows (one chain of 5 nodes: 12.0 us, from Python 12.9).  Otherwise k_tree_join, chained by programmatic
//    dependent launch, joins them in order from memory, a thread per row and eight columns (the same chain 12.5, from Python
//    17.3, the second launch's time on the host).
//  * Every wait is bounded: one that runs out raises a status bit and an abort flag, every role then leaves, copies and
//    MMAs in flight are drained and tensor memory is freed.
//
// Measured (head size 128, full rings).  128 sequences of 16 nodes, groups of 7, four rings of 2048 slots: 571 MB in 107 us,
// 5.3 TB/s; an item costs about 10000 cycles beside the 33000 of its tiles (description, set-up, the last product, the rows' way
// out).  64 sequences of 64 nodes, groups of 4, eight rings of 4096 slots: 277 GFLOP in 303 us, 0.9 PFLOP/s; there the
// tensor pipe is 44 % busy, the exponentials' unit 45 %, the issue slots 46 %: the bound is a stream's chain, about 3800
// cycles a tile, of which both products take 1100, the maximum 630, its exchange 180, P 1650 and handing over the rest.  One
// chain of 5 nodes over 1024 slots: 12 us, most of it set-up and the join.  What did not shorten the chain: tiles of 64
// tokens (a 64-column product costs as much as one of 128), a second warp issuing products (334 us), part of the exponentials
// on the FMA pipe, reading the scores 16 at a time with the next ones in flight, exchanging between the two warps of a row
// alone, and the weights in one pass against the running maximum (twice the time: P in registers until the maximum is known
// spills).
#include <cooperative_groups.h>
#include <string.h>
#include <type_traits>

#include "ptenc_tree.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr uint32_t TT_POLLS = 2000;             // bounded wait: tries of up to a millisecond each before giving up
constexpr int TN = 128;                        // slots per K/V tile
constexpr int TH = 64;                         // tokens of a softmax thread: half a tile
constexpr int TM = 128;                        // rows of a row tile = TMEM lanes
constexpr int TT_THREADS = 640;                // producer, MMA, two patch warps, 2 x 8 softmax warps
constexpr int TT_SOFT = 512;
constexpr int TT_LEAD = 128;                   // the softmax thread that speaks for all of them
// Registers: 640 threads are launched with 96 each (61440); the first four warps give up 32 so that a softmax thread can hold
// its 64 scores: 128 * 64 + 512 * 104 = 61440.
constexpr int TT_REGS_LOW = 64, TT_REGS_HIGH = 104;
static_assert(128 * TT_REGS_LOW + 512 * TT_REGS_HIGH <= 640 * 96, "the split waits for registers that do not exist");
constexpr int HALF = TN * 128;                 // 64 columns of a 128-row tile
constexpr int TT_MAX_PIECES = 16;

// ------------------------------------------------------------------------------------------------ PTX
__device__ __forceinline__ uint32_t tt_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Lets the hardware park the thread for up to a millisecond instead of spinning: the waiting warps share their schedulers
// with the softmax warps.
__device__ __forceinline__ uint32_t bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000000u) : "memory");
  return ok;
}
// Bounded wait that also gives up when another role has raised the abort flag.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (bar_try(bar, parity)) return true;
  for (uint32_t i = 0; i < TT_POLLS; ++i) {
    if (bar_try(bar, parity)) return true;
    if (*abort_flag != 0) return false;
  }
  return false;
}
// Bounded wait for what completes by itself: copies and products in flight.
__device__ __forceinline__ void bar_drain(uint32_t bar, uint32_t parity) {
  for (uint32_t i = 0; i < TT_POLLS; ++i)
    if (bar_try(bar, parity)) return;
}
// True in one lane of the (converged) warp.
__device__ __forceinline__ bool tt_elect() {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
  return is != 0;
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// A and B from shared memory.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
// A from tensor memory.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
// 32 consecutive 32-bit columns of this thread's lane.
__device__ __forceinline__ void ld32(uint32_t t, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(t) : "memory");
}
__device__ __forceinline__ void ld16(uint32_t t, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(t) : "memory");
}
__device__ __forceinline__ void st16(uint32_t t, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      ::"r"(t), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// The hardware's 2^x: a relative error of about 2^-22, far below the rounding of P, and zero below 2^-126, where the weight would be
// lost in its row's sum anyhow (the row's largest is between 1 and 2^8).
__device__ __forceinline__ float tt_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t tt_two(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void tt_both(uint64_t d, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(d));
}
__device__ __forceinline__ uint64_t tt_fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t tt_add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// NaN if any of the three is.
__device__ __forceinline__ float tt_max3(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ uint32_t tt_pack(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
// Sixteen outputs of a row.  The rows of a warp lie apart, so a store costs a cycle per row whatever its width: 32 bytes at a
// time where the tensor is aligned for it.
__device__ __forceinline__ void tt_store(__nv_bfloat16* to, const uint32_t (&r)[8], bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
  } else {
    reinterpret_cast<uint4*>(to)[0] = make_uint4(r[0], r[1], r[2], r[3]);
    reinterpret_cast<uint4*>(to)[1] = make_uint4(r[4], r[5], r[6], r[7]);
  }
}
__device__ __forceinline__ void soft_sync() { asm volatile("bar.sync 1, %0;" ::"n"(TT_SOFT) : "memory"); }
__device__ __forceinline__ void stream_sync(int st) {                        // the eight warps of a stream
  asm volatile("bar.sync %0, %1;" ::"r"(2 + st), "n"(TT_SOFT / 2) : "memory");
}

// Shared-memory descriptors of bf16 tiles of 128-byte rows with the 128-byte swizzle.
// K-major (the contraction index runs along the row): groups of 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_k(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)2 << 61);
}
// MN-major (the contraction index counts rows): the next 64 columns one HALF on, the next 8 rows 1024 bytes on.
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(HALF >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// D fp32, A and B bf16, M = 128; b_mn: B is MN-major.
__host__ __device__ constexpr uint32_t tt_idesc(int n, int b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(TM >> 4) << 24);
}

// ------------------------------------------------------------------------------------------------ layout
// Item description words in shared memory; I_LB is layer of the call * batch + sequence.
enum { I_KIND, I_LB, I_H, I_NODE0, I_N, I_TWO, I_HEAD, I_COUNT, I_SINK, I_CHUNK, I_T0, I_LEN2, I_LO, I_CNT, I_NT, I_PIECES,
       I_PIECE, I_SPLIT, I_EVMAX, I_VALID, I_ODD, I_WORDS };
template <int D>
struct TSmem {
  static constexpr int TILE = (D / 64) * HALF;                       // bytes of a 128-row tile
  static constexpr int STAGES = D == 128 ? 5 : 10;
  static constexpr int OFF_Q = STAGES * TILE;                        // two Q tiles
  static constexpr int OFF_VIS = OFF_Q + 2 * TILE;                   // u64 [64] what each node sees of the draft
  static constexpr int OFF_ML = OFF_VIS + TREE_MAX * 8;              // exchange: float [2][2][128] maxima, float2 [128]
  static constexpr int OFF_DESC = OFF_ML + 4 * TM * 4;               // int [2][I_WORDS] items
  static constexpr int OFF_BAR = OFF_DESC + 2 * I_WORDS * 4;
  static constexpr int N_BAR = 3 * STAGES + 18;
  static constexpr int OFF_DEPTH = OFF_BAR + N_BAR * 8;              // u8 [64]: first the doubled parents, then the depths
  static constexpr int OFF_MISC = OFF_DEPTH + TREE_MAX;              // int [4]
  static constexpr int TOTAL = OFF_MISC + 16;
  static_assert(OFF_BAR % 8 == 0 && OFF_MISC % 4 == 0, "alignment");
  static_assert(TOTAL <= 232448, "shared memory of one CTA");
};

struct TreeTcArgs {
  int l0, NT;                      // first layer; nodes per sequence in the call's tensors
  int npt, tpb, nqp;               // nodes per row tile, row tiles per block (1 or 2), row blocks per unit
  int nb;                          // rows of the draft tile: NT rounded up to 16
  int ring_box;                    // rows of a ring box
  int n_full, n_items, P;          // items that are whole blocks; all items; pieces of the other blocks
  const int32_t* parent;
  const int32_t* n_nodes;
  const uint8_t* active;
  __nv_bfloat16* out;
  float* lse;
  const __nv_bfloat16* v_tree;
  float* part;                     // [slot][2][D / 4][128][4]
  float2* part_ml;                 // [slot][2][128]
  int* pieces;                     // [block that is split]: its parts, 0 if there is nothing to join
};

// Tiles of a ring that hold slots some node sees: the pinned entries [0, sink) and `count` slots from sink + head on, wrapping
// inside [sink, W).  Enumerated from the tile of the first sliding slot upwards, then from tile 0.
__device__ __forceinline__ int tt_tiles(int sink, int head, int count, int W, int* t0, int* len2) {
  int low = sink, high = 0;                              // slots [0, low) and [sink + head, sink + head + high)
  const int first = W - sink - head;
  if (count > first) { low = sink + count - first; high = first; } else { high = count; }
  *t0 = 0;
  *len2 = 0;
  const int e1 = (low + TN - 1) / TN;                    // tiles of the low part
  if (high == 0) return e1;
  *t0 = (sink + head) / TN;
  *len2 = (sink + head + high - 1) / TN - *t0 + 1;
  return *len2 + min(e1, *t0);
}

// Bits of columns [lo, hi) in the word of columns [at, at + 32).
__device__ __forceinline__ uint32_t run_mask(int lo, int hi, int at) {
  const int a = max(lo - at, 0), b = min(hi - at, 32);
  return a >= b ? 0u : (~0u >> (32 - (b - a))) << a;
}

// Adds the non-finite values of the V rows that this row sees and others do not (they were taken out of the products) to 16 of
// its columns.
__device__ __noinline__ void add_not_finite(float* o, int c, const PtencDev& p, const __nv_bfloat16* vt, size_t ring, TreeRing r,
                                            int ev, int ev_max, unsigned long long vis, int nodes, int lo, int n, int nt, int t0,
                                            int len2) {
  for (int i = 0; i < n; ++i) {
    const int u = lo + i;
    const int slot0 = (u < len2 ? t0 + u : u - len2) * TN;
    const bool draft = u == nt - 1;
    for (int t = 0; t < (draft ? nodes : TN); ++t) {
      const __nv_bfloat16* v;
      if (draft) {
        if (!((vis >> t) & 1ull)) continue;
        v = vt + (size_t)t * p.Hkv * p.D;
      } else {
        int dd = slot0 + t - r.sink - r.head;
        if (dd < 0) dd += r.cap;
        if (slot0 + t < r.sink || slot0 + t >= p.W || dd < ev || dd >= ev_max || dd >= r.count) continue;
        v = reinterpret_cast<const __nv_bfloat16*>(p.V) + ring + (size_t)(slot0 + t) * p.D;
      }
      for (int y = 0; y < 16; ++y) {
        const float x = __bfloat162float(v[c + y]);
        if (!isfinite(x)) o[y] += x;
      }
    }
  }
}

// Eight columns of one row of block n_full + split, x counting rows, then columns, then row tiles: the parts' sums weighted by
// 2^(m - max), four parts requested together.  ml(part, tile, row) and sums(part, tile, column / 4 * 128 + row) fetch them.
template <int D, typename ML, typename SUMS>
__device__ __forceinline__ void join_row(const TreeTcArgs& a, int B, int Hkv, int g, int split, int x, int pieces, ML ml, SUMS sums) {
  const int row = x % TM, c = 8 * (x / TM % (D / 8)), tile = x / (TM * (D / 8));
  const int blk = a.n_full + split;
  const int unit = blk / a.nqp, qp = blk - unit * a.nqp;
  const int e = unit / Hkv, h = unit - e * Hkv, b = e % B;
  const int n = a.n_nodes != nullptr ? a.n_nodes[b] : a.NT;
  const int node = qp * 2 * a.npt + tile * a.npt + row / g;
  if (row >= a.npt * g || node >= n) return;
  float mm = -INFINITY, ll = 0.f;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int q = 0; q < pieces; q += 4) {
    float2 v[4];
    float4 f[4][2];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = min(q + k, pieces - 1);
      v[k] = ml(at, tile, row);
#pragma unroll
      for (int y = 0; y < 2; ++y) f[k][y] = sums(at, tile, ((c >> 2) + y) * TM + row);
    }
    float mn = mm;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (q + k < pieces) mn = tt_max3(mn, v[k].x, v[k].x);
    const float corr = mm == -INFINITY ? 0.f : tt_ex2(mm - mn);
    ll *= corr;
#pragma unroll
    for (int y = 0; y < 8; ++y) acc[y] *= corr;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (q + k < pieces && v[k].x != -INFINITY) {       // a part in which the row sees nothing does not count
        const float w = tt_ex2(v[k].x - mn);
        ll = fmaf(w, v[k].y, ll);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          acc[4 * y] = fmaf(w, f[k][y].x, acc[4 * y]);
          acc[4 * y + 1] = fmaf(w, f[k][y].y, acc[4 * y + 1]);
          acc[4 * y + 2] = fmaf(w, f[k][y].z, acc[4 * y + 2]);
          acc[4 * y + 3] = fmaf(w, f[k][y].w, acc[4 * y + 3]);
        }
      }
    }
    mm = mn;
  }
  const size_t o = ((size_t)e * a.NT + node) * (size_t)(Hkv * g) + (size_t)h * g + row % g;
  const float linv = 1.f / ll;                           // nothing but -inf: 0 * inf, NaN
  *reinterpret_cast<uint4*>(a.out + o * D + c) = make_uint4(tt_pack(acc[0] * linv, acc[1] * linv), tt_pack(acc[2] * linv, acc[3] * linv),
                                                            tt_pack(acc[4] * linv, acc[5] * linv), tt_pack(acc[6] * linv, acc[7] * linv));
  if (c == 0 && a.lse != nullptr) a.lse[o] = (mm + log2f(ll)) * 0.6931471805599453f;
}

// ------------------------------------------------------------------------------------------------ kernel
template <int D, bool CL>
__global__ void __launch_bounds__(TT_THREADS, 1)
k_tree_tc(const __grid_constant__ PtencDev p, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
          const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmKt,
          const __grid_constant__ CUtensorMap tmVt, const __grid_constant__ TreeTcArgs a) {
  using SM = TSmem<D>;
  constexpr int NS = SM::STAGES, TILE = SM::TILE, DH = D / 64;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sb = tt_u32(smem);
  volatile int* desc = reinterpret_cast<volatile int*>(smem + SM::OFF_DESC);
  unsigned long long* s_vis = reinterpret_cast<unsigned long long*>(smem + SM::OFF_VIS);
  float2* s_ml = reinterpret_cast<float2*>(smem + SM::OFF_ML);
  float* s_mx = reinterpret_cast<float*>(smem + SM::OFF_ML);
  uint8_t* s_depth = smem + SM::OFF_DEPTH;
  int8_t* s_jump = reinterpret_cast<int8_t*>(smem + SM::OFF_DEPTH);
  volatile int* misc = reinterpret_cast<volatile int*>(smem + SM::OFF_MISC);
  // misc[1]: TMEM base, misc[2]: verdict on the next item, misc[3]: with CL, the parts that make up the block
  volatile int* abort_flag = misc;
  const uint32_t full = sb + SM::OFF_BAR, empty = full + 8 * NS, ready = empty + 8 * NS;
  // barriers with two entries: [stream], [Q tile] or [item slot]
  const uint32_t s_full = ready + 8 * NS, p_full = s_full + 16, o_full = p_full + 16, q_full = o_full + 16,
                 q_empty = q_full + 16, item_full = q_empty + 16, item_empty = item_full + 16, o_empty = item_empty + 16,
                 info_full = o_empty + 8, info_empty = info_full + 8, drain = info_empty + 8;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int W = p.W, B = p.B, Hkv = p.Hkv, g = p.g;

  if (tid == 0) {
    for (int s = 0; s < NS; ++s) { bar_init(full + 8 * s, 1); bar_init(empty + 8 * s, 3); bar_init(ready + 8 * s, 2); }
    for (int s = 0; s < 2; ++s) {
      bar_init(s_full + 8 * s, 1);
      bar_init(p_full + 8 * s, 8);
      bar_init(o_full + 8 * s, 1);
      bar_init(q_full + 8 * s, 1);
      bar_init(q_empty + 8 * s, 1);
      bar_init(item_full + 8 * s, 1);
      bar_init(item_empty + 8 * s, 1 + 2 + 16);          // MMA, patch and softmax warps
    }
    bar_init(o_empty, 16);
    bar_init(info_full, 1);
    bar_init(info_empty, 1 + 16);
    bar_init(drain, 1);
    *abort_flag = 0;
    misc[3] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sb + SM::OFF_MISC + 4), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // What the producer has to know of an item's sequence; the first item's is requested while tensor memory is allocated.
  struct Words { int act, n, head, count, sink; };
  auto words_of = [&](int item) -> Words {
    const int blk = item < a.n_full ? item : a.n_full + (item - a.n_full) / a.P;
    const int e = blk / a.nqp / Hkv, li = e / B, b = e - li * B;
    const size_t lb = (size_t)(a.l0 + li) * B + b;
    Words w;
    w.act = a.active != nullptr ? a.active[b] : 1;
    w.n = a.n_nodes != nullptr ? a.n_nodes[b] : a.NT;
    w.head = p.head[lb];
    w.count = p.count[lb];
    w.sink = p.n_sink[lb];
    return w;
  };
  Words words = {0, 0, 0, 0, 0};
  tree_after_previous();
  tree_let_next_start();
  if (tid == 0) words = words_of((int)blockIdx.x);       // gridDim.x <= n_items
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = (uint32_t)misc[1];
  const uint32_t tS = tmem, tO = tmem + 2 * TN;          // S [stream] of 128 columns, O [stream] of D columns

  // Ring position of an item's K and V tiles, counted from its first: with two row tiles K0 V0 K1 V1 ..; with one, the next
  // K tile of a stream is wanted before the V tile of the other: K0 K1 V0 K2 V1 K3 ..
  auto pos_k = [](int i, bool two) -> int { return two ? 2 * i : (i < 2 ? i : 2 * i - 1); };
  auto pos_v = [](int i, int n, bool two) -> int { return two ? 2 * i + 1 : (i == n - 1 ? 2 * n - 1 : 2 * i + 2); };

  if (warp < 4) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TT_REGS_LOW));
  if (warp == 0) {
    // ================================================================ producer
    if (lane == 0) {
      uint32_t pos = 0, qn = 0, seq = 0;                 // ring entries, Q tiles and items so far
      bool okay = true;
      int item = (int)blockIdx.x;
      bool fresh = true;
      while (okay) {
        const int last_grab = a.n_items + (int)gridDim.x - 1;
        if (item >= a.n_items) {
          if (!CL && item == last_grab) *p.work = 0;            // the launch's last grab rewinds the counter
          if (bar_wait(item_empty + 8 * (seq & 1), ((seq >> 1) & 1) ^ 1, abort_flag)) {
            desc[(seq & 1) * I_WORDS + I_KIND] = 0;
            bar_arrive(item_full + 8 * (seq & 1));
          } else {
            okay = false;
          }
          break;
        }
        const int next = CL ? a.n_items : atomicAdd(p.work, 1) + (int)gridDim.x;     // a CTA of a cluster has one part
        int blk, piece = 0, pieces = 1, split = -1;
        if (item < a.n_full) {
          blk = item;
        } else {
          split = (item - a.n_full) / a.P;
          piece = item - a.n_full - split * a.P;
          pieces = a.P;
          blk = a.n_full + split;
        }
        const Words w = fresh ? words : words_of(item);
        fresh = false;
        item = next;
        const int unit = blk / a.nqp, qp = blk - unit * a.nqp;
        const int e = unit / Hkv, h = unit - e * Hkv;
        const int li = e / B, b = e - li * B;
        const size_t lb = (size_t)(a.l0 + li) * B + b;
        const int n = w.n;
        TreeRing r;
        r.head = w.head; r.count = w.count; r.sink = w.sink; r.cap = W - w.sink; r.e = min(p.E, r.cap);
        if (!CL && split >= 0 && piece == 0) a.pieces[split] = 0;           // until its rows say otherwise
        if (w.act == 0) continue;
        if (r.sink < 0 || r.cap < 1 || r.head < 0 || r.head >= r.cap || r.count < 0 || r.count > r.cap || n < 0 || n > a.NT) {
          atomicOr(p.status, PTENC_ST_BAD_INDEX);
          continue;
        }
        const int node0 = qp * 2 * a.npt;
        if (node0 >= n) continue;
        const int ev0 = min(tree_evicted(r.count, r.cap, r.e, 1), r.count);
        int t0, len2;
        int head2 = r.head + ev0;
        if (head2 >= r.cap) head2 -= r.cap;
        const int nt = tt_tiles(r.sink, head2, r.count - ev0, W, &t0, &len2) + 1;     // the draft's own tile is the last
        if (pieces > nt) pieces = nt;
        if (piece >= pieces) continue;
        const int lo = (int)((long long)piece * nt / pieces);
        const int cnt = (int)((long long)(piece + 1) * nt / pieces) - lo;
        const bool two = n - node0 > a.npt;
        const uint32_t slot = seq & 1;
        if (!bar_wait(item_empty + 8 * slot, ((seq >> 1) & 1) ^ 1, abort_flag)) { okay = false; break; }
        volatile int* d = desc + slot * I_WORDS;
        d[I_LB] = li * B + b; d[I_H] = h; d[I_NODE0] = node0; d[I_N] = n; d[I_TWO] = two ? 1 : 0;
        d[I_HEAD] = r.head; d[I_COUNT] = r.count; d[I_SINK] = r.sink; d[I_CHUNK] = r.e; d[I_T0] = t0; d[I_LEN2] = len2;
        d[I_LO] = lo; d[I_CNT] = cnt; d[I_NT] = nt; d[I_PIECES] = pieces; d[I_PIECE] = piece;
        d[I_SPLIT] = pieces > 1 ? split : -1;
        d[I_KIND] = 1;
        bar_arrive(item_full + 8 * slot);
        ++seq;
        const int row = (li * B + b) * a.NT;             // first node of the sequence in the call's tensors
        for (int t = 0; t < (two ? 2 : 1); ++t, ++qn) {
          const uint32_t qs = qn & 1;
          if (!bar_wait(q_empty + 8 * qs, ((qn >> 1) & 1) ^ 1, abort_flag)) { okay = false; break; }
          bar_expect(q_full + 8 * qs, (uint32_t)(DH * g * a.npt * 128));
          for (int hf = 0; hf < DH; ++hf)
            tma_3d(sb + SM::OFF_Q + qs * TILE + hf * HALF, &tmQ, hf * 64, h * g, row + node0 + t * a.npt, q_full + 8 * qs);
        }
        if (!okay) break;
        const int z = (int)(lb * Hkv + h);
        for (int k = 0; k < 2 * cnt; ++k, ++pos) {
          // entry k of the item: which tile, and whether its K or its V
          int i;
          bool is_v;
          if (two) { i = k >> 1; is_v = k & 1; }
          else if (k < 2 && cnt > 1) { i = k; is_v = false; }
          else if (k == 2 * cnt - 1) { i = cnt - 1; is_v = true; }
          else if (k & 1) { i = (k + 1) >> 1; is_v = false; }
          else { i = cnt > 1 ? (k - 2) >> 1 : 0; is_v = cnt > 1; }
          const uint32_t s = pos % NS, bar = full + 8 * s, dst = sb + s * TILE;
          if (!bar_wait(empty + 8 * s, ((pos / NS) & 1) ^ 1, abort_flag)) { okay = false; break; }
          if (lo + i == nt - 1) {
            bar_expect(bar, (uint32_t)(DH * a.nb * 128));
            for (int hf = 0; hf < DH; ++hf) tma_3d(dst + hf * HALF, is_v ? &tmVt : &tmKt, hf * 64, h, row, bar);
          } else {
            const int u = lo + i;
            const int j = u < len2 ? t0 + u : u - len2;
            bar_expect(bar, (uint32_t)(DH * a.ring_box * 128));
            for (int hf = 0; hf < DH; ++hf) tma_3d(dst + hf * HALF, is_v ? &tmV : &tmK, hf * 64, j * TN, z, bar);
          }
        }
      }
      if (!okay) { atomicOr(p.status, PTENC_ST_WAIT_TIMEOUT); *abort_flag = 1; }
      // whatever the other roles did, copies in flight land before the shared memory goes away
      for (uint32_t i = 1; i <= (uint32_t)NS && i <= pos; ++i) bar_drain(full + 8 * ((pos - i) % NS), ((pos - i) / NS) & 1);
      for (uint32_t i = 1; i <= 2 && i <= qn; ++i) bar_drain(q_full + 8 * ((qn - i) & 1), ((qn - i) >> 1) & 1);
    }
  } else if (warp == 1) {
    // ================================================================ MMA issuer
    // The whole warp takes every step, so that addresses, descriptors and counters are alike in all lanes and can live in
    // uniform registers, which the MMA instruction takes its operands from; one elected lane issues.  With the steps
    // behind `lane == 0` an MMA cost about 100 cycles to issue, more than it takes to run.
    const bool leader = tt_elect();
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
      return __all_sync(0xffffffffu, bar_wait(bar, parity, abort_flag));
    };
    constexpr uint32_t ID_QK = tt_idesc(TN, 0), ID_PV = tt_idesc(D, 1);
    const uint32_t ID_QKD = tt_idesc(a.nb, 0);
    uint32_t base = 0, qn = 0, seq = 0, items = 0;
    uint32_t np0 = 0, np1 = 0;                           // tiles of the streams whose P has been taken
    bool okay = true;
    while (okay) {
      if (!wait(item_full + 8 * (seq & 1), (seq >> 1) & 1)) { okay = false; break; }
      volatile int* d = desc + (seq & 1) * I_WORDS;
      const int kind = __shfl_sync(0xffffffffu, d[I_KIND], 0);
      if (kind == 0) break;
      const bool two = __shfl_sync(0xffffffffu, d[I_TWO], 0) != 0;
      const int n = __shfl_sync(0xffffffffu, d[I_CNT], 0);
      const int draft = __shfl_sync(0xffffffffu, d[I_NT] - 1 - d[I_LO], 0);   // the draft's tile, if the item has it
      __syncwarp();
      if (leader) bar_arrive(item_empty + 8 * (seq & 1));
      ++seq;
      const uint32_t q0 = qn, nq = two ? 2 : 1;
      const int stride = two ? 1 : 2;                    // a stream's next tile
      const int off1 = two ? 0 : 1;                      // with one row tile the second stream takes the odd tiles
      // S = Q K^T of tile i; whoever sees it done knows that the stream's products before it are done too
      auto issue_s = [&](auto ST, int i) {
        constexpr int st = decltype(ST)::value;
        const uint32_t s = (base + pos_k(i, two)) % NS;
        const uint64_t dq = desc_k(sb + SM::OFF_Q + ((q0 + (two ? st : 0)) & 1) * TILE), dk = desc_k(sb + s * TILE);
        const uint32_t id = i == draft ? ID_QKD : ID_QK;
        if (leader) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint64_t off = ((k >> 2) * HALF + (k & 3) * 32) >> 4;        // the address field counts 16 bytes
            mma_ss(tS + st * TN, dq + off, dk + off, id, k > 0);
          }
          commit(s_full + 8 * st);
        }
        __syncwarp();
      };
      auto wait_k = [&](int i) -> bool {
        if (i >= n) return true;
        const uint32_t ps = base + pos_k(i, two);
        return wait(full + 8 * (ps % NS), (ps / NS) & 1);
      };
      bool first = true;
      // O += P V of the stream's tile i, then S of its next tile.  What does not depend on P is waited for first.
      auto step = [&](auto ST, int i, uint32_t& np) -> bool {
        constexpr int st = decltype(ST)::value;
        if (i >= n) return true;
        const uint32_t ps = base + pos_v(i, n, two), s = ps % NS;
        const uint64_t dv = desc_mn(sb + s * TILE);
        const uint32_t start = i < stride ? 0u : 1u;                           // 0: the product replaces what O holds
        const int ks = i == draft ? a.nb / 16 : TN / 16;
        if (first && !wait(o_empty, (items & 1) ^ 1)) return false;            // O of the item before is out
        first = false;
        if (!wait(ready + 8 * s, (ps / NS) & 1) || !wait_k(i + stride)) return false;
        if (!wait(p_full + 8 * st, np & 1)) return false;
        ++np;
        fence_after();
        if (leader) {
#pragma unroll
          for (int k = 0; k < TN / 16; ++k)
            if (k < ks)                                  // P lies at the start of each half of S
              mma_ts(tO + st * D, tS + st * TN + (k >> 2) * TH + (k & 3) * 8, dv + (k * 2048 >> 4), ID_PV, k > 0 ? 1u : start);
          if (!two) commit(empty + 8 * s);               // the V tile is this stream's alone and free when that is done
          if (i + stride >= n) commit(o_full + 8 * st);
        }
        __syncwarp();
        if (i + stride < n) issue_s(ST, i + stride);
        return true;
      };
      using S0 = std::integral_constant<int, 0>;
      using S1 = std::integral_constant<int, 1>;
      for (uint32_t t = 0; t < nq && okay; ++t) okay = wait(q_full + 8 * ((q0 + t) & 1), ((q0 + t) >> 1) & 1);
      okay = okay && wait_k(0);
      fence_after();
      if (okay) issue_s(S0(), 0);
      if (okay && off1 < n) {
        okay = wait_k(off1);
        fence_after();
        if (okay) issue_s(S1(), off1);
      }
      for (int i = 0; i < n && okay; i += stride) okay = step(S0(), i, np0) && step(S1(), i + off1, np1);
      if (okay && leader)
        for (uint32_t t = 0; t < nq; ++t) commit(q_empty + 8 * ((q0 + t) & 1));
      __syncwarp();
      qn += nq;
      base += 2 * n;
      ++items;
    }
    if (leader) {
      if (!okay) { atomicOr(p.status, PTENC_ST_WAIT_TIMEOUT); *abort_flag = 1; }
      commit(drain);                                     // MMAs still in flight finish before tensor memory is freed
      bar_drain(drain, 0);
    }
    __syncwarp();
  } else {
    // ================================================================ patch warps
    const int me = warp - 2;
    uint32_t base = 0, seq = 0;
    bool okay = true;
    // the lanes give up together, or not at all
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
      return __all_sync(0xffffffffu, bar_wait(bar, parity, abort_flag));
    };
    while (okay) {
      if (!wait(item_full + 8 * (seq & 1), (seq >> 1) & 1)) { okay = false; break; }
      volatile int* d = desc + (seq & 1) * I_WORDS;
      if (d[I_KIND] == 0) break;
      const bool two = d[I_TWO] != 0;
      const int n = d[I_CNT], nodes = d[I_N], lo = d[I_LO], nt = d[I_NT], t0 = d[I_T0], len2 = d[I_LEN2];
      TreeRing r;
      r.head = d[I_HEAD]; r.count = d[I_COUNT]; r.sink = d[I_SINK]; r.cap = W - r.sink; r.e = d[I_CHUNK];
      const int ev0 = min(tree_evicted(r.count, r.cap, r.e, 1), r.count);
      int ev_max;
      if (me == 0) {
        // ---- what each node sees: the parent relation closed by pointer doubling, two nodes per lane ---------------------
        const int32_t* par = a.parent + (size_t)(d[I_LB] % B) * a.NT;
        int pa[2];
        unsigned long long anc[2] = {0ull, 0ull};
        int bad = 0;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int i = lane + 32 * x;
          pa[x] = -1;
          if (i < nodes) {
            const int v = par[i];
            if (v < -1 || v >= i) bad = 1; else pa[x] = v;
            anc[x] = 1ull << i;
          }
        }
        bad = __any_sync(0xffffffffu, bad);
        if (bad) { pa[0] = pa[1] = -1; }
        if (!wait(info_empty, (seq & 1) ^ 1)) { okay = false; break; }   // the rows have what they need of the last item
        for (int s = 1; s < nodes; s <<= 1) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            s_vis[lane + 32 * x] = anc[x];
            s_jump[lane + 32 * x] = (int8_t)pa[x];
          }
          __syncwarp();
#pragma unroll
          for (int x = 0; x < 2; ++x)
            if (pa[x] >= 0) { anc[x] |= s_vis[pa[x]]; pa[x] = s_jump[pa[x]]; }
          __syncwarp();
        }
        int deepest = 0;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int depth = __popcll(anc[x]) - 1;
          s_depth[lane + 32 * x] = (uint8_t)(depth < 0 ? 0 : depth);
          deepest = max(deepest, depth);
        }
        __syncwarp();
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int gone = tree_evicted(r.count, r.cap, r.e, __popcll(anc[x]));
          unsigned long long v = anc[x];
          if (gone > r.count) {                          // a path longer than the ring: its first tokens have left again
            v = 0;
            for (unsigned long long m = anc[x]; m != 0; m &= m - 1) {
              const int j = __ffsll((long long)m) - 1;
              if (r.count + s_depth[j] >= gone) v |= 1ull << j;
            }
          }
          s_vis[lane + 32 * x] = v;
        }
        deepest = __reduce_max_sync(0xffffffffu, deepest);
        ev_max = tree_evicted(r.count, r.cap, r.e, deepest + 1);
        if (lane == 0) {
          if (bad) atomicOr(p.status, PTENC_ST_BAD_INDEX);
          d[I_EVMAX] = ev_max;
          d[I_VALID] = bad ? 0 : 1;
          d[I_ODD] = 0;
        }
        __syncwarp();
        if (lane == 0) bar_arrive(info_full);
      } else {
        if (!wait(info_full, seq & 1)) { okay = false; break; }
        ev_max = d[I_EVMAX];
        __syncwarp();
        if (lane == 0) bar_arrive(info_empty);
      }
      // ---- pass the stages on, in ring order --------------------------------------------------------------------------------
      for (int k = 0; k < 2 * n; ++k) {
        int i = -1;                                      // the tile whose V this entry is, if it is one
        if (two) { if (k & 1) i = k >> 1; }
        else if (k == 2 * n - 1) i = n - 1;
        else if (k >= 2 && (k & 1) == 0) i = (k - 2) >> 1;
        const uint32_t ps = base + k, s = ps % NS;
        if (!wait(full + 8 * s, (ps / NS) & 1)) { okay = false; break; }
        if (i >= 0) {
          const int u = lo + i;
          const bool draft = u == nt - 1;
          const int slot0 = (u < len2 ? t0 + u : u - len2) * TN;
          bool clean = false;
          if (!draft) {
            int d0 = slot0 - r.sink - r.head;
            if (d0 < 0) d0 += r.cap;
            clean = slot0 + TN <= r.sink ||
                    (slot0 >= r.sink && slot0 + TN <= W &&
                     ((d0 >= ev_max && d0 + TN <= r.count) || (ev_max == 0 && r.count == r.cap)));
          }
          if (!clean) {
            // which rows nobody sees and which only some nodes see, 32 at a time; then 16 bytes per lane of those rows
            uint8_t* v = smem + s * TILE;
            constexpr int VPR = DH * 8;                  // 16-byte vectors of a row
            const int rows = draft ? a.nb : TN;
            int odd = 0;
            for (int rb = 32 * me; rb < rows; rb += 64) {          // the two warps take turns
              const int t = rb + lane;
              bool dead, some;
              if (draft) {
                dead = t >= nodes;
                some = !dead;
              } else {
                const int slot = slot0 + t;
                int dd = slot - r.sink - r.head;
                if (dd < 0) dd += r.cap;
                dead = slot >= r.sink && (slot >= W || dd < ev0 || dd >= r.count);
                some = !dead && slot >= r.sink && dd < ev_max;
              }
              const unsigned m_dead = __ballot_sync(0xffffffffu, dead && t < rows);
              unsigned todo = m_dead | __ballot_sync(0xffffffffu, some && t < rows);
              while (todo != 0) {
                // 32 / VPR rows at a time: this lane's is the (lane / VPR)-th of those left
                int at = __ffs(todo) - 1;
                unsigned rest = todo & (todo - 1);
#pragma unroll
                for (int y = 1; y < 32 / VPR; ++y) {
                  if (lane / VPR >= y) at = rest != 0 ? __ffs(rest) - 1 : -1;
                  rest &= rest - 1;
                }
                todo = rest;
                if (at < 0) continue;
                const int c = lane % VPR;
                uint4* vec = reinterpret_cast<uint4*>(v + (c >> 3) * HALF + (rb + at) * 128 + (c & 7) * 16);
                if ((m_dead >> at) & 1u) {
                  *vec = make_uint4(0u, 0u, 0u, 0u);
                } else {
                  uint4 w = *vec;
                  uint32_t* e = reinterpret_cast<uint32_t*>(&w);
                  uint32_t top = 0;                      // exponent bits all set, infinity or NaN, carry into the sign's place
#pragma unroll
                  for (int y = 0; y < 4; ++y) top |= (e[y] & 0x7fff7fffu) + 0x00800080u;
                  int hit = 0;
                  if ((top & 0x80008000u) != 0) {
                    hit = 1;
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                      if ((e[y] & 0x7f80u) == 0x7f80u) e[y] &= 0xffff0000u;
                      if ((e[y] & 0x7f800000u) == 0x7f800000u) e[y] &= 0x0000ffffu;
                    }
                  }
                  if (hit) { *vec = w; odd = 1; }
                }
              }
            }
            if (__any_sync(0xffffffffu, odd) && lane == 0) d[I_ODD] = 1;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
          }
        }
        if (lane == 0) { bar_arrive(ready + 8 * s); bar_arrive(empty + 8 * s); }
      }
      if (!okay) break;
      __syncwarp();
      if (lane == 0) bar_arrive(item_empty + 8 * (seq & 1));
      ++seq;
      base += 2 * n;
    }
    if (!okay && lane == 0) { atomicOr(p.status, PTENC_ST_WAIT_TIMEOUT); *abort_flag = 1; }
  }
  } else {
    // ================================================================ softmax: stream st, a row per thread
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(TT_REGS_HIGH));
    const int st = (warp - 4) >> 3, half = ((warp - 4) >> 2) & 1, quarter = warp & 3;
    const int lrow = 32 * quarter + lane;
    const uint32_t lane_off = (uint32_t)(32 * quarter) << 16;
    const bool passes = tid == TT_LEAD + 256 * st;       // the thread of the stream that gives stages back
    const float sl2 = 1.4426950408889634f / sqrtf((float)D), slack = 8.f / sl2;
    uint32_t seq = 0, ntile = 0, base = 0;               // items; tiles of this stream; ring entries
    uint32_t no0 = 0, no1 = 0;                           // items in which the streams had tiles
    bool fine = true;                                    // a wait that ran out: go through the motions, never wait again
    auto wait = [&](uint32_t bar, uint32_t parity) {
      if (fine && !bar_wait(bar, parity, abort_flag)) {
        fine = false;
        atomicOr(p.status, PTENC_ST_WAIT_TIMEOUT);
        *abort_flag = 1;
      }
    };
    while (true) {
      // one thread waits for the item and posts what all warps then read, so that they agree on going on
      if (tid == TT_LEAD) {
        int v = 0;
        if (*abort_flag == 0 && bar_wait(item_full + 8 * (seq & 1), (seq >> 1) & 1, abort_flag)) v = desc[(seq & 1) * I_WORDS + I_KIND];
        misc[2] = v;
      }
      soft_sync();
      if (misc[2] != 1) break;
      wait(item_full + 8 * (seq & 1), (seq >> 1) & 1);
      wait(info_full, seq & 1);
      volatile int* d = desc + (seq & 1) * I_WORDS;
      const bool two = d[I_TWO] != 0;
      const int n = d[I_CNT], nodes = d[I_N], lo = d[I_LO], nt = d[I_NT], t0 = d[I_T0], len2 = d[I_LEN2];
      const int ev_max = d[I_EVMAX], valid = d[I_VALID];
      TreeRing r;
      r.head = d[I_HEAD]; r.count = d[I_COUNT]; r.sink = d[I_SINK]; r.cap = W - r.sink; r.e = d[I_CHUNK];
      const int node_l = lrow / g, hh = lrow - node_l * g;
      const int node = d[I_NODE0] + (two ? st * a.npt : 0) + node_l;
      const bool real = node_l < a.npt && node < nodes;
      const unsigned long long vis = real ? s_vis[node] : 0ull;
      const int ev = real ? tree_evicted(r.count, r.cap, r.e, s_depth[node] + 1) : 0;
      const bool idle = __all_sync(0xffffffffu, !real);  // a warp without rows only keeps the barriers going
      __syncwarp();
      if (lane == 0) bar_arrive(info_empty);
      float m = -INFINITY, l = 0.f;                      // running maximum (of the raw scores) and this half's sum
      const int stride = two ? 1 : 2;
#pragma unroll 1
      for (int i = two ? 0 : st; i < n; i += stride, ++ntile) {
        const int u = lo + i;
        const bool draft = u == nt - 1;
        const int slot0 = (u < len2 ? t0 + u : u - len2) * TN + half * TH;
        bool clean = false;
        uint32_t keep0 = 0, keep1 = 0;                   // columns the row sees
        if (draft) {
          if (half == 0) { keep0 = (uint32_t)vis; keep1 = (uint32_t)(vis >> 32); }
        } else {
          int d0 = slot0 - r.sink - r.head;
          if (d0 < 0) d0 += r.cap;
          clean = slot0 + TH <= r.sink ||
                  (slot0 >= r.sink && slot0 + TH <= W &&
                   ((d0 >= ev_max && d0 + TH <= r.count) || (ev_max == 0 && r.count == r.cap)));
          if (!clean) {
            // three runs of slots: pinned; from the oldest one seen to the end of the ring; what has wrapped round
            const int z = r.sink + r.head - slot0;
            const int lo1 = z + ev, hi1 = min(z + r.count, W - slot0);
            const int lo2 = max(z - r.cap + ev, r.sink - slot0), hi2 = min(z - r.cap + r.count, z);
            keep0 = run_mask(-slot0, r.sink - slot0, 0) | run_mask(lo1, hi1, 0) | run_mask(lo2, hi2, 0);
            keep1 = run_mask(-slot0, r.sink - slot0, 32) | run_mask(lo1, hi1, 32) | run_mask(lo2, hi2, 32);
          }
        }
        wait(s_full + 8 * st, ntile & 1);
        fence_after();
        if (passes && (!two || st == 1)) {               // S is done, and with two row tiles both streams' products with the V before it
          bar_arrive(empty + 8 * ((base + pos_k(i, two)) % NS));
          if (two && i > 0) bar_arrive(empty + 8 * ((base + pos_v(i - 1, n, two)) % NS));
        }
        const bool some = !idle && !(draft && half == 1);          // uniform over the warp
        // The scores are read from tensor memory twice, 32 at a time, once for the maximum and once for P: held in registers
        // they would push everything else out of them.
        const uint32_t ts = tS + st * TN + half * TH + lane_off;
        float mine = -INFINITY;
        if (some) {
#pragma unroll 1
          for (int c = 0; c < TH; c += 32) {
            float x[32];
            ld32(ts + c, x);
            wait_ld();
            if (!clean) {
              const uint32_t keep = c == 0 ? keep0 : keep1;
#pragma unroll
              for (int y = 0; y < 32; ++y)
                if (!(keep & (1u << y))) x[y] = -INFINITY;
            }
            float mx[4] = {mine, x[0], x[1], x[2]};
#pragma unroll
            for (int y = 3; y < 31; y += 2) mx[(y >> 1) & 3] = tt_max3(mx[(y >> 1) & 3], x[y], x[y + 1]);
            mine = tt_max3(tt_max3(mx[0], mx[1], mx[2]), mx[3], x[31]);
          }
        }
        s_mx[(2 * st + half) * TM + lrow] = mine;        // the halves agree on a maximum
        stream_sync(st);
        const float mnew = tt_max3(m, mine, s_mx[(2 * st + 1 - half) * TM + lrow]);
        if (i < stride) {
          m = mnew;
        } else {
          const bool grown = !(mnew <= m + slack);       // NaN counts; nothing seen yet and nothing now (-inf) does not
          if (!idle && __any_sync(0xffffffffu, grown)) {
            // between the references as they were rounded, which for large scores is not their distance
            const float corr = grown ? tt_ex2(__fmul_rn(m, sl2) - __fmul_rn(mnew, sl2)) : 1.f;
            if (grown) m = mnew;
            l *= corr;
            // O is at rest; each half of the threads rescales half of the columns
#pragma unroll 1
            for (int c = half * (D / 2); c < (half + 1) * (D / 2); c += 16) {
              float o[16];
              ld16(tO + st * D + lane_off + c, o);
              wait_ld();
#pragma unroll
              for (int y = 0; y < 16; ++y) o[y] *= corr;
              st16(tO + st * D + lane_off + c, reinterpret_cast<uint32_t*>(o));
            }
          }
        }
        if (some) {
          // an infinite maximum makes the row NaN, as inf - inf does
          const float neg = m == -INFINITY ? 0.f : m == INFINITY ? __int_as_float(0x7fffffff) : -__fmul_rn(m, sl2);
          const uint64_t neg2 = tt_two(neg, neg), scl2 = tt_two(sl2, sl2);
          uint64_t sum[2] = {0ull, 0ull};
#pragma unroll 1
          for (int c = 0; c < TH; c += 32) {
            float x[32];
            uint32_t pk[16];
            ld32(ts + c, x);
            wait_ld();
            if (!clean) {
              const uint32_t keep = c == 0 ? keep0 : keep1;
#pragma unroll
              for (int y = 0; y < 32; ++y)
                if (!(keep & (1u << y))) x[y] = -INFINITY;
            }
#pragma unroll
            for (int y = 0; y < 32; y += 2) {
              float e0, e1;
              tt_both(tt_fma2(tt_two(x[y], x[y + 1]), scl2, neg2), e0, e1);
              e0 = tt_ex2(e0);
              e1 = tt_ex2(e1);
              sum[(y >> 1) & 1] = tt_add2(sum[(y >> 1) & 1], tt_two(e0, e1));
              // P in bf16, half a step of 2^-8 per weight: the product's operands are of one type and V is bf16.  The sum is of
              // the weights as they were.  Outputs are off by 2.3e-3 of their size instead of 1.7e-3 (the output's own
              // rounding); a second product for what the rounding cuts off would double half of the tensor work.
              pk[y >> 1] = tt_pack(e0, e1);
            }
            st16(ts + c / 2, pk);                        // over this half's own scores, those that have been read
          }
          float s0, s1;
          tt_both(tt_add2(sum[0], sum[1]), s0, s1);
          l += s0 + s1;
        }
        wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(p_full + 8 * st);
      }
      // ---- the item's rows ------------------------------------------------------------------------------------------------
      const bool both = two || n > 1;                    // the second stream had tiles
      if (!two || st == 0) wait(o_full, no0 & 1);
      if (both && (!two || st == 1)) wait(o_full + 8, no1 & 1);
      ++no0;
      if (both) ++no1;
      fence_after();
      if (passes && two && st == 1) bar_arrive(empty + 8 * ((base + pos_v(n - 1, n, two)) % NS));
      base += 2 * n;
      // (m, l) of both streams for everybody: first the halves' sums, then the streams' values
      float m0, l0, m1, l1;
      m = __fmul_rn(m, sl2);                             // base-2 units from here on (-inf stays)
      {
        float* s_l = reinterpret_cast<float*>(s_ml);
        stream_sync(st);                                 // the maxima of the last tile have been read
        soft_sync();
        if (half == 1) s_l[2 * lrow + st] = l;
        soft_sync();
        if (half == 0) l += s_l[2 * lrow + st];
        soft_sync();
        if (half == 0 && st == 1) s_ml[lrow] = make_float2(m, l);
        soft_sync();
        { const float2 v = s_ml[lrow]; m1 = v.x; l1 = v.y; }
        soft_sync();
        if (half == 0 && st == 0) s_ml[lrow] = make_float2(m, l);
        soft_sync();
        { const float2 v = s_ml[lrow]; m0 = v.x; l0 = v.y; }
      }
      const bool odd = d[I_ODD] != 0;
      const int split = d[I_SPLIT], pieces = d[I_PIECES], piece = d[I_PIECE];
      const int e = d[I_LB], h = d[I_H];
      const size_t lb = (size_t)a.l0 * B + e;
      // With one row tile both streams hold parts of the same rows; the columns are dealt to the groups of warps.
      float w0 = 1.f, w1 = 0.f;
      int c_lo, c_hi;
      if (two) {
        m = st == 0 ? m0 : m1;
        l = st == 0 ? l0 : l1;
        c_lo = half * (D / 2);
        c_hi = c_lo + D / 2;
      } else {
        m = fmaxf(m0, m1);
        w0 = m0 == -INFINITY ? 0.f : tt_ex2(m0 - m);
        w1 = m1 == -INFINITY ? 0.f : tt_ex2(m1 - m);
        l = w0 * l0 + w1 * l1;
        if (m0 != m0 || m1 != m1) m = l = __int_as_float(0x7fffffff);
        c_lo = D == 128 ? (2 * st + half) * 32 : (half == 0 ? st * 32 : D);
        c_hi = D == 128 ? c_lo + 32 : min(c_lo + 32, D);
      }
      const size_t orow = ((size_t)e * a.NT + node) * p.Hq + (size_t)h * g + hh;
      const float inv = m == -INFINITY ? __int_as_float(0x7fffffff) : 1.f / l;      // every score -inf: NaN
      const int tile_i = two ? st : 0;
      const size_t pslot = split >= 0 ? (((size_t)split * a.P + piece) * a.tpb + tile_i) : 0;
      float4* part = reinterpret_cast<float4*>(a.part) + pslot * (D / 4) * TM;
      const bool wide = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0;
      float4* s_part = reinterpret_cast<float4*>(smem);  // over the stages, whose products are done
#pragma unroll 1
      for (int c = c_lo; c < c_hi; c += 16) {
        float o[16];
        if (idle) continue;
        if (two) {
          ld16(tO + st * D + lane_off + c, o);
          wait_ld();
        } else {
          float o1[16];
          ld16(tO + lane_off + c, o);
          if (both) ld16(tO + D + lane_off + c, o1);
          wait_ld();
#pragma unroll
          for (int y = 0; y < 16; ++y) o[y] = both ? fmaf(o1[y], w1, o[y] * w0) : o[y] * w0;
        }
        if (odd && real) {                               // rare, and out of line: it would cost the tile loop its registers
          float x[16];
#pragma unroll
          for (int y = 0; y < 16; ++y) x[y] = o[y];
          add_not_finite(x, c, p, a.v_tree + ((size_t)e * a.NT * Hkv + h) * D, (lb * Hkv + h) * (size_t)W * D, r, ev, ev_max,
                         vis, nodes, lo, n, nt, t0, len2);
#pragma unroll
          for (int y = 0; y < 16; ++y) o[y] = x[y];
        }
        if (split >= 0) {
          if (real)
#pragma unroll
            for (int y = 0; y < 16; y += 4)
              (CL ? s_part + tile_i * (D / 4) * TM : part)[((c + y) >> 2) * TM + lrow] = make_float4(o[y], o[y + 1], o[y + 2], o[y + 3]);
        } else if (real && valid) {
          uint32_t pk[8];
#pragma unroll
          for (int y = 0; y < 16; y += 2) pk[y >> 1] = tt_pack(o[y] * inv, o[y + 1] * inv);
          tt_store(a.out + orow * D + c, pk, wide);
        }
      }
      fence_before();
      __syncwarp();
      if (lane == 0) { bar_arrive(o_empty); bar_arrive(item_empty + 8 * (seq & 1)); }
      if (CL) soft_sync();                               // the exchange is over
      if (real && half == 0 && (two || st == 0)) {       // once per row
        if (split >= 0) (CL ? s_ml + tile_i * TM : a.part_ml + pslot * TM)[lrow] = make_float2(m, l);
        else if (valid && a.lse != nullptr) a.lse[orow] = (m + log2f(l)) * 0.6931471805599453f;
      }
      if (tid == TT_LEAD && split >= 0 && piece == 0) (CL ? misc + 3 : a.pieces + split)[0] = valid ? pieces : 0;
      ++seq;
      soft_sync();                                       // misc[2] and the exchange buffer are free again
    }
  }

  fence_before();
  __syncthreads();
  if (warp == 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
  if (CL) {
    // the parts of the block lie in the CTAs of the cluster: everybody adds some of the rows
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    if (warp >= 4) {
      const int pieces = *cluster.map_shared_rank(const_cast<const int*>(misc) + 3, 0);
      const int total = pieces > 1 ? a.tpb * TM * (D / 8) : 0;
      for (int x = (int)cluster.block_rank() * TT_SOFT + tid - TT_LEAD; x < total; x += (int)cluster.num_blocks() * TT_SOFT)
        join_row<D>(a, p.B, Hkv, g, (int)blockIdx.x / a.P, x, pieces,
                    [&](int q, int tile, int at) { return *cluster.map_shared_rank(s_ml + tile * TM + at, q); },
                    [&](int q, int tile, int at) { return *cluster.map_shared_rank(reinterpret_cast<float4*>(smem) + tile * (D / 4) * TM + at, q); });
    }
    __syncwarp();
    cluster.sync();                                      // nobody leaves while its rows may still be read
  }
}

constexpr int TJ_THREADS = 256;

// Joins the parts of the blocks that were split.
template <int D>
__global__ void __launch_bounds__(TJ_THREADS)
k_tree_join(const __grid_constant__ TreeTcArgs a, int B, int Hkv, int g) {
  tree_after_previous();                                 // the parts are written
  tree_let_next_start();
  const int per = a.tpb * TM * (D / 8) / TJ_THREADS;     // CTAs per block
  const int split = blockIdx.x / per;
  const int pieces = a.pieces[split];
  if (pieces <= 1) return;
  const float4* part = reinterpret_cast<const float4*>(a.part) + (size_t)split * a.P * a.tpb * (D / 4) * TM;
  const float2* ml = a.part_ml + (size_t)split * a.P * a.tpb * TM;
  join_row<D>(a, B, Hkv, g, split, (blockIdx.x - split * per) * TJ_THREADS + threadIdx.x, pieces,
              [&](int q, int tile, int at) { return __ldcg(ml + (q * a.tpb + tile) * TM + at); },
              [&](int q, int tile, int at) { return __ldcg(part + (q * a.tpb + tile) * (D / 4) * TM + at); });
}

// ------------------------------------------------------------------------------------------------ host
typedef CUresult (*TtEncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                               const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                               CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

TtEncodeFn tt_encode_fn() {
  static std::atomic<TtEncodeFn> fn;
  if (fn != nullptr) return fn;
  void* ptr = nullptr;
  cudaDriverEntryPointQueryResult qres;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) != cudaSuccess ||
      qres != cudaDriverEntryPointSuccess)
    return nullptr;
  fn = reinterpret_cast<TtEncodeFn>(ptr);
  return fn;
}

// bf16 [n2][n1][D], box [b2][b1][64], 128-byte swizzle; what lies outside the tensor reads as zero.
bool tt_map(CUtensorMap* map, const void* base, int D, long long n1, long long n2, int b1, int b2) {
  TtEncodeFn fn = tt_encode_fn();
  if (fn == nullptr) return false;
  cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)n1, (cuuint64_t)n2};
  cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)n1 * D * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)b1, (cuuint32_t)b2};
  cuuint32_t estr[3] = {1, 1, 1};
  return ptenc_encode_map([&] {
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  });
}

template <int D>
cudaError_t tt_attributes(int device) {
  static PtencOnce once;
  return ptenc_first_use(once, device, [] {
    const cudaError_t e = ptenc_allow_smem(k_tree_tc<D, false>, TSmem<D>::TOTAL);
    return e != cudaSuccess ? e : ptenc_allow_smem(k_tree_tc<D, true>, TSmem<D>::TOTAL);
  });
}

template <int D>
cudaError_t tt_launch(ptenc_cache* c, const CUtensorMap& q, const CUtensorMap& kt, const CUtensorMap& vt,
                      const TreeTcArgs& a, int grid, bool clusters, cudaStream_t st) {
  cudaError_t e = tt_attributes<D>(c->cfg.device);
  if (e != cudaSuccess) return e;
  c->launches++;
  if (clusters)
    return tree_launch(k_tree_tc<D, true>, dim3(grid), TT_THREADS, TSmem<D>::TOTAL, a.P, st, c->dev, c->tmTreeK, c->tmTreeV, q, kt, vt, a);
  e = tree_launch(k_tree_tc<D, false>, dim3(grid), TT_THREADS, TSmem<D>::TOTAL, 0, st, c->dev, c->tmTreeK, c->tmTreeV, q, kt, vt, a);
  if (e != cudaSuccess || a.P == 1 || a.n_items == a.n_full) return e;
  c->launches++;
  return tree_launch(k_tree_join<D>, dim3((unsigned)((a.n_items - a.n_full) / a.P * (a.tpb * TM * (D / 8) / TJ_THREADS))), TJ_THREADS,
                     0, 0, st, a, c->dev.B, c->dev.Hkv, c->dev.g);
}

// Clusters of `size` CTAs that the device holds at a time (one CTA per SM), -1 if it cannot say.
template <int D>
int tt_clusters(int device, int size) {
  if (tt_attributes<D>(device) != cudaSuccess) {
    cudaGetLastError();
    return -1;
  }
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3(size);
  cfg.blockDim = dim3(TT_THREADS);
  cfg.dynamicSmemBytes = TSmem<D>::TOTAL;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, k_tree_tc<D, true>, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return -1;
  }
  return n;
}

}  // namespace

// Bytes of the scratch that the parts of split blocks need: partial rows and their (m, l).
bool ptenc_tree_tc_shape(const ptenc_config* c) {
  return c->dtype == PTENC_DTYPE_BF16 && (c->head_dim == 64 || c->head_dim == 128) && c->policy == PTENC_POLICY_FIFO &&
         c->n_q_heads / c->n_kv_heads <= TM;
}
size_t ptenc_tree_part_bytes(const ptenc_config* c) { return (size_t)PTENC_TREE_SLOTS * TM * c->head_dim * 4; }
size_t ptenc_tree_ml_bytes(const ptenc_config*) { return (size_t)PTENC_TREE_SLOTS * TM * 8; }

bool ptenc_tree_tc_prepare(ptenc_cache* c) {
  c->tree_tc = false;
  if (!ptenc_tree_tc_shape(&c->cfg)) return false;
  const PtencDev& p = c->dev;
  const long long units = (long long)p.L * p.B * p.Hkv;
  const int box = p.W < TN ? p.W : TN;
  c->tree_tc = tt_map(&c->tmTreeK, p.K, p.D, p.W, units, box, 1) && tt_map(&c->tmTreeV, p.V, p.D, p.W, units, box, 1);
  // 1 + clusters of 2, 4, 8 CTAs; alike for every handle on the device, so threads that find none ask for the same
  static std::atomic<int> held[PTENC_MAX_DEVICES][2][3];
  for (int i = 0; i < 3; ++i) {
    int x = 0;
    const bool keep = c->cfg.device < PTENC_MAX_DEVICES;
    if (keep) x = held[c->cfg.device][p.D == 128][i];
    if (x == 0) x = 1 + (p.D == 128 ? tt_clusters<128>(c->cfg.device, 2 << i) : tt_clusters<64>(c->cfg.device, 2 << i));
    if (keep) held[c->cfg.device][p.D == 128][i] = x;    // 0: the next handle asks again
    c->tree_clusters[i] = x > 0 ? x - 1 : 0;
  }
  return c->tree_tc;
}

cudaError_t ptenc_launch_tree(ptenc_cache* c, int l0, int nl, const void* q, const void* k_tree, const void* v_tree,
                              const int32_t* parent, const int32_t* n_nodes, int max_nodes, const uint8_t* active, void* out,
                              float* lse, cudaStream_t st) {
  const PtencDev& p = c->dev;
  CUtensorMap mq, mk, mv;
  const long long nodes = (long long)nl * p.B * max_nodes;
  const int npt = c->tree_tc ? TM / p.g : 0, nb = (max_nodes + 15) / 16 * 16;
  if (!c->tree_tc || nodes >= (1ll << 31) || !tt_map(&mq, q, p.D, p.Hq, nodes, p.g, npt) ||
      !tt_map(&mk, k_tree, p.D, p.Hkv, nodes, 1, nb) || !tt_map(&mv, v_tree, p.D, p.Hkv, nodes, 1, nb))
    return ptenc_launch_tree_generic(c, l0, nl, q, k_tree, v_tree, parent, n_nodes, max_nodes, active, out, lse, st);
  TreeTcArgs a;
  memset(&a, 0, sizeof(a));
  a.l0 = l0; a.NT = max_nodes; a.npt = npt; a.tpb = max_nodes > npt ? 2 : 1;
  a.nqp = (max_nodes + 2 * npt - 1) / (2 * npt);
  a.nb = nb;
  a.ring_box = p.W < TN ? p.W : TN;
  a.parent = parent; a.n_nodes = n_nodes; a.active = active;
  a.out = static_cast<__nv_bfloat16*>(out); a.lse = lse; a.v_tree = static_cast<const __nv_bfloat16*>(v_tree);
  a.part = c->tree_part; a.part_ml = reinterpret_cast<float2*>(c->tree_ml); a.pieces = c->tree_pieces;
  // Whole rounds of blocks, one block per SM; the blocks of the last, partial round are cut into P parts each, so that
  // they fill the SMs too.  Microseconds: an item costs about 4 and 1.2 per tile (1.6 with two row tiles), the join 3.  The host
  // does not know the ring words: every block counts as a full window of nodes that are all there, so uneven batches are cut
  // worse than this says (23 sequences of 1 to 13 nodes and all lengths: 25 us by it, 38 to 44 measured).
  const long long blocks = (long long)nl * p.B * p.Hkv * a.nqp;
  if (blocks > (1ll << 30)) return cudaErrorInvalidValue;
  const int sms = c->sm_count, rem = (int)(blocks % sms), nt = (p.W + TN - 1) / TN + 1;
  a.n_full = (int)(blocks - rem);
  a.P = 1;
  float best = 1e30f;
  for (int P = 1; P <= TT_MAX_PIECES && P <= nt && (rem * P * a.tpb <= PTENC_TREE_SLOTS || P == 1); ++P) {
    const float cost = (float)((rem * P + sms - 1) / sms) * (4.f + (a.tpb == 2 ? 1.6f : 1.2f) * (float)((nt + P - 1) / P)) + (P > 1 ? 3.f : 0.f);
    if (cost < best) { best = cost; a.P = P; }
  }
  // Where a cluster can hold every block's parts, they are joined in its shared memory instead, without a second kernel.
  bool clusters = false;
  for (int i = 0; i < 3 && a.n_full == 0; ++i) {
    const int P = 2 << i;
    if (P > nt || rem > c->tree_clusters[i]) continue;
    const float cost = 4.f + (a.tpb == 2 ? 1.6f : 1.2f) * (float)((nt + P - 1) / P) + 1.f;
    if (cost < best) { best = cost; a.P = P; clusters = true; }
  }
  a.n_items = a.n_full + rem * a.P;
  const int grid = clusters || a.n_items < sms ? a.n_items : sms;
  return p.D == 128 ? tt_launch<128>(c, mq, mk, mv, a, grid, clusters, st) : tt_launch<64>(c, mq, mk, mv, a, grid, clusters, st);
}

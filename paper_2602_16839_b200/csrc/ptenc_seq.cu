// Attention over whole sequences: the entry points, and the shape-generic kernels (fp32, head sizes above 128).
//
//   s_ij = scale q_i . k_j,  p_ij = exp(s_ij - lse_i),  o_i = sum_j p_ij v_j  over the j that i sees;
//   dv_j = sum_i p_ij do_i,  ds_ij = p_ij (do_i . v_j - do_i . o_i),  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i.
//
// A CTA has a tile of M rows (64, or 32 where a head is wider than 128) and goes through the tiles of the other side, all in
// fp32 from shared memory, an (M / 16) x (M / 16) block of scores and (M / 16) x (D / 16) of sums per thread.  The backward pass is
// two kernels, one per side, each recomputing the scores: seven products instead of five, but no sums in an order that changes, so
// results have the same bits every time.  The tiles of the other side are copied a tile ahead where shared memory has room for
// two.  Where there are few tiles of rows, the tiles of the other side (for keys and values: of all heads of the group) are dealt to a
// cluster of CTAs, which join their sums in order through distributed shared memory.
//
// Bound by what a tile takes one CTA alone, 7 us where its multiply-adds are 2 (eight warps do not hide the latencies of shared memory
// and of the row sums), times the longest sequence's tiles: nine fp32 sequences of 3001 tokens in all, 4 + 1 heads of 64, forward 68 us,
// dq 90, dk and dv 140.
#include <cooperative_groups.h>

#include "ptenc_seq.cuh"
#include "ptenc_tc.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int SG_THREADS = 256, SG_MAX_CLUSTER = 8;
// In a tile that some rows see in part, what a row does not see is marked by this NaN, which arithmetic does not produce, and
// left out of the sums: a product by zero would carry the infinities and NaN of unseen tokens along.
constexpr unsigned SG_UNSEEN = 0xFFFFDEADu;

template <int DP>
struct SgShape {
  static constexpr int M = DP <= 128 ? 64 : 32;
  static constexpr int R = M / 16;               // rows, and columns of scores, of a thread
  static constexpr int LD = DP + 4;              // row pitch: rows 4 banks apart, so 16-byte reads of 8 rows fill all banks
  static constexpr int LP = M + 4;
  static constexpr int TILE = M * LD;
  // floats of shared memory with `bufs` buffers for the tiles of the other side
  static constexpr int fwd(int bufs) { return (1 + 2 * bufs) * TILE + M * LP; }
  static constexpr int dq(int bufs) { return (2 + 2 * bufs) * TILE + M * LP; }
  static constexpr int dkv(int bufs) { return (2 + 2 * bufs) * TILE + 2 * M * LP + bufs * 2 * M; }
  static constexpr int room = 232448 / 4, half = (233472 / 2 - 1024) / 4;
  // One buffer where two CTAs share an SM then, two otherwise: eight fp32 sequences of 2048 tokens, 8 + 2 heads of 64, dq 1505 us so, 1735
  // with two buffers, dk and dv 2664 and 2725.
  static constexpr int bufs(int two, int one) { return two <= half ? 2 : one <= half ? 1 : two <= room ? 2 : 1; }
  static constexpr int BF = bufs(fwd(2), fwd(1)), BQ = bufs(dq(2), dq(1)), BK = bufs(dkv(2), dkv(1));
  static_assert(fwd(BF) <= room && dq(BQ) <= room && dkv(BK) <= room, "shared memory of one CTA");
};

// Rows [row0, row0 + M) of a sequence's tensor to shared memory; rows past `rows` and columns past D are zero.  fp32 is copied
// asynchronously: sg_arrived() waits for everything asked for.
template <typename T, int DP>
__device__ __forceinline__ void sg_load(float* to, const T* base, long long stride, int row0, int rows, int D) {
  using S = SgShape<DP>;
  constexpr int N = 16 / sizeof(T);
  for (int x = threadIdx.x; x < S::M * (DP / N); x += SG_THREADS) {
    const int r = x / (DP / N), c = (x - r * (DP / N)) * N;
    const bool there = row0 + r < rows && c < D;
    const T* from = base + (there ? (long long)(row0 + r) * stride + c : 0);
    float* at = to + r * S::LD + c;
    if constexpr (sizeof(T) == 4) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                   ::"r"((uint32_t)__cvta_generic_to_shared(at)), "l"(from), "r"(there ? 16 : 0) : "memory");
    } else {
      const uint4 w = there ? *reinterpret_cast<const uint4*>(from) : make_uint4(0u, 0u, 0u, 0u);
      const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int y = 0; y < N; y += 4)
        *reinterpret_cast<float4*>(at + y) =
            make_float4(ptenc_to_float(e[y]), ptenc_to_float(e[y + 1]), ptenc_to_float(e[y + 2]), ptenc_to_float(e[y + 3]));
    }
  }
}
__device__ __forceinline__ void sg_arrived() {
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
}

// acc[i][j] = row (ty + 16 i) of A . row (tx + 16 j) of B.  Two multiply-adds per instruction, here and below: with one the kernels
// were bound by issuing them.
template <int DP>
__device__ __forceinline__ void sg_dot(float (&acc)[SgShape<DP>::R][SgShape<DP>::R], const float* A, const float* B, int tx, int ty, int D) {
  using S = SgShape<DP>;
  uint64_t two[S::R][S::R];                      // sums over the even and over the odd places
#pragma unroll
  for (int i = 0; i < S::R; ++i)
#pragma unroll
    for (int j = 0; j < S::R; ++j) two[i][j] = 0ull;
#pragma unroll 4
  for (int c = 0; c < D; c += 4) {
    ulonglong2 x[S::R], y[S::R];
#pragma unroll
    for (int i = 0; i < S::R; ++i) {
      x[i] = *reinterpret_cast<const ulonglong2*>(A + (ty + 16 * i) * S::LD + c);
      y[i] = *reinterpret_cast<const ulonglong2*>(B + (tx + 16 * i) * S::LD + c);
    }
#pragma unroll
    for (int i = 0; i < S::R; ++i)
#pragma unroll
      for (int j = 0; j < S::R; ++j) two[i][j] = tt_fma2(x[i].x, y[j].x, tt_fma2(x[i].y, y[j].y, two[i][j]));
  }
#pragma unroll
  for (int i = 0; i < S::R; ++i)
#pragma unroll
    for (int j = 0; j < S::R; ++j) {
      float lo, hi;
      tt_both(two[i][j], lo, hi);
      acc[i][j] = lo + hi;
    }
}

// acc[i][4 c + y] += sum_m P[ty + 16 i][m] * B[m][4 tx + 64 c + y]
template <int DP, bool SOME>
__device__ __forceinline__ void sg_add_t(uint64_t (&acc)[SgShape<DP>::R][DP / 32], const float* P, const float* B, int tx, int ty) {
  using S = SgShape<DP>;
#pragma unroll 2
  for (int m = 0; m < S::M; m += 4) {
    float4 p[S::R];
#pragma unroll
    for (int i = 0; i < S::R; ++i) p[i] = *reinterpret_cast<const float4*>(P + (ty + 16 * i) * S::LP + m);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int c = 0; c < DP / 64; ++c) {
        const ulonglong2 b = *reinterpret_cast<const ulonglong2*>(B + (m + k) * S::LD + 4 * tx + 64 * c);
#pragma unroll
        for (int i = 0; i < S::R; ++i) {
          const float w = k == 0 ? p[i].x : k == 1 ? p[i].y : k == 2 ? p[i].z : p[i].w;
          if (SOME && __float_as_uint(w) == SG_UNSEEN) continue;
          const uint64_t w2 = tt_two(w, w);
          acc[i][2 * c] = tt_fma2(w2, b.x, acc[i][2 * c]);
          acc[i][2 * c + 1] = tt_fma2(w2, b.y, acc[i][2 * c + 1]);
        }
      }
    }
  }
}
// A tile's sum is formed by itself and then added: the error of a sum over n tokens grows with n / M + M instead of n (gradients of
// keys over four heads of 976 tokens: 1.1e-6 of their size in one chain of additions, and less than the scores' own 6e-7 so).
template <int DP>
__device__ __forceinline__ void sg_add(float (&acc)[SgShape<DP>::R][DP / 16], const float* P, const float* B, int tx, int ty, bool all) {
  uint64_t sum[SgShape<DP>::R][DP / 32];
#pragma unroll
  for (int i = 0; i < SgShape<DP>::R; ++i)
#pragma unroll
    for (int c = 0; c < DP / 32; ++c) sum[i][c] = 0ull;
  if (all) sg_add_t<DP, false>(sum, P, B, tx, ty); else sg_add_t<DP, true>(sum, P, B, tx, ty);
#pragma unroll
  for (int i = 0; i < SgShape<DP>::R; ++i)
#pragma unroll
    for (int c = 0; c < DP / 32; ++c) {
      float lo, hi;
      tt_both(sum[i][c], lo, hi);
      acc[i][2 * c] += lo;
      acc[i][2 * c + 1] += hi;
    }
}

template <typename T, int DP>
__device__ __forceinline__ void sg_store(T* base, long long stride, const float (&acc)[SgShape<DP>::R][DP / 16], const float (&f)[SgShape<DP>::R],
                                         int row0, int rows, int D, int tx, int ty) {
  using S = SgShape<DP>;
#pragma unroll
  for (int i = 0; i < S::R; ++i) {
    const int r = row0 + ty + 16 * i;
    if (r >= rows) continue;
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) {
      const int d = 4 * tx + 64 * c;
      if (d >= D) continue;
      T* to = base + (long long)r * stride + d;
#pragma unroll
      for (int y = 0; y < 4; ++y) to[y] = ptenc_from_float<T>(acc[i][4 * c + y] * f[i]);
    }
  }
}

__device__ __forceinline__ float sg_row_sum(float v) {           // over the 16 threads of a row
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A CTA's sums to its shared memory, for the cluster.
template <int DP>
__device__ __forceinline__ void sg_leave(float* to, const float (&acc)[SgShape<DP>::R][DP / 16], int tx, int ty) {
  using S = SgShape<DP>;
#pragma unroll
  for (int i = 0; i < S::R; ++i)
#pragma unroll
    for (int c = 0; c < DP / 64; ++c)
      *reinterpret_cast<float4*>(to + (ty + 16 * i) * S::LD + 4 * tx + 64 * c) =
          make_float4(acc[i][4 * c], acc[i][4 * c + 1], acc[i][4 * c + 2], acc[i][4 * c + 3]);
}
// Four values of a row, summed over the cluster's CTAs in order, each times its factor f[q].
__device__ __forceinline__ float4 sg_joined(cg::cluster_group& cluster, float* mine, int cs, const float* f) {
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int q = 0; q < SG_MAX_CLUSTER; ++q) {
    if (q >= cs) break;
    const float4 v = *reinterpret_cast<const float4*>(cluster.map_shared_rank(mine, q));
    sum.x = fmaf(v.x, f[q], sum.x); sum.y = fmaf(v.y, f[q], sum.y); sum.z = fmaf(v.z, f[q], sum.z); sum.w = fmaf(v.w, f[q], sum.w);
  }
  return sum;
}
template <typename T>
__device__ __forceinline__ void sg_put(T* to, const float4& v, float f) {
  to[0] = ptenc_from_float<T>(v.x * f); to[1] = ptenc_from_float<T>(v.y * f);
  to[2] = ptenc_from_float<T>(v.z * f); to[3] = ptenc_from_float<T>(v.w * f);
}

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// The last launch bound, here and below: how many CTAs of an SM the registers are to allow where the compiler's own choice (0) was the
// slower one.  Five fp32 sequences of 8000 tokens in all, 5839 the longest, 12 + 4 heads of
// 128: forward 3395 us with 1, 3834 with 0.
template <typename T, int DP>
__global__ void __launch_bounds__(SG_THREADS, SgShape<DP>::fwd(SgShape<DP>::BF) <= SgShape<DP>::half ? 0 : 1)
k_seq_fwd(const __grid_constant__ SeqArgs a) {
  using S = SgShape<DP>;
  extern __shared__ __align__(16) float sm[];
  float* sQ = sm;
  float* sKV = sQ + S::TILE;                             // [buffer][K, V]
  float* sP = sKV + 2 * S::BF * S::TILE;
  cg::cluster_group cluster = cg::this_cluster();
  const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int item = (int)(gridDim.x - 1 - blockIdx.x) / cs, h = item % a.Hq, hk = h / a.g, D = a.D;
  tree_after_previous();
  SeqView s;
  int tile;
  if (!seq_find(a, item / a.Hq, S::M, &s, &tile)) return;               // late tiles, which see most, first; a cluster agrees
  const int i0 = tile * S::M, i1 = min(i0 + S::M, s.len) - 1;
  const T* q = static_cast<const T*>(a.q) + s.start * a.qs + (long long)h * D;
  const T* k = static_cast<const T*>(a.k) + s.start * a.ks + (long long)hk * D;
  const T* v = static_cast<const T*>(a.v) + s.start * a.vs + (long long)hk * D;
  sg_load<T, DP>(sQ, q, a.qs, i0, s.len, D);
  const float c2 = a.scale * LOG2E;
  float m[S::R], l[S::R], o[S::R][DP / 16], lowest[S::R];
#pragma unroll
  for (int i = 0; i < S::R; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
    lowest[i] = __int_as_float(s.low(i0 + ty + 16 * i));
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) o[i][c] = 0.f;
  }
  const SeqRange r = seq_keys(s, i0, i1, S::M);
  const int nt = seq_count(r), low1 = s.low(i0 + S::M - 1);
  auto fetch = [&](int t, int buf) {
    const int j0 = seq_at(r, t) * S::M;
    float* to = sKV + (S::BF == 2 ? buf * 2 * S::TILE : 0);
    sg_load<T, DP>(to, k, a.ks, j0, s.len, D);
    sg_load<T, DP>(to + S::TILE, v, a.vs, j0, s.len, D);
  };
  int buf = 0;
  if (rank < nt) fetch(rank, 0);
  for (int t = rank; t < nt; t += cs, buf ^= 1) {
    const int j0 = seq_at(r, t) * S::M;
    if (S::BF == 1 && t > rank) { __syncthreads(); fetch(t, 0); }
    sg_arrived();                                        // also: the other buffer's tile and P are not needed any more
    if (S::BF == 2 && t + cs < nt) fetch(t + cs, buf ^ 1);
    const float* sK = sKV + (S::BF == 2 ? buf * 2 * S::TILE : 0);
    const float* sV = sK + S::TILE;
    const bool all = seq_all(s, i0, low1, j0, j0 + S::M - 1);
    float x[S::R][S::R];
    sg_dot<DP>(x, sQ, sK, tx, ty, D);
#pragma unroll
    for (int i = 0; i < S::R; ++i) {
      const int row = i0 + ty + 16 * i;
      float mx = -INFINITY;
      unsigned unseen = 0;
#pragma unroll
      for (int j = 0; j < S::R; ++j) {
        const int col = j0 + tx + 16 * j;
        if (!all && !(col <= row && (col < s.pin || col >= __float_as_int(lowest[i])))) unseen |= 1u << j;
        else mx = fmaxf(mx, x[i][j]);
      }
#pragma unroll
      for (int y = 8; y > 0; y >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, y));
      // references as they are rounded: with a fused product the factor of an unchanged maximum would not be one
      const float mn = fmaxf(m[i], mx), ref = mn == -INFINITY ? 0.f : __fmul_rn(mn, c2);
      const float corr = m[i] == -INFINITY ? 0.f : exp2f(__fmul_rn(m[i], c2) - ref);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < S::R; ++j) {
        float p = exp2f(fmaf(x[i][j], c2, -ref));
        if ((unseen >> j) & 1u) p = __uint_as_float(SG_UNSEEN); else sum += p;
        sP[(ty + 16 * i) * S::LP + tx + 16 * j] = p;
      }
      l[i] = l[i] * corr + sg_row_sum(sum);
      m[i] = mn;
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) o[i][c] *= corr;
    }
    __syncthreads();
    sg_add<DP>(o, sP, sV, tx, ty, all);
  }
  if (cs > 1) {
    // sums over Q, and their rows' maxima and weights over P
    sg_arrived();
    sg_leave<DP>(sQ, o, tx, ty);
    float2* sRow = reinterpret_cast<float2*>(sP);
#pragma unroll
    for (int i = 0; i < S::R; ++i)
      if (tx == 0) sRow[ty + 16 * i] = make_float2(m[i], l[i]);
    cluster.sync();
    const int quads = D / 4;
    const long long os = (long long)a.Hq * D;
    for (int x = rank * SG_THREADS + threadIdx.x; x < S::M * quads; x += cs * SG_THREADS) {
      const int row = x / quads, c = 4 * (x - row * quads);
      if (i0 + row >= s.len) continue;
      float f[SG_MAX_CLUSTER], w[SG_MAX_CLUSTER], mx = -INFINITY, sum = 0.f;
#pragma unroll
      for (int q = 0; q < SG_MAX_CLUSTER; ++q) {
        if (q >= cs) break;
        const float2 ml = *cluster.map_shared_rank(sRow + row, q);
        f[q] = ml.x;
        w[q] = ml.y;
        mx = fmaxf(mx, ml.x);
      }
      const float ref = mx == -INFINITY ? 0.f : __fmul_rn(mx, c2);
#pragma unroll
      for (int q = 0; q < SG_MAX_CLUSTER; ++q) {
        if (q >= cs) break;
        f[q] = f[q] == -INFINITY ? 0.f : exp2f(__fmul_rn(f[q], c2) - ref);
        sum = fmaf(w[q], f[q], sum);
      }
      const float4 v = sg_joined(cluster, sQ + row * S::LD + c, cs, f);
      sg_put(static_cast<T*>(a.out) + (s.start + i0 + row) * os + (long long)h * D + c, v, 1.f / sum);
      if (c == 0 && a.lse != nullptr) a.lse[(long long)(s.start + i0 + row) * a.Hq + h] = (__fmul_rn(mx, c2) + log2f(sum)) * LN2;
    }
    cluster.sync();                                      // nobody leaves while its sums may be read
    return;
  }
  float f[S::R];
#pragma unroll
  for (int i = 0; i < S::R; ++i) {
    f[i] = 1.f / l[i];
    const int row = i0 + ty + 16 * i;
    if (tx == 0 && row < s.len && a.lse != nullptr)
      a.lse[(long long)(s.start + row) * a.Hq + h] = (__fmul_rn(m[i], c2) + log2f(l[i])) * LN2;
  }
  const long long os = (long long)a.Hq * D;
  sg_store<T, DP>(static_cast<T*>(a.out) + s.start * os + (long long)h * D, os, o, f, i0, s.len, D, tx, ty);
}

// dq of a tile of rows, and delta for the other kernel.
template <typename T, int DP>
__global__ void __launch_bounds__(SG_THREADS, SgShape<DP>::dq(SgShape<DP>::BQ) <= SgShape<DP>::half ? 2 : 1)
k_seq_dq(const __grid_constant__ SeqArgs a) {
  using S = SgShape<DP>;
  extern __shared__ __align__(16) float sm[];
  float* sQ = sm;
  float* sG = sQ + S::TILE;
  float* sKV = sG + S::TILE;                             // [buffer][K, V]; first O
  float* sP = sKV + 2 * S::BQ * S::TILE;
  cg::cluster_group cluster = cg::this_cluster();
  const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int item = (int)(gridDim.x - 1 - blockIdx.x) / cs, h = item % a.Hq, hk = h / a.g, D = a.D;
  tree_after_previous();
  SeqView s;
  int tile;
  if (!seq_find(a, item / a.Hq, S::M, &s, &tile)) return;
  const int i0 = tile * S::M, i1 = min(i0 + S::M, s.len) - 1;
  const long long os = (long long)a.Hq * D, first = s.start * os + (long long)h * D;
  const T* k = static_cast<const T*>(a.k) + s.start * a.ks + (long long)hk * D;
  const T* v = static_cast<const T*>(a.v) + s.start * a.vs + (long long)hk * D;
  sg_load<T, DP>(sQ, static_cast<const T*>(a.q) + s.start * a.qs + (long long)h * D, a.qs, i0, s.len, D);
  sg_load<T, DP>(sG, static_cast<const T*>(a.dout) + first, os, i0, s.len, D);
  sg_load<T, DP>(sKV, static_cast<const T*>(a.out) + first, os, i0, s.len, D);
  sg_arrived();
  const float c2 = a.scale * LOG2E;
  float acc[S::R][DP / 16], lse2[S::R], delta[S::R];
#pragma unroll
  for (int i = 0; i < S::R; ++i) {
    const int row = ty + 16 * i;
    float sum = 0.f;
    for (int c = 4 * tx; c < D; c += 64)
#pragma unroll
      for (int y = 0; y < 4; ++y) sum = fmaf(sG[row * S::LD + c + y], sKV[row * S::LD + c + y], sum);
    delta[i] = sg_row_sum(sum);
    const long long at = (long long)(s.start + i0 + row) * a.Hq + h;
    lse2[i] = 0.f;
    if (i0 + row < s.len) {
      lse2[i] = a.lse[at] * LOG2E;
      if (tx == 0 && rank == 0) a.delta[at] = delta[i];
    }
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) acc[i][c] = 0.f;
  }
  const SeqRange r = seq_keys(s, i0, i1, S::M);
  const int nt = seq_count(r), low1 = s.low(i0 + S::M - 1);
  auto fetch = [&](int t, int buf) {
    const int j0 = seq_at(r, t) * S::M;
    float* to = sKV + (S::BQ == 2 ? buf * 2 * S::TILE : 0);
    sg_load<T, DP>(to, k, a.ks, j0, s.len, D);
    sg_load<T, DP>(to + S::TILE, v, a.vs, j0, s.len, D);
  };
  __syncthreads();                                       // O has been read
  int buf = 0;
  if (rank < nt) fetch(rank, 0);
  for (int t = rank; t < nt; t += cs, buf ^= 1) {
    const int j0 = seq_at(r, t) * S::M;
    if (S::BQ == 1 && t > rank) { __syncthreads(); fetch(t, 0); }
    sg_arrived();
    if (S::BQ == 2 && t + cs < nt) fetch(t + cs, buf ^ 1);
    const float* sK = sKV + (S::BQ == 2 ? buf * 2 * S::TILE : 0);
    const float* sV = sK + S::TILE;
    const bool all = seq_all(s, i0, low1, j0, j0 + S::M - 1);
    float x[S::R][S::R], y[S::R][S::R];
    sg_dot<DP>(x, sQ, sK, tx, ty, D);
    sg_dot<DP>(y, sG, sV, tx, ty, D);
#pragma unroll
    for (int i = 0; i < S::R; ++i) {
      const int row = i0 + ty + 16 * i, lo = all ? 0 : s.low(row);
      const bool alone = !all && s.alone(row);
#pragma unroll
      for (int j = 0; j < S::R; ++j) {
        const int col = j0 + tx + 16 * j;
        float ds = exp2f(fmaf(x[i][j], c2, -lse2[i])) * (y[i][j] - delta[i]);
        if (alone) ds = 0.f;
        if (!all && !(col <= row && (col < s.pin || col >= lo))) ds = __uint_as_float(SG_UNSEEN);
        sP[(ty + 16 * i) * S::LP + tx + 16 * j] = ds;
      }
    }
    __syncthreads();
    sg_add<DP>(acc, sP, sK, tx, ty, all);
  }
  if (cs > 1) {
    sg_arrived();
    sg_leave<DP>(sQ, acc, tx, ty);
    cluster.sync();
    const float one[SG_MAX_CLUSTER] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    const int quads = D / 4;
    for (int x = rank * SG_THREADS + threadIdx.x; x < S::M * quads; x += cs * SG_THREADS) {
      const int row = x / quads, c = 4 * (x - row * quads);
      if (i0 + row >= s.len) continue;
      const float4 sum = sg_joined(cluster, sQ + row * S::LD + c, cs, one);
      sg_put(static_cast<T*>(a.dq) + (s.start + i0 + row) * a.dqs + (long long)h * D + c, sum, a.scale);
    }
    cluster.sync();
    return;
  }
  float f[S::R];
#pragma unroll
  for (int i = 0; i < S::R; ++i) f[i] = a.scale;
  sg_store<T, DP>(static_cast<T*>(a.dq) + s.start * a.dqs + (long long)h * D, a.dqs, acc, f, i0, s.len, D, tx, ty);
}

// dk and dv of a tile of tokens: tiles of queries of the group's heads, one head after another.
template <typename T, int DP>
__global__ void __launch_bounds__(SG_THREADS, SgShape<DP>::dkv(SgShape<DP>::BK) <= SgShape<DP>::half ? 0 : 1)
k_seq_dkv(const __grid_constant__ SeqArgs a) {
  using S = SgShape<DP>;
  extern __shared__ __align__(16) float sm[];
  float* sK = sm;
  float* sV = sK + S::TILE;
  float* sQG = sV + S::TILE;                             // [buffer][Q, dO]
  float* sP = sQG + 2 * S::BK * S::TILE;
  float* sD = sP + S::M * S::LP;
  float* sStat = sD + S::M * S::LP;                      // [buffer][lse (base 2), delta][M]
  cg::cluster_group cluster = cg::this_cluster();
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int item = (int)blockIdx.x / cs, hk = item % a.Hkv, D = a.D;
  tree_after_previous();
  SeqView s;
  int tile;
  if (!seq_find(a, item / a.Hkv, S::M, &s, &tile)) return;      // early tiles are seen by most; a cluster agrees
  const int j0 = tile * S::M, j1 = min(j0 + S::M, s.len) - 1;
  sg_load<T, DP>(sK, static_cast<const T*>(a.k) + s.start * a.ks + (long long)hk * D, a.ks, j0, s.len, D);
  sg_load<T, DP>(sV, static_cast<const T*>(a.v) + s.start * a.vs + (long long)hk * D, a.vs, j0, s.len, D);
  const float c2 = a.scale * LOG2E;
  const long long os = (long long)a.Hq * D;
  float dk[S::R][DP / 16], dv[S::R][DP / 16];
#pragma unroll
  for (int i = 0; i < S::R; ++i)
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) dk[i][c] = dv[i][c] = 0.f;
  const int last = j0 < s.pin ? s.len - 1 : s.last(j1), until = seq_seen_until(s, j0, j0 + S::M - 1);
  const int tiles = last / S::M - tile + 1, nt = tiles * a.g;
  auto fetch = [&](int t, int buf) {
    const int hh = t / tiles, i0 = (tile + t - hh * tiles) * S::M, h = hk * a.g + hh;
    float* to = sQG + (S::BK == 2 ? buf * 2 * S::TILE : 0);
    float* st = sStat + (S::BK == 2 ? buf * 2 * S::M : 0);
    sg_load<T, DP>(to, static_cast<const T*>(a.q) + s.start * a.qs + (long long)h * D, a.qs, i0, s.len, D);
    sg_load<T, DP>(to + S::TILE, static_cast<const T*>(a.dout) + s.start * os + (long long)h * D, os, i0, s.len, D);
    if (threadIdx.x < S::M) {
      const int row = i0 + threadIdx.x;
      const long long at = (long long)(s.start + row) * a.Hq + h;
      st[threadIdx.x] = row < s.len ? a.lse[at] * LOG2E : 0.f;
      st[S::M + threadIdx.x] = row < s.len ? a.delta[at] : 0.f;
    }
  };
  int buf = 0;
  if (rank < nt) fetch(rank, 0);
  for (int t = rank; t < nt; t += cs, buf ^= 1) {
    const int i0 = (tile + t % tiles) * S::M;
    if (S::BK == 1 && t > rank) { __syncthreads(); fetch(t, 0); }
    sg_arrived();
    if (S::BK == 2 && t + cs < nt) fetch(t + cs, buf ^ 1);
    const float* sQ = sQG + (S::BK == 2 ? buf * 2 * S::TILE : 0);
    const float* sG = sQ + S::TILE;
    const float* st = sStat + (S::BK == 2 ? buf * 2 * S::M : 0);
    const bool all = i0 + S::M <= s.len && j0 + S::M - 1 <= i0 && i0 + S::M - 1 <= until;
    float x[S::R][S::R], y[S::R][S::R];
    sg_dot<DP>(x, sK, sQ, tx, ty, D);
    sg_dot<DP>(y, sV, sG, tx, ty, D);
#pragma unroll
    for (int j = 0; j < S::R; ++j) {                     // queries run along the row
      const int c = tx + 16 * j, row = i0 + c;
      const float lse2 = st[c], delta = st[S::M + c];
      const int lo = all ? 0 : s.low(row);
      const bool alone = !all && s.alone(row);
#pragma unroll
      for (int i = 0; i < S::R; ++i) {
        const int col = j0 + ty + 16 * i;
        float p = exp2f(fmaf(x[i][j], c2, -lse2)), ds = alone ? 0.f : p * (y[i][j] - delta);
        if (!all && !(row < s.len && col <= row && (col < s.pin || col >= lo))) p = ds = __uint_as_float(SG_UNSEEN);
        sP[(ty + 16 * i) * S::LP + c] = p;
        sD[(ty + 16 * i) * S::LP + c] = ds;
      }
    }
    __syncthreads();
    sg_add<DP>(dv, sP, sG, tx, ty, all);
    sg_add<DP>(dk, sD, sQ, tx, ty, all);
  }
  if (cs > 1) {
    // over K and V; each then adds a share of the rows of all, in order
    sg_arrived();
    float* mine[2] = {sK, sV};
    sg_leave<DP>(sK, dk, tx, ty);
    sg_leave<DP>(sV, dv, tx, ty);
    cluster.sync();
    const float one[SG_MAX_CLUSTER] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    T* to[2] = {static_cast<T*>(a.dk) + s.start * a.dks + (long long)hk * D, static_cast<T*>(a.dv) + s.start * a.dvs + (long long)hk * D};
    const int quads = D / 4;
    for (int x = rank * SG_THREADS + threadIdx.x; x < 2 * S::M * quads; x += cs * SG_THREADS) {
      const int which = x / (S::M * quads), rem = x - which * S::M * quads, row = rem / quads, c = 4 * (rem - row * quads);
      if (j0 + row >= s.len) continue;
      const float4 sum = sg_joined(cluster, mine[which] + row * S::LD + c, cs, one);
      sg_put(to[which] + (long long)(j0 + row) * (which == 0 ? a.dks : a.dvs) + c, sum, which == 0 ? a.scale : 1.f);
    }
    cluster.sync();                                      // nobody leaves while its sums may be read
    return;
  }
  float one[S::R], f[S::R];
#pragma unroll
  for (int i = 0; i < S::R; ++i) { one[i] = 1.f; f[i] = a.scale; }
  sg_store<T, DP>(static_cast<T*>(a.dv) + s.start * a.dvs + (long long)hk * D, a.dvs, dv, one, j0, s.len, D, tx, ty);
  sg_store<T, DP>(static_cast<T*>(a.dk) + s.start * a.dks + (long long)hk * D, a.dks, dk, f, j0, s.len, D, tx, ty);
}

template <typename T, int DP>
cudaError_t sg_attributes(int dev) {
  static PtencOnce once;
  return ptenc_first_use(once, dev, [] {
    using S = SgShape<DP>;
    cudaError_t e = ptenc_allow_smem(k_seq_fwd<T, DP>, S::fwd(S::BF) * 4);
    if (e == cudaSuccess) e = ptenc_allow_smem(k_seq_dq<T, DP>, S::dq(S::BQ) * 4);
    return e == cudaSuccess ? ptenc_allow_smem(k_seq_dkv<T, DP>, S::dkv(S::BK) * 4) : e;
  });
}

// CTAs of a cluster: doubled until the SMs have two CTAs each for so many items, and never more than the tiles that an item could have
// at most.  Nine fp32 sequences of 3001 tokens, 4 + 1 heads of 64, forward, dq and dkv: 108, 120 and 608 us without clusters, 68, 99 and
// 150 so; until one CTA each 108, 120 and 178, four 73, 133 and 150, eight 107, 234 and 150.
int sg_cluster(long long items, long long most, int sms) {
  int cs = 1;
  while (cs < SG_MAX_CLUSTER && items * cs < 2ll * sms && 2 * cs <= most) cs *= 2;
  return cs;
}

template <typename T, int DP>
cudaError_t sg_fwd(const SeqArgs& a, int dev, int sms, cudaStream_t st) {
  using S = SgShape<DP>;
  const cudaError_t e = sg_attributes<T, DP>(dev);
  if (e != cudaSuccess) return e;
  const unsigned items = (unsigned)seq_numbers(a.n, a.B, S::M) * a.Hq;
  const int cs = sg_cluster(items, (a.n + S::M - 1) / S::M, sms);
  return tree_launch(k_seq_fwd<T, DP>, dim3(items * cs), SG_THREADS, S::fwd(S::BF) * 4, cs, st, a);
}

template <typename T, int DP>
cudaError_t sg_bwd(const SeqArgs& a, int dev, int sms, cudaStream_t st) {
  using S = SgShape<DP>;
  cudaError_t e = sg_attributes<T, DP>(dev);
  if (e != cudaSuccess) return e;
  const unsigned numbers = (unsigned)seq_numbers(a.n, a.B, S::M);
  const long long tiles = (a.n + S::M - 1) / S::M;
  int cs = sg_cluster((long long)numbers * a.Hq, tiles, sms);
  e = tree_launch(k_seq_dq<T, DP>, dim3(numbers * a.Hq * cs), SG_THREADS, S::dq(S::BQ) * 4, cs, st, a);
  if (e != cudaSuccess) return e;
  cs = sg_cluster((long long)numbers * a.Hkv, tiles * a.g, sms);
  return tree_launch(k_seq_dkv<T, DP>, dim3(numbers * a.Hkv * cs), SG_THREADS, S::dkv(S::BK) * 4, cs, st, a);
}

template <typename T>
cudaError_t sg_any(const SeqArgs& a, bool back, int dev, cudaStream_t st) {
  int sms = 0;
  const cudaError_t e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  if (a.D <= 64) return back ? sg_bwd<T, 64>(a, dev, sms, st) : sg_fwd<T, 64>(a, dev, sms, st);
  if (a.D <= 128) return back ? sg_bwd<T, 128>(a, dev, sms, st) : sg_fwd<T, 128>(a, dev, sms, st);
  return back ? sg_bwd<T, 256>(a, dev, sms, st) : sg_fwd<T, 256>(a, dev, sms, st);
}

inline bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
inline bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; }

int check_config(const ptenc_seq_config* c, int32_t batch, int64_t n) {
  if (c == nullptr || batch < 0 || n < 0) return PTENC_EINVAL;
  if (c->dtype != PTENC_DTYPE_FP32 && c->dtype != PTENC_DTYPE_BF16) return PTENC_EINVAL;
  if (c->n_q_heads < 1 || c->n_kv_heads < 1 || c->head_dim < 1 || c->window < 0) return PTENC_EINVAL;
  if (c->window > 0 && (c->evict_chunk < 1 || c->evict_chunk > c->window)) return PTENC_EINVAL;
  if (!(c->scale >= 0.f) || c->scale > 2e38f) return PTENC_EINVAL;
  if (c->head_dim % 8 != 0 || c->head_dim > 256 || c->n_q_heads > 16384 || c->n_q_heads % c->n_kv_heads != 0) return PTENC_ESHAPE;
  if (n >= (1ll << 31) - 512 || batch > (1 << 24)) return PTENC_ESHAPE;
  if ((n / 32 + batch) * c->n_q_heads >= (1ll << 31)) return PTENC_ESHAPE;      // numbers of tiles and heads, of any of the kernels
  return PTENC_OK;
}

int check_stride(long long stride, int heads, const ptenc_seq_config* c) {
  if (stride < (long long)heads * c->head_dim || stride > (1ll << 38)) return PTENC_ESHAPE;
  return stride * (c->dtype == PTENC_DTYPE_FP32 ? 4 : 2) % 16 != 0 ? PTENC_EALIGN : PTENC_OK;
}

void fill(SeqArgs& a, const ptenc_seq_config* c, const void* q, int64_t qs, const void* k, int64_t ks, const void* v, int64_t vs,
          const int32_t* cu, const int32_t* pinned, int32_t batch, int64_t n) {
  memset(&a, 0, sizeof(a));
  a.Hq = c->n_q_heads; a.Hkv = c->n_kv_heads; a.D = c->head_dim; a.g = a.Hq / a.Hkv; a.B = batch;
  a.window = c->window; a.chunk = c->evict_chunk;
  a.scale = c->scale > 0.f ? c->scale : 1.f / sqrtf((float)c->head_dim);
  a.n = n; a.q = q; a.k = k; a.v = v; a.qs = qs; a.ks = ks; a.vs = vs; a.cu = cu; a.pinned = pinned;
}

}  // namespace

cudaError_t seq_forward_any(const SeqArgs& a, int dtype, int dev, cudaStream_t st) {
  return dtype == PTENC_DTYPE_FP32 ? sg_any<float>(a, false, dev, st) : sg_any<__nv_bfloat16>(a, false, dev, st);
}
cudaError_t seq_backward_any(const SeqArgs& a, int dtype, int dev, cudaStream_t st) {
  return dtype == PTENC_DTYPE_FP32 ? sg_any<float>(a, true, dev, st) : sg_any<__nv_bfloat16>(a, true, dev, st);
}

extern "C" int ptenc_seq_attn(const ptenc_seq_config* cfg, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                              const void* v, int64_t v_stride, const int32_t* cu_seqlens, const int32_t* n_pinned, int32_t batch,
                              int64_t n_tokens, void* out, float* lse_out, void* stream) {
  int rc = check_config(cfg, batch, n_tokens);
  if (rc != PTENC_OK || batch == 0 || n_tokens == 0) return rc;
  if (q == nullptr || k == nullptr || v == nullptr || cu_seqlens == nullptr || out == nullptr) return PTENC_EINVAL;
  if ((rc = check_stride(q_stride, cfg->n_q_heads, cfg)) != PTENC_OK || (rc = check_stride(k_stride, cfg->n_kv_heads, cfg)) != PTENC_OK ||
      (rc = check_stride(v_stride, cfg->n_kv_heads, cfg)) != PTENC_OK)
    return rc;
  if (off16(q) || off16(k) || off16(v) || off16(out) || off4(cu_seqlens) || off4(n_pinned) || off4(lse_out)) return PTENC_EALIGN;
  SeqArgs a;
  fill(a, cfg, q, q_stride, k, k_stride, v, v_stride, cu_seqlens, n_pinned, batch, n_tokens);
  a.out = out;
  a.lse = lse_out;
  ptenc_drop_old_error();
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return PTENC_ECUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (!seq_forward_tc(a, cfg->dtype, dev, st, &e)) e = seq_forward_any(a, cfg->dtype, dev, st);
  return e == cudaSuccess ? PTENC_OK : PTENC_ECUDA;
}

extern "C" int ptenc_seq_attn_workspace_bytes(int64_t n_tokens, int32_t n_q_heads, size_t* bytes) {
  if (bytes == nullptr || n_tokens < 0 || n_q_heads < 1) return PTENC_EINVAL;
  if (n_tokens >= (1ll << 31) - 512 || n_q_heads > 16384) return PTENC_ESHAPE;
  *bytes = (size_t)n_tokens * n_q_heads * 2 * sizeof(float);
  return PTENC_OK;
}

extern "C" int ptenc_seq_attn_backward(const ptenc_seq_config* cfg, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                       const void* v, int64_t v_stride, const void* out, const float* lse, const void* dout,
                                       const int32_t* cu_seqlens, const int32_t* n_pinned, int32_t batch, int64_t n_tokens,
                                       void* dq, int64_t dq_stride, void* dk, int64_t dk_stride, void* dv, int64_t dv_stride,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_config(cfg, batch, n_tokens);
  if (rc != PTENC_OK || batch == 0 || n_tokens == 0) return rc;
  if (q == nullptr || k == nullptr || v == nullptr || out == nullptr || lse == nullptr || dout == nullptr || cu_seqlens == nullptr ||
      dq == nullptr || dk == nullptr || dv == nullptr || workspace == nullptr)
    return PTENC_EINVAL;
  if ((rc = check_stride(q_stride, cfg->n_q_heads, cfg)) != PTENC_OK || (rc = check_stride(k_stride, cfg->n_kv_heads, cfg)) != PTENC_OK ||
      (rc = check_stride(v_stride, cfg->n_kv_heads, cfg)) != PTENC_OK || (rc = check_stride(dq_stride, cfg->n_q_heads, cfg)) != PTENC_OK ||
      (rc = check_stride(dk_stride, cfg->n_kv_heads, cfg)) != PTENC_OK || (rc = check_stride(dv_stride, cfg->n_kv_heads, cfg)) != PTENC_OK)
    return rc;
  if (off16(q) || off16(k) || off16(v) || off16(out) || off16(dout) || off16(dq) || off16(dk) || off16(dv) || off16(workspace) ||
      off4(cu_seqlens) || off4(n_pinned) || off4(lse))
    return PTENC_EALIGN;
  size_t need = 0;
  ptenc_seq_attn_workspace_bytes(n_tokens, cfg->n_q_heads, &need);
  if (workspace_bytes < need) return PTENC_EWORKSPACE;
  SeqArgs a;
  fill(a, cfg, q, q_stride, k, k_stride, v, v_stride, cu_seqlens, n_pinned, batch, n_tokens);
  a.out = const_cast<void*>(out);
  a.lse = const_cast<float*>(lse);
  a.dout = dout;
  a.dq = dq; a.dk = dk; a.dv = dv; a.dqs = dq_stride; a.dks = dk_stride; a.dvs = dv_stride;
  a.delta = static_cast<float*>(workspace);
  ptenc_drop_old_error();
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return PTENC_ECUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (!seq_backward_tc(a, cfg->dtype, dev, st, &e)) e = seq_backward_any(a, cfg->dtype, dev, st);
  return e == cudaSuccess ? PTENC_OK : PTENC_ECUDA;
}

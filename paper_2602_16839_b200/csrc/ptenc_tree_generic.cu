// Attention of a draft tree over the cache, shape-generic kernel: fp32 or bf16 storage, any head_dim <= 256 that is a
// multiple of 8, any query group size.
//
// out[i,h] = softmax(q[i,h] . K^T / sqrt(D)) V over the tokens node i sees (ptenc_tree.cuh).  A CTA takes 32 query rows
// (row = node * g + head of the group) of one (layer, sequence, KV head).  Two sets of four warps walk its tokens in turn, 64 at
// a time, each set with a tile buffer of its own, so that one set's copies run under the other's arithmetic (one set where
// two buffers do not fit).  A warp owns eight rows: a thread scores 4 rows x 4 tokens, the running maximum and sum of the
// softmax stay in registers, and the outputs are 4 rows x 4 D / 64 dims per thread, so that every 16-byte read of shared
// memory feeds 8 (scores) to 16 (outputs) multiply-adds.  fp32 FMA throughout (no TF32): the bound is the FMA pipe for many
// rows and latency for few, so when the call has fewer CTAs than the machine has room for, the tokens are split over a cluster
// of CTAs as well; sets and CTAs join their rows through (distributed) shared memory.  Loops stay rolled: a small call runs
// from cold instruction memory.
//
// Measured (fp32, head size 64, 16 sequences of 8 nodes, 4 heads over one ring of 1024 slots): 27 us, of which set-up takes 2, the
// loads' way 4, each pair of a tile's scores and outputs 6, the join 3; 8.7 MB and 0.13 GFLOP would take 2.  With one set per CTA
// 32 us.  Calls that read more are far from the copy bandwidth, because a CTA scores 32 rows however few there are and has one tile
// of a set on its way: fp32, 36 sequences of 2 nodes, 28 heads over 4 rings of 1024 slots of 128 dims (153 MB) 156 us, 1.0 TB/s;
// bf16, 32 sequences of 8 nodes, 16 heads over 4 rings of 2048 slots, 198 us at D = 96 (103 MB) and 515 us at D = 256 (274 MB).
#include <cooperative_groups.h>
#include <string.h>

#include "ptenc_tree.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int TG_SET = 128;          // threads of a set
constexpr int TG_SETS = 2;
constexpr int TG_ROWS = 32;
constexpr int TG_TOK = 64;
constexpr int TG_PP = TG_TOK + 4;    // pitch of the probabilities
constexpr int TG_CLUSTER = 8;

__device__ __forceinline__ float4 tg_ld4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 tg_ld4(const __nv_bfloat16* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                     __uint_as_float(u.y & 0xffff0000u));
}
__device__ __forceinline__ void tg_async16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
               ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(dst))), "l"(src) : "memory");
}
__device__ __forceinline__ void tg_fma4(float4& a, float s, const float4& v) {
  a.x = fmaf(s, v.x, a.x); a.y = fmaf(s, v.y, a.y); a.z = fmaf(s, v.z, a.z); a.w = fmaf(s, v.w, a.w);
}

__device__ __forceinline__ void tg_set_sync(int set) { asm volatile("bar.sync %0, %1;" ::"r"(1 + set), "n"(TG_SET) : "memory"); }

// Shared memory in bytes: a K and a V tile and probabilities per set, Q rows.
template <typename T>
__host__ __device__ inline int tg_pitch(int D) { return D + 16 / (int)sizeof(T); }
template <typename T>
inline size_t tg_smem(int D, int sets) {
  return (size_t)sets * (2 * TG_TOK * tg_pitch<T>(D) * sizeof(T) + sizeof(float) * TG_ROWS * TG_PP) +
         sizeof(float) * TG_ROWS * (D + 4);
}

// J = 64-dim blocks of a row (D <= 64 J).
template <typename T, int J>
__global__ void __launch_bounds__(TG_SET * TG_SETS)
k_tree_generic(PtencDev p, int l0, const T* __restrict__ q, const T* __restrict__ k_tree, const T* __restrict__ v_tree,
               const int32_t* __restrict__ parent, const int32_t* __restrict__ n_nodes, int NT,
               const uint8_t* __restrict__ active, T* __restrict__ out, float* __restrict__ lse, int n_groups) {
  extern __shared__ __align__(16) uint8_t tg_sm[];
  const int D = p.D, g = p.g, W = p.W, Hkv = p.Hkv;
  const int KP = tg_pitch<T>(D), QP = D + 4;
  const int sets = (int)blockDim.x / TG_SET, threads = (int)blockDim.x;
  const int tid = threadIdx.x, lane = tid & 31, set = tid / TG_SET, st = tid - set * TG_SET, warp = st >> 5;
  const size_t kv_bytes = (size_t)2 * TG_TOK * KP * sizeof(T);
  float* s_q = reinterpret_cast<float*>(tg_sm + sets * kv_bytes);                                // [TG_ROWS][QP]
  float* s_p = s_q + TG_ROWS * QP + set * TG_ROWS * TG_PP;                                       // [sets][TG_ROWS][TG_PP]
  T* s_k = reinterpret_cast<T*>(tg_sm + set * kv_bytes);                                         // [sets][K, V][TG_TOK][KP]
  T* s_v = s_k + TG_TOK * KP;
  __shared__ float2 s_ml[TG_SETS][TG_ROWS];
  __shared__ unsigned long long s_anc[TREE_MAX], s_vis[TREE_MAX];
  __shared__ int s_ev[TREE_MAX], s_jump[TREE_MAX];

  cg::cluster_group cluster = cg::this_cluster();
  const int CS = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  int idx = blockIdx.x / CS;
  const int grp = idx % n_groups; idx /= n_groups;
  const int hkv = idx % Hkv; idx /= Hkv;
  const int b = idx % p.B;
  const int li = idx / p.B;
  tree_after_previous();
  if (active != nullptr && active[b] == 0) return;        // these verdicts are alike for the CTAs of a cluster
  const int n = n_nodes != nullptr ? n_nodes[b] : NT;
  const size_t lb = (size_t)(l0 + li) * p.B + b;
  const size_t ob = (size_t)li * p.B + b;
  TreeRing r;
  const bool fine = tree_ring(p, lb, &r) && n >= 0 && n <= NT;
  if (!fine) {
    if (threadIdx.x == 0) atomicOr(p.status, PTENC_ST_BAD_INDEX);
    return;
  }
  const int row0 = grp * TG_ROWS;
  if (row0 >= n * g) return;                              // rows of nodes that do not exist stay as they are
  if (!tree_setup(parent + (size_t)b * NT, n, r, s_anc, s_vis, s_ev, s_jump)) {
    if (threadIdx.x == 0) atomicOr(p.status, PTENC_ST_BAD_INDEX);
    return;
  }

  // tokens of the unit: pinned entries, then the ring from the oldest token that any node sees, then the nodes
  const int ev0 = min(tree_evicted(r.count, r.cap, r.e, 1), r.count);
  const int n_cache = r.sink + r.count - ev0;
  const int n_tok = n_cache + n;
  const int tiles = (n_tok + TG_TOK - 1) / TG_TOK;
  // this set's tiles: rank * sets + set of CS * sets shares
  const int share = rank * sets + set, shares = CS * sets;
  const int t_lo = share * tiles / shares, t_hi = (share + 1) * tiles / shares;      // tiles < 2^19, shares <= 16
  const T* Kb = reinterpret_cast<const T*>(p.K) + (lb * Hkv + hkv) * (size_t)W * D;
  const T* Vb = reinterpret_cast<const T*>(p.V) + (lb * Hkv + hkv) * (size_t)W * D;
  const int vpr = D * (int)sizeof(T) / 16;                // 16-byte vectors of a row
  // Where the tile's tokens lie is worked out a token per lane (slot, or -1 - node, or nothing); then a token per warp and
  // turn, the lanes taking the vectors of its K row and of its V row.
  auto place = [&](int i) -> int {
    if (i < r.sink) return i;
    if (i < n_cache) return tree_slot(r, ev0 + (i - r.sink));
    return i < n_tok ? -1 - (i - n_cache) : -1000;
  };
  const T* Kt = k_tree + (ob * NT * Hkv + hkv) * (size_t)D;
  const T* Vt = v_tree + (ob * NT * Hkv + hkv) * (size_t)D;
  auto fetch = [&](int tile) {
    const int pl0 = place(tile * TG_TOK + lane), pl1 = place(tile * TG_TOK + 32 + lane);
#pragma unroll 4
    for (int t = warp; t < TG_TOK; t += TG_SET / 32) {
      const int at = __shfl_sync(0xffffffffu, t < 32 ? pl0 : pl1, t & 31);
      const size_t off = at >= 0 ? (size_t)at * D : (size_t)(-1 - at) * Hkv * D;
      for (int x = lane; x < 2 * vpr; x += 32) {
        const bool is_v = x >= vpr;
        const int v = 16 * (is_v ? x - vpr : x);
        uint8_t* dst = reinterpret_cast<uint8_t*>((is_v ? s_v : s_k) + t * KP) + v;
        const T* src = (at >= 0 ? (is_v ? Vb : Kb) : (is_v ? Vt : Kt)) + off;
        if (at != -1000) tg_async16(dst, reinterpret_cast<const uint8_t*>(src) + v);
        else *reinterpret_cast<uint4*>(dst) = make_uint4(0u, 0u, 0u, 0u);      // past the end: the products stay finite
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (t_lo < t_hi) fetch(t_lo);
#pragma unroll 4
  for (int rr = tid >> 5; rr < TG_ROWS; rr += threads >> 5) {
    const int row = row0 + rr, node = row / g, h = row - node * g;
    const T* src = q + ((ob * NT + node) * p.Hq + (size_t)hkv * g + h) * D;
#pragma unroll
    for (int j = 0; j < (64 * J + 127) / 128; ++j) {
      const int d = 4 * lane + 128 * j;
      if (d < D) *reinterpret_cast<float4*>(s_q + rr * QP + d) = node < n ? tg_ld4(src + d) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  __syncthreads();

  const float scale = 1.0f / sqrtf((float)D);
  const int rb = 8 * warp + 4 * (lane >> 4);              // this thread's four rows
  const int tk = lane & 15;
  float m[4], l[4];
  float4 acc[4][J];
  int ev[4], node_of[4];
  int ev_max = ev0;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    m[x] = -INFINITY;
    l[x] = 0.f;
    const int node = (row0 + rb + x) / g;
    node_of[x] = node < n ? node : -1;
    ev[x] = node < n ? s_ev[node] : ev0;
#pragma unroll
    for (int j = 0; j < J; ++j) acc[x][j] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
#pragma unroll 1
  for (int i = 0; i < n; ++i) ev_max = max(ev_max, s_ev[i]);

#pragma unroll 1
  for (int tile = t_lo; tile < t_hi; ++tile) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    tg_set_sync(set);
    const T *sk = s_k, *sv = s_v;
    const int t0 = tile * TG_TOK;
    // every row sees every token of the tile
    const bool clean = t0 + TG_TOK <= n_cache && (ev_max == ev0 || t0 >= r.sink + ev_max - ev0 || t0 + TG_TOK <= r.sink);
    // ---- scores: 4 rows x tokens tk, tk + 16, .. -----------------------------------------------------------------------
    float s[4][4];
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int y = 0; y < 4; ++y) s[x][y] = 0.f;
#pragma unroll 2
    for (int d = 0; d < D; d += 4) {
      float4 qq[4], kk[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) qq[x] = tg_ld4(s_q + (rb + x) * QP + d);
#pragma unroll
      for (int y = 0; y < 4; ++y) kk[y] = tg_ld4(sk + (tk + 16 * y) * KP + d);
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y)
          s[x][y] = fmaf(qq[x].x, kk[y].x, fmaf(qq[x].y, kk[y].y, fmaf(qq[x].z, kk[y].z, fmaf(qq[x].w, kk[y].w, s[x][y]))));
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      unsigned seen = 0xfu;
      if (!clean) {
        const unsigned long long vis = node_of[x] >= 0 ? s_vis[node_of[x]] : ~0ull;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int i = t0 + tk + 16 * y;
          const bool is = i < r.sink || (i < n_cache ? ev0 + (i - r.sink) >= ev[x] : (i < n_tok && ((vis >> ((i - n_cache) & 63)) & 1ull)));
          if (!is) seen &= ~(1u << y);
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        s[x][y] = ((seen >> y) & 1u) ? s[x][y] * scale : -INFINITY;
        mx = fmaxf(mx, s[x][y]);
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float m_new = fmaxf(m[x], mx);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      const float corr = m[x] == -INFINITY ? 0.f : expf(m[x] - m_use);
      float sum = 0.f;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const float e = ((seen >> y) & 1u) ? expf(s[x][y] - m_use) : 0.f;
        sum += e;
        s_p[(rb + x) * TG_PP + tk + 16 * y] = e;
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      l[x] = l[x] * corr + sum;
      m[x] = m_new;
#pragma unroll
      for (int j = 0; j < J; ++j) { acc[x][j].x *= corr; acc[x][j].y *= corr; acc[x][j].z *= corr; acc[x][j].w *= corr; }
    }
    __syncwarp();                                         // a warp reads the probabilities it wrote
    // ---- outputs: 4 rows x dims 4 tk + 64 j -----------------------------------------------------------------------------
#pragma unroll 1
    for (int t = 0; t < TG_TOK; t += 4) {
      float4 pp[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) pp[x] = tg_ld4(s_p + (rb + x) * TG_PP + t);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int d = 4 * tk + 64 * j;
        if (d < D) {
          float4 vv[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) vv[y] = tg_ld4(sv + (t + y) * KP + d);
          if (clean) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              tg_fma4(acc[x][j], pp[x].x, vv[0]); tg_fma4(acc[x][j], pp[x].y, vv[1]);
              tg_fma4(acc[x][j], pp[x].z, vv[2]); tg_fma4(acc[x][j], pp[x].w, vv[3]);
            }
          } else {                                        // a token the row does not see may hold anything, NaN included
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              if (pp[x].x != 0.f) tg_fma4(acc[x][j], pp[x].x, vv[0]);
              if (pp[x].y != 0.f) tg_fma4(acc[x][j], pp[x].y, vv[1]);
              if (pp[x].z != 0.f) tg_fma4(acc[x][j], pp[x].z, vv[2]);
              if (pp[x].w != 0.f) tg_fma4(acc[x][j], pp[x].w, vv[3]);
            }
          }
        }
      }
    }
    tg_set_sync(set);                                     // the tile's buffer is free
    if (tile + 1 < t_hi) fetch(tile + 1);
  }

  if (shares == 1) {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (node_of[x] < 0) continue;
      const size_t at = (ob * NT + node_of[x]) * p.Hq + (size_t)hkv * g + (row0 + rb + x) % g;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int d = 4 * tk + 64 * j;
        if (d < D) {
          T* o = out + at * D + d;
          o[0] = ptenc_from_float<T>(acc[x][j].x / l[x]); o[1] = ptenc_from_float<T>(acc[x][j].y / l[x]);
          o[2] = ptenc_from_float<T>(acc[x][j].z / l[x]); o[3] = ptenc_from_float<T>(acc[x][j].w / l[x]);
        }
      }
      if (lse != nullptr && tk == 0) lse[at] = m[x] + logf(l[x]);
    }
    return;
  }
  // ---- the sets and CTAs join their rows: sums in the place of the set's tile, (m, l) beside them -----------------------------
  float* s_o = reinterpret_cast<float*>(s_k);             // [TG_ROWS][QP], no larger than the tiles
#pragma unroll
  for (int x = 0; x < 4; ++x) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int d = 4 * tk + 64 * j;
      if (d < D) *reinterpret_cast<float4*>(s_o + (rb + x) * QP + d) = acc[x][j];
    }
    if (tk == 0) s_ml[set][rb + x] = make_float2(m[x], l[x]);
  }
  if (CS > 1) cluster.sync(); else __syncthreads();
  // a row per warp: a lane per share looks at its (m, l), then a lane per four dims adds the shares' sums
  for (int rr = rank * (threads >> 5) + (tid >> 5); rr < TG_ROWS; rr += CS * (threads >> 5)) {
    const int row = row0 + rr, node = row / g;
    if (node >= n) continue;                              // uniform over the warp
    const int from = lane / sets, ss = lane - from * sets;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < shares) ml = cluster.map_shared_rank(&s_ml[ss][0], from)[rr];
    float mt = ml.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, o));
    const float w = ml.x == -INFINITY ? 0.f : expf(ml.x - mt);
    float lt = w * ml.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) lt += __shfl_xor_sync(0xffffffffu, lt, o);
    const size_t at = (ob * NT + node) * p.Hq + (size_t)hkv * g + row % g;
    for (int d0 = 0; d0 < D; d0 += 128) {
      const int d = min(d0 + 4 * lane, D - 4);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int c = 0; c < shares; ++c) {
        const int cf = c / sets, cs = c - cf * sets;
        const float4 v = *reinterpret_cast<const float4*>(
            cluster.map_shared_rank(reinterpret_cast<float*>(tg_sm + cs * kv_bytes), cf) + rr * QP + d);
        const float wc = __shfl_sync(0xffffffffu, w, c);
        if (wc != 0.f) tg_fma4(o, wc, v);                 // a share in which the row sees nothing does not count
      }
      if (d0 + 4 * lane < D) {
        T* dst = out + at * D + d;
        dst[0] = ptenc_from_float<T>(o.x / lt); dst[1] = ptenc_from_float<T>(o.y / lt);
        dst[2] = ptenc_from_float<T>(o.z / lt); dst[3] = ptenc_from_float<T>(o.w / lt);
      }
    }
    if (lse != nullptr && lane == 0) lse[at] = mt + logf(lt);
  }
  if (CS > 1) cluster.sync();                             // nobody leaves while its rows may still be read
}

template <typename T, int J>
cudaError_t launch_tree_j(ptenc_cache* c, int l0, int nl, const void* q, const void* kt, const void* vt,
                          const int32_t* parent, const int32_t* n_nodes, int NT, const uint8_t* active, void* out,
                          float* lse, cudaStream_t st) {
  const PtencDev& p = c->dev;
  const int n_groups = (NT * p.g + TG_ROWS - 1) / TG_ROWS;
  const long long blocks = (long long)nl * p.B * p.Hkv * n_groups;
  // Tokens over up to eight CTAs while that does not exceed two CTAs per SM and each still has a tile of 64.  Two CTAs fit an SM
  // where they take up to 113 KB and 128 registers each (fp32 at D <= 64, bf16 at D <= 128); of the larger ones one fits, and
  // such a call may be split into two rounds.
  int cs = 1;
  while (cs < TG_CLUSTER && blocks * cs * 2 <= 2 * c->sm_count && cs * 2 * TG_TOK <= p.W) cs *= 2;
  if (blocks * cs > 0x7fffffffll) return cudaErrorInvalidValue;
  const int sets = tg_smem<T>(p.D, 2) > 200 * 1024 ? 1 : 2;
  const size_t smem = tg_smem<T>(p.D, sets);
  static PtencOnce once;
  const cudaError_t e = ptenc_first_use(once, c->cfg.device, [] { return ptenc_allow_smem(k_tree_generic<T, J>, 216 * 1024); });
  if (e != cudaSuccess) return e;
  c->launches++;
  return tree_launch(k_tree_generic<T, J>, dim3((unsigned)(blocks * cs)), TG_SET * sets, smem, cs, st, p, l0, (const T*)q,
                     (const T*)kt, (const T*)vt, parent, n_nodes, NT, active, (T*)out, lse, n_groups);
}
template <typename T>
cudaError_t launch_tree_t(ptenc_cache* c, int l0, int nl, const void* q, const void* kt, const void* vt,
                          const int32_t* parent, const int32_t* n_nodes, int NT, const uint8_t* active, void* out,
                          float* lse, cudaStream_t st) {
  if (c->dev.D <= 64) return launch_tree_j<T, 1>(c, l0, nl, q, kt, vt, parent, n_nodes, NT, active, out, lse, st);
  if (c->dev.D <= 128) return launch_tree_j<T, 2>(c, l0, nl, q, kt, vt, parent, n_nodes, NT, active, out, lse, st);
  return launch_tree_j<T, 4>(c, l0, nl, q, kt, vt, parent, n_nodes, NT, active, out, lse, st);
}

}  // namespace

cudaError_t ptenc_launch_tree_generic(ptenc_cache* c, int l0, int nl, const void* q, const void* k_tree,
                                      const void* v_tree, const int32_t* parent, const int32_t* n_nodes, int max_nodes,
                                      const uint8_t* active, void* out, float* lse, cudaStream_t st) {
  if (c->cfg.dtype == PTENC_DTYPE_FP32)
    return launch_tree_t<float>(c, l0, nl, q, k_tree, v_tree, parent, n_nodes, max_nodes, active, out, lse, st);
  return launch_tree_t<__nv_bfloat16>(c, l0, nl, q, k_tree, v_tree, parent, n_nodes, max_nodes, active, out, lse, st);
}

// The accepted path of a draft enters the cache: as many appends, evictions and folds as the path has tokens, in one call.
//
// The same result as ptenc_append_evict and ptenc_encode once per token of the path.  The ring words follow from counts
// alone (ptenc_tree.cuh): after m arrivals ev(m) tokens have left, in events of e; event k takes the arrival numbers
// [k e, (k + 1) e), which are cache tokens or, when the ring is shorter than the path, the path's own first tokens.  The
// state is normalised after every event, so events are folded in order; the rows of an event are summed,
//   S <- Normalize(S + sum_i (Q_a k_a,i) v_a,i^T)   (Sec. 3.3, Eq. (3) and the sentence after it).
#include <type_traits>

#include "ptenc_tree.cuh"

namespace {

constexpr int CM_THREADS = 256;

template <typename T> struct CmVec;
template <> struct CmVec<float> { static constexpr int N = 4; };
template <> struct CmVec<__nv_bfloat16> { static constexpr int N = 8; };

template <typename T>
__device__ __forceinline__ float cm_dot16(const T* __restrict__ w, const float* x) {
  constexpr int N = CmVec<T>::N;
  const uint4 raw = *reinterpret_cast<const uint4*>(w);
  const T* e = reinterpret_cast<const T*>(&raw);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) s = fmaf(ptenc_to_float(e[i]), x[i], s);
  return s;
}

// The end of a commit, alike for every kernel: the last event's rows to the staging area, the tokens that stay into the
// slots the evicted ones left, the ring words.  All threads of the CTA; every row has been folded before.
template <typename T>
__device__ __forceinline__ void cm_store(const PtencDev& p, size_t lb, size_t ob, const TreeRing& rg, int m, int gone,
                                         int events, long long n0, const T* __restrict__ k_tree,
                                         const T* __restrict__ v_tree, int NT, const int* s_path, int32_t* n_evicted_out) {
  const int D = p.D, Hkv = p.Hkv, W = p.W, tid = threadIdx.x;
  const T* ringK = reinterpret_cast<const T*>(p.K);
  const T* ringV = reinterpret_cast<const T*>(p.V);
  auto row = [&](int o, const T* ring, const T* fresh, size_t* stride) -> const T* {
    if (o < rg.count) { *stride = (size_t)W * D; return ring + (lb * Hkv * (size_t)W + tree_slot(rg, o)) * D; }
    *stride = D;
    return fresh + (ob * NT + s_path[o - rg.count]) * (size_t)Hkv * D;
  };
  // ---- what the last arrival evicted stays staged, as after ptenc_append_evict ---------------------------------------
  const int vph = D * (int)sizeof(T) / 16, vpr = Hkv * vph;
  const bool last_evicts = events > 0 && rg.cap - rg.count + (events - 1) * rg.e == m - 1;
  if (last_evicts) {
    for (int i = tid; i < rg.e * vpr; i += CM_THREADS) {
      const int rr = i / vpr, v = i - rr * vpr, h = v / vph, vv = v - h * vph;
      size_t ks, vs;
      const int o = (events - 1) * rg.e + rr;
      const T* kr = row(o, ringK, k_tree, &ks);
      const T* vr = row(o, ringV, v_tree, &vs);
      kr += h * ks;
      vr += h * vs;
      const size_t dst = ((lb * p.E + rr) * Hkv + h) * (size_t)D * sizeof(T) + (size_t)vv * 16;
      *reinterpret_cast<uint4*>(p.stageK + dst) = reinterpret_cast<const uint4*>(kr)[vv];
      *reinterpret_cast<uint4*>(p.stageV + dst) = reinterpret_cast<const uint4*>(vr)[vv];
    }
  }
  // ---- the tokens that stay, into the slots the evicted ones left (all of those have been read above) ------------------
  __syncthreads();
  const int first = gone > rg.count ? gone - rg.count : 0;         // a path longer than the ring keeps its newest tokens
  for (int i = first * vpr + tid; i < m * vpr; i += CM_THREADS) {
    const int j = i / vpr, v = i - j * vpr, h = v / vph, vv = v - h * vph;
    const size_t src = ((ob * NT + s_path[j]) * Hkv + h) * (size_t)D * sizeof(T) + (size_t)vv * 16;
    const size_t dst = ((lb * Hkv + h) * (size_t)W + tree_slot(rg, rg.count + j)) * D * sizeof(T) + (size_t)vv * 16;
    *reinterpret_cast<uint4*>(p.K + dst) = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(k_tree) + src);
    *reinterpret_cast<uint4*>(p.V + dst) = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(v_tree) + src);
  }
  if (tid == 0) {
    p.head[lb] = (int)(((long long)rg.head + gone) % rg.cap);
    p.count[lb] = rg.count + m - gone;
    p.n_app[lb] = n0 + m;
    p.n_staged[lb] = last_evicts ? rg.e : 0;
    p.evict_first[lb] = last_evicts ? n0 - rg.count + (long long)(events - 1) * rg.e : -1;
    if (n_evicted_out) n_evicted_out[ob] = gone;
  }
}

// Shape-generic kernel: a CTA per (layer, sequence), rows one after another.
template <typename T>
__global__ void __launch_bounds__(CM_THREADS)
k_commit(PtencDev p, int l0, const T* __restrict__ k_tree, const T* __restrict__ v_tree, int NT,
         const int32_t* __restrict__ path, const int32_t* __restrict__ n_path, const uint8_t* __restrict__ active,
         int32_t* n_evicted_out) {
  extern __shared__ float cm_sm[];
  __shared__ int s_path[TREE_MAX];
  const int G = p.G, r = p.r, d_kv = p.d_kv, D = p.D, Hkv = p.Hkv, W = p.W;
  const int li = blockIdx.x / p.B;
  const int b = blockIdx.x - li * p.B;
  const int l = l0 + li;
  const size_t lb = (size_t)l * p.B + b;
  const size_t ob = (size_t)li * p.B + b;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nwarps = CM_THREADS / 32;
  const int m = (active != nullptr && active[b] == 0) ? 0 : n_path[b];
  TreeRing rg;
  int bad = !tree_ring(p, lb, &rg) || m < 0 || m > NT;
  if (!bad && tid < m) {
    const int at = path[(size_t)b * NT + tid];
    s_path[tid] = at;
    bad = at < 0 || at >= NT;
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) {
      atomicOr(p.status, PTENC_ST_BAD_INDEX);
      if (n_evicted_out) n_evicted_out[ob] = 0;
    }
    return;
  }
  if (m == 0) {
    if (tid == 0) {
      p.n_staged[lb] = 0;
      p.evict_first[lb] = -1;
      if (n_evicted_out) n_evicted_out[ob] = 0;
    }
    return;
  }
  const int gone = tree_evicted(rg.count, rg.cap, rg.e, m);
  const int events = gone / rg.e;
  const long long n0 = p.n_app[lb];
  // rows of the token with arrival number o: head h at + h * stride
  auto row = [&](int o, const T* ring, const T* fresh, size_t* stride) -> const T* {
    if (o < rg.count) { *stride = (size_t)W * D; return ring + (lb * Hkv * (size_t)W + tree_slot(rg, o)) * D; }
    *stride = D;
    return fresh + (ob * NT + s_path[o - rg.count]) * (size_t)Hkv * D;
  };
  const T* ringK = reinterpret_cast<const T*>(p.K);
  const T* ringV = reinterpret_cast<const T*>(p.V);

  // ---- fold the events ---------------------------------------------------------------------------------------------
  if (events > 0 && p.encode_enabled && p.enc_set[l]) {
    float* xk = cm_sm;
    float* xv = xk + d_kv;
    float* ka = xv + d_kv;           // k_a [r], v_a [r]
    float* pg = ka + 2 * r;
    float* qa = pg + G;
    float* acc = qa + G * r;
    float* red = acc + G * r;        // G + 1
    const T* Wk = reinterpret_cast<const T*>(p.Wk) + (size_t)l * r * d_kv;
    const T* Wv = reinterpret_cast<const T*>(p.Wv) + (size_t)l * r * d_kv;
    const int gr = G * r;
    float* S = p.S + lb * gr;
    for (int i = tid; i < gr; i += CM_THREADS) { qa[i] = p.Qa[(size_t)l * gr + i]; acc[i] = S[i]; }
    constexpr int N = CmVec<T>::N;
    for (int ev = 0; ev < events; ++ev) {
      for (int i = 0; i < rg.e; ++i) {
        size_t ks, vs;
        const T* kr = row(ev * rg.e + i, ringK, k_tree, &ks);
        const T* vr = row(ev * rg.e + i, ringV, v_tree, &vs);
        __syncthreads();
        for (int d = tid; d < d_kv; d += CM_THREADS) {
          const int h = d / D, dd = d - h * D;
          xk[d] = ptenc_to_float(kr[h * ks + dd]);
          xv[d] = ptenc_to_float(vr[h * vs + dd]);
        }
        __syncthreads();
        for (int j = warp; j < 2 * r; j += nwarps) {
          const T* wrow = (j < r) ? (Wk + (size_t)j * d_kv) : (Wv + (size_t)(j - r) * d_kv);
          const float* x = (j < r) ? xk : xv;
          float s = 0.f;
          for (int d = lane * N; d < d_kv; d += 32 * N) s += cm_dot16<T>(wrow + d, x + d);
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
          if (lane == 0) ka[j] = s;
        }
        __syncthreads();
        for (int gi = tid; gi < G; gi += CM_THREADS) {
          float s = 0.f;
          for (int j = 0; j < r; ++j) s = fmaf(qa[gi * r + j], ka[j], s);
          pg[gi] = s;
        }
        __syncthreads();
        for (int x = tid; x < gr; x += CM_THREADS) acc[x] = fmaf(pg[x / r], ka[r + x % r], acc[x]);
      }
      __syncthreads();
      if (p.norm_mode != PTENC_NORM_NONE) {
        for (int gi = warp; gi < G; gi += nwarps) {
          float s = 0.f;
          for (int j = lane; j < r; j += 32) s = fmaf(acc[gi * r + j], acc[gi * r + j], s);
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
          if (lane == 0) red[gi] = s;
        }
        __syncthreads();
        if (tid == 0 && p.norm_mode == PTENC_NORM_FROBENIUS) {
          float s = 0.f;
          for (int gi = 0; gi < G; ++gi) s += red[gi];
          red[G] = s;
        }
        __syncthreads();
        for (int x = tid; x < gr; x += CM_THREADS)
          acc[x] *= 1.f / fmaxf(sqrtf(red[p.norm_mode == PTENC_NORM_ROW_L2 ? x / r : G]), 1e-12f);
      }
    }
    __syncthreads();
    for (int i = tid; i < gr; i += CM_THREADS) S[i] = acc[i];
  }
  cm_store(p, lb, ob, rg, m, gone, events, n0, k_tree, v_tree, NT, s_path, n_evicted_out);
}

// ------------------------------------------------------------------------------------------------ bf16, tensor cores
__device__ __forceinline__ void cm_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                       uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cm_async16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
               ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(dst))), "l"(src) : "memory");
}

// The same for bf16 storage, row-normalised or unnormalised states, r a multiple of 8, H_kv D a multiple of 32: a CTA per
// (layer, sequence), the evicted rows 16 MT at a time in order of arrival.
//  * k_a and v_a of a tile come from mma.m16n8k16, a warp per eight outputs.  A lane reads its pieces of rows and weights as
//    16-byte vectors straight from memory: eight consecutive values serve two mma steps, the contraction index permuted
//    alike on both operands, so nothing is staged.
//  * p = Q_a k_a for all rows of the tile, then S += p v_a^T row by row, a warp per four state rows and a lane per
//    column, with the state rows in registers; behind the last row of an event the rows are normalised.
//  RJ = columns per lane (r <= 32 RJ), MT = 16-row blocks per tile.
template <int RJ, int MT>
__global__ void __launch_bounds__(CM_THREADS, MT == 1 ? 3 : 2)
k_commit_bf16(PtencDev p, int l0, const __nv_bfloat16* __restrict__ k_tree, const __nv_bfloat16* __restrict__ v_tree, int NT,
              const int32_t* __restrict__ path, const int32_t* __restrict__ n_path, const uint8_t* __restrict__ active,
              int32_t* n_evicted_out) {
  extern __shared__ __align__(16) float cm_sm[];
  __shared__ int s_path[TREE_MAX];
  constexpr int RT = 16 * MT;
  const int G = p.G, r = p.r, d_kv = p.d_kv, D = p.D, Hkv = p.Hkv, W = p.W;
  const int li = blockIdx.x / p.B;
  const int b = blockIdx.x - li * p.B;
  const int l = l0 + li;
  const size_t lb = (size_t)l * p.B + b;
  const size_t ob = (size_t)li * p.B + b;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int KP = 2 * r + 4, QP = r + 4, GP = (G + 31) / 32 * 32 + 4;  // row pitches
  float* s_kv = cm_sm;                                     // [RT][KP] k_a, v_a
  float* s_p = s_kv + RT * KP;                             // [RT][GP] Q_a k_a
  float* s_q = s_p + RT * GP;                              // [G][QP] Q_a
  float* s_s = s_q + G * QP;                               // [G][r] state
  const bool enc = p.encode_enabled != 0;
  float* S = p.S + lb * G * r;
  if (enc) {                                               // Q_a and the state travel while the ring words are looked at
    for (int i = tid; i < G * r / 4; i += CM_THREADS) {
      cm_async16(s_q + (4 * i / r) * QP + 4 * i % r, p.Qa + (size_t)l * G * r + 4 * i);
      cm_async16(s_s + 4 * i, S + 4 * i);
    }
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
  const int m = (active != nullptr && active[b] == 0) ? 0 : n_path[b];
  const bool folds = enc && p.enc_set[l] != 0;
  TreeRing rg;
  int bad = !tree_ring(p, lb, &rg) || m < 0 || m > NT;
  const long long n0 = p.n_app[lb];
  if (tid < NT) {
    const int at = path[(size_t)b * NT + tid];
    s_path[tid] = at;
    bad |= tid < m && (at < 0 || at >= NT);
  }
  if (__syncthreads_or(bad)) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (tid == 0) {
      atomicOr(p.status, PTENC_ST_BAD_INDEX);
      if (n_evicted_out) n_evicted_out[ob] = 0;
    }
    return;
  }
  if (m == 0) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (tid == 0) {
      p.n_staged[lb] = 0;
      p.evict_first[lb] = -1;
      if (n_evicted_out) n_evicted_out[ob] = 0;
    }
    return;
  }
  const int gone = tree_evicted(rg.count, rg.cap, rg.e, m);
  const int events = gone / rg.e;
  const __nv_bfloat16* ringK = reinterpret_cast<const __nv_bfloat16*>(p.K);
  const __nv_bfloat16* ringV = reinterpret_cast<const __nv_bfloat16*>(p.V);
  auto row = [&](int o, const __nv_bfloat16* ring, const __nv_bfloat16* fresh, size_t* stride) -> const __nv_bfloat16* {
    if (o < rg.count) { *stride = (size_t)W * D; return ring + (lb * Hkv * (size_t)W + tree_slot(rg, o)) * D; }
    *stride = D;
    return fresh + (ob * NT + s_path[o - rg.count]) * (size_t)Hkv * D;
  };

  if (folds && gone > 0) {
    const int tiles_n = r >> 2;                            // 8-output tiles of W^a_K and W^a_V
    const int fr = lane >> 2, fq = lane & 3;               // fragment row and quarter
    for (int t0 = 0; t0 < gone; t0 += RT) {
      for (int x = warp; x < tiles_n; x += CM_THREADS / 32) {
        const bool is_v = x >= (r >> 3);
        const int j0 = (is_v ? x - (r >> 3) : x) * 8;
        const __nv_bfloat16* w = reinterpret_cast<const __nv_bfloat16*>(is_v ? p.Wv : p.Wk) +
                                 ((size_t)l * r + j0 + fr) * d_kv + 8 * fq;
        const __nv_bfloat16* src[2 * MT];
        size_t hs[2 * MT];
#pragma unroll
        for (int y = 0; y < 2 * MT; ++y) {
          const int o = t0 + fr + 8 * y;
          src[y] = nullptr;
          hs[y] = 0;
          if (o < gone) src[y] = row(o, is_v ? ringV : ringK, is_v ? v_tree : k_tree, &hs[y]);
        }
        float acc[MT][4];
#pragma unroll
        for (int y = 0; y < MT; ++y) { acc[y][0] = acc[y][1] = acc[y][2] = acc[y][3] = 0.f; }
        constexpr int U = MT == 1 ? 4 : 2;                 // 32-value steps whose loads are in flight together
        int h = (8 * fq) / D, dd = 8 * fq - h * D;
        for (int k0 = 0; k0 < d_kv; k0 += 32 * U) {
          uint4 bw[U], aw[U][2 * MT];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const bool in = k0 + 32 * u < d_kv;
            bw[u] = make_uint4(0u, 0u, 0u, 0u);
            if (in) bw[u] = __ldg(reinterpret_cast<const uint4*>(w + k0 + 32 * u));
#pragma unroll
            for (int y = 0; y < 2 * MT; ++y) {
              aw[u][y] = make_uint4(0u, 0u, 0u, 0u);
              if (in && src[y] != nullptr) aw[u][y] = *reinterpret_cast<const uint4*>(src[y] + h * hs[y] + dd);
            }
            dd += 32;
            while (dd >= D) { dd -= D; ++h; }
          }
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int y = 0; y < MT; ++y) {
              cm_mma(acc[y], aw[u][2 * y].x, aw[u][2 * y + 1].x, aw[u][2 * y].y, aw[u][2 * y + 1].y, bw[u].x, bw[u].y);
              cm_mma(acc[y], aw[u][2 * y].z, aw[u][2 * y + 1].z, aw[u][2 * y].w, aw[u][2 * y + 1].w, bw[u].z, bw[u].w);
            }
        }
        float* dst = s_kv + (is_v ? r : 0) + j0 + 2 * fq;
#pragma unroll
        for (int y = 0; y < MT; ++y) {
          *reinterpret_cast<float2*>(dst + (16 * y + fr) * KP) = make_float2(acc[y][0], acc[y][1]);
          *reinterpret_cast<float2*>(dst + (16 * y + fr + 8) * KP) = make_float2(acc[y][2], acc[y][3]);
        }
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      __syncthreads();
      const int rows = min(RT, gone - t0);
      // p[i][g] = Q_a[g] . k_a[i]: a lane per state row, 2 MT rows of the tile per warp
      for (int g0 = 0; g0 < G; g0 += 32) {
        const int g = min(g0 + lane, G - 1);
        float acc[2 * MT];
#pragma unroll
        for (int y = 0; y < 2 * MT; ++y) acc[y] = 0.f;
        for (int j = 0; j < r; j += 4) {
          const float4 q4 = *reinterpret_cast<const float4*>(s_q + g * QP + j);
#pragma unroll
          for (int y = 0; y < 2 * MT; ++y) {
            const float4 k4 = *reinterpret_cast<const float4*>(s_kv + (warp + 8 * y) * KP + j);
            acc[y] = fmaf(q4.x, k4.x, fmaf(q4.y, k4.y, fmaf(q4.z, k4.z, fmaf(q4.w, k4.w, acc[y]))));
          }
        }
#pragma unroll
        for (int y = 0; y < 2 * MT; ++y) s_p[(warp + 8 * y) * GP + g0 + lane] = acc[y];
      }
      __syncthreads();
      // S += p v_a^T, normalised behind each event's last row; warp w holds state rows g0 + 4 w .. + 3
      for (int g0 = 0; g0 < G; g0 += 32) {
        const int gw = g0 + 4 * warp;
        if (gw >= G) break;                                // uniform over the warp
        float s[4][RJ];
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int jj = 0; jj < RJ; ++jj) {
            const int j = lane + 32 * jj;
            s[x][jj] = (gw + x < G && j < r) ? s_s[(gw + x) * r + j] : 0.f;
          }
        int left = rg.e - t0 % rg.e;                       // rows until the current event is complete
        for (int i = 0; i < rows; ++i) {
          const float4 pv = *reinterpret_cast<const float4*>(s_p + i * GP + gw);
#pragma unroll
          for (int jj = 0; jj < RJ; ++jj) {
            const int j = lane + 32 * jj;
            const float va = j < r ? s_kv[i * KP + r + j] : 0.f;
            s[0][jj] = fmaf(pv.x, va, s[0][jj]);
            s[1][jj] = fmaf(pv.y, va, s[1][jj]);
            s[2][jj] = fmaf(pv.z, va, s[2][jj]);
            s[3][jj] = fmaf(pv.w, va, s[3][jj]);
          }
          if (--left == 0) {
            left = rg.e;
            if (p.norm_mode == PTENC_NORM_ROW_L2) {
              float q2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int jj = 0; jj < RJ; ++jj) q2[x] = fmaf(s[x][jj], s[x][jj], q2[x]);
#pragma unroll
              for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                for (int x = 0; x < 4; ++x) q2[x] += __shfl_xor_sync(0xffffffffu, q2[x], o);
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const float sc = 1.f / fmaxf(sqrtf(q2[x]), 1e-12f);
#pragma unroll
                for (int jj = 0; jj < RJ; ++jj) s[x][jj] *= sc;
              }
            }
          }
        }
        const bool done = t0 + RT >= gone;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int jj = 0; jj < RJ; ++jj) {
            const int j = lane + 32 * jj;
            if (gw + x < G && j < r) {
              if (done) S[(gw + x) * r + j] = s[x][jj];
              else s_s[(gw + x) * r + j] = s[x][jj];
            }
          }
      }
      __syncthreads();                                     // the tile's buffers are free
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  cm_store(p, lb, ob, rg, m, gone, events, n0, k_tree, v_tree, NT, s_path, n_evicted_out);
}

template <typename T>
cudaError_t launch_commit_t(ptenc_cache* c, int l0, int nl, const void* kt, const void* vt, int NT, const int32_t* path,
                            const int32_t* n_path, const uint8_t* active, int32_t* n_evicted_out, cudaStream_t st) {
  const PtencDev& p = c->dev;
  const size_t smem = sizeof(float) * (size_t)(2 * p.d_kv + 2 * p.r + p.G + 2 * p.G * p.r + p.G + 1);
  static bool attr_done[PTENC_MAX_DEVICES] = {};
  if (smem > 40 * 1024 && ptenc_first_use(attr_done, c->cfg.device)) {
    cudaError_t e = cudaFuncSetAttribute(k_commit<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
    if (e != cudaSuccess) return e;
  }
  k_commit<T><<<nl * c->cfg.batch, CM_THREADS, smem, st>>>(p, l0, (const T*)kt, (const T*)vt, NT, path, n_path, active,
                                                           n_evicted_out);
  c->launches++;
  return cudaGetLastError();
}

constexpr size_t CM_SMEM = 220 * 1024;
size_t commit_smem(const PtencDev& p, int mt) {
  const size_t rt = 16 * (size_t)mt, gp = (p.G + 31) / 32 * 32 + 4;
  return sizeof(float) * (rt * (2 * p.r + 4) + rt * gp + (size_t)p.G * (p.r + 4) + (size_t)p.G * p.r);
}

template <int RJ, int MT>
cudaError_t launch_commit_bf16(ptenc_cache* c, int l0, int nl, const void* kt, const void* vt, int NT, const int32_t* path,
                               const int32_t* n_path, const uint8_t* active, int32_t* n_evicted_out, cudaStream_t st) {
  const size_t smem = commit_smem(c->dev, MT);
  static bool attr_done[PTENC_MAX_DEVICES] = {};
  if (smem > 40 * 1024 && ptenc_first_use(attr_done, c->cfg.device)) {
    cudaError_t e = cudaFuncSetAttribute(k_commit_bf16<RJ, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)CM_SMEM);
    if (e != cudaSuccess) return e;
  }
  k_commit_bf16<RJ, MT><<<nl * c->cfg.batch, CM_THREADS, smem, st>>>(
      c->dev, l0, (const __nv_bfloat16*)kt, (const __nv_bfloat16*)vt, NT, path, n_path, active, n_evicted_out);
  c->launches++;
  return cudaGetLastError();
}

}  // namespace

cudaError_t ptenc_launch_commit(ptenc_cache* c, int l0, int nl, const void* k_tree, const void* v_tree, int max_nodes,
                                const int32_t* path, const int32_t* n_path, const uint8_t* active,
                                int32_t* n_evicted_out, cudaStream_t st) {
  const PtencDev& p = c->dev;
  if (c->cfg.dtype == PTENC_DTYPE_BF16 && p.r % 8 == 0 && p.d_kv % 32 == 0 && p.norm_mode != PTENC_NORM_FROBENIUS) {
    // one token per event: 16 rows cover most paths; chunks: 64 rows share each weight vector
    const bool many = p.E > 1 && commit_smem(p, 4) <= CM_SMEM;
    const int rj = p.r <= 32 ? 1 : p.r <= 64 ? 2 : 4;
    auto go = [&](auto RJ, auto MT) {
      return launch_commit_bf16<decltype(RJ)::value, decltype(MT)::value>(c, l0, nl, k_tree, v_tree, max_nodes, path, n_path,
                                                                          active, n_evicted_out, st);
    };
    using std::integral_constant;
    if (many)
      return rj == 1 ? go(integral_constant<int, 1>(), integral_constant<int, 4>())
             : rj == 2 ? go(integral_constant<int, 2>(), integral_constant<int, 4>())
                       : go(integral_constant<int, 4>(), integral_constant<int, 4>());
    return rj == 1 ? go(integral_constant<int, 1>(), integral_constant<int, 1>())
           : rj == 2 ? go(integral_constant<int, 2>(), integral_constant<int, 1>())
                     : go(integral_constant<int, 4>(), integral_constant<int, 1>());
  }
  if (c->cfg.dtype == PTENC_DTYPE_FP32)
    return launch_commit_t<float>(c, l0, nl, k_tree, v_tree, max_nodes, path, n_path, active, n_evicted_out, st);
  return launch_commit_t<__nv_bfloat16>(c, l0, nl, k_tree, v_tree, max_nodes, path, n_path, active, n_evicted_out, st);
}

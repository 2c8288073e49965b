// The accepted path of a draft enters the cache: as many appends, evictions and folds as the path has tokens, in one call.
//
// The same result as ptenc_append_evict and ptenc_encode once per token of the path.  The ring words follow from counts
// alone (ptenc_tree.cuh): after m arrivals ev(m) tokens have left, in events of e; event k takes the arrival numbers
// [k e, (k + 1) e), which are cache tokens or, when the ring is shorter than the path, the path's own first tokens.  The
// state is normalised after every event, so events are folded in order; the rows of an event are summed,
//   S <- Normalize(S + sum_i (Q_a k_a,i) v_a,i^T)   (Sec. 3.3, Eq. (3) and the sentence after it).
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

}  // namespace

cudaError_t ptenc_launch_commit(ptenc_cache* c, int l0, int nl, const void* k_tree, const void* v_tree, int max_nodes,
                                const int32_t* path, const int32_t* n_path, const uint8_t* active,
                                int32_t* n_evicted_out, cudaStream_t st) {
  if (c->cfg.dtype == PTENC_DTYPE_FP32)
    return launch_commit_t<float>(c, l0, nl, k_tree, v_tree, max_nodes, path, n_path, active, n_evicted_out, st);
  return launch_commit_t<__nv_bfloat16>(c, l0, nl, k_tree, v_tree, max_nodes, path, n_path, active, n_evicted_out, st);
}

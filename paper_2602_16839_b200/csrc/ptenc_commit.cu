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
constexpr int CM_KC = 512;             // columns of the evicted rows in shared memory at a time
constexpr int CM_KP = CM_KC + 32;      // and their pitch, 64 bytes past whole rounds of the banks: 64-byte pieces of two rows side by side

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

// Rows [r0, r1) of the last event to the staging area, oldest first and KV heads concatenated.  All threads of the CTA.
template <typename T>
__device__ __forceinline__ void cm_stage(const PtencDev& p, size_t lb, size_t ob, const TreeRing& rg, int events, int r0, int r1,
                                         const T* __restrict__ k_tree, const T* __restrict__ v_tree, int NT,
                                         const int* s_path) {
  const int D = p.D, Hkv = p.Hkv, W = p.W, tid = threadIdx.x;
  const int vph = D * (int)sizeof(T) / 16, vpr = Hkv * vph;
  auto row = [&](int o, const char* ring, const T* fresh, size_t* stride) -> const T* {
    if (o < rg.count) {
      *stride = (size_t)W * D;
      return reinterpret_cast<const T*>(ring) + (lb * Hkv * (size_t)W + tree_slot(rg, o)) * D;
    }
    *stride = D;
    return fresh + (ob * NT + s_path[o - rg.count]) * (size_t)Hkv * D;
  };
  // four vectors of K and of V per thread and turn, all requested before any is stored
  constexpr int U = 4;
  for (int rb = r0; rb < r1; rb += PTENC_ROW_BLOCK) {
    const int total = min(r1 - rb, PTENC_ROW_BLOCK) * vpr, o0 = (events - 1) * rg.e + rb;
    const size_t to = (lb * p.E + rb) * vpr;               // rows of the staging area are Hkv D long
    for (int i0 = tid; i0 < total; i0 += U * CM_THREADS) {
      uint4 kv[U], vv[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = min(i0 + u * CM_THREADS, total - 1);
        const int rr = i / vpr, v = i - rr * vpr, h = v / vph;
        size_t ks, vs;
        const T* kr = row(o0 + rr, p.K, k_tree, &ks);
        const T* vr = row(o0 + rr, p.V, v_tree, &vs);
        kv[u] = reinterpret_cast<const uint4*>(kr + h * ks)[v - h * vph];
        vv[u] = reinterpret_cast<const uint4*>(vr + h * vs)[v - h * vph];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * CM_THREADS;
        if (i < total) {
          reinterpret_cast<uint4*>(p.stageK)[to + i] = kv[u];
          reinterpret_cast<uint4*>(p.stageV)[to + i] = vv[u];
        }
      }
    }
  }
}

// The end of a commit, alike for every kernel: the last event's rows to the staging area, the tokens that stay into the
// slots the evicted ones left, the ring words.  All threads of the CTA; every row has been folded before, and with `staged`
// the last event's rows are in the staging area already.
template <typename T>
__device__ __forceinline__ void cm_store(const PtencDev& p, size_t lb, size_t ob, const TreeRing& rg, int m, int gone,
                                         int events, long long n0, const T* __restrict__ k_tree,
                                         const T* __restrict__ v_tree, int NT, const int* s_path, int32_t* n_evicted_out,
                                         bool staged = false) {
  const int D = p.D, Hkv = p.Hkv, W = p.W, tid = threadIdx.x;
  const int vph = D * (int)sizeof(T) / 16, vpr = Hkv * vph;
  const bool last_evicts = events > 0 && rg.cap - rg.count + (events - 1) * rg.e == m - 1;
  if (last_evicts && !staged) cm_stage(p, lb, ob, rg, events, 0, rg.e, k_tree, v_tree, NT, s_path);
  // ---- the tokens that stay, into the slots the evicted ones left (all of those have been read above) ------------------
  __syncthreads();
  const int first = gone > rg.count ? gone - rg.count : 0;         // a path longer than the ring keeps its newest tokens
  constexpr int NW = CM_THREADS / 32;
  for (int v = tid & 31; v < vpr; v += 32) {               // a lane per 16 bytes of a row, a token per warp, two at a time
    const int h = v / vph;
    const size_t at = ((lb * Hkv + h) * (size_t)W) * vph + (v - h * vph);
    for (int j0 = first + (tid >> 5); j0 < m; j0 += 2 * NW) {
      uint4 kv[2], vv[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const size_t src = (ob * NT + s_path[min(j0 + u * NW, m - 1)]) * (size_t)vpr + v;
        kv[u] = reinterpret_cast<const uint4*>(k_tree)[src];
        vv[u] = reinterpret_cast<const uint4*>(v_tree)[src];
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int j = j0 + u * NW;
        if (j < m) {
          const size_t dst = at + (size_t)tree_slot(rg, rg.count + j) * vph;
          reinterpret_cast<uint4*>(p.K)[dst] = kv[u];
          reinterpret_cast<uint4*>(p.V)[dst] = vv[u];
        }
      }
    }
  }
  if (tid == 0) {
    p.head[lb] = (rg.head + gone) % rg.cap;              // gone <= window + nodes
    p.count[lb] = rg.count + m - gone;
    p.n_app[lb] = n0 + m;
    p.n_staged[lb] = last_evicts ? rg.e : 0;
    p.evict_first[lb] = last_evicts ? n0 - rg.count + (long long)(events - 1) * rg.e : -1;
    if (n_evicted_out) n_evicted_out[ob] = gone;
  }
}

// Shape-generic kernel (fp32 storage, Frobenius norm, ranks or rows that k_commit_bf16 does not take): a CTA per (layer, sequence),
// rows one after another, four block barriers and the weights read anew for each.  That chain is the bound: 28 layers x 32
// sequences, paths of up to 8 tokens that each evict one, 203 us in fp32 (61 MB, 9 us of copy bandwidth) and 265 us in bf16
// with the Frobenius norm; chunks of 129 rows in fp32 815 us.  The tiling of k_commit_bf16 has not been carried over to it.
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
  tree_after_previous();
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
// (layer, sequence), the evicted rows 16 at a time in order of arrival.  A commit is a chain of round trips (ring words, rows
// and weights, the events one after another, the stores), so each link asks for all it needs at once:
//  * rows come to shared memory by asynchronous copies while the first weights are requested; k_a and v_a of the 16 rows are
//    mma.m16n8k16 products, a warp per eight outputs.  A lane reads 16-byte vectors of rows and weights: eight consecutive
//    values serve two mma steps, the contraction index permuted alike on both operands.
//  * p = Q_a k_a for all rows, then S += p v_a^T row by row, a warp per four state rows and a lane per column, with the
//    state rows in registers; behind the last row of an event the rows are normalised, four at a time.
// With `defer` the last event is left out: its rows are in the staging area (k_commit_stage) for the chunk encoder.
//  RJ = columns per lane (r <= 32 RJ).
// Measured (G = r = 32, four KV heads of 128): 28 layers x 32 sequences, paths of up to 8 tokens that each evict one, 30 us
// (34 MB that have to move, 5 us of copy bandwidth); one layer of 8 sequences 8 us.  The bound is the chain of round trips
// and the instructions of many small steps (issue slots 40 % busy, DRAM 8 %), so four CTAs share an SM: three, with twice the
// weights in flight, 32 us.
template <int RJ>
__global__ void __launch_bounds__(CM_THREADS, 4)
k_commit_bf16(PtencDev p, int l0, const __nv_bfloat16* __restrict__ k_tree, const __nv_bfloat16* __restrict__ v_tree, int NT,
              const int32_t* __restrict__ path, const int32_t* __restrict__ n_path, const uint8_t* __restrict__ active,
              int32_t* n_evicted_out, bool defer) {
  extern __shared__ __align__(16) float cm_sm[];
  __shared__ int s_path[TREE_MAX];
  __shared__ const __nv_bfloat16* s_src[32];
  __shared__ size_t s_hs[32];
  constexpr int RT = 16;
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
  __nv_bfloat16* s_row = reinterpret_cast<__nv_bfloat16*>(s_s + G * r);    // [K, V][RT][CM_KP] columns of the evicted rows
  const bool enc = p.encode_enabled != 0;
  float* S = p.S + lb * G * r;
  tree_after_previous();
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

  const int fold = defer && events > 0 ? gone - rg.e : gone;       // rows to fold here
  if (folds && fold > 0) {
    const int tiles_n = r >> 2;                            // 8-output tiles of W^a_K and W^a_V
    const int fr = lane >> 2, fq = lane & 3;               // fragment row and quarter
    for (int t0 = 0; t0 < fold; t0 += RT) {
      const int here = min(RT, fold - t0);
      if (tid < 2 * RT) {                                  // where the tile's rows lie
        size_t hs = 0;
        const __nv_bfloat16* src = nullptr;
        const int o = t0 + tid % RT;
        if (o < fold) src = row(o, tid < RT ? ringK : ringV, tid < RT ? k_tree : v_tree, &hs);
        s_src[tid] = src;
        s_hs[tid] = hs;
      }
      __syncthreads();
      for (int kc = 0; kc < d_kv; kc += CM_KC) {
        const int kn = min(CM_KC, d_kv - kc);
        // the columns [kc, kc + kn) of the tile's rows, a row of K or V per warp and turn; what lies behind the last row is
        // whatever it was: it reaches only the products of rows that nobody reads
        for (int w = warp; w < 2 * here; w += CM_THREADS / 32) {
          const int is_v = w >= here, rr = is_v ? w - here : w;
          const __nv_bfloat16* src = s_src[is_v * RT + rr];
          const size_t hs = s_hs[is_v * RT + rr];
          __nv_bfloat16* dst = s_row + (is_v * RT + rr) * CM_KP;
          for (int d = 8 * lane; d < kn; d += 256) {
            const int h = (kc + d) / D;
            cm_async16(dst + d, src + h * hs + (kc + d - h * D));
          }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        bool there = false;
        for (int x = warp; x < tiles_n; x += CM_THREADS / 32) {
          const bool is_v = x >= (r >> 3);
          const int j0 = (is_v ? x - (r >> 3) : x) * 8;
          const __nv_bfloat16* w = reinterpret_cast<const __nv_bfloat16*>(is_v ? p.Wv : p.Wk) +
                                   ((size_t)l * r + j0 + fr) * d_kv + kc + 8 * fq;
          float acc[4] = {0.f, 0.f, 0.f, 0.f};
          float* dst = s_kv + fr * KP + (is_v ? r : 0) + j0 + 2 * fq;
          if (kc > 0) { acc[0] = dst[0]; acc[1] = dst[1]; acc[2] = dst[8 * KP]; acc[3] = dst[8 * KP + 1]; }
          constexpr int U = 4;                             // 32-value steps whose weights are in flight together
          for (int k0 = 0; k0 < kn; k0 += 32 * U) {
            uint4 bw[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
              bw[u] = k0 + 32 * u < kn ? __ldg(reinterpret_cast<const uint4*>(w + k0 + 32 * u)) : make_uint4(0u, 0u, 0u, 0u);
            if (!there) {                                  // the first weights are on their way: now wait for the rows
              there = true;
              asm volatile("cp.async.wait_group 0;" ::: "memory");
              asm volatile("bar.sync 0;" ::: "memory");
            }
            const __nv_bfloat16* ar = s_row + ((is_v ? RT : 0) + fr) * CM_KP + k0 + 8 * fq;
#pragma unroll
            for (int u = 0; u < U; ++u) {
              if (k0 + 32 * u < kn) {
                const uint4 lo = *reinterpret_cast<const uint4*>(ar + 32 * u);
                uint4 hi = make_uint4(0u, 0u, 0u, 0u);
                if (here > 8) hi = *reinterpret_cast<const uint4*>(ar + 8 * CM_KP + 32 * u);
                cm_mma(acc, lo.x, hi.x, lo.y, hi.y, bw[u].x, bw[u].y);
                cm_mma(acc, lo.z, hi.z, lo.w, hi.w, bw[u].z, bw[u].w);
              }
            }
          }
          *reinterpret_cast<float2*>(dst) = make_float2(acc[0], acc[1]);
          *reinterpret_cast<float2*>(dst + 8 * KP) = make_float2(acc[2], acc[3]);
        }
        if (!there) {                                      // a warp without outputs still takes part
          asm volatile("cp.async.wait_group 0;" ::: "memory");
          asm volatile("bar.sync 0;" ::: "memory");
        }
        __syncthreads();                                   // products stored, row buffer free
      }
      // p[i][g] = Q_a[g] . k_a[i]: a lane per state row, two rows of the tile per warp
      for (int g0 = 0; g0 < G; g0 += 32) {
        const int g = min(g0 + lane, G - 1);
        float acc[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) acc[y] = 0.f;
        for (int j = 0; j < r; j += 4) {
          const float4 q4 = *reinterpret_cast<const float4*>(s_q + g * QP + j);
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float4 k4 = *reinterpret_cast<const float4*>(s_kv + (warp + 8 * y) * KP + j);
            acc[y] = fmaf(q4.x, k4.x, fmaf(q4.y, k4.y, fmaf(q4.z, k4.z, fmaf(q4.w, k4.w, acc[y]))));
          }
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) s_p[(warp + 8 * y) * GP + g0 + lane] = acc[y];
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
        for (int i = 0; i < here; ++i) {
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
              // four sums over the warp: each exchange halves the values a lane carries, eight lanes finish a row
              const bool up = lane & 16, right = lane & 8;
              const float a = (up ? q2[2] : q2[0]) + __shfl_xor_sync(0xffffffffu, up ? q2[0] : q2[2], 16);
              const float b = (up ? q2[3] : q2[1]) + __shfl_xor_sync(0xffffffffu, up ? q2[1] : q2[3], 16);
              float n2 = (right ? b : a) + __shfl_xor_sync(0xffffffffu, right ? a : b, 8);
#pragma unroll
              for (int o = 4; o > 0; o >>= 1) n2 += __shfl_xor_sync(0xffffffffu, n2, o);
              // 1 / max(|row|, 1e-12) by rsqrtf, within two units in the last place of the square root and division, which would
              // sit in the chain between two events: a state after eight events is off by 6e-7 of its size
              n2 = rsqrtf(fmaxf(n2, 1e-24f));
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const float sc = __shfl_sync(0xffffffffu, n2, 8 * x);
#pragma unroll
                for (int jj = 0; jj < RJ; ++jj) s[x][jj] *= sc;
              }
            }
          }
        }
        const bool done = t0 + RT >= fold;
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
  cm_store(p, lb, ob, rg, m, gone, events, n0, k_tree, v_tree, NT, s_path, n_evicted_out, defer);
}

// The staging of a chunk in front of the commit itself, 16 rows per CTA: one CTA per sequence would copy 129 rows of 512
// columns in 18 us.  deferred[] receives the number of rows staged; paths that the commit refuses are left alone here.  `groups`
// CTAs per sequence, all in the grid's first direction, since a chunk may have more groups than the second one has places.
constexpr int CM_STAGE = 16;
__global__ void __launch_bounds__(CM_THREADS)
k_commit_stage(PtencDev p, int l0, const __nv_bfloat16* __restrict__ k_tree, const __nv_bfloat16* __restrict__ v_tree, int NT,
               const int32_t* __restrict__ path, const int32_t* __restrict__ n_path, const uint8_t* __restrict__ active,
               int32_t* __restrict__ deferred, int groups) {
  __shared__ int s_path[TREE_MAX];
  const int seq = blockIdx.x / groups, group = blockIdx.x - seq * groups;
  const int li = seq / p.B, b = seq - li * p.B, tid = threadIdx.x;
  const size_t lb = (size_t)(l0 + li) * p.B + b, ob = (size_t)li * p.B + b;
  tree_after_previous();
  const int m = (active != nullptr && active[b] == 0) ? 0 : n_path[b];
  TreeRing rg;
  int bad = !tree_ring(p, lb, &rg) || m < 0 || m > NT;
  if (tid < NT) {
    const int at = path[(size_t)b * NT + tid];
    s_path[tid] = at;
    bad |= tid < m && (at < 0 || at >= NT);
  }
  bad = __syncthreads_or(bad);
  const int events = bad ? 0 : tree_evicted(rg.count, rg.cap, rg.e, m) / rg.e;
  if (group == 0 && tid == 0) deferred[ob] = events > 0 ? rg.e : 0;
  const int r0 = group * CM_STAGE;
  if (events == 0 || r0 >= rg.e) return;
  cm_stage(p, lb, ob, rg, events, r0, min(r0 + CM_STAGE, rg.e), k_tree, v_tree, NT, s_path);
}

template <typename T>
cudaError_t launch_commit_t(ptenc_cache* c, int l0, int nl, const void* kt, const void* vt, int NT, const int32_t* path,
                            const int32_t* n_path, const uint8_t* active, int32_t* n_evicted_out, cudaStream_t st) {
  const PtencDev& p = c->dev;
  const size_t smem = sizeof(float) * (size_t)(2 * p.d_kv + 2 * p.r + p.G + 2 * p.G * p.r + p.G + 1);
  static PtencOnce once;
  if (smem > 40 * 1024) {
    const cudaError_t e = ptenc_first_use(once, c->cfg.device, [] { return ptenc_allow_smem(k_commit<T>, 200 * 1024); });
    if (e != cudaSuccess) return e;
  }
  c->launches++;
  return tree_launch(k_commit<T>, dim3(nl * c->cfg.batch), CM_THREADS, smem, 0, st, p, l0, (const T*)kt, (const T*)vt, NT, path,
                     n_path, active, n_evicted_out);
}

constexpr size_t CM_SMEM = 220 * 1024;
size_t commit_smem(const PtencDev& p) {
  const size_t gp = (p.G + 31) / 32 * 32 + 4;
  return sizeof(float) * (16 * (size_t)(2 * p.r + 4) + 16 * gp + (size_t)p.G * (p.r + 4) + (size_t)p.G * p.r) +
         (size_t)2 * 16 * CM_KP * 2;
}

template <int RJ>
cudaError_t launch_commit_bf16(ptenc_cache* c, int l0, int nl, const void* kt, const void* vt, int NT, const int32_t* path,
                               const int32_t* n_path, const uint8_t* active, int32_t* n_evicted_out, bool defer,
                               cudaStream_t st) {
  const size_t smem = commit_smem(c->dev);
  static PtencOnce once;
  if (smem > 40 * 1024) {
    const cudaError_t e = ptenc_first_use(once, c->cfg.device, [] { return ptenc_allow_smem(k_commit_bf16<RJ>, CM_SMEM); });
    if (e != cudaSuccess) return e;
  }
  c->launches++;
  return tree_launch(k_commit_bf16<RJ>, dim3(nl * c->cfg.batch), CM_THREADS, smem, 0, st, c->dev, l0, (const __nv_bfloat16*)kt,
                     (const __nv_bfloat16*)vt, NT, path, n_path, active, n_evicted_out, defer);
}

}  // namespace

cudaError_t ptenc_launch_commit(ptenc_cache* c, int l0, int nl, const void* k_tree, const void* v_tree, int max_nodes,
                                const int32_t* path, const int32_t* n_path, const uint8_t* active,
                                int32_t* n_evicted_out, cudaStream_t st) {
  const PtencDev& p = c->dev;
  if (c->cfg.dtype == PTENC_DTYPE_BF16 && p.r % 8 == 0 && p.d_kv % 32 == 0 && p.norm_mode != PTENC_NORM_FROBENIUS) {
    // Chunks of evicted tokens (E >= 16, a tile of the fold here) are folded by the chunk encoder, which reads them from the
    // staging area: 192 sequences of which 40 % evict 129 rows 56 us by k_commit_bf16 alone, 29 us with the encoder.  The encoder
    // loads boxes of up to 128 rows, which the staged rows of the call's layers have to be as many as.
    const bool chunks = p.E >= 16 && c->tc_encode && c->cfg.encode_enabled && (long long)nl * p.B * p.E >= 128;
    int32_t* deferred = c->commit_rows;
    cudaError_t e;
    if (chunks) {
      c->launches++;
      const int groups = (p.E + CM_STAGE - 1) / CM_STAGE;          // nl B E < 2^31: the grid's size fits
      e = tree_launch(k_commit_stage, dim3(nl * p.B * groups), CM_THREADS, 0, 0, st, p, l0, (const __nv_bfloat16*)k_tree,
                      (const __nv_bfloat16*)v_tree, max_nodes, path, n_path, active, deferred, groups);
      if (e != cudaSuccess) return e;
    }
    if (p.r <= 32) e = launch_commit_bf16<1>(c, l0, nl, k_tree, v_tree, max_nodes, path, n_path, active, n_evicted_out, chunks, st);
    else if (p.r <= 64) e = launch_commit_bf16<2>(c, l0, nl, k_tree, v_tree, max_nodes, path, n_path, active, n_evicted_out, chunks, st);
    else e = launch_commit_bf16<4>(c, l0, nl, k_tree, v_tree, max_nodes, path, n_path, active, n_evicted_out, chunks, st);
    if (e != cudaSuccess || !chunks) return e;
    const size_t rows = (size_t)l0 * p.B * p.E * p.d_kv * p.elt;
    return ptenc_launch_encode_tc(c, l0, nl, p.stageK + rows, p.stageV + rows, deferred, p.E, st);
  }
  if (c->cfg.dtype == PTENC_DTYPE_FP32)
    return launch_commit_t<float>(c, l0, nl, k_tree, v_tree, max_nodes, path, n_path, active, n_evicted_out, st);
  return launch_commit_t<__nv_bfloat16>(c, l0, nl, k_tree, v_tree, max_nodes, path, n_path, active, n_evicted_out, st);
}

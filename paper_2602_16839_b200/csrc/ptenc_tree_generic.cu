// Attention of a draft tree over the cache, shape-generic kernel: fp32 or bf16 storage, any head_dim <= 256 that is a
// multiple of 8, any query group size.
//
// out[i,h] = softmax(q[i,h] . K^T / sqrt(D)) V over the tokens node i sees (ptenc_tree.cuh).  A CTA takes 16 query rows
// (row = node * g + head of the group) of one (layer, sequence, KV head) and walks the tokens 32 at a time: K and V rows
// as fp32 in shared memory, a score per (lane = token, four rows per warp), the running maximum and sum of the softmax
// per row, and the outputs of a row in the registers of eight threads.  fp32 FMA throughout (no TF32).
#include "ptenc_tree.cuh"

namespace {

constexpr int TG_THREADS = 128;
constexpr int TG_ROWS = 16;
constexpr int TG_TOK = 32;
constexpr int TG_MAXJ = 32;          // head_dim <= 8 * TG_MAXJ

template <typename T>
__global__ void __launch_bounds__(TG_THREADS)
k_tree_generic(PtencDev p, int l0, const T* __restrict__ q, const T* __restrict__ k_tree, const T* __restrict__ v_tree,
               const int32_t* __restrict__ parent, const int32_t* __restrict__ n_nodes, int NT,
               const uint8_t* __restrict__ active, T* __restrict__ out, float* __restrict__ lse, int n_groups) {
  extern __shared__ float tg_sm[];
  const int D = p.D, g = p.g, W = p.W, Hkv = p.Hkv;
  const int KP = D + 4;                                  // K row pitch: 16-byte loads of 32 rows without bank conflicts
  float* s_k = tg_sm;                                    // [TG_TOK][KP]
  float* s_v = s_k + TG_TOK * KP;                        // [TG_TOK][D]
  float* s_q = s_v + TG_TOK * D;                         // [TG_ROWS][D]
  __shared__ float s_p[TG_ROWS][TG_TOK + 1];
  __shared__ float s_m[TG_ROWS], s_l[TG_ROWS], s_c[TG_ROWS];
  __shared__ unsigned long long s_anc[TREE_MAX], s_vis[TREE_MAX];
  __shared__ int s_ev[TREE_MAX], s_jump[TREE_MAX];

  int idx = blockIdx.x;
  const int grp = idx % n_groups; idx /= n_groups;
  const int hkv = idx % Hkv; idx /= Hkv;
  const int b = idx % p.B;
  const int li = idx / p.B;
  if (active != nullptr && active[b] == 0) return;
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
  if (row0 >= n * g) return;                             // rows of nodes that do not exist stay as they are
  if (!tree_setup(parent + (size_t)b * NT, n, r, s_anc, s_vis, s_ev, s_jump)) {
    if (threadIdx.x == 0) atomicOr(p.status, PTENC_ST_BAD_INDEX);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int i = tid; i < TG_ROWS * D; i += TG_THREADS) {
    const int rr = i / D, d = i - rr * D, row = row0 + rr;
    const int node = row / g, h = row - node * g;
    s_q[i] = node < n ? ptenc_to_float(q[((ob * NT + node) * p.Hq + (size_t)hkv * g + h) * D + d]) : 0.f;
  }
  if (tid < TG_ROWS) { s_m[tid] = -INFINITY; s_l[tid] = 0.f; }

  // tokens of the unit: pinned entries, then the ring from the oldest token that any node sees, then the nodes
  const int ev0 = min(tree_evicted(r.count, r.cap, r.e, 1), r.count);
  const int n_ring = r.count - ev0;
  const int n_cache = r.sink + n_ring;
  const int n_tok = n_cache + n;
  const T* Kb = reinterpret_cast<const T*>(p.K) + (lb * Hkv + hkv) * (size_t)W * D;
  const T* Vb = reinterpret_cast<const T*>(p.V) + (lb * Hkv + hkv) * (size_t)W * D;
  const float scale = 1.0f / sqrtf((float)D);
  const int orow = tid >> 3, od = tid & 7;
  float acc[TG_MAXJ];
#pragma unroll
  for (int j = 0; j < TG_MAXJ; ++j) acc[j] = 0.f;

  for (int t0 = 0; t0 < n_tok; t0 += TG_TOK) {
    __syncthreads();
    for (int tt = warp; tt < TG_TOK; tt += TG_THREADS / 32) {
      const int i = t0 + tt;
      const T *kr = nullptr, *vr = nullptr;
      if (i < n_cache) {
        const int slot = i < r.sink ? i : tree_slot(r, ev0 + (i - r.sink));
        kr = Kb + (size_t)slot * D;
        vr = Vb + (size_t)slot * D;
      } else if (i < n_tok) {
        const size_t at = ((ob * NT + (i - n_cache)) * Hkv + hkv) * (size_t)D;
        kr = k_tree + at;
        vr = v_tree + at;
      }
      for (int d = lane; d < D; d += 32) {
        s_k[tt * KP + d] = kr != nullptr ? ptenc_to_float(kr[d]) : 0.f;
        s_v[tt * D + d] = kr != nullptr ? ptenc_to_float(vr[d]) : 0.f;
      }
    }
    __syncthreads();
    // scores: lane = token, rows 4 warp .. 4 warp + 3
    {
      float s[4] = {0.f, 0.f, 0.f, 0.f};
      const float4* kr = reinterpret_cast<const float4*>(s_k + lane * KP);
      for (int d4 = 0; d4 < D / 4; ++d4) {
        const float4 kk = kr[d4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float4 qq = *reinterpret_cast<const float4*>(s_q + (4 * warp + x) * D + 4 * d4);
          s[x] = fmaf(qq.x, kk.x, fmaf(qq.y, kk.y, fmaf(qq.z, kk.z, fmaf(qq.w, kk.w, s[x]))));
        }
      }
      const int i = t0 + lane;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int rr = 4 * warp + x;
        const int node = (row0 + rr) / g;
        bool seen = false;
        if (node < n && i < n_tok) {
          if (i < r.sink) seen = true;
          else if (i < n_cache) seen = ev0 + (i - r.sink) >= s_ev[node];
          else seen = (s_vis[node] >> (i - n_cache)) & 1ull;
        }
        const float v = seen ? s[x] * scale : -INFINITY;
        float mx = v;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float m_old = s_m[rr], m_new = fmaxf(m_old, mx);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float e = seen ? expf(v - m_use) : 0.f;
        float sum = e;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        s_p[rr][lane] = e;
        __syncwarp();                                     // every lane has read the row's old maximum
        if (lane == 0) {
          const float corr = m_old == -INFINITY ? 0.f : expf(m_old - m_use);
          s_c[rr] = corr;
          s_l[rr] = s_l[rr] * corr + sum;
          s_m[rr] = m_new;
        }
      }
    }
    __syncthreads();
    // outputs: eight threads per row, every eighth dim
    {
      const float corr = s_c[orow];
#pragma unroll
      for (int j = 0; j < TG_MAXJ; ++j) acc[j] *= corr;
      const int last = min(TG_TOK, n_tok - t0);
      for (int tt = 0; tt < last; ++tt) {
        const float e = s_p[orow][tt];
        if (e != 0.f) {                                   // a token the row does not see may hold anything, NaN included
#pragma unroll
          for (int j = 0; j < TG_MAXJ; ++j)
            if (od + 8 * j < D) acc[j] = fmaf(e, s_v[tt * D + od + 8 * j], acc[j]);
        }
      }
    }
  }
  const int row = row0 + orow;
  const int node = row / g, h = row - node * g;
  if (node < n) {
    const float l = s_l[orow];
    const size_t at = (ob * NT + node) * p.Hq + (size_t)hkv * g + h;
#pragma unroll
    for (int j = 0; j < TG_MAXJ; ++j)
      if (od + 8 * j < D) out[at * D + od + 8 * j] = ptenc_from_float<T>(acc[j] / l);
    if (lse != nullptr && od == 0) lse[at] = s_m[orow] + logf(l);
  }
}

template <typename T>
cudaError_t launch_tree_t(ptenc_cache* c, int l0, int nl, const void* q, const void* kt, const void* vt,
                          const int32_t* parent, const int32_t* n_nodes, int NT, const uint8_t* active, void* out,
                          float* lse, cudaStream_t st) {
  const PtencDev& p = c->dev;
  const int n_groups = (NT * p.g + TG_ROWS - 1) / TG_ROWS;
  const long long grid = (long long)nl * p.B * p.Hkv * n_groups;
  if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
  const size_t smem = sizeof(float) * ((size_t)TG_TOK * (2 * p.D + 4) + (size_t)TG_ROWS * p.D);
  static bool attr_done[PTENC_MAX_DEVICES] = {};
  if (smem > 40 * 1024 && ptenc_first_use(attr_done, c->cfg.device)) {
    cudaError_t e = cudaFuncSetAttribute(k_tree_generic<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 96 * 1024);
    if (e != cudaSuccess) return e;
  }
  k_tree_generic<T><<<(unsigned)grid, TG_THREADS, smem, st>>>(p, l0, (const T*)q, (const T*)kt, (const T*)vt, parent,
                                                              n_nodes, NT, active, (T*)out, lse, n_groups);
  c->launches++;
  return cudaGetLastError();
}

}  // namespace

cudaError_t ptenc_launch_tree_generic(ptenc_cache* c, int l0, int nl, const void* q, const void* k_tree,
                                      const void* v_tree, const int32_t* parent, const int32_t* n_nodes, int max_nodes,
                                      const uint8_t* active, void* out, float* lse, cudaStream_t st) {
  if (c->cfg.dtype == PTENC_DTYPE_FP32)
    return launch_tree_t<float>(c, l0, nl, q, k_tree, v_tree, parent, n_nodes, max_nodes, active, out, lse, st);
  return launch_tree_t<__nv_bfloat16>(c, l0, nl, q, k_tree, v_tree, parent, n_nodes, max_nodes, active, out, lse, st);
}

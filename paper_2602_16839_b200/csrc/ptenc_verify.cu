// Verification of a draft tree against the target's probabilities, from given random numbers.
//
// Scan, per sequence: the walk stands at node cur (the root at first) with r = p[cur].  The children of cur are judged in
// order of their index; child i with token x was drawn from q[cur] and is accepted when u[i] q[cur](x) < r(x): the walk
// moves to i and r = p[i].  Otherwise r <- max(r - q[cur], 0) / sum, the distribution that makes the procedure as a whole
// sample from the target's rows (nothing left, i.e. a sum that is not positive: r = p[cur]).  When the children are used
// up the next token is the first x whose cumulative sum of r exceeds u[0] times the total.
//
// What it costs.  Judging a first child needs two numbers of a row; only a rejection or the last draw needs whole rows,
// and those are rows of one node.  So a sequence reads its tree, one number of p and q per node (all requested together),
// and then one row of p, and of q if a child was rejected there, once per rejected child that has a younger sibling and
// once for the draw; the repeats come from the caches.  The rows are spread over a cluster of CTAs.
//
// Arithmetic: r, its sums and the border of the draw are held in 64 bits.  Neighbouring borders of a row of 10^5 entries
// are about as close as a 32-bit sum of them is wrong, so a 32-bit cumulative sum would draw another token now and then.
#include <cooperative_groups.h>
#include <string.h>

#include "ptenc_tree.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int VF_THREADS = 512;
constexpr int VF_WARPS = VF_THREADS / 32;
constexpr int VF_CLUSTER = 8;

struct VerifyArgs {
  const void* p;
  const void* q;                 // null: the drafted token had probability one
  const int32_t* tokens;
  const int32_t* parent;
  const int32_t* n_nodes;
  const float* u;
  const uint8_t* active;
  int T;
  long long V, total;            // entries of a row, entries of the whole tensor
  int32_t* path;
  int32_t* n_path;
  int32_t* next;
};

// Sixteen bytes' worth of consecutive entries, as they lie in memory.
template <typename T> struct VfVec {
  static constexpr int N = 16 / (int)sizeof(T);
  T e[N];
};
// Entries [at, at + N) of a tensor of `total` entries; at is a multiple of N, at >= 0.
template <typename T>
__device__ __forceinline__ VfVec<T> vf_load(const T* base, long long at, long long total) {
  VfVec<T> v;
  if (at + VfVec<T>::N <= total) {
    *reinterpret_cast<uint4*>(v.e) = __ldg(reinterpret_cast<const uint4*>(base + at));
  } else {
#pragma unroll
    for (int i = 0; i < VfVec<T>::N; ++i) v.e[i] = at + i < total ? base[at + i] : ptenc_from_float<T>(0.f);
  }
  return v;
}

template <typename T>
__global__ void __launch_bounds__(VF_THREADS)
k_verify_tree(const VerifyArgs a) {
  constexpr int N = VfVec<T>::N;
  cg::cluster_group cluster = cg::this_cluster();
  const int CS = (int)cluster.num_blocks();
  const int rank = (int)cluster.block_rank();
  const int b = blockIdx.x / CS;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  __shared__ int s_par[TREE_MAX], s_tok[TREE_MAX], s_path[TREE_MAX];
  __shared__ double s_pv[TREE_MAX], s_qv[TREE_MAX], s_u[TREE_MAX];
  __shared__ double s_norm[TREE_MAX];              // sums of the levels of r at the current node
  __shared__ int s_rej[TREE_MAX];                  // tokens rejected at the current node
  __shared__ double s_warp[VF_WARPS];
  __shared__ double s_cta[2];                      // this CTA's sum, read by the other CTAs; passes alternate
  __shared__ double s_all[VF_CLUSTER];

  if (a.active != nullptr && a.active[b] == 0) return;            // the whole cluster
  const int n = a.n_nodes != nullptr ? a.n_nodes[b] : a.T;
  const T* P = static_cast<const T*>(a.p);
  const T* Q = static_cast<const T*>(a.q);
  int bad = n < 1 || n > a.T;
  if (!bad && tid < n) {
    const size_t at = (size_t)b * a.T + tid;
    const int par = a.parent[at];
    const int tok = a.tokens[at];
    s_par[tid] = par;
    s_tok[tid] = tok;
    s_u[tid] = (double)a.u[at];
    bad = tid == 0 ? par != -1 : (par < 0 || par >= tid || tok < 0 || tok >= a.V);
    if (!bad && tid > 0) {
      const long long x = ((long long)b * a.T + par) * a.V + tok;
      s_pv[tid] = (double)ptenc_to_float(P[x]);
      s_qv[tid] = Q != nullptr ? (double)ptenc_to_float(Q[x]) : 1.0;
    }
  }
  if (__syncthreads_or(bad)) {                                    // the same verdict in every CTA of the cluster
    if (rank == 0) {
      for (int i = tid; i < a.T; i += VF_THREADS) a.path[(size_t)b * a.T + i] = -1;
      if (tid == 0) { a.n_path[b] = 0; a.next[b] = -1; }
    }
    return;
  }

  // r after `levels` rejections at the current node, for an entry with p, q and index x; a level whose sum was not
  // positive starts over from p
  int levels = 0;
  auto level = [&](double pv, double qv, long long x, int upto) -> double {
    double r = pv;
    for (int k = 0; k < upto; ++k) {
      const double qk = Q != nullptr ? qv : (x == (long long)s_rej[k] ? 1.0 : 0.0);
      const double s = s_norm[k];
      r = s > 0.0 ? fmax(r - qk, 0.0) / s : pv;
    }
    return r;
  };
  // weight of an entry in a pass: the last rejection's subtraction is not normalised yet
  auto weight = [&](double pv, double qv, long long x, bool open) -> double {
    if (!open) return level(pv, qv, x, levels);
    const double qk = Q != nullptr ? qv : (x == (long long)s_rej[levels - 1] ? 1.0 : 0.0);
    return fmax(level(pv, qv, x, levels - 1) - qk, 0.0);
  };

  int cur = 0;
  int pass = 0;
  const long long wslot = (long long)rank * VF_WARPS + warp, wslots = (long long)CS * VF_WARPS;
  // One pass over the current node's row: every warp sums a stretch of its own, the sums of all CTAs end up in s_all.
  // Vectors are aligned in memory, so the row's first one may begin inside the row before it.
  auto row_total = [&](bool open) -> double {
    const long long row = ((long long)b * a.T + cur) * a.V;
    const long long v0 = row / N, v1 = (row + a.V + N - 1) / N;
    const long long per = (v1 - v0 + wslots - 1) / wslots;
    const long long lo = v0 + wslot * per, hi = min(lo + per, v1);
    const bool need_q = Q != nullptr && levels > 0;
    double sum = 0.0;
#pragma unroll 4
    for (long long v = lo + lane; v < hi; v += 32) {
      const VfVec<T> pv = vf_load(P, v * N, a.total);
      VfVec<T> qv = pv;
      if (need_q) qv = vf_load(Q, v * N, a.total);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const long long x = v * N + i - row;
        if (x >= 0 && x < a.V) sum += weight((double)ptenc_to_float(pv.e[i]), (double)ptenc_to_float(qv.e[i]), x, open);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    __syncthreads();                                              // the pass before is done with s_warp and s_all
    if (lane == 0) s_warp[warp] = sum;
    __syncthreads();
    if (tid == 0) {
      double t = 0.0;
      for (int w = 0; w < VF_WARPS; ++w) t += s_warp[w];
      s_cta[pass & 1] = t;
    }
    cluster.sync();
    if (tid < CS) s_all[tid] = *cluster.map_shared_rank(&s_cta[pass & 1], tid);
    __syncthreads();
    ++pass;
    double t = 0.0;
    for (int c = 0; c < CS; ++c) t += s_all[c];
    return t;
  };

  // ---- the walk: every thread of the cluster takes the same one --------------------------------------------------------
  int len = 1;
  bool open = false;                                              // a rejection whose sum has not been formed
  if (tid == 0) s_path[0] = 0;
  for (int i = 1; i < n; ++i) {
    if (s_par[i] != cur) continue;
    if (open) {
      const double t = row_total(true);
      if (tid == 0) s_norm[levels - 1] = t;
      __syncthreads();
      open = false;
    }
    const double r = level(s_pv[i], s_qv[i], s_tok[i], levels);
    if (s_u[i] * s_qv[i] < r) {
      if (tid == 0) s_path[len] = i;
      ++len;
      cur = i;
      levels = 0;
    } else {
      __syncthreads();
      if (tid == 0) s_rej[levels] = s_tok[i];
      __syncthreads();
      ++levels;
      open = true;
    }
  }
  // ---- the draw ------------------------------------------------------------------------------------------------------------
  double total = row_total(open);
  if (open && !(total > 0.0)) {                                   // nothing left of r: the target's own row
    levels = 0;
    open = false;
    total = row_total(false);
  }
  const double border = s_u[0] * total;
  if (rank == 0) {
    for (int i = tid; i < a.T; i += VF_THREADS) a.path[(size_t)b * a.T + i] = i < len ? s_path[i] : -1;
    if (tid == 0) {
      a.n_path[b] = len;
      if (!(total > 0.0)) a.next[b] = -1;
    }
  }
  if (total > 0.0) {
    // the CTA and the warp whose stretch holds the border; the last one with any weight if rounding puts it past the end
    int owner = -1, last = 0;
    double before = 0.0, cum = 0.0, before_last = 0.0;
    for (int c = 0; c < CS; ++c) {
      if (s_all[c] > 0.0) { last = c; before_last = cum; }
      if (owner < 0 && cum + s_all[c] > border) { owner = c; before = cum; }
      cum += s_all[c];
    }
    if (owner < 0) { owner = last; before = before_last; }
    if (owner == rank) {
      int mine = -1;
      last = 0;
      cum = before_last = before;
      for (int w = 0; w < VF_WARPS; ++w) {
        if (s_warp[w] > 0.0) { last = w; before_last = cum; }
        if (mine < 0 && cum + s_warp[w] > border) { mine = w; before = cum; }
        cum += s_warp[w];
      }
      if (mine < 0) { mine = last; before = before_last; }
      if (mine == warp) {
        const long long row = ((long long)b * a.T + cur) * a.V;
        const long long v0 = row / N, v1 = (row + a.V + N - 1) / N;
        const long long per = (v1 - v0 + wslots - 1) / wslots;
        const long long lo = v0 + wslot * per, hi = min(lo + per, v1);
        const bool need_q = Q != nullptr && levels > 0;
        long long found = -1, tail = -1;                          // tail: the last entry with any weight so far
        for (long long vb = lo; vb < hi && found < 0; vb += 32) {
          const long long v = vb + lane;
          double w[N], sum = 0.0;
          long long my_tail = -1;
          VfVec<T> pv, qv;
          if (v < hi) {
            pv = vf_load(P, v * N, a.total);
            qv = pv;
            if (need_q) qv = vf_load(Q, v * N, a.total);
          }
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const long long x = v * N + i - row;
            w[i] = 0.0;
            if (v < hi && x >= 0 && x < a.V)
              w[i] = weight((double)ptenc_to_float(pv.e[i]), (double)ptenc_to_float(qv.e[i]), x, open);
            if (w[i] > 0.0) my_tail = x;
            sum += w[i];
          }
          double inc = sum;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const double t = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += t;
          }
          double c = before + (inc - sum);
          long long x_hit = -1;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            c += w[i];
            if (x_hit < 0 && w[i] > 0.0 && c > border) x_hit = v * N + i - row;
          }
          const unsigned hit = __ballot_sync(0xffffffffu, x_hit >= 0);
          if (hit != 0) found = __shfl_sync(0xffffffffu, x_hit, __ffs(hit) - 1);
          const unsigned some = __ballot_sync(0xffffffffu, my_tail >= 0);
          if (some != 0) tail = __shfl_sync(0xffffffffu, my_tail, 31 - __clz(some));
          before += __shfl_sync(0xffffffffu, inc, 31);
        }
        if (lane == 0) a.next[b] = (int32_t)(found >= 0 ? found : tail);
      }
    }
  }
  cluster.sync();                                                 // nobody leaves while its sum may still be read
}

template <typename T>
cudaError_t launch_verify_t(const VerifyArgs& a, int batch, cudaStream_t st) {
  // A CTA's share of a row should be worth its start: at least 4096 entries, eight CTAs at most.
  int cs = 1;
  while (cs < VF_CLUSTER && a.V >= 8192ll * cs) cs *= 2;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3((unsigned)batch * cs);
  cfg.blockDim = dim3(VF_THREADS);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cs;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, k_verify_tree<T>, a);
  return e != cudaSuccess ? e : cudaGetLastError();
}

inline bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
inline bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; }

}  // namespace

extern "C" int ptenc_verify_tree(const void* p, const void* q, int dtype, const int32_t* tokens, const int32_t* parent,
                                 const int32_t* n_nodes, const float* u, const uint8_t* active, int32_t batch,
                                 int32_t max_nodes, int32_t vocab, int32_t* path, int32_t* n_path, int32_t* next_token,
                                 void* stream) {
  if (p == nullptr || tokens == nullptr || parent == nullptr || u == nullptr || path == nullptr || n_path == nullptr ||
      next_token == nullptr)
    return PTENC_EINVAL;
  if (dtype != PTENC_DTYPE_FP32 && dtype != PTENC_DTYPE_BF16) return PTENC_EINVAL;
  if (batch < 1 || max_nodes < 1 || vocab < 1) return PTENC_EINVAL;
  if (max_nodes > PTENC_MAX_TREE || batch > (1 << 24)) return PTENC_ESHAPE;
  if (off16(p) || off16(q) || off4(tokens) || off4(parent) || off4(n_nodes) || off4(u) || off4(path) || off4(n_path) ||
      off4(next_token))
    return PTENC_EALIGN;
  VerifyArgs a;
  a.p = p; a.q = q; a.tokens = tokens; a.parent = parent; a.n_nodes = n_nodes; a.u = u; a.active = active;
  a.T = max_nodes; a.V = vocab; a.total = (long long)batch * max_nodes * vocab;
  a.path = path; a.n_path = n_path; a.next = next_token;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == PTENC_DTYPE_FP32 ? launch_verify_t<float>(a, batch, st)
                                                  : launch_verify_t<__nv_bfloat16>(a, batch, st);
  return e == cudaSuccess ? PTENC_OK : PTENC_ECUDA;
}

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
// and then, per rejection, one row of p and q (of p alone at a node without a rejection); the repeats at a node come from
// the caches.  A row is spread over a cluster of CTAs, a stretch per warp; the draw finds the CTA, the warp and the vector
// that hold the border from the sums of the last pass, so it re-reads one warp's stretch, a vector per thread.
//
// Arithmetic: with c_0 = 1 and q >= 0, k rejections of the same row leave r = w / c_k with
//   w = max(p - C q, 0),  C = c_0 + .. + c_(k-1),  c_k = sum of w
// (max(max(a - b, 0) - c, 0) = max(a - b - c, 0)), so a pass costs one multiply-add per entry however many siblings have
// been rejected, and no division.  w, its sums and the border of the draw are held in 64 bits: neighbouring borders of a
// row of 10^5 entries are about as close as a 32-bit sum of them is wrong, so a 32-bit cumulative sum would draw another
// token now and then.
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
// Vector v of a row whose storage starts at `base` (16-byte aligned, up to N - 1 entries before the row's first); `room`
// entries of the tensor lie from there on.
template <typename T>
__device__ __forceinline__ VfVec<T> vf_load(const T* base, int v, long long room) {
  constexpr int N = VfVec<T>::N;
  VfVec<T> x;
  const long long at = (long long)v * N;
  if (at + N <= room) {
    *reinterpret_cast<uint4*>(x.e) = __ldg(reinterpret_cast<const uint4*>(base) + v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x.e[i] = at + i < room ? base[at + i] : ptenc_from_float<T>(0.f);
  }
  return x;
}
// Inclusive sums over the lanes of a warp.
__device__ __forceinline__ double vf_scan(double x, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double t = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += t;
  }
  return x;
}

template <typename T>
__global__ void __launch_bounds__(VF_THREADS, 2)
k_verify_tree(const VerifyArgs a) {
  constexpr int N = VfVec<T>::N;
  cg::cluster_group cluster = cg::this_cluster();
  const int CS = (int)cluster.num_blocks();
  const int rank = (int)cluster.block_rank();
  const int b = blockIdx.x / CS;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  __shared__ int s_par[TREE_MAX], s_tok[TREE_MAX];
  __shared__ double s_pv[TREE_MAX], s_qv[TREE_MAX];
  __shared__ float s_u[TREE_MAX];
  __shared__ int s_rej[TREE_MAX];                  // certain drafts: tokens rejected at the current node,
  __shared__ double s_left[TREE_MAX];              // and what is left of their entries
  __shared__ double s_warp[VF_WARPS];
  __shared__ double s_cta[2];                      // this CTA's sum, read by the other CTAs; passes alternate
  __shared__ double s_all[VF_CLUSTER];
  __shared__ int s_hit, s_tail;

  if (a.active != nullptr && a.active[b] == 0) return;            // the whole cluster
  const T* P = static_cast<const T*>(a.p);
  const T* Q = static_cast<const T*>(a.q);
  const int n = a.n_nodes != nullptr ? a.n_nodes[b] : a.T;
  int bad = 0;
  if (tid < a.T) {
    const size_t at = (size_t)b * a.T + tid;
    const int par = a.parent[at], tok = a.tokens[at];
    s_u[tid] = a.u[at];
    s_par[tid] = par;
    s_tok[tid] = tok;
    if (tid < n) {
      bad = tid == 0 ? par != -1 : (par < 0 || par >= tid || tok < 0 || tok >= a.V);
      if (!bad && tid > 0) {
        const long long x = ((long long)b * a.T + par) * a.V + tok;
        const T pv = P[x], qv = Q != nullptr ? Q[x] : ptenc_from_float<T>(1.f);
        s_pv[tid] = (double)ptenc_to_float(pv);
        s_qv[tid] = (double)ptenc_to_float(qv);
      }
    }
  }
  bad |= n < 1 || n > a.T;
  if (__syncthreads_or(bad)) {                                    // the same verdict in every CTA of the cluster
    if (rank == 0) {
      for (int i = tid; i < a.T; i += VF_THREADS) a.path[(size_t)b * a.T + i] = -1;
      if (tid == 0) { a.n_path[b] = 0; a.next[b] = -1; }
    }
    return;
  }

  // ---- a pass over the current node's row: weights max(p - C q, 0), a stretch of vectors per warp -----------------------
  const int V = (int)a.V;
  int cur = 0, pass = 0, nrej = 0;
  double C = 0.0;
  const T *pr = nullptr, *qr = nullptr;
  int off = 0, nv = 0, per = 0;
  long long room = 0;
  auto take_row = [&]() {
    const long long row = ((long long)b * a.T + cur) * a.V;
    off = (int)(row % N);                                         // entries of the first vector that belong to the row before
    pr = P + (row - off);
    qr = Q != nullptr ? Q + (row - off) : nullptr;
    room = a.total - (row - off);
    nv = (off + V + N - 1) / N;
    per = (nv + CS * VF_WARPS - 1) / (CS * VF_WARPS);
  };
  // weights of vector v; x0: index of its first entry in the row
  auto weigh = [&](const VfVec<T>& pv, const VfVec<T>& qv, int v, double (&w)[N]) {
    const int x0 = v * N - off;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = (double)ptenc_to_float(pv.e[i]);
    if (C != 0.0) {
      if (Q != nullptr) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const double d = fma(-C, (double)ptenc_to_float(qv.e[i]), w[i]);
          w[i] = d > 0.0 ? d : 0.0;
        }
      } else {
        for (int k = 0; k < nrej; ++k) {
          const int at = s_rej[k] - x0;
#pragma unroll
          for (int i = 0; i < N; ++i) if (at == i) w[i] = s_left[k];
        }
      }
    }
    if (x0 < 0 || x0 + N > V) {
#pragma unroll
      for (int i = 0; i < N; ++i) if (x0 + i < 0 || x0 + i >= V) w[i] = 0.0;
    }
  };
  auto row_total = [&]() -> double {
    const int lo = (rank * VF_WARPS + warp) * per, hi = min(lo + per, nv);
    const bool need_q = Q != nullptr && C != 0.0;
    double sum = 0.0;
    constexpr int U = N == 4 ? 4 : 2;                             // vectors of p and of q in flight per lane: what 64 registers hold
    for (int v0 = lo + lane; v0 < hi; v0 += 32 * U) {
      VfVec<T> pv[U], qv[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int v = min(v0 + 32 * j, hi - 1);
        pv[j] = vf_load(pr, v, room);
        qv[j] = pv[j];
        if (need_q) qv[j] = vf_load(qr, v, room);
      }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (v0 + 32 * j < hi) {
          double w[N];
          weigh(pv[j], qv[j], v0 + 32 * j, w);
#pragma unroll
          for (int i = 0; i < N; ++i) sum += w[i];
        }
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    __syncthreads();                                              // the pass before is done with s_warp and s_all
    if (lane == 0) s_warp[warp] = sum;
    __syncthreads();
    if (warp == 0) {
      double t = lane < VF_WARPS ? s_warp[lane] : 0.0;
#pragma unroll
      for (int o = VF_WARPS / 2; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
      if (lane == 0) s_cta[pass & 1] = t;
    }
    if (CS > 1) {
      cluster.sync();
      if (tid < CS) s_all[tid] = *cluster.map_shared_rank(&s_cta[pass & 1], tid);
    } else if (tid == 0) {
      s_all[0] = s_cta[pass & 1];
    }
    __syncthreads();
    ++pass;
    double t = 0.0;
    for (int c = 0; c < CS; ++c) t += s_all[c];
    return t;
  };

  // ---- the walk: every warp of the cluster takes the same one ------------------------------------------------------------
  const int par0 = lane < n ? s_par[lane] : -2, par1 = lane + 32 < n ? s_par[lane + 32] : -2;
  unsigned long long line = 1ull;                                 // the path's nodes; they come in rising order
  double c = 1.0;                                                 // r = w / c
  bool moved = true, summed = false;
  while (moved) {
    moved = false;
    summed = false;
    C = 0.0;
    c = 1.0;
    nrej = 0;
    unsigned long long kids = (unsigned long long)__ballot_sync(0xffffffffu, par0 == cur) |
                              (unsigned long long)__ballot_sync(0xffffffffu, par1 == cur) << 32;
    for (; kids != 0 && !moved; kids &= kids - 1) {
      const int i = __ffsll((long long)kids) - 1;
      double w = s_pv[i];
      int same = -1;                                              // certain drafts: the token was rejected before, as entry `same`
      if (Q != nullptr) {
        w = fmax(fma(-C, s_qv[i], w), 0.0);
      } else {
        for (int k = 0; k < nrej; ++k) if (s_rej[k] == s_tok[i]) { same = k; w = s_left[k]; }
      }
      if ((double)s_u[i] * s_qv[i] < w / c) {
        line |= 1ull << i;
        cur = i;
        moved = true;
        break;
      }
      take_row();
      C += c;
      if (Q == nullptr) {
        __syncthreads();
        if (tid == 0) {
          const int k = same >= 0 ? same : nrej;
          s_rej[k] = s_tok[i];
          s_left[k] = fmax(w - c, 0.0);
        }
        if (same < 0) ++nrej;
        __syncthreads();
      }
      c = row_total();
      summed = c > 0.0;
      if (!summed) { C = 0.0; c = 1.0; nrej = 0; }                // nothing left: the target's own row
    }
  }
  // ---- the draw ------------------------------------------------------------------------------------------------------------
  if (!summed) {
    take_row();
    c = row_total();
  }
  const double border = (double)s_u[0] * c;
  const int len = __popcll(line);
  if (rank == 0) {
    if (tid < a.T) {
      a.path[(size_t)b * a.T + tid] = -1;
    }
    __syncthreads();
    if (tid < a.T && ((line >> tid) & 1ull)) a.path[(size_t)b * a.T + __popcll(line & ((1ull << tid) - 1))] = tid;
    if (tid == 0) {
      a.n_path[b] = len;
      if (!(c > 0.0)) a.next[b] = -1;
    }
  }
  if (c > 0.0) {
    // the CTA and the warp whose stretch holds the border; the last one with any weight if rounding puts it past the end
    auto holder = [&](double x, double start, double* before) -> int {
      const double inc = start + vf_scan(x, lane);
      unsigned m = __ballot_sync(0xffffffffu, x > 0.0 && inc > border);
      const unsigned some = __ballot_sync(0xffffffffu, x > 0.0);
      const int at = m != 0 ? __ffs(m) - 1 : 31 - __clz(some);
      *before = __shfl_sync(0xffffffffu, inc - x, at);
      return at;
    };
    double before;
    const int owner = holder(lane < CS ? s_all[lane] : 0.0, 0.0, &before);
    if (owner == rank) {
      const int mine = holder(lane < VF_WARPS ? s_warp[lane] : 0.0, before, &before);
      const int lo = (rank * VF_WARPS + mine) * per, hi = min(lo + per, nv);
      const bool need_q = Q != nullptr && C != 0.0;
      if (tid == 0) { s_hit = 0x7fffffff; s_tail = -1; }
      __syncthreads();                                            // s_warp is free too
      for (int vb = lo; vb < hi; vb += VF_THREADS) {
        const int v = vb + tid;
        double w[N], sum = 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = 0.0;
        if (v < hi) {
          const VfVec<T> pv = vf_load(pr, v, room);
          VfVec<T> qv = pv;
          if (need_q) qv = vf_load(qr, v, room);
          weigh(pv, qv, v, w);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) sum += w[i];
        const double inc = vf_scan(sum, lane);
        if (lane == 31) s_warp[warp] = inc;
        __syncthreads();
        const double wsum = vf_scan(lane < VF_WARPS ? s_warp[lane] : 0.0, lane);
        double at = before + (inc - sum);
        const double prev = __shfl_sync(0xffffffffu, wsum, warp > 0 ? warp - 1 : 0);
        if (warp > 0) at += prev;
        int hit = 0x7fffffff, tail = -1;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          at += w[i];
          if (w[i] > 0.0) {
            tail = v * N + i - off;
            if (at > border && hit == 0x7fffffff) hit = tail;
          }
        }
        hit = __reduce_min_sync(0xffffffffu, hit);
        tail = __reduce_max_sync(0xffffffffu, tail);
        if (lane == 0) {
          if (hit != 0x7fffffff) atomicMin(&s_hit, hit);
          if (tail >= 0) atomicMax(&s_tail, tail);
        }
        before += __shfl_sync(0xffffffffu, wsum, 31);
        __syncthreads();
        if (s_hit != 0x7fffffff) break;                           // uniform: nobody writes it before the next barrier
      }
      if (tid == 0) a.next[b] = s_hit != 0x7fffffff ? s_hit : s_tail;
    }
  }
  if (CS > 1) cluster.sync();                                     // nobody leaves while its sum may still be read
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
  if (max_nodes > PTENC_MAX_TREE || batch > (1 << 24) || vocab > (1 << 28)) return PTENC_ESHAPE;
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

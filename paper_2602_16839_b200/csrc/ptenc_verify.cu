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
// the caches.  A row is spread over a cluster of CTAs, a stretch per warp.  Every warp stores its sum into the shared memory
// of all the cluster's CTAs, so that behind one cluster barrier each CTA has all sums and finds the total, the warp and
// (re-reading that warp's stretch, a vector per thread) the entry that hold the border.  The code is kept short: a launch
// starts from cold instruction memory, and a pass unrolled for throughput cost 5 us in a call for one sequence.
//
// Arithmetic: with c_0 = 1 and q >= 0, k rejections of the same row leave r = w / c_k with
//   w = max(p - C q, 0),  C = c_0 + .. + c_(k-1),  c_k = sum of w
// (max(max(a - b, 0) - c, 0) = max(a - b - c, 0)), so a pass costs one multiply-add per entry however many siblings have
// been rejected, and no division.  w, its sums and the border of the draw are held in 64 bits: neighbouring borders of a
// row of 10^5 entries are about as close as a 32-bit sum of them is wrong, so a 32-bit cumulative sum would draw another
// token now and then.
//
// Measured: one sequence of 5 nodes and 32000 entries 6 us; 128 sequences, 152000 fp32 entries, at least 156 MB of rows: 53 us,
// 2.9 TB/s.  The bound is the passes' arithmetic in 64 bits and their barriers (issue slots 36 % busy, DRAM 27 %): a row that
// is read again for the next sibling comes from L2.  Certain drafts need one pass per node: 8.6 us where reading the row for
// every rejection took 22.
#include <cooperative_groups.h>
#include <string.h>

#include "ptenc_tree.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int VF_THREADS = 256;
constexpr int VF_WARPS = VF_THREADS / 32;
constexpr int VF_CLUSTER = 8;
constexpr int VF_DEPTH = 4;          // vectors of p and of q that a thread keeps in flight
constexpr int VF_SMEM = VF_DEPTH * 2 * VF_THREADS * 16;

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
__device__ __forceinline__ void vf_async(uint4* dst, const void* src, int bytes) {        // the rest of the 16 bytes reads as zero
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
               ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(dst))), "l"(src), "r"(bytes) : "memory");
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

// QROWS: the draft's rows are given; otherwise the drafted tokens were certain.
template <typename T, bool QROWS>
__global__ void __launch_bounds__(VF_THREADS, 4)
k_verify_tree(const VerifyArgs a) {
  constexpr int N = VfVec<T>::N;
  cg::cluster_group cluster = cg::this_cluster();
  const int CS = (int)cluster.num_blocks();
  const int rank = (int)cluster.block_rank();
  const int b = blockIdx.x / CS;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  extern __shared__ __align__(16) uint4 s_ring[];  // [VF_DEPTH][p, q][VF_THREADS]
  __shared__ int s_par[TREE_MAX], s_tok[TREE_MAX];
  __shared__ double s_pv[TREE_MAX], s_qv[TREE_MAX];
  __shared__ float s_u[TREE_MAX];
  __shared__ int s_rej[TREE_MAX];                  // certain drafts: tokens rejected at the current node,
  __shared__ double s_left[TREE_MAX];              // and what is left of their entries
  __shared__ double s_sum[2][VF_CLUSTER * VF_WARPS];              // the warps' sums of a pass; passes alternate
  __shared__ double s_raw[VF_CLUSTER * VF_WARPS];  // certain drafts: the warps' sums of the row as it is
  __shared__ double s_warp[VF_WARPS];
  __shared__ int s_hit, s_tail;

  tree_after_previous();
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
        const T pv = P[x], qv = QROWS ? Q[x] : ptenc_from_float<T>(1.f);
        s_pv[tid] = (double)ptenc_to_float(pv);
        s_qv[tid] = (double)ptenc_to_float(qv);
      }
    }
  }
  for (int i = tid; i < 2 * VF_CLUSTER * VF_WARPS; i += VF_THREADS) (&s_sum[0][0])[i] = 0.0;
  bad |= n < 1 || n > a.T;
  bad = __syncthreads_or(bad);                                    // the same verdict in every CTA of the cluster
  if (CS > 1) cluster.sync();                                     // all CTAs run and their sums are clear before any is stored
  if (bad) {
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
    if (QROWS) qr = Q + (row - off);
    room = a.total - (row - off);
    nv = (off + V + N - 1) / N;
    per = (nv + CS * VF_WARPS - 1) / (CS * VF_WARPS);
  };
  // weights of vector v
  auto weigh = [&](const VfVec<T>& pv, const VfVec<T>& qv, int v, double (&w)[N]) {
    const int x0 = v * N - off;                                   // index of its first entry in the row
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = (double)ptenc_to_float(pv.e[i]);
    if (QROWS) {
      if (C != 0.0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const double d = fma(-C, (double)ptenc_to_float(qv.e[i]), w[i]);
          w[i] = d > 0.0 ? d : 0.0;
        }
      }
    } else {
#pragma unroll 1
      for (int k = 0; k < nrej; ++k) {
        const int at = s_rej[k] - x0;
#pragma unroll
        for (int i = 0; i < N; ++i) if (at == i) w[i] = s_left[k];
      }
    }
    if (x0 < 0 || x0 + N > V) {
#pragma unroll
      for (int i = 0; i < N; ++i) if (x0 + i < 0 || x0 + i >= V) w[i] = 0.0;
    }
  };
  auto row_total = [&]() -> double {
    const int lo = (rank * VF_WARPS + warp) * per, hi = min(lo + per, nv);
    const bool need_q = QROWS && C != 0.0;
    double sum = 0.0;
    // Every thread keeps VF_DEPTH vectors of its own on their way through shared memory: with two or three in registers a row
    // alone on the machine took 9 us a pass.
    auto fetch = [&](int v, int slot) {
      if (v < hi) {
        const int bytes = (int)min(16ll, (room - (long long)v * N) * (long long)sizeof(T));
        vf_async(s_ring + slot * 2 * VF_THREADS + tid, pr + (size_t)v * N, bytes);
        if (need_q) vf_async(s_ring + (slot * 2 + 1) * VF_THREADS + tid, qr + (size_t)v * N, bytes);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // this lane's next vector that holds a rejected token of a certain draft
    auto next_rejected = [&](int from) -> int {
      int best = 0x7fffffff;
      for (int k = 0; k < nrej; ++k) {
        const int v = (s_rej[k] + off) / N;
        if (v >= from && v < best && ((v - lo) & 31) == lane) best = v;
      }
      return best;
    };
    int rejected = QROWS ? 0x7fffffff : next_rejected(lo);
#pragma unroll 1
    for (int k = 0; k < VF_DEPTH; ++k) fetch(lo + lane + 32 * k, k);
    int slot = 0;
#pragma unroll 1
    for (int v = lo + lane; v < hi; v += 32) {
      asm volatile("cp.async.wait_group %0;" ::"n"(VF_DEPTH - 1) : "memory");
      VfVec<T> p0, q0;
      *reinterpret_cast<uint4*>(p0.e) = s_ring[slot * 2 * VF_THREADS + tid];
      q0 = p0;
      if (need_q) *reinterpret_cast<uint4*>(q0.e) = s_ring[(slot * 2 + 1) * VF_THREADS + tid];
      fetch(v + 32 * VF_DEPTH, slot);
      slot = slot + 1 == VF_DEPTH ? 0 : slot + 1;
      if (v == 0 || v == nv - 1 || v == rejected) {               // the ends of the row, entries to replace
        double w[N];
        weigh(p0, q0, v, w);
#pragma unroll
        for (int i = 0; i < N; ++i) sum += w[i];
        if (!QROWS && v == rejected) rejected = next_rejected(v + 1);
      } else if (need_q) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const double d = fma(-C, (double)ptenc_to_float(q0.e[i]), (double)ptenc_to_float(p0.e[i]));
          if (__double2hiint(d) >= 0) sum += d;                   // max(d, 0) joins the sum
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) sum += (double)ptenc_to_float(p0.e[i]);
      }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    double* to = &s_sum[pass & 1][rank * VF_WARPS + warp];
    if (CS > 1) {
      if (lane < CS) *cluster.map_shared_rank(to, lane) = sum;
      cluster.sync();
    } else {
      if (lane == 0) *to = sum;
      __syncthreads();
    }
    const double* all = s_sum[pass & 1];
    ++pass;
    double t = 0.0;                                               // every lane adds the same four warps' sums everywhere
#pragma unroll
    for (int i = 0; i < VF_CLUSTER * VF_WARPS / 32; ++i) t += all[lane * (VF_CLUSTER * VF_WARPS / 32) + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    return t;
  };

  // ---- the walk: every warp of the cluster takes the same one ------------------------------------------------------------
  const int par0 = lane < n ? s_par[lane] : -2, par1 = lane + 32 < n ? s_par[lane + 32] : -2;
  unsigned long long line = 1ull;                                 // the path's nodes; they come in rising order
  double c = 1.0;                                                 // r = w / c
  double raw = 0.0, mass = 0.0;                                   // certain drafts: sums of the row as it is, and of w
  bool summed = false, stale = false;                             // stale: some warp's sum is to be taken again before the draw
  unsigned long long kids = 0;
  auto children = [&]() {
    kids = (unsigned long long)__ballot_sync(0xffffffffu, par0 == cur) |
           (unsigned long long)__ballot_sync(0xffffffffu, par1 == cur) << 32;
  };
  children();
  // one step: the next child is judged, or there is none left and the last pass is made
#pragma unroll 1
  while (true) {
    if (kids != 0) {
      const int i = __ffsll((long long)kids) - 1;
      kids &= kids - 1;
      double w = s_pv[i];
      int same = -1;                                              // certain drafts: the token was rejected before, as entry `same`
      if (QROWS) {
        w = fmax(fma(-C, s_qv[i], w), 0.0);
      } else {
        for (int k = 0; k < nrej; ++k) if (s_rej[k] == s_tok[i]) { same = k; w = s_left[k]; }
      }
      if ((double)s_u[i] * s_qv[i] < w / c) {
        line |= 1ull << i;
        cur = i;
        C = raw = 0.0;
        c = 1.0;
        nrej = 0;
        summed = stale = false;
        children();
        continue;
      }
      C += c;
      if (!QROWS) {
        // A certain draft changes one entry, so the sums follow from those of the row as it is, as long as what is left is
        // no small part of it (1e-3 leaves thirteen digits); otherwise the row is summed again without the entries.  The same
        // holds of the sum of the warp that had the entry, which only the draw looks at: where little is left of it, down
        // to a residue of the rounding or nothing beside entries that were too small to count, the row is summed once more before
        // the draw.
        if (raw == 0.0) {
          take_row();
          raw = mass = row_total();
          if (tid < VF_CLUSTER * VF_WARPS) s_raw[tid] = s_sum[(pass - 1) & 1][tid];
        }
        const double left = fmax(w - c, 0.0);
        __syncthreads();
        if (tid == 0) {
          const int k = same >= 0 ? same : nrej;
          s_rej[k] = s_tok[i];
          s_left[k] = left;
        }
        if (same < 0) ++nrej;
        mass -= w - left;
        if (mass > 1e-3 * raw) {
          const int at = (s_tok[i] + off) / N / per;
          if (tid == 0) s_sum[(pass - 1) & 1][at] -= w - left;
          c = mass;
          summed = true;
          __syncthreads();
          stale |= w > left && !(s_sum[(pass - 1) & 1][at] > 1e-3 * s_raw[at]);
          continue;
        }
        __syncthreads();
      }
    } else if (summed && !stale) {
      break;
    }
    stale = false;
    const bool last = kids == 0 && C == 0.0;                      // no rejection to account for: the row as it is, for the draw
    take_row();
    c = mass = row_total();
    summed = true;
    if (last) break;
    if (!(c > 0.0)) { C = raw = 0.0; c = 1.0; nrej = 0; summed = false; } // nothing left: the target's own row
  }
  // ---- the draw ------------------------------------------------------------------------------------------------------------
  const double border = (double)s_u[0] * c;
  if (rank == 0 && tid < a.T) {
    const int len = __popcll(line);
    // the path, node by node, and -1 behind it
    int node = -1;
    if (tid < len) {
      unsigned long long m = line;
      for (int k = 0; k < tid; ++k) m &= m - 1;
      node = __ffsll((long long)m) - 1;
    }
    a.path[(size_t)b * a.T + tid] = node;
    if (tid == 0) {
      a.n_path[b] = len;
      if (!(c > 0.0)) a.next[b] = -1;
    }
  }
  if (c > 0.0) {
    // the warp whose stretch holds the border; the last one with any weight if rounding puts it past the end
    constexpr int PL = VF_CLUSTER * VF_WARPS / 32;
    const double* all = s_sum[(pass - 1) & 1];
    double x[PL], mine = 0.0;
#pragma unroll
    for (int i = 0; i < PL; ++i) { x[i] = all[lane * PL + i]; mine += x[i]; }
    double at = vf_scan(mine, lane) - mine;
    int hit = 0x7fffffff, tail = -1;
    double before_hit = 0.0, before_tail = 0.0;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      if (x[i] > 0.0) {
        tail = lane * PL + i;
        before_tail = at;
        if (hit == 0x7fffffff && at + x[i] > border) { hit = tail; before_hit = at; }
      }
      at += x[i];
    }
    const int h = __reduce_min_sync(0xffffffffu, hit), tl = __reduce_max_sync(0xffffffffu, tail);
    const int holder = h != 0x7fffffff ? h : tl;
    double before = __shfl_sync(0xffffffffu, h != 0x7fffffff ? before_hit : before_tail, holder / PL);
    if (holder < 0) {                                             // only with sums that are no numbers
      if (rank == 0 && tid == 0) a.next[b] = -1;
    } else if (holder / VF_WARPS == rank) {
      const int lo = holder * per, hi = min(lo + per, nv);
      const bool need_q = QROWS && C != 0.0;
      if (tid == 0) { s_hit = 0x7fffffff; s_tail = -1; }
      __syncthreads();
#pragma unroll 1
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
        double pos = before + (inc - sum);
        const double prev = __shfl_sync(0xffffffffu, wsum, warp > 0 ? warp - 1 : 0);
        if (warp > 0) pos += prev;
        int first = 0x7fffffff, some = -1;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          pos += w[i];
          if (w[i] > 0.0) {
            some = v * N + i - off;
            if (pos > border && first == 0x7fffffff) first = some;
          }
        }
        first = __reduce_min_sync(0xffffffffu, first);
        some = __reduce_max_sync(0xffffffffu, some);
        if (lane == 0) {
          if (first != 0x7fffffff) atomicMin(&s_hit, first);
          if (some >= 0) atomicMax(&s_tail, some);
        }
        before += __shfl_sync(0xffffffffu, wsum, 31);
        __syncthreads();
        if (s_hit != 0x7fffffff) break;                           // uniform: nobody writes it before the next barrier
      }
      if (tid == 0) a.next[b] = s_hit != 0x7fffffff ? s_hit : s_tail;
    }
  }
}

template <typename T>
cudaError_t launch_verify_t(const VerifyArgs& a, int batch, int dev, int sms, cudaStream_t st) {
  // A row over up to eight CTAs: a CTA's share should be worth its start, 2048 entries at least, and the batch should not
  // need more than two rounds of the four CTAs that an SM holds (64 registers x 256 threads).  128 rows of 152000 entries: 53 us
  // with eight CTAs each (1.7 rounds), 65 us with four.  The rule steps at whole rounds: 149 sequences on 148 SMs get four CTAs
  // each, which is one round and four CTAs.
  int cs = 1;
  while (cs < VF_CLUSTER && a.V >= 4096ll * cs && (long long)batch * cs * 2 <= 8 * sms) cs *= 2;
  static PtencOnce once;
  const cudaError_t e = ptenc_first_use(once, dev, [] {
    const cudaError_t err = ptenc_allow_smem(k_verify_tree<T, true>, VF_SMEM);
    return err != cudaSuccess ? err : ptenc_allow_smem(k_verify_tree<T, false>, VF_SMEM);
  });
  if (e != cudaSuccess) return e;
  return tree_launch(a.q != nullptr ? k_verify_tree<T, true> : k_verify_tree<T, false>, dim3((unsigned)batch * cs), VF_THREADS,
                     VF_SMEM, cs, st, a);
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
  ptenc_drop_old_error();
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int dev = -1, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return PTENC_ECUDA;
  const cudaError_t e = dtype == PTENC_DTYPE_FP32 ? launch_verify_t<float>(a, batch, dev, sms, st)
                                                  : launch_verify_t<__nv_bfloat16>(a, batch, dev, sms, st);
  return e == cudaSuccess ? PTENC_OK : PTENC_ECUDA;
}

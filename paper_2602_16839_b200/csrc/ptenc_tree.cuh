// What the kernels of the speculative step share: the description of a draft tree, and which tokens a node sees.
//
// A sequence's draft is a tree of n <= 64 nodes in topological order (parent[i] < i, -1 for a root).  Node i stands for
// the sequence after the tokens on its path (its ancestors and itself) have been appended one by one.  Appending m
// tokens to a ring that holds c of C sliding tokens evicts, oldest first and e = min(E, C) at a time,
//   ev(m) = e * ceil(max(0, c + m - C) / e)
// tokens (a full ring makes room before each arrival).  Numbering tokens by arrival -- cache tokens 0..c-1, the path's
// token at depth d is c + d -- node i at depth d_i therefore sees the pinned entries and every token on its path or in
// the ring whose number is at least ev(d_i + 1): exactly what a token-by-token decode step would see there.
#pragma once

#include <string.h>

#include "ptenc_internal.h"

constexpr int TREE_MAX = PTENC_MAX_TREE;

// The calls of a speculative step take a few microseconds each, about as long as a launch, so their kernels are launched ahead
// of the end of the one in front of them on the stream (programmatic dependent launch): every thread waits here, in front of
// its first access to memory, until that kernel has completed.  From Python, back to back: one chain's attention 16.4 -> 13.5
// us, one layer's commit 10.3 -> 7.9.
__device__ __forceinline__ void tree_after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Lets the next kernel become resident before this one ends: for kernels with one CTA per SM and their joins.  Where several
// CTAs share an SM the next kernel's would crowd on the SMs that are done first (fp32 attention 27.3 -> 29.4 us, verification
// of 61 rows 18.8 -> 19.5).
__device__ __forceinline__ void tree_let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
template <typename... KArgs, typename... Args>
cudaError_t tree_launch(void (*kernel)(KArgs...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 0 ? 2 : 1;                    // 0: a kernel that knows no clusters
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// One sequence's ring as a tree kernel needs it.
struct TreeRing {
  int head, count, sink, cap, e;
};

__host__ __device__ inline int tree_evicted(int count, int cap, int e, int m) {
  const int over = count + m - cap;
  return over > 0 ? (over + e - 1) / e * e : 0;
}

// Ring words of (layer, sequence) lb; false when they are out of range (corrupt workspace).
__device__ __forceinline__ bool tree_ring(const PtencDev& p, size_t lb, TreeRing* r) {
  r->head = p.head[lb];
  r->count = p.count[lb];
  r->sink = p.n_sink[lb];
  r->cap = p.W - r->sink;
  r->e = p.E < r->cap ? p.E : r->cap;
  return !(r->sink < 0 || r->cap < 1 || r->head < 0 || r->head >= r->cap || r->count < 0 || r->count > r->cap);
}

// Slot of the token with arrival number o (counted from the oldest sliding token).
__device__ __forceinline__ int tree_slot(const TreeRing& r, int o) {
  int s = r.head + o;                                    // o is below cap + TREE_MAX, so a few turns at most where cap is small
  if (s >= 2 * r.cap) s %= r.cap;
  else if (s >= r.cap) s -= r.cap;
  return r.sink + s;
}

// Fills, for the n nodes of a sequence, anc[i] (bit j: node j is on node i's path, i included), ev[i] (tokens gone when
// the path has arrived) and vis[i] (the path's nodes that are still there).  All threads of the CTA call it; the path
// relation is closed by pointer doubling, six rounds for 64 nodes.  Returns false (for every thread) when a parent is out
// of order.  jump: scratch of TREE_MAX ints.
__device__ __forceinline__ bool tree_setup(const int32_t* __restrict__ parent, int n, const TreeRing& r,
                                           unsigned long long* anc, unsigned long long* vis, int* ev, int* jump) {
  const int i = threadIdx.x;
  int bad = 0;
  if (i < n) {
    const int pa = parent[i];
    bad = pa < -1 || pa >= i;
    anc[i] = 1ull << i;
    jump[i] = bad ? -1 : pa;
  }
  if (__syncthreads_or(bad)) return false;
  for (int s = 1; s < n; s <<= 1) {
    unsigned long long a = 0;
    int j = -1;
    if (i < n) {
      a = anc[i];
      j = jump[i];
      if (j >= 0) { a |= anc[j]; j = jump[j]; }
    }
    __syncthreads();
    if (i < n) { anc[i] = a; jump[i] = j; }
    __syncthreads();
  }
  if (i < n) {
    const int gone = tree_evicted(r.count, r.cap, r.e, __popcll(anc[i]));
    ev[i] = gone;
    unsigned long long v = anc[i];
    if (gone > r.count) {                       // so many arrivals that the path's first tokens have left again
      v = 0;
      for (unsigned long long m = anc[i]; m != 0; m &= m - 1) {
        const int j = __ffsll((long long)m) - 1;
        if (r.count + __popcll(anc[j]) - 1 >= gone) v |= 1ull << j;
      }
    }
    vis[i] = v;
  }
  __syncthreads();
  return true;
}

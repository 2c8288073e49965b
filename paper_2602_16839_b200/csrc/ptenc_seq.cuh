// What the kernels of attention over whole sequences share: which tokens a token sees, and how tiles of packed sequences are found.
#pragma once

#include "ptenc_tree.cuh"

struct SeqArgs {
  int Hq, Hkv, D, g, B;
  int window, chunk;               // window 0: none
  int pins;                        // tiles of a sequence that may be pinned and are numbered by themselves (gradients of keys and values)
  float scale;
  long long n;
  const void* q;
  const void* k;
  const void* v;
  long long qs, ks, vs;            // elements from token to token
  const int32_t* cu;
  const int32_t* pinned;
  void* out;
  float* lse;                      // forward: nullable output; backward: input
  const void* dout;
  void* dq;
  void* dk;
  void* dv;
  long long dqs, dks, dvs;
  float* delta;                    // backward scratch, 2 n Hq: sums of dout * out (and lse, in the tensor-core kernels)
};

// A sequence as its tiles see it.  Token i sees j <= i with j < pin or j >= low(i); token j is seen by i >= j with i <= last(j).
struct SeqView {
  int start, len;                  // first row in the packed tensors, tokens
  int pin, cap, e;                 // pinned tokens, sliding capacity, chunk; cap 0: no window

  __device__ __forceinline__ int low(int i) const {
    if (cap == 0 || i < pin) return 0;
    const int over = i - pin + 1 - cap;
    return pin + (over > 0 ? (over + e - 1) / e * e : 0);      // below i + e, and i < 2^31 - 512
  }
  // Token i sees itself alone: its weight is one whatever its score, and its score has a gradient of exactly zero, not what the
  // roundings of two equal sums leave.
  __device__ __forceinline__ bool alone(int i) const { return i == 0 || (cap != 0 && pin == 0 && low(i) == i); }
  __device__ __forceinline__ int last(int j) const {
    if (cap == 0 || j < pin) return len - 1;
    const long long x = (long long)pin + cap - 1 + (long long)((j - pin) / e) * e;
    return x < len - 1 ? (int)x : len - 1;
  }
};

// Describes sequence b; false where its bounds or its pinned tokens are out of range.
__device__ __forceinline__ bool seq_at_start(const SeqArgs& a, int b, SeqView* s) {
  const int c0 = a.cu[b], c1 = a.cu[b + 1];
  if (c0 < 0 || c1 < c0 || c1 > a.n) return false;
  s->start = c0;
  s->len = c1 - c0;
  s->pin = s->cap = 0;
  s->e = 1;
  if (a.window > 0) {
    const int pin = a.pinned != nullptr ? a.pinned[b] : 0;
    if (pin < 0 || pin >= a.window) return false;
    s->pin = pin;
    s->cap = a.window - pin;
    s->e = min(a.chunk, s->cap);
  }
  return true;
}

// Tile numbers.  Tile t of sequence b has number cu[b] / M + b + t: since cu[b + 1] / M + 1 - cu[b] / M is at least the number
// of tiles of M tokens that sequence b needs, numbers are never shared, and a call has at most n / M + B of them -- the host
// needs to know no length.  Some numbers belong to no tile.  Finds the sequence by binary search and checks everything read.
__device__ __forceinline__ bool seq_find(const SeqArgs& a, int number, int M, SeqView* s, int* tile) {
  int lo = 0, hi = a.B;            // the last b with cu[b] / M + b <= number is in [lo, hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.cu[mid] / M + mid <= number) lo = mid; else hi = mid;
  }
  if (!seq_at_start(a, lo, s)) return false;
  const int t = number - (s->start / M + lo);
  if (t < 0 || (long long)t * M >= s->len) return false;
  *tile = t;
  return true;
}
inline long long seq_numbers(long long n, int B, int M) { return n / M + B; }

// The tiles of M keys that the query rows [i0, i1] see some of: pinned ones [0, np), then [s0, s1].
struct SeqRange { int np, s0, s1; };
__device__ __forceinline__ SeqRange seq_keys(const SeqView& s, int i0, int i1, int M) {
  SeqRange r;
  const int pinned = s.cap == 0 ? 0 : min(s.pin, i1 + 1);
  r.np = (pinned + M - 1) / M;
  r.s0 = max(r.np, max(s.low(i0), pinned) / M);
  r.s1 = i1 / M;
  return r;
}
__device__ __forceinline__ int seq_count(const SeqRange& r) { return r.np + max(0, r.s1 - r.s0 + 1); }
__device__ __forceinline__ int seq_at(const SeqRange& r, int k) { return k < r.np ? k : r.s0 + k - r.np; }
// Whether every row of [i0, i1] sees every key of [j0, j1], low1 = low(i1): a division that is not done once per tile (in the
// tensor-core kernels it and the tests row by row had cost a third of the time under a window).
__device__ __forceinline__ bool seq_all(const SeqView& s, int i0, int low1, int j0, int j1) {
  return j1 <= i0 && (j1 < s.pin || j0 >= low1);
}
// The same from the keys' side: every row of [i0, i1] sees every key of [j0, j1] if j1 <= i0 and i1 <= seq_seen_until(j0, j1).
__device__ __forceinline__ int seq_seen_until(const SeqView& s, int j0, int j1) {
  if (s.cap == 0 || j1 < s.pin) return 0x7fffffff;
  if (j0 < s.pin) return s.pin - 1;                // rows of the prompt alone
  const long long x = (long long)s.pin + s.cap - 1 + (long long)((j0 - s.pin) / s.e) * s.e;
  return x < 0x7fffffff ? (int)x : 0x7fffffff;
}

cudaError_t seq_forward_any(const SeqArgs& a, int dtype, int dev, cudaStream_t st);
cudaError_t seq_backward_any(const SeqArgs& a, int dtype, int dev, cudaStream_t st);
// The tensor-core kernels; false: they do not cover the call.
bool seq_forward_tc(const SeqArgs& a, int dtype, int dev, cudaStream_t st, cudaError_t* e);
bool seq_backward_tc(const SeqArgs& a, int dtype, int dev, cudaStream_t st, cudaError_t* e);

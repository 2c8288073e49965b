// The clipped policy loss with a KL term, from logits to their gradient.
//
// Per token: lp = z_y / T - log sum exp(z / T), r = exp(lp - old), loss = -min(r A, clip(r) A) + beta (exp(ref - lp) - (ref - lp) - 1),
// d loss / d z_x = (d loss / d lp) / T * ((x == y) - softmax_x).
//
// Bound by memory: a row is read once and its gradient written once.  A row's maximum and sum have to be known before any of its
// gradient is, so the row stays in shared memory in between: a cluster of one to eight CTAs per row holds a slice each (bulk copies
// in two chunks, the maximum and the sum of a chunk while the next ones arrive), exchanges (maximum, sum) through distributed shared
// memory, works the loss out in 64 bits, and writes the gradient from shared memory.  Rows need not be aligned: the values in front of
// the first and behind the last 16-byte boundary are held by the first CTA's threads, one each.  Rows that eight CTAs cannot hold
// are read three times.
//
// 4096 rows of 152000 bf16, loss and gradient: 547 us, 4.55 TB/s; the exponentials, two per logit, keep their unit busy for half of that.  1001
// rows of 65537 fp32, none but the first aligned, a third masked: 92 us.  Log-probabilities of 16 rows of 32000 fp32: 6.4 us.
#include <cooperative_groups.h>

#include "ptenc_tc.cuh"
#include "ptenc_tree.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int PL_THREADS = 256;
constexpr int PL_CHUNKS = 2;
constexpr int PL_CTAS = 3;                       // CTAs per SM
// Most bytes of a row in a CTA: so that three share an SM (228 KB, of which a CTA takes 1 KB and its static part besides), or two.
constexpr int PL_SLICE3 = 76544, PL_SLICE2 = 112 * 1024;

struct PolicyArgs {
  const void* z;
  long long zs;
  const int32_t* tok;
  const float* old_lp;
  const float* ref_lp;
  const float* adv;
  const float* weight;
  long long n;
  int V;
  float inv_t, c2;                               // 1 / T, and log2(e) / T
  float clip_low, clip_high, kl;
  float* logp;
  float* token_loss;
  float* token_kl;
  void* dz;
  long long dzs;
};

// exp(x) - 1 in 64 bits: x = k ln 2 + r, the Taylor series of r to its 13th term (|r| <= 0.35: below 2^-53), 2^k (exp(r) - 1) + 2^k - 1.
// One chain for the ratio and the KL term, in two lanes: with the library's functions a row's arithmetic kept its CTA waiting longer.
__device__ __forceinline__ double pl_expm1(double x) {
  const double k = fmin(fmax(rint(x * 1.44269504088896340736), -1000.0), 1023.0);
  const double r = fma(-k, 0.69314718055994530942, x);
  double p = 1.0 / 6227020800.0;
  const double inv[11] = {1.0 / 479001600.0, 1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0,
                          1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5};
#pragma unroll
  for (int i = 0; i < 11; ++i) p = fma(p, r, inv[i]);
  p = fma(p * r, r, r);
  const double s = __longlong_as_double((long long)(1023 + (int)k) << 52);
  const double y = fma(s, p, s - 1.0);
  return x < -690.0 ? -1.0 : x > 709.0 ? (double)INFINITY : y;          // NaN stays
}
// log2 of a positive finite number: the fp32 logarithm of its fraction, corrected by what 2^-y0 leaves of it.
__device__ __forceinline__ double pl_log2(float l) {
  if (!(l >= 1.17549435e-38f) || l > 3e38f) return log2((double)l);
  const int e = (int)(__float_as_uint(l) >> 23) - 127;
  const double m = (double)__uint_as_float((__float_as_uint(l) & 0x7fffffu) | 0x3f800000u);
  const float y0 = log2f((float)m);
  const double q = fma(m, pl_expm1(-(double)y0 * 0.69314718055994530942), m - 1.0);
  return (double)e + (double)y0 + q * 1.44269504088896340736 * (1.0 - 0.5 * q);
}

struct PolicyRow { float lp, loss, kl, grad; };  // grad: d (weight * loss) / d z_y without the softmax's part

// What follows from a row's log-probability, in 64 bits: a ratio's side of the clip border decides a whole row of the gradient.  A
// warp calls it; lane 0 has the answer.
__device__ __forceinline__ PolicyRow pl_row(const PolicyArgs& a, long long t, double lp, float w) {
  PolicyRow o = {(float)lp, 0.f, 0.f, 0.f};
  if (a.adv == nullptr) return o;
  const int lane = threadIdx.x & 31;
  const double adv = a.adv[t], ref = a.ref_lp != nullptr ? (double)a.ref_lp[t] : lp, old = a.old_lp != nullptr ? (double)a.old_lp[t] : lp;
  const double over = ref - lp;
  const double em1 = pl_expm1(lane == 0 ? lp - old : over);
  const double rk = __shfl_sync(0xffffffffu, em1, 1);    // exp(ref - lp) - 1
  const double r = a.old_lp != nullptr ? em1 + 1.0 : 1.0;
  const double lo = 1.0 - (double)a.clip_low, hi = 1.0 + (double)a.clip_high;
  const double rc = r < lo ? lo : r > hi ? hi : r;       // NaN stays
  const double s0 = r * adv, s1 = rc * adv;
  double loss = -(s1 < s0 ? s1 : s0);
  const bool cut = (adv > 0.0 && r > hi) || (adv < 0.0 && r < lo);
  double d = cut ? 0.0 : -s0;
  if (a.ref_lp != nullptr) {
    const double kl = rk - over;
    o.kl = (float)kl;
    loss += (double)a.kl * kl;
    d -= (double)a.kl * rk;
  }
  o.loss = (float)loss;
  o.grad = (float)((double)w * d * (double)a.inv_t);
  return o;
}

// Rows of any width, read from memory three times.  A thread adds PL_BLOCK weights in fp32 and the blocks in 64 bits: in one fp32 chain of up to
// 2^20 weights log-probabilities were off by 9e-3 at 2^28 columns and 3e-4 at 2 * 10^7.
constexpr int PL_BLOCK = 16;
template <typename T>
__global__ void __launch_bounds__(PL_THREADS)
k_policy_row(const __grid_constant__ PolicyArgs a) {
  __shared__ float s_m[PL_THREADS / 32];
  __shared__ double s_l[PL_THREADS / 32];
  __shared__ float s_out;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  tree_after_previous();
  const long long t = blockIdx.x;
  const int y = a.tok[t];
  const float w = a.weight != nullptr ? a.weight[t] : 1.f;
  const T* z = static_cast<const T*>(a.z) + t * a.zs;
  T* dz = a.dz != nullptr ? static_cast<T*>(a.dz) + t * a.dzs : nullptr;
  if (w == 0.f || y < 0 || y >= a.V) {
    if (tid == 0) {
      a.logp[t] = 0.f;
      if (a.token_loss != nullptr) a.token_loss[t] = 0.f;
      if (a.token_kl != nullptr) a.token_kl[t] = 0.f;
    }
    if (dz != nullptr)
      for (int x = tid; x < a.V; x += PL_THREADS) dz[x] = ptenc_from_float<T>(0.f);
    return;
  }
  const float zy = ptenc_to_float(z[y]);
  float m = zy;
  bool nan = zy != zy;
  for (int x = tid; x < a.V; x += PL_THREADS) { const float v = ptenc_to_float(z[x]); m = fmaxf(m, v); nan |= v != v; }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) s_m[warp] = m;
  __syncthreads();
  for (int i = 0; i < PL_THREADS / 32; ++i) m = fmaxf(m, s_m[i]);
  const float ref = m == -INFINITY ? 0.f : m;
  double sum = nan ? (double)__int_as_float(0x7fffffff) : 0.0;
  int x0 = tid;
  for (; x0 + PL_THREADS * (PL_BLOCK - 1) < a.V; x0 += PL_THREADS * PL_BLOCK) {      // a.V is at most 2^28
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < PL_BLOCK; ++i) {
      const float p = exp2f((ptenc_to_float(z[x0 + PL_THREADS * i]) - ref) * a.c2);
      l += x0 + PL_THREADS * i == y ? 0.f : p;
    }
    sum += (double)l;
  }
  float rest = 0.f;                                      // less than a block
  for (; x0 < a.V; x0 += PL_THREADS)
    if (x0 != y) rest += exp2f((ptenc_to_float(z[x0]) - ref) * a.c2);
  sum += (double)rest;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_l[warp] = sum;
  __syncthreads();
  sum = 0.0;                                             // without the token's own weight, see k_policy
  for (int i = 0; i < PL_THREADS / 32; ++i) sum += s_l[i];
  const float others = (float)sum, l = (float)(sum + (double)exp2f((zy - ref) * a.c2));
  if (warp == 0) {
    const double lp = (((double)zy - (double)ref) * (double)a.c2 - pl_log2(l)) * 0.69314718055994530942;
    const PolicyRow o = pl_row(a, t, lp, w);
    if (tid == 0) {
      a.logp[t] = o.lp;
      if (a.token_loss != nullptr) a.token_loss[t] = o.loss;
      if (a.token_kl != nullptr) a.token_kl[t] = o.kl;
      s_out = o.grad;
    }
  }
  if (dz == nullptr) return;
  __syncthreads();                                       // also: everybody has read the row before it may be overwritten
  const float grad = s_out, scale = -grad / l;
  for (int x = tid; x < a.V; x += PL_THREADS)
    dz[x] = ptenc_from_float<T>(x == y ? grad * (others / l) : exp2f((ptenc_to_float(z[x]) - ref) * a.c2) * scale);
}

// ------------------------------------------------------------------------------------------------ a row per cluster
__device__ __forceinline__ void pl_bulk(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// A vector's values, two to a register pair.
__device__ __forceinline__ void pl_unpack(const uint4& w, uint64_t (&f)[4], __nv_bfloat16) {
  const uint32_t e[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int y = 0; y < 4; ++y) f[y] = tt_two(__uint_as_float(e[y] << 16), __uint_as_float(e[y] & 0xffff0000u));
}
__device__ __forceinline__ void pl_unpack(const uint4& w, uint64_t (&f)[2], float) {
  f[0] = tt_two(__uint_as_float(w.x), __uint_as_float(w.y));
  f[1] = tt_two(__uint_as_float(w.z), __uint_as_float(w.w));
}
__device__ __forceinline__ uint4 pl_pack(const float (&f)[8], __nv_bfloat16) {
  return make_uint4(tt_pack(f[0], f[1]), tt_pack(f[2], f[3]), tt_pack(f[4], f[5]), tt_pack(f[6], f[7]));
}
__device__ __forceinline__ uint4 pl_pack(const float (&f)[4], float) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
// A vector with its e-th value put to -inf.
__device__ __forceinline__ uint4 pl_without(const uint4& w, int e, __nv_bfloat16) {
  const uint32_t keep = (e & 1) ? 0xffffu : 0xffff0000u, inf = (e & 1) ? 0xff800000u : 0xff80u;
  return make_uint4((e >> 1) == 0 ? (w.x & keep) | inf : w.x, (e >> 1) == 1 ? (w.y & keep) | inf : w.y,
                    (e >> 1) == 2 ? (w.z & keep) | inf : w.z, (e >> 1) == 3 ? (w.w & keep) | inf : w.w);
}
__device__ __forceinline__ uint4 pl_without(const uint4& w, int e, float) {
  const uint32_t inf = 0xff800000u;
  return make_uint4(e == 0 ? inf : w.x, e == 1 ? inf : w.y, e == 2 ? inf : w.z, e == 3 ? inf : w.w);
}
// A vector's largest value, not counting NaN.
__device__ __forceinline__ float pl_max(const uint4& w, __nv_bfloat16) {
  const __nv_bfloat162* e = reinterpret_cast<const __nv_bfloat162*>(&w);
  const __nv_bfloat162 m = __hmax2(__hmax2(e[0], e[1]), __hmax2(e[2], e[3]));
  return fmaxf(__low2float(m), __high2float(m));
}
__device__ __forceinline__ float pl_max(const uint4& w, float) {
  return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
}
// 2^((z - ref) c2) of two values.  The difference comes first: ref c2 would pass the range of fp32 in a row of the type's lowest values.
__device__ __forceinline__ void pl_weights(uint64_t z, uint64_t neg_ref, uint64_t c2, float& lo, float& hi) {
  tt_both(tt_mul2(tt_add2(z, neg_ref), c2), lo, hi);
  lo = tt_ex2(lo);
  hi = tt_ex2(hi);
}
// Running maximum and sum of 2^((z - ref) c2), ref the maximum, 0 while nothing but -inf has been seen.
struct PlSum {
  float m, l;
  __device__ __forceinline__ float ref() const { return m == -INFINITY ? 0.f : m; }
  __device__ __forceinline__ void grow(float mn, float c2) {
    if (mn > m) {
      l = l == 0.f ? 0.f : l * tt_ex2((ref() - mn) * c2);          // NaN stays
      m = mn;
    }
  }
  __device__ __forceinline__ void join(float om, float ol, float c2) {
    const PlSum o = {om, ol};
    const float mn = fmaxf(m, om), to = mn == -INFINITY ? 0.f : mn;
    l = (l == 0.f ? 0.f : l * tt_ex2((ref() - to) * c2)) + (ol == 0.f ? 0.f : ol * tt_ex2((o.ref() - to) * c2));
    m = mn;
  }
};

// The token's own weight is left out of the sums and added at the end: where it is nearly one, its gradient, which is the sum of the
// others over the whole, would be the difference of two numbers that are the same but for their last bits.  (4096 rows of 152000 bf16
// 547 us so, 539 with one sum.)
template <typename T>
__global__ void __launch_bounds__(PL_THREADS, PL_CTAS)
k_policy(const __grid_constant__ PolicyArgs a) {
  constexpr int N = 16 / sizeof(T);
  extern __shared__ __align__(16) uint8_t s_row[];
  __shared__ __align__(8) uint64_t s_bar[PL_CHUNKS];
  __shared__ float2 s_part[PL_THREADS / 32], s_all;      // s_all: read by the cluster
  __shared__ float s_out[3];
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const long long t = blockIdx.x / cs;
  const uint32_t bar = tt_u32(s_bar);
  if (tid == 0) {
    for (int c = 0; c < PL_CHUNKS; ++c) bar_init(bar + 8 * c, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tree_after_previous();
  const int y = a.tok[t];
  const float w = a.weight != nullptr ? a.weight[t] : 1.f;
  const T* z = static_cast<const T*>(a.z) + t * a.zs;
  T* dz = a.dz != nullptr ? static_cast<T*>(a.dz) + t * a.dzs : nullptr;
  // values [0, head) and [head + N nv, V) lie outside the row's 16-byte vectors; this CTA's vectors are [v0, v0 + mine)
  const int off = (int)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T)), head = min(a.V, off == 0 ? 0 : N - off);
  const int nv = (a.V - head) / N, per = (nv + cs - 1) / cs, v0 = min(nv, rank * per), mine = min(per, nv - v0);
  const int loose = a.V - N * nv, lx = tid < head ? tid : tid + N * nv;        // this thread's value outside them: index lx
  const bool has = rank == 0 && tid < loose;
  const bool same = dz != nullptr && ((reinterpret_cast<uintptr_t>(dz) ^ reinterpret_cast<uintptr_t>(z)) & 15) == 0;
  const T* body = z + head + (long long)N * v0;
  if (w == 0.f || y < 0 || y >= a.V) {                   // the whole cluster agrees
    if (rank == 0 && tid == 0) {
      a.logp[t] = 0.f;
      if (a.token_loss != nullptr) a.token_loss[t] = 0.f;
      if (a.token_kl != nullptr) a.token_kl[t] = 0.f;
    }
    if (dz != nullptr) {
      if (has) dz[lx] = ptenc_from_float<T>(0.f);
      T* to = dz + head + (long long)N * v0;
      if (same)
        for (int v = tid; v < mine; v += PL_THREADS) reinterpret_cast<uint4*>(to)[v] = make_uint4(0u, 0u, 0u, 0u);
      else
        for (int x = tid; x < mine * N; x += PL_THREADS) to[x] = ptenc_from_float<T>(0.f);
    }
    return;
  }
  const int chunk = (mine + PL_CHUNKS - 1) / PL_CHUNKS;
  if (tid == 0) {
    for (int c = 0; c < PL_CHUNKS; ++c) {
      const int first = min(mine, c * chunk), count = min(chunk, mine - first);
      if (count == 0) continue;
      bar_expect(bar + 8 * c, (uint32_t)count * 16);
      pl_bulk(tt_u32(s_row) + (uint32_t)first * 16, body + (long long)N * first, (uint32_t)count * 16, bar + 8 * c);
    }
  }
  const float zy = ptenc_to_float(z[y]);
  const float zl = has ? ptenc_to_float(z[lx]) : -INFINITY;
  const float c2 = a.c2;
  const uint64_t c22 = tt_two(c2, c2);
  PlSum sum = {-INFINITY, 0.f};
  const int yb = y - head - N * v0, yv = yb >= 0 && yb < N * mine ? yb / N : -1, ye = yb & (N - 1);      // where y lies in this CTA's slice
  if (has && lx != y) {
    sum.grow(zl, c2);
    sum.l += tt_ex2((zl - sum.ref()) * c2);
  }
  __syncthreads();                                       // the barriers are there
  bool late = false;
  const uint4* row = reinterpret_cast<const uint4*>(s_row);
  for (int c = 0; c < PL_CHUNKS; ++c) {
    const int first = min(mine, c * chunk), end = min(mine, first + chunk);
    if (first == end) continue;
    bool there = false;
    for (uint32_t i = 0; i < TT_POLLS && !there; ++i) there = bar_try(bar + 8 * c, 0) != 0;
    late |= !there;
    int v = first + tid;
    // four vectors at a time: their maximum, then their weights
    for (; v + 3 * PL_THREADS < end; v += 4 * PL_THREADS) {
      uint4 r[4];
      float mx[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) r[k] = row[v + k * PL_THREADS];
      if ((unsigned)(yv - v) < 4u * PL_THREADS) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (v + k * PL_THREADS == yv) r[k] = pl_without(r[k], ye, T());
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) mx[k] = pl_max(r[k], T());
      sum.grow(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), c2);
      const float nr = -sum.ref();
      const uint64_t nr2 = tt_two(nr, nr);
      uint64_t add[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint64_t f[N / 2];
        pl_unpack(r[k], f, T());
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
          float lo, hi;
          pl_weights(f[e], nr2, c22, lo, hi);
          add[k] = tt_add2(add[k], tt_two(lo, hi));
        }
      }
      float lo, hi;
      tt_both(tt_add2(tt_add2(add[0], add[1]), tt_add2(add[2], add[3])), lo, hi);
      sum.l += lo + hi;
    }
    for (; v < end; v += PL_THREADS) {
      uint4 r = row[v];
      if (v == yv) r = pl_without(r, ye, T());
      sum.grow(pl_max(r, T()), c2);
      const float nr = -sum.ref();
      const uint64_t nr2 = tt_two(nr, nr);
      uint64_t f[N / 2], add = 0ull;
      pl_unpack(r, f, T());
      float lo, hi;
#pragma unroll
      for (int e = 0; e < N / 2; ++e) {
        pl_weights(f[e], nr2, c22, lo, hi);
        add = tt_add2(add, tt_two(lo, hi));
      }
      tt_both(add, lo, hi);
      sum.l += lo + hi;
    }
  }
  if (late) {                                            // a copy that did not come: the row becomes NaN, and the copies are waited for again
    sum.l = __int_as_float(0x7fffffff);
    for (int c = 0; c < PL_CHUNKS; ++c)
      if (c * chunk < mine) bar_drain(bar + 8 * c, 0);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    sum.join(__shfl_xor_sync(0xffffffffu, sum.m, o), __shfl_xor_sync(0xffffffffu, sum.l, o), c2);
  if (lane == 0) s_part[warp] = make_float2(sum.m, sum.l);
  __syncthreads();
  sum.m = s_part[0].x; sum.l = s_part[0].y;
#pragma unroll
  for (int i = 1; i < PL_THREADS / 32; ++i) sum.join(s_part[i].x, s_part[i].y, c2);
  if (cs > 1) {
    if (tid == 0) s_all = make_float2(sum.m, sum.l);
    cluster.sync();                                      // also: every CTA has read what it needs of the row
  }
  if (warp == 0) {
    if (cs > 1) {
      const float2 own = *cluster.map_shared_rank(&s_all, lane < cs ? lane : 0);
      sum.m = __shfl_sync(0xffffffffu, own.x, 0);
      sum.l = __shfl_sync(0xffffffffu, own.y, 0);
      for (int i = 1; i < cs; ++i)                       // in the same order everywhere
        sum.join(__shfl_sync(0xffffffffu, own.x, i), __shfl_sync(0xffffffffu, own.y, i), c2);
    }
    // the others' weights and the token's own, by the larger maximum
    const float m_o = sum.ref(), some = sum.l;
    sum.join(zy, zy == -INFINITY ? 0.f : zy - zy + 1.f, c2);             // NaN and inf become NaN
    const float others = some == 0.f ? 0.f : some * tt_ex2((m_o - sum.ref()) * c2);
    const double lp = (((double)zy - (double)sum.ref()) * (double)c2 - pl_log2(sum.l)) * 0.69314718055994530942;
    const PolicyRow o = pl_row(a, t, lp, w);
    if (lane == 0) {
      if (rank == 0) {
        a.logp[t] = o.lp;
        if (a.token_loss != nullptr) a.token_loss[t] = o.loss;
        if (a.token_kl != nullptr) a.token_kl[t] = o.kl;
      }
      s_out[0] = -sum.ref(); s_out[1] = o.grad * (others / sum.l); s_out[2] = -o.grad / sum.l;
    }
    __syncwarp();
  }
  if (cs > 1) asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");      // nobody leaves while its sum may be read
  __syncthreads();
  if (dz != nullptr) {
    const float nr = s_out[0], grad = s_out[1], scale = s_out[2];
    const uint64_t nr2 = tt_two(nr, nr);
    if (has) dz[lx] = ptenc_from_float<T>(lx == y ? grad : tt_ex2((zl + nr) * c2) * scale);
    T* to = dz + head + (long long)N * v0;
    if (same) {
#pragma unroll 2
      for (int v = tid; v < mine; v += PL_THREADS) {
        uint64_t x[N / 2];
        float f[N];
        pl_unpack(row[v], x, T());
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          pl_weights(x[e >> 1], nr2, c22, f[e], f[e + 1]);
          f[e] *= scale;
          f[e + 1] *= scale;
        }
        if ((unsigned)(yb - N * v) < (unsigned)N) {      // one vector of the row
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (yb - N * v == e) f[e] = grad;
        }
        reinterpret_cast<uint4*>(to)[v] = pl_pack(f, T());
      }
    } else {
      const T* from = reinterpret_cast<const T*>(s_row);
      for (int x = tid; x < mine * N; x += PL_THREADS)
        to[x] = ptenc_from_float<T>(x == yb ? grad : tt_ex2((ptenc_to_float(from[x]) + nr) * c2) * scale);
    }
  }
  if (cs > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}

// loss = sum of weight * token_loss, every thread its tokens in order, then the threads in a fixed tree.
__global__ void __launch_bounds__(1024)
k_policy_sum(const float* __restrict__ token_loss, const float* __restrict__ weight, long long n, float* out) {
  __shared__ double s[32];
  tree_after_previous();
  double sum = 0.0;
  for (long long t = threadIdx.x; t < n; t += 1024) {
    const double w = weight != nullptr ? (double)weight[t] : 1.0;
    if (w != 0.0) sum += w * (double)token_loss[t];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x < 32) {
    sum = s[threadIdx.x];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (threadIdx.x == 0) out[0] = (float)sum;
  }
}

template <typename T>
cudaError_t policy_launch(const PolicyArgs& a, float* loss, int dev, int sms, cudaStream_t st) {
  const long long row = (long long)a.V * sizeof(T);
  int cs = 1;
  // Slices that let three CTAs share an SM, so that one's copies run under another's arithmetic; smaller ones, down to 16 KB, while
  // the call has too few rows to fill the SMs.  4096 rows of 152000 bf16: 548 us with clusters of four; 651 to 723 with eight; more
  // threads per CTA 598 to 1322; clusters that stay and load the next row behind the gradient of the one before 585.
  while (cs < 8 && (row > (long long)cs * PL_SLICE3 || (row > cs * 32ll * 1024 && a.n * cs * 2 <= 4ll * sms))) cs *= 2;
  cudaError_t e;
  if (row > 8ll * PL_SLICE2) {
    e = tree_launch(k_policy_row<T>, dim3((unsigned)a.n), PL_THREADS, 0, 0, st, a);
  } else {
    static PtencOnce once;
    e = ptenc_first_use(once, dev, [] { return ptenc_allow_smem(k_policy<T>, PL_SLICE2); });
    const size_t smem = (size_t)((row / 16 + cs - 1) / cs * 16);
    if (e == cudaSuccess) e = tree_launch(k_policy<T>, dim3((unsigned)(a.n * cs)), PL_THREADS, smem, cs, st, a);
  }
  if (e != cudaSuccess || loss == nullptr) return e;
  return tree_launch(k_policy_sum, dim3(1), 1024, 0, 0, st, (const float*)a.token_loss, a.weight, a.n, loss);
}

inline bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
inline bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; }

}  // namespace

extern "C" int ptenc_policy_loss(const ptenc_policy_config* cfg, const void* logits, int64_t logits_stride, const int32_t* tokens,
                                 const float* old_logp, const float* ref_logp, const float* advantage, const float* weight,
                                 int64_t n_tokens, float* logp, float* token_loss, float* token_kl, float* loss, void* dlogits,
                                 int64_t dlogits_stride, void* stream) {
  if (cfg == nullptr || n_tokens < 0) return PTENC_EINVAL;
  if (cfg->dtype != PTENC_DTYPE_FP32 && cfg->dtype != PTENC_DTYPE_BF16) return PTENC_EINVAL;
  if (cfg->vocab < 1 || !(cfg->temperature >= 1.17549435e-38f) || cfg->temperature > 3e38f) return PTENC_EINVAL;
  if (cfg->vocab > (1 << 28) || n_tokens >= (1ll << 28)) return PTENC_ESHAPE;
  if (advantage != nullptr && (!(cfg->clip_low >= 0.f) || !(cfg->clip_high >= 0.f))) return PTENC_EINVAL;
  if (advantage != nullptr && ref_logp != nullptr && !(cfg->kl_coef >= 0.f)) return PTENC_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (n_tokens == 0) {
    ptenc_drop_old_error();
    if (off4(loss)) return PTENC_EALIGN;
    return loss == nullptr || cudaMemsetAsync(loss, 0, sizeof(float), st) == cudaSuccess ? PTENC_OK : PTENC_ECUDA;
  }
  if (advantage == nullptr && (old_logp != nullptr || ref_logp != nullptr || token_loss != nullptr || token_kl != nullptr ||
                               loss != nullptr || dlogits != nullptr))
    return PTENC_EINVAL;
  if (loss != nullptr && token_loss == nullptr) return PTENC_EINVAL;
  if (off4(tokens) || off4(old_logp) || off4(ref_logp) || off4(advantage) || off4(weight) || off4(logp) || off4(token_loss) ||
      off4(token_kl) || off4(loss) || off16(logits) || off16(dlogits))
    return PTENC_EALIGN;
  if (logits == nullptr || tokens == nullptr || logp == nullptr) return PTENC_EINVAL;
  if (logits_stride < cfg->vocab || logits_stride > (1ll << 40)) return PTENC_ESHAPE;
  if (dlogits != nullptr && (dlogits_stride < cfg->vocab || dlogits_stride > (1ll << 40))) return PTENC_ESHAPE;
  if (dlogits == logits && dlogits_stride != logits_stride) return PTENC_EINVAL;
  PolicyArgs a;
  a.z = logits; a.zs = logits_stride; a.tok = tokens; a.old_lp = old_logp; a.ref_lp = ref_logp; a.adv = advantage;
  a.weight = weight; a.n = n_tokens; a.V = cfg->vocab;
  a.inv_t = 1.f / cfg->temperature;
  a.c2 = (float)(1.44269504088896340736 / (double)cfg->temperature);
  a.clip_low = cfg->clip_low; a.clip_high = cfg->clip_high; a.kl = cfg->kl_coef;
  a.logp = logp; a.token_loss = token_loss; a.token_kl = token_kl; a.dz = dlogits; a.dzs = dlogits_stride;
  ptenc_drop_old_error();
  int dev = -1, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return PTENC_ECUDA;
  const cudaError_t e = cfg->dtype == PTENC_DTYPE_FP32 ? policy_launch<float>(a, loss, dev, sms, st)
                                                       : policy_launch<__nv_bfloat16>(a, loss, dev, sms, st);
  return e == cudaSuccess ? PTENC_OK : PTENC_ECUDA;
}

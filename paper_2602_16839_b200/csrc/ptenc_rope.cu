// Norms of query and key heads and the rotation by position, forward and backward.
//
//   n = x / sqrt(mean(x^2) + eps),  y = w n,  (a, b) -> (a cos - b sin, b cos + a sin)  for each pair of the rotated values.
// Backward, with g the gradient turned back by the same angles (a rotation's inverse is its transpose):
//   dw = sum g n,  dx = (w g - n mean(w g n)) / sqrt(mean(x^2) + eps).
//
// Bound by memory: every value is read and written once, a few operations each.  A CTA takes a few tokens with all their query heads
// or all their key heads at a step; their angles, in 64 bits, are worked out once for all heads, one by each thread, while the next
// step's values are on their way.  A head is a group of lanes
// (a power of two) with two 16-byte vectors each, chosen so that both values of a pair are in the same lane.
//
// bf16: 32768 tokens of 28 + 4 heads of 128, rotation alone, 107 us, 5.0 TB/s; 16384 tokens of 32 + 8 with norms, forward and
// backward, 179 us, 4.7 TB/s; 16 tokens of 16 + 2 heads 2.9 us.
#include <string.h>

#include "ptenc_tc.cuh"
#include "ptenc_tree.cuh"

namespace {

constexpr int RP_MAX_D = 256;
constexpr int RP_BLOCKS = 592;                   // most CTAs of a backward launch, each with a partial sum of dw
constexpr int RP_THREADS = 256;
constexpr int RP_TOK = 8;                        // most tokens of a CTA at a time
// CTAs per SM, forward and backward: what 64 and 128 registers per thread allow.  Each thread has the next step's row in flight, 32 or
// 64 bytes.  32768 tokens of 28 + 4 heads, forward: 108 us so, 122 with three CTAs, 117 with five (spills), 115 with two rows in
// flight; without a next step in flight, a CTA per step, 126; angles of eight steps at a time, one barrier for them, 135.  Backward,
// 16384 tokens of 32 + 8 heads: 110 us; 163 with one CTA per SM, 153 with three (spills).
constexpr int RP_CTAS_F = 4, RP_CTAS_B = 2;
constexpr int RP_WARPS = 8;

struct RopeArgs {
  int Hq, Hkv, D, rot, inter;
  float eps;
  long long n;
  const void* x[2];                              // q, k
  long long xs[2];
  const void* w[2];
  const void* g[2];                              // gradients of the outputs
  long long gs[2];
  void* y[2];                                    // outputs (forward) or gradients of the inputs (backward)
  long long ys[2];
  const int32_t* pos;
  const float* freq;
  float* part;                                   // [CTA][2][D] partial sums of dw
};

// Cosine and sine of pos * freq, turns = freq / (2 pi).  The product is taken in 64 bits and brought to a fraction of a turn there: in 32 bits the
// angle of position 60000 would be off by 2e-3.  `fast`: the hardware's sine and cosine, off by 2^-20.5 at most within half a turn, for
// results that are rounded to bf16 (2^-8) anyhow; the weights' gradients, which are fp32 sums over bf16 values, take them too.
__device__ __forceinline__ void rp_angle(int pos, double turns, float* s, float* c, bool fast) {
  double t = (double)pos * turns;
  t -= rint(t);
  if (fast) {
    const float x = (float)t * 6.2831853071795864769f;
    *s = __sinf(x);
    *c = __cosf(x);
  } else {
    sincospif(2.f * (float)t, s, c);
  }
}

__device__ __forceinline__ float rp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The shape-generic form: a warp per token and head, values 32 apart in a lane, pairs through shared memory.
template <typename T, bool BWD>
__global__ void __launch_bounds__(32 * RP_WARPS)
k_rope_any(const __grid_constant__ RopeArgs a) {
  __shared__ float s_row[RP_WARPS][RP_MAX_D];
  __shared__ float s_sum[RP_WARPS][RP_MAX_D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int H = a.Hq + a.Hkv, D = a.D, half = a.rot >> 1;
  float* row = s_row[warp];
  float dw[2][RP_MAX_D / 32];
#pragma unroll
  for (int i = 0; i < RP_MAX_D / 32; ++i) dw[0][i] = dw[1][i] = 0.f;
  tree_after_previous();
  for (long long it = (long long)blockIdx.x * RP_WARPS + warp; it < a.n * H; it += (long long)gridDim.x * RP_WARPS) {
    const long long t = it / H;
    const int hh = (int)(it - t * H), side = hh >= a.Hq ? 1 : 0, h = side ? hh - a.Hq : hh;
    const T* x = static_cast<const T*>(a.x[side]) + t * a.xs[side] + (long long)h * D;
    const T* w = static_cast<const T*>(a.w[side]);
    const int pos = a.pos[t];
    float v[RP_MAX_D / 32], g[RP_MAX_D / 32];
    float inv = 1.f;
    if (!BWD || w != nullptr) {
      float sq = 0.f;
#pragma unroll
      for (int i = 0; i < RP_MAX_D / 32; ++i) {
        const int d = lane + 32 * i;
        v[i] = d < D ? ptenc_to_float(x[d]) : 0.f;
        sq = fmaf(v[i], v[i], sq);
      }
      if (w != nullptr) inv = 1.f / sqrtf(rp_sum(sq) / (float)D + a.eps);
    }
    const T* gr = BWD ? static_cast<const T*>(a.g[side]) + t * a.gs[side] + (long long)h * D : nullptr;
#pragma unroll
    for (int i = 0; i < RP_MAX_D / 32; ++i) {
      const int d = lane + 32 * i;
      if (d < D) row[d] = BWD ? ptenc_to_float(gr[d]) : w != nullptr ? v[i] * inv * ptenc_to_float(w[d]) : v[i];
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < RP_MAX_D / 32; ++i) {
      const int d = lane + 32 * i;
      g[i] = 0.f;
      if (d < D) {
        g[i] = row[d];
        if (d < a.rot) {
          const int f = a.inter ? d >> 1 : (d < half ? d : d - half);
          const bool second = a.inter ? (d & 1) != 0 : d >= half;
          const float other = row[a.inter ? d ^ 1 : (second ? d - half : d + half)];
          float sn, cs;
          rp_angle(pos, (double)a.freq[f] * 0.15915494309189533577, &sn, &cs, false);
          if (BWD) sn = -sn;
          g[i] = fmaf(g[i], cs, second ? other * sn : -other * sn);
        }
      }
    }
    __syncwarp();
    T* y = static_cast<T*>(a.y[side]) + t * a.ys[side] + (long long)h * D;
    float dot = 0.f;
    if (BWD && w != nullptr) {
#pragma unroll
      for (int i = 0; i < RP_MAX_D / 32; ++i) {
        const int d = lane + 32 * i;
        if (d < D) {
          v[i] *= inv;
          const float add = g[i] * v[i];
          if (side) dw[1][i] += add; else dw[0][i] += add;
          g[i] *= ptenc_to_float(w[d]);
          dot = fmaf(g[i], v[i], dot);
        }
      }
      dot = rp_sum(dot) / (float)D;
    }
#pragma unroll
    for (int i = 0; i < RP_MAX_D / 32; ++i) {
      const int d = lane + 32 * i;
      if (d < D) y[d] = ptenc_from_float<T>(BWD && w != nullptr ? inv * (g[i] - v[i] * dot) : g[i]);
    }
  }
  if (BWD && a.part != nullptr) {
    for (int side = 0; side < 2; ++side) {
#pragma unroll
      for (int i = 0; i < RP_MAX_D / 32; ++i) s_sum[warp][lane + 32 * i] = dw[side][i];
      __syncthreads();
      if (threadIdx.x < D) {
        float sum = 0.f;
        for (int k = 0; k < RP_WARPS; ++k) sum += s_sum[k][threadIdx.x];
        a.part[((size_t)side * RP_BLOCKS + blockIdx.x) * D + threadIdx.x] = sum;
      }
      __syncthreads();
    }
  }
}

// ------------------------------------------------------------------------------------------------ vectors
struct RopeShape {
  int lanes;                                     // of a head: a power of two up to 32
  // of the queries and of the keys: tokens of a step, steps that the heads of a step's tokens are cut into
  int tok[2], chunks[2];
  int first[2], ctas[2];                         // and the CTAs that take them: all take both, in small calls each takes one side
  unsigned inv[2];                               // ceil(2^32 / heads): x / heads = umulhi(x, inv) for x heads < 2^32
};

template <typename T> struct RpVec { static constexpr int N = 16 / sizeof(T); };

// A vector's values, two to a register pair, for packed arithmetic: taken one by one the kernel was bound by its instructions.
__device__ __forceinline__ void rp_unpack(const uint4& w, uint64_t (&f)[8], int at, __nv_bfloat16) {
  const uint32_t e[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int y = 0; y < 4; ++y) f[at + y] = tt_two(__uint_as_float(e[y] << 16), __uint_as_float(e[y] & 0xffff0000u));
}
__device__ __forceinline__ void rp_unpack(const uint4& w, uint64_t (&f)[4], int at, float) {
  f[at] = tt_two(__uint_as_float(w.x), __uint_as_float(w.y));
  f[at + 1] = tt_two(__uint_as_float(w.z), __uint_as_float(w.w));
}
__device__ __forceinline__ uint4 rp_pack(const uint64_t (&f)[8], int at, __nv_bfloat16) {
  uint32_t e[4];
#pragma unroll
  for (int y = 0; y < 4; ++y) {
    float lo, hi;
    tt_both(f[at + y], lo, hi);
    e[y] = tt_pack(lo, hi);
  }
  return make_uint4(e[0], e[1], e[2], e[3]);
}
__device__ __forceinline__ uint4 rp_pack(const uint64_t (&f)[4], int at, float) {
  float a, b, c, d;
  tt_both(f[at], a, b);
  tt_both(f[at + 1], c, d);
  return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
}
__device__ __forceinline__ float rp_group_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Lane l of a head holds pairs N l .. N l + N - 1 (N = values of a vector) as vectors va and vb: with halves as pairs the same place
// in both halves, and behind those lanes values that are not rotated, two vectors each; with neighbours as pairs two vectors in a row.
template <typename T, bool BWD, bool INTER>
__global__ void __launch_bounds__(RP_THREADS, BWD ? RP_CTAS_B : RP_CTAS_F)
k_rope(const __grid_constant__ RopeArgs a, const __grid_constant__ RopeShape sh) {
  constexpr int N = RpVec<T>::N;
  extern __shared__ __align__(16) float s_trig[];        // [2][tok][cos, sin][lanes * N]
  __shared__ float s_sum[RP_THREADS / 32][RP_MAX_D];
  const int tid = threadIdx.x, l = tid & (sh.lanes - 1), groups = RP_THREADS / sh.lanes, grp = tid / sh.lanes;
  const int D = a.D, half = a.rot >> 1, nv = D / N, P = half / N, np = sh.lanes * N;
  const int va = INTER || l >= P ? 2 * l : l, vb = INTER || l >= P ? 2 * l + 1 : l + P;
  const bool ha = va < nv, hb = vb < nv;
  const bool turns = N * l < half;                       // some of the lane's pairs are rotated: all of them, with halves
  const float rD = 1.f / (float)D;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  tree_after_previous();
  int turn = 0;
  // first the CTA's share of the queries' steps, then of the keys'
#pragma unroll 1
  for (int side = 0; side < 2; ++side) {
    const int H = side ? a.Hkv : a.Hq, tok = sh.tok[side], chunks = sh.chunks[side];
    const unsigned inv_h = sh.inv[side];
    const long long steps = (a.n + tok - 1) / tok * chunks;
    const int cta = (int)blockIdx.x - sh.first[side], ctas = sh.ctas[side];
    if (cta < 0 || cta >= ctas) continue;
    const T* w = static_cast<const T*>(a.w[side]);
    const bool norm = w != nullptr, need_x = !BWD || norm;
    const T* X = static_cast<const T*>(a.x[side]);
    const T* G = static_cast<const T*>(a.g[side]);
    T* Y = static_cast<T*>(a.y[side]);
    const long long xs = a.xs[side], gs = a.gs[side], ys = a.ys[side];
    // this thread's angle of a step: pair my_p of the step's token my_t, in turns; where it goes: four pairs of a lane next to each
    // other, the lanes behind one another, for 16-byte reads without bank conflicts
    const int my_t = half > 0 ? tid / half : tok, my_p = half > 0 ? tid - my_t * half : 0;
    const int my_at = my_t * 2 * np + (my_p / N) * 4 + (my_p & 3) + (N == 8 ? ((my_p >> 2) & 1) * (np / 2) : 0);
    uint64_t dw[N], w2[N];
#pragma unroll
    for (int y = 0; y < N; ++y) dw[y] = w2[y] = 0ull;
    uint4 x[2], g[2];
    int my_pos = 0;
    // asks for the values and the position of step s
    auto fetch = [&](long long s) {
      const long long tg = chunks == 1 ? s : s / chunks, t0 = tg * tok;
      const int toks = (int)(a.n - t0 < tok ? a.n - t0 : tok), items = toks * H;
      const int it = (int)(s - tg * chunks) * groups + grp, t = H == 1 ? it : (int)__umulhi((unsigned)it, inv_h), h = it - t * H;
      const bool on = it < items;
      if (my_t < toks) my_pos = a.pos[t0 + my_t];
      x[0] = x[1] = g[0] = g[1] = zero;
      if (need_x && on) {
        const uint4* from = reinterpret_cast<const uint4*>(X + (t0 + t) * xs + (long long)h * D);
        if (ha) x[0] = from[va];
        if (hb) x[1] = from[vb];
      }
      if (BWD && on) {
        const uint4* from = reinterpret_cast<const uint4*>(G + (t0 + t) * gs + (long long)h * D);
        if (ha) g[0] = from[va];
        if (hb) g[1] = from[vb];
      }
    };
    if (cta < steps) fetch(cta);
    const double my_freq = my_t < tok ? (double)a.freq[my_p] * 0.15915494309189533577 : 0.0;
    if (norm) {
      rp_unpack(ha ? reinterpret_cast<const uint4*>(w)[va] : zero, w2, 0, T());
      rp_unpack(hb ? reinterpret_cast<const uint4*>(w)[vb] : zero, w2, N / 2, T());
    }
    for (long long s = cta; s < steps; s += ctas, turn ^= 1) {
      const long long tg = chunks == 1 ? s : s / chunks, t0 = tg * tok;
      const int toks = (int)(a.n - t0 < tok ? a.n - t0 : tok), items = toks * H;
      const int it = (int)(s - tg * chunks) * groups + grp, t = H == 1 ? it : (int)__umulhi((unsigned)it, inv_h), h = it - t * H;
      const bool on = it < items;
      float* trig = s_trig + turn * RP_TOK * 2 * np;         // the other copy may still be read
      if (my_t < toks) {
        float sn, cs;
        rp_angle(my_pos, my_freq, &sn, &cs, sizeof(T) == 2);
        trig[my_at] = cs;
        trig[my_at + np] = BWD ? -sn : sn;
      }
      __syncthreads();
      const uint4 x0 = x[0], x1 = x[1], g0 = g[0], g1 = g[1];
      if (s + ctas < steps) fetch(s + ctas);
      uint64_t v[N], o[N];
      float inv = 1.f;
      if (need_x) {
        rp_unpack(x0, v, 0, T());
        rp_unpack(x1, v, N / 2, T());
        if (norm) {
          uint64_t sq = 0ull;
#pragma unroll
          for (int y = 0; y < N; ++y) sq = tt_fma2(v[y], v[y], sq);
          float lo, hi;
          tt_both(sq, lo, hi);
          inv = rsqrtf(rp_group_sum(lo + hi, sh.lanes) * rD + a.eps);      // groups of a warp take the same steps
          const uint64_t inv2 = tt_two(inv, inv);
#pragma unroll
          for (int y = 0; y < N; ++y) v[y] = tt_mul2(v[y], inv2);
        }
      }
      if (BWD) {
        rp_unpack(g0, o, 0, T());
        rp_unpack(g1, o, N / 2, T());
      } else {
#pragma unroll
        for (int y = 0; y < N; ++y) o[y] = norm ? tt_mul2(v[y], w2[y]) : v[y];
      }
      if (turns && on) {
        const float* at = trig + t * 2 * np + l * 4;
#pragma unroll
        for (int q = 0; q < N; q += 4) {
          const float4 c4 = *reinterpret_cast<const float4*>(at + q / 4 * (np / 2));
          const float4 s4 = *reinterpret_cast<const float4*>(at + np + q / 4 * (np / 2));
          if (INTER) {
            const float cs[4] = {c4.x, c4.y, c4.z, c4.w}, sn[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
            for (int y = q; y < q + 4; ++y) {
              if (N * l + y >= half) continue;
              float p, r;
              tt_both(o[y], p, r);
              o[y] = tt_fma2(o[y], tt_two(cs[y - q], cs[y - q]), tt_mul2(tt_two(r, p), tt_two(-sn[y - q], sn[y - q])));
            }
          } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int i = q / 2 + k, j = i + N / 2;
              const uint64_t cs = k ? tt_two(c4.z, c4.w) : tt_two(c4.x, c4.y), sn = k ? tt_two(s4.z, s4.w) : tt_two(s4.x, s4.y);
              const uint64_t ns = k ? tt_two(-s4.z, -s4.w) : tt_two(-s4.x, -s4.y);
              const uint64_t p = o[i], r = o[j];
              o[i] = tt_fma2(r, ns, tt_mul2(p, cs));
              o[j] = tt_fma2(p, sn, tt_mul2(r, cs));
            }
          }
        }
      }
      if (BWD && norm) {
        uint64_t dot2 = 0ull;
#pragma unroll
        for (int y = 0; y < N; ++y) {
          if (on) dw[y] = tt_fma2(o[y], v[y], dw[y]);    // with eps = 0 the zeros of a group without a head have the norm 0 * inf
          o[y] = tt_mul2(o[y], w2[y]);
          dot2 = tt_fma2(o[y], v[y], dot2);
        }
        float lo, hi;
        tt_both(dot2, lo, hi);
        const float dot = -rp_group_sum(lo + hi, sh.lanes) * rD * inv;
        const uint64_t d2 = tt_two(dot, dot), inv2 = tt_two(inv, inv);
#pragma unroll
        for (int y = 0; y < N; ++y) o[y] = tt_fma2(v[y], d2, tt_mul2(o[y], inv2));
      }
      if (on) {
        uint4* to = reinterpret_cast<uint4*>(Y + (t0 + t) * ys + (long long)h * D);
        if (ha) to[va] = rp_pack(o, 0, T());
        if (hb) to[vb] = rp_pack(o, N / 2, T());
      }
    }
    if (BWD && a.part != nullptr) {
      // groups of a warp, then the warps, in a fixed order
#pragma unroll
      for (int y = 0; y < 2 * N; ++y) {
        float lo, hi;
        tt_both(dw[y >> 1], lo, hi);
        float v = (y & 1) ? hi : lo;
        for (int o = 16; o >= sh.lanes; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        const int at = (y < N ? va : vb) * N + (y & (N - 1));
        if ((tid & 31) < sh.lanes && (y < N ? ha : hb)) s_sum[tid >> 5][at] = v;
      }
      __syncthreads();
      for (int d = tid; d < D; d += RP_THREADS) {
        float sum = 0.f;
        for (int k = 0; k < RP_THREADS / 32; ++k) sum += s_sum[k][d];
        a.part[((size_t)side * RP_BLOCKS + cta) * D + d] = sum;
      }
      __syncthreads();
    }
  }
}

// dw of both sides: the CTAs' partial sums, each thread those of every 32nd CTA in order, then the threads of a column.
__global__ void __launch_bounds__(1024)
k_rope_weights(const float* __restrict__ part, int nq, int nk, int D, float* dwq, float* dwk) {
  __shared__ double s[32][33];
  const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, side = blockIdx.y;
  float* to = side ? dwk : dwq;
  tree_after_previous();
  if (to == nullptr) return;
  const float* from = part + (size_t)side * RP_BLOCKS * D;
  const int n = side ? nk : nq;
  double sum = 0.0;
  if (c < D) {
#pragma unroll 8
    for (int b = grp; b < n; b += 32) sum += (double)from[(size_t)b * D + c];
  }
  s[grp][lane] = sum;
  __syncthreads();
  if (grp == 0 && c < D) {
    sum = 0.0;
    for (int k = 0; k < 32; ++k) sum += s[k][lane];
    to[c] = (float)sum;
  }
}

inline bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
inline bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; }

int check_config(const ptenc_rope_config* c, long long n) {
  if (c == nullptr || n < 0) return PTENC_EINVAL;
  if (c->dtype != PTENC_DTYPE_FP32 && c->dtype != PTENC_DTYPE_BF16) return PTENC_EINVAL;
  if (c->n_q_heads < 1 || c->n_kv_heads < 1 || c->head_dim < 1) return PTENC_EINVAL;
  if (c->interleaved != 0 && c->interleaved != 1) return PTENC_EINVAL;
  if (!(c->eps >= 0.f) || c->eps > 3e38f) return PTENC_EINVAL;
  if (c->head_dim % 8 != 0 || c->head_dim > RP_MAX_D || c->n_q_heads > 16384 || c->n_q_heads % c->n_kv_heads != 0)
    return PTENC_ESHAPE;
  if (c->rotary_dim < 0 || c->rotary_dim > c->head_dim || c->rotary_dim % 2 != 0) return PTENC_ESHAPE;
  if (n >= (1ll << 31) - 512) return PTENC_ESHAPE;
  return PTENC_OK;
}

// A stride in elements: room for the heads, and every token's row 16-byte aligned.
int check_stride(long long stride, int heads, int D, int dtype) {
  if (stride < (long long)heads * D || stride > (1ll << 40)) return PTENC_ESHAPE;
  return stride * (dtype == PTENC_DTYPE_FP32 ? 4 : 2) % 16 != 0 ? PTENC_EALIGN : PTENC_OK;
}

template <typename T, bool BWD>
cudaError_t rope_launch(const RopeArgs& a, int sms, float* dwq, float* dwk, cudaStream_t st) {
  const int N = 16 / (int)sizeof(T), H = a.Hq + a.Hkv;
  cudaError_t e;
  int ctas[2];
  if (!a.inter && (a.rot / 2) % N != 0) {
    // halves that do not start on a vector
    const long long want = (a.n * H + RP_WARPS - 1) / RP_WARPS;
    ctas[0] = ctas[1] = (int)(want < RP_BLOCKS ? want : RP_BLOCKS);
    e = tree_launch(k_rope_any<T, BWD>, dim3(ctas[0]), 32 * RP_WARPS, 0, 0, st, a);
  } else {
    RopeShape sh;
    const int pairs = (a.D / N + 1) / 2;
    for (sh.lanes = 1; sh.lanes < pairs; sh.lanes *= 2) {}
    const int fly = RP_THREADS / sh.lanes, per_sm = BWD ? RP_CTAS_B : RP_CTAS_F;
    const int resident = per_sm * sms < RP_BLOCKS ? per_sm * sms : RP_BLOCKS;
    long long steps[2];
    for (int side = 0; side < 2; ++side) {
      // tokens of a step: as many as its groups have in flight, no more than its threads have angles for, fewer where that would
      // leave CTAs without work
      const int heads = side ? a.Hkv : a.Hq;
      int tok = fly / heads;
      if (tok > RP_TOK) tok = RP_TOK;
      if (a.rot > 0 && tok > RP_THREADS / (a.rot / 2)) tok = RP_THREADS / (a.rot / 2);
      while (tok > 1 && a.n / tok < resident) tok /= 2;
      sh.tok[side] = tok < 1 ? 1 : tok;
      sh.chunks[side] = (sh.tok[side] * heads + fly - 1) / fly;
      sh.inv[side] = heads > 1 ? (unsigned)(((1ull << 32) + heads - 1) / heads) : 0u;
      steps[side] = (a.n + sh.tok[side] - 1) / sh.tok[side] * sh.chunks[side];
    }
    const bool small = steps[0] + steps[1] <= resident;  // each step has a CTA of its own: 16 tokens of 16 + 2 heads 3.6 -> 2.8 us
    for (int side = 0; side < 2; ++side) sh.ctas[side] = ctas[side] = (int)(steps[side] < resident ? steps[side] : resident);
    sh.first[0] = 0;
    sh.first[1] = small ? ctas[0] : 0;
    const int grid = small ? ctas[0] + ctas[1] : ctas[0] > ctas[1] ? ctas[0] : ctas[1];
    const size_t smem = (size_t)2 * RP_TOK * 2 * sh.lanes * N * sizeof(float);
    e = tree_launch(a.inter ? k_rope<T, BWD, true> : k_rope<T, BWD, false>, dim3(grid), RP_THREADS, smem, 0, st, a, sh);
  }
  if (e != cudaSuccess || !BWD || a.part == nullptr) return e;
  return tree_launch(k_rope_weights, dim3((a.D + 31) / 32, 2), 1024, 0, 0, st, (const float*)a.part, ctas[0], ctas[1], a.D, dwq, dwk);
}

template <bool BWD>
int rope_run(const ptenc_rope_config* cfg, const RopeArgs& a, float* dwq, float* dwk, cudaStream_t st) {
  ptenc_drop_old_error();
  int dev = -1, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return PTENC_ECUDA;
  const cudaError_t e = cfg->dtype == PTENC_DTYPE_FP32 ? rope_launch<float, BWD>(a, sms, dwq, dwk, st)
                                                       : rope_launch<__nv_bfloat16, BWD>(a, sms, dwq, dwk, st);
  return e == cudaSuccess ? PTENC_OK : PTENC_ECUDA;
}

RopeArgs rope_args(const ptenc_rope_config* c, const void* q, int64_t qs, const void* k, int64_t ks, const void* wq, const void* wk,
                   const int32_t* pos, const float* freq, long long n) {
  RopeArgs a;
  memset(&a, 0, sizeof(a));
  a.Hq = c->n_q_heads; a.Hkv = c->n_kv_heads; a.D = c->head_dim; a.rot = c->rotary_dim; a.inter = c->interleaved;
  a.eps = c->eps; a.n = n;
  a.x[0] = q; a.x[1] = k; a.xs[0] = qs; a.xs[1] = ks; a.w[0] = wq; a.w[1] = wk;
  a.pos = pos; a.freq = freq;
  return a;
}

}  // namespace

extern "C" int ptenc_head_norm_rope(const ptenc_rope_config* cfg, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                    const void* q_weight, const void* k_weight, const int32_t* positions, const float* inv_freq,
                                    int64_t n_tokens, void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride,
                                    void* stream) {
  int rc = check_config(cfg, n_tokens);
  if (rc != PTENC_OK || n_tokens == 0) return rc;
  if (q == nullptr || k == nullptr || q_out == nullptr || k_out == nullptr || positions == nullptr ||
      (inv_freq == nullptr && cfg->rotary_dim > 0))
    return PTENC_EINVAL;
  const int Hq = cfg->n_q_heads, Hkv = cfg->n_kv_heads, D = cfg->head_dim, dt = cfg->dtype;
  if ((rc = check_stride(q_stride, Hq, D, dt)) != PTENC_OK || (rc = check_stride(k_stride, Hkv, D, dt)) != PTENC_OK ||
      (rc = check_stride(q_out_stride, Hq, D, dt)) != PTENC_OK || (rc = check_stride(k_out_stride, Hkv, D, dt)) != PTENC_OK)
    return rc;
  if (off16(q) || off16(k) || off16(q_out) || off16(k_out) || off16(q_weight) || off16(k_weight) || off4(positions) || off4(inv_freq))
    return PTENC_EALIGN;
  if ((q_out == q && q_out_stride != q_stride) || (k_out == k && k_out_stride != k_stride)) return PTENC_EINVAL;
  RopeArgs a = rope_args(cfg, q, q_stride, k, k_stride, q_weight, k_weight, positions, inv_freq, n_tokens);
  a.y[0] = q_out; a.y[1] = k_out; a.ys[0] = q_out_stride; a.ys[1] = k_out_stride;
  return rope_run<false>(cfg, a, nullptr, nullptr, static_cast<cudaStream_t>(stream));
}

extern "C" int ptenc_head_norm_rope_workspace_bytes(int32_t head_dim, size_t* bytes) {
  if (bytes == nullptr || head_dim < 1) return PTENC_EINVAL;
  if (head_dim % 8 != 0 || head_dim > RP_MAX_D) return PTENC_ESHAPE;
  *bytes = (size_t)RP_BLOCKS * 2 * head_dim * sizeof(float);
  return PTENC_OK;
}

extern "C" int ptenc_head_norm_rope_backward(const ptenc_rope_config* cfg, const void* q, int64_t q_stride, const void* k,
                                             int64_t k_stride, const void* q_weight, const void* k_weight, const int32_t* positions,
                                             const float* inv_freq, int64_t n_tokens, const void* dq_out, int64_t dq_out_stride,
                                             const void* dk_out, int64_t dk_out_stride, void* dq, int64_t dq_stride, void* dk,
                                             int64_t dk_stride, float* dq_weight, float* dk_weight, void* workspace,
                                             size_t workspace_bytes, void* stream) {
  int rc = check_config(cfg, n_tokens);
  if (rc != PTENC_OK) return rc;
  if ((q_weight != nullptr && dq_weight == nullptr) || (k_weight != nullptr && dk_weight == nullptr)) return PTENC_EINVAL;
  if (n_tokens > 0 && ((dq_weight != nullptr && q_weight == nullptr) || (dk_weight != nullptr && k_weight == nullptr)))
    return PTENC_EINVAL;
  if (off16(dq_weight) || off16(dk_weight)) return PTENC_EALIGN;
  const int Hq = cfg->n_q_heads, Hkv = cfg->n_kv_heads, D = cfg->head_dim, dt = cfg->dtype;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (n_tokens == 0) {                                   // a sum over nothing
    ptenc_drop_old_error();
    if ((dq_weight != nullptr && cudaMemsetAsync(dq_weight, 0, D * sizeof(float), st) != cudaSuccess) ||
        (dk_weight != nullptr && cudaMemsetAsync(dk_weight, 0, D * sizeof(float), st) != cudaSuccess))
      return PTENC_ECUDA;
    return PTENC_OK;
  }
  if (q == nullptr || k == nullptr || dq_out == nullptr || dk_out == nullptr || dq == nullptr || dk == nullptr ||
      positions == nullptr || (inv_freq == nullptr && cfg->rotary_dim > 0))
    return PTENC_EINVAL;
  if ((rc = check_stride(q_stride, Hq, D, dt)) != PTENC_OK || (rc = check_stride(k_stride, Hkv, D, dt)) != PTENC_OK ||
      (rc = check_stride(dq_out_stride, Hq, D, dt)) != PTENC_OK || (rc = check_stride(dk_out_stride, Hkv, D, dt)) != PTENC_OK ||
      (rc = check_stride(dq_stride, Hq, D, dt)) != PTENC_OK || (rc = check_stride(dk_stride, Hkv, D, dt)) != PTENC_OK)
    return rc;
  if (off16(q) || off16(k) || off16(dq_out) || off16(dk_out) || off16(dq) || off16(dk) || off16(q_weight) || off16(k_weight) ||
      off4(positions) || off4(inv_freq) || off16(workspace))
    return PTENC_EALIGN;
  if ((dq == dq_out && dq_stride != dq_out_stride) || (dk == dk_out && dk_stride != dk_out_stride)) return PTENC_EINVAL;
  RopeArgs a = rope_args(cfg, q, q_stride, k, k_stride, q_weight, k_weight, positions, inv_freq, n_tokens);
  a.g[0] = dq_out; a.g[1] = dk_out; a.gs[0] = dq_out_stride; a.gs[1] = dk_out_stride;
  a.y[0] = dq; a.y[1] = dk; a.ys[0] = dq_stride; a.ys[1] = dk_stride;
  if (q_weight != nullptr || k_weight != nullptr) {
    size_t need = 0;
    ptenc_head_norm_rope_workspace_bytes(D, &need);
    if (workspace == nullptr) return PTENC_EINVAL;
    if (workspace_bytes < need) return PTENC_EWORKSPACE;
    a.part = static_cast<float*>(workspace);
  }
  return rope_run<true>(cfg, a, dq_weight, dk_weight, st);
}

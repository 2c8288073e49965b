// The clipped policy loss with a KL term, from logits to their gradient.
//
// Per token: lp = z_y / T - log sum exp(z / T), r = exp(lp - old), loss = -min(r A, clip(r) A) + beta (exp(ref - lp) - (ref - lp) - 1),
// d loss / d z_x = (d loss / d lp) / T * ((x == y) - softmax_x).
#include "ptenc_tree.cuh"

namespace {

constexpr int PL_THREADS = 256;

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

struct PolicyRow { float lp, loss, kl, grad; };  // grad: d (weight * loss) / d z_y without the softmax's part

// What follows from a row's log-probability, in 64 bits: a ratio's side of the clip border decides a whole row of the gradient.
__device__ __forceinline__ PolicyRow pl_row(const PolicyArgs& a, long long t, double lp, float w) {
  PolicyRow o = {(float)lp, 0.f, 0.f, 0.f};
  if (a.adv == nullptr) return o;
  const double adv = a.adv[t];
  const double r = a.old_lp != nullptr ? exp(lp - (double)a.old_lp[t]) : 1.0;
  const double lo = 1.0 - (double)a.clip_low, hi = 1.0 + (double)a.clip_high;
  const double rc = r < lo ? lo : r > hi ? hi : r;       // NaN stays
  const double s0 = r * adv, s1 = rc * adv;
  double loss = -(s1 < s0 ? s1 : s0);
  const bool cut = (adv > 0.0 && r > hi) || (adv < 0.0 && r < lo);
  double d = cut ? 0.0 : -s0;
  if (a.ref_lp != nullptr) {
    const double over = (double)a.ref_lp[t] - lp;
    const double kl = expm1(over) - over;
    o.kl = (float)kl;
    loss += (double)a.kl * kl;
    d -= (double)a.kl * expm1(over);
  }
  o.loss = (float)loss;
  o.grad = (float)((double)w * d * (double)a.inv_t);
  return o;
}

template <typename T>
__global__ void __launch_bounds__(PL_THREADS)
k_policy_row(const __grid_constant__ PolicyArgs a) {
  __shared__ float s_m[PL_THREADS / 32], s_l[PL_THREADS / 32];
  __shared__ float s_out[3];
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
  float m = -INFINITY;
  bool nan = false;
  for (int x = tid; x < a.V; x += PL_THREADS) { const float v = ptenc_to_float(z[x]); m = fmaxf(m, v); nan |= v != v; }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) s_m[warp] = m;
  __syncthreads();
  for (int i = 0; i < PL_THREADS / 32; ++i) m = fmaxf(m, s_m[i]);
  const float mc = m * a.c2;
  float l = 0.f;
  for (int x = tid; x < a.V; x += PL_THREADS) l += exp2f(fmaf(ptenc_to_float(z[x]), a.c2, -mc));
  l = nan ? __int_as_float(0x7fffffff) : l;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  if (lane == 0) s_l[warp] = l;
  __syncthreads();
  l = 0.f;
  for (int i = 0; i < PL_THREADS / 32; ++i) l += s_l[i];
  if (tid == 0) {
    const double lp = ((double)zy * (double)a.c2 - (double)mc - log2((double)l)) * 0.69314718055994530942;
    const PolicyRow o = pl_row(a, t, lp, w);
    a.logp[t] = o.lp;
    if (a.token_loss != nullptr) a.token_loss[t] = o.loss;
    if (a.token_kl != nullptr) a.token_kl[t] = o.kl;
    s_out[0] = o.grad;
  }
  if (dz == nullptr) return;
  __syncthreads();                                       // also: everybody has read the row before it may be overwritten
  const float grad = s_out[0], scale = -grad / l;
  for (int x = tid; x < a.V; x += PL_THREADS) {
    float v = exp2f(fmaf(ptenc_to_float(z[x]), a.c2, -mc)) * scale;
    if (x == y) v += grad;
    dz[x] = ptenc_from_float<T>(v);
  }
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
cudaError_t policy_launch(const PolicyArgs& a, float* loss, cudaStream_t st) {
  cudaError_t e = tree_launch(k_policy_row<T>, dim3((unsigned)a.n), PL_THREADS, 0, 0, st, a);
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
  if (cfg->vocab < 1 || !(cfg->temperature > 0.f) || cfg->temperature > 3e38f) return PTENC_EINVAL;
  if (cfg->vocab > (1 << 28) || n_tokens >= (1ll << 31) - 512) return PTENC_ESHAPE;
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
  const cudaError_t e = cfg->dtype == PTENC_DTYPE_FP32 ? policy_launch<float>(a, loss, st) : policy_launch<__nv_bfloat16>(a, loss, st);
  return e == cudaSuccess ? PTENC_OK : PTENC_ECUDA;
}

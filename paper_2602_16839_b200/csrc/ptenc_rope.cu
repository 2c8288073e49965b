// Norms of query and key heads and the rotation by position, forward and backward.
//
//   n = x / sqrt(mean(x^2) + eps),  y = w n,  (a, b) -> (a cos - b sin, b cos + a sin)  for each pair of the rotated values.
// Backward, with g the gradient turned back by the same angles (a rotation's inverse is its transpose):
//   dw = sum g n,  dx = (w g - n mean(w g n)) / sqrt(mean(x^2) + eps).
#include <string.h>

#include "ptenc_tree.cuh"

namespace {

constexpr int RP_MAX_D = 256;
constexpr int RP_BLOCKS = 592;                   // most CTAs of a backward launch, each with a partial sum of dw
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

// Cosine and sine of pos * freq.  The product is taken in 64 bits and brought to a fraction of a turn there: in 32 bits the
// angle of position 60000 would be off by 2e-3.
__device__ __forceinline__ void rp_angle(int pos, float freq, float* s, float* c) {
  double t = (double)pos * (double)freq * 0.15915494309189533577;
  t -= rint(t);
  sincospif(2.f * (float)t, s, c);
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
          rp_angle(pos, a.freq[f], &sn, &cs);
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
        a.part[((size_t)blockIdx.x * 2 + side) * D + threadIdx.x] = sum;
      }
      __syncthreads();
    }
  }
}

// dw of both sides: the CTAs' partial sums, added in order, eight groups of CTAs at a time.
__global__ void __launch_bounds__(256)
k_rope_weights(const float* __restrict__ part, int blocks, int D, float* dwq, float* dwk) {
  __shared__ double s[8][32];
  const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  tree_after_previous();
  double sum = 0.0;
  if (c < 2 * D)
    for (int b = grp; b < blocks; b += 8) sum += (double)part[(size_t)b * 2 * D + c];
  s[grp][lane] = sum;
  __syncthreads();
  if (grp == 0 && c < 2 * D) {
    for (int k = 1; k < 8; ++k) sum += s[k][lane];
    float* to = c < D ? dwq : dwk;
    if (to != nullptr) to[c < D ? c : c - D] = (float)sum;
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
  const long long items = a.n * (a.Hq + a.Hkv);
  const long long want = (items + RP_WARPS - 1) / RP_WARPS;
  const int grid = (int)(want < RP_BLOCKS ? want : RP_BLOCKS);
  (void)sms;
  cudaError_t e = tree_launch(k_rope_any<T, BWD>, dim3(grid), 32 * RP_WARPS, 0, 0, st, a);
  if (e != cudaSuccess || !BWD || a.part == nullptr) return e;
  return tree_launch(k_rope_weights, dim3((2 * a.D + 31) / 32), 256, 0, 0, st, (const float*)a.part, grid, a.D, dwq, dwk);
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

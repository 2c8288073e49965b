// What the tensor-core kernels of attention over whole sequences share.
#pragma once

#include "ptenc_seq.cuh"
#include "ptenc_tc.cuh"

namespace {

constexpr int SN = 128;                        // tokens of a K/V tile
constexpr int ST_THREADS = 384;                // producer, MMA, two patch warps, 2 x 4 softmax warps
// Registers: 384 threads are launched with 168 each (64512); the first four warps give up 96 for the softmax threads' scores.
constexpr int ST_REGS_LOW = 72, ST_REGS_HIGH = 216;
static_assert(128 * ST_REGS_LOW + 256 * ST_REGS_HIGH <= 384 * 168, "the split waits for registers that do not exist");
constexpr float ST_LOG2E = 1.4426950408889634f, ST_LN2 = 0.6931471805599453f;

// Bits of positions [lo, hi) in the word of positions [at, at + 32).
__device__ __forceinline__ uint32_t st_run(int lo, int hi, int at) {
  const int a = max(lo - at, 0), b = min(hi - at, 32);
  return a >= b ? 0u : (~0u >> (32 - (b - a))) << a;
}

// ------------------------------------------------------------------------------------------------ taking over CTAs
// Asks for a CTA of the grid that has not started yet; 16 bytes of answer arrive at `to` and count at the barrier.
__device__ __forceinline__ void clc_ask(uint32_t to, uint32_t bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
               ::"r"(to), "r"(bar) : "memory");
}
// The x coordinate of the CTA that was taken over, or -1: none was left.
__device__ __forceinline__ int clc_answer(uint32_t at) {
  int x;
  asm volatile(
      "{\n\t.reg .b128 h;\n\t.reg .pred p;\n\t.reg .b32 y;\n\t"
      "ld.shared.b128 h, [%1];\n\t"
      "mov.b32 y, -1;\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 y, h;\n\t"
      "mov.b32 %0, y;\n\t}"
      : "=r"(x) : "r"(at) : "memory");
  return x;
}

// Rows [row0, row0 + 128) of a 128-row tile of bf16 columns in shared memory: those past `rows` become zero, non-finite values of the
// others too.  `me` of `of` warps.  True in every lane if something was taken out; bad (nullable): a bit per row it was.
// A row's products with zero, added up, are NaN exactly if it holds an infinity or a NaN: four packed instructions per 16 bytes, so
// that the pass hides under a tile's products (tested bit by bit it took 4000 cycles, more than they do, and bounded the kernels).
__device__ __forceinline__ bool patch_tile(uint8_t* tile, int halves, int row0, int rows, int me, int of, uint32_t* bad) {
  const int lane = threadIdx.x & 31;
  auto place = [&](int x) { return reinterpret_cast<uint4*>(tile + (x >> 10) * HALF + ((x >> 3) & (TM - 1)) * 128 + (x & 7) * 16); };
  const int total = halves * TM * 8;
  if (row0 + TM > rows)
    for (int x = me * 32 + lane; x < total; x += of * 32)
      if (row0 + ((x >> 3) & (TM - 1)) >= rows) *place(x) = make_uint4(0u, 0u, 0u, 0u);
  const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
  __nv_bfloat162 acc[2] = {zero, zero};
  for (int x0 = me * 32 + lane; x0 < total; x0 += of * 32 * 8) {       // a multiple of eight steps: 512 or 1024 vectors per warp
    uint4 w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = *place(x0 + k * of * 32);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const __nv_bfloat162* e = reinterpret_cast<const __nv_bfloat162*>(&w[k]);
#pragma unroll
      for (int y = 0; y < 4; ++y) acc[y & 1] = __hfma2(e[y], zero, acc[y & 1]);
    }
  }
  acc[0] = __hadd2(acc[0], acc[1]);
  const bool odd = __any_sync(0xffffffffu, !(__low2float(acc[0]) == 0.f) || !(__high2float(acc[0]) == 0.f));
  if (odd) {
#pragma unroll 1
    for (int x = me * 32 + lane; x < total; x += of * 32) {
      uint4 w = *place(x);
      uint32_t* e = reinterpret_cast<uint32_t*>(&w);
      bool hit = false;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        if ((e[y] & 0x7f80u) == 0x7f80u) { e[y] &= 0xffff0000u; hit = true; }
        if ((e[y] & 0x7f800000u) == 0x7f800000u) { e[y] &= 0x0000ffffu; hit = true; }
      }
      if (hit) {
        *place(x) = w;
        if (bad != nullptr) atomicOr(bad + ((x >> 8) & 3), 1u << ((x >> 3) & 31));
      }
    }
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  return odd;
}

// Waits for a CTA's next item for as long as its producer, which counts the numbers it has looked at, gets on: a bounded wait lasts 8 ms,
// and numbers that belong to no tile (one per empty sequence and head) can take longer than that together.
__device__ __forceinline__ bool item_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, volatile int* looks) {
  for (int seen = -1;;) {
    if (bar_wait(bar, parity, abort_flag)) return true;
    const int now = *looks;
    if (*abort_flag != 0 || now == seen) return false;
    seen = now;
  }
}

// ------------------------------------------------------------------------------------------------ host
// bf16 [n][heads][D] with `stride` elements from token to token, box of 128 tokens x 1 head x 64 columns, 128-byte swizzle; what lies
// outside the tensor reads as zero.
bool seq_map(CUtensorMap* map, const void* base, int D, int heads, long long n, long long stride) {
  TtEncodeFn fn = tt_encode_fn();
  if (fn == nullptr) return false;
  cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)n};
  cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)stride * 2};
  cuuint32_t box[3] = {64, 1, SN};
  cuuint32_t estr[3] = {1, 1, 1};
  return ptenc_encode_map([&] {
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  });
}

}  // namespace

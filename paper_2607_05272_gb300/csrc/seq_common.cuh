// seq_common.cuh — shared by the operators of sequence policies (seq_loss.cu, seq_scan.cu,
// seq_norm.cu): element types, block sums, and the running maximum and sums of a softmax.
//
// Tensors hold fp32 or bf16; every value is widened to fp32 on load and rounded once, to nearest
// even, on store.  exp, sigmoid and 1/x here are the hardware approximations (relative error about
// 2^-22, far below the 1e-5 that these operators are held to); logarithms of sums use logf.
#pragma once
#include <cuda_bf16.h>

#include <cstdint>

#include "devmath.cuh"

namespace simx {
namespace seq {

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T>
__device__ __forceinline__ T narrow(float x);
template <>
__device__ __forceinline__ float narrow<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// 2^x and 1/x, one special-function instruction each (subnormal results flush to zero).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kMost = 3.402823466e+38f;  // the largest finite fp32
__device__ __forceinline__ float inf() { return __int_as_float(0x7F800000); }
__device__ __forceinline__ float nan() { return __int_as_float(0x7FC00000); }

// Sums over a row of logits with its maximum m: s = sum e^((x - m) / T), t = sum e^((x - m) / T) (x - m).
// The maximum is taken over the whole row first, so that partial sums are only added: rescaling them by
// ex2 on the way would give each its error again.  A row with nothing above -inf has x - m = NaN, and
// so have its sums.
struct Part {
  float m, s, t;
};

// Term j of the sums; k = log2(e) / T.
__device__ __forceinline__ float part_term(float x, float m, float k, float& t) {
  const float d = __fsub_rn(x, m);
  const float e = ex2(__fmul_rn(d, k));
  t = __fmaf_rn(e, fmaxf(d, -kMost), t);  // x = -inf: e is 0, and so is the product
  return e;
}

__device__ __forceinline__ float max_lanes(float v) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
  return v;
}
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) v = __fadd_rn(v, __shfl_xor_sync(0xffffffffu, v, d));
  return v;
}

// Lets the next kernel of the stream start its preamble; waits for the previous one's results.
__device__ __forceinline__ void pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

}  // namespace seq
}  // namespace simx

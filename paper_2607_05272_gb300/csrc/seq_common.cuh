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
#include "tc_common.cuh"

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

// Clusters: this block's rank, a barrier of all their threads, and a store of 8 bytes into block `rank`'s
// shared memory that counts them on a barrier of that block: the data carries its own signal, where a
// cluster barrier's release would wait for every global store on its way.
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void post_peer(float2* slot, uint64_t* bar, uint32_t rank, float2 v) {
  uint32_t at, on;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(tcx::su32(slot)), "r"(rank));
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(on) : "r"(tcx::su32(bar)), "r"(rank));
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(at), "f"(v.x),
               "f"(v.y), "r"(on)
               : "memory");
}
constexpr long long kPeerCycles = 2000000000ll;  // a peer's posts take microseconds: a second is a failure

// Asynchronous copies into a thread's own places in shared memory (BYTES 4, 8 or 16).
template <int BYTES>
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
  if (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tcx::su32(dst)), "l"(src) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(tcx::su32(dst)), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_wait_all() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Lets the next kernel of the stream start its preamble; waits for the previous one's results.
__device__ __forceinline__ void pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// A sum as hi + lo, each addition's rounding error kept (Knuth's two-sum): about 46 bits.  fp64 runs at a
// sixty-fourth of the fp32 rate here, and the few thousand additions of a call's statistics took longer in it than its rows.
struct Sum2 {
  float hi, lo;
  __device__ __forceinline__ void add(float v, float rest) {
    const float s = __fadd_rn(hi, v), b = __fsub_rn(s, hi);
    const float e = __fadd_rn(__fsub_rn(hi, __fsub_rn(s, b)), __fsub_rn(v, b));
    hi = s;
    lo = __fadd_rn(lo, __fadd_rn(e, rest));
  }
  // a sum that is not finite has no rounding error to give back
  __device__ __forceinline__ float value() const { return fabsf(hi) < inf() ? __fadd_rn(hi, lo) : hi; }
};

// out[c] = the sum over the rows of part [rows][cols]: a block of 1024 threads for the 32 columns from c0
// on, 32 rows at a time, joined in a fixed order.
__device__ __forceinline__ void column_sums(const float* part, int64_t rows, int64_t cols, int64_t c0, float* out) {
  __shared__ float sh[32][33];
  const int cl = threadIdx.x & 31, rl = (int)threadIdx.x / 32;
  const int64_t c = c0 + cl;
  Sum2 t = {};
  if (c < cols) {
    int64_t r = rl;
    for (; r + 96 < rows; r += 128) {
      float v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = part[(r + 32 * u) * cols + c];
      t.add(__fadd_rn(__fadd_rn(v[0], v[1]), __fadd_rn(v[2], v[3])), 0.0f);
    }
    for (; r < rows; r += 32) t.add(part[r * cols + c], 0.0f);
  }
  sh[rl][cl] = t.value();
  __syncthreads();
  const float s = sum_lanes(sh[cl][rl]);
  if (cl == 0 && c0 + rl < cols) out[c0 + rl] = s;
}

}  // namespace seq
}  // namespace simx

// seq_norm.cu — dropout of a branch, its addition to the residual stream and the root-mean-square
// norm of the sum, forward and backward, with a mask drawn from Philox counters in both passes
// instead of being stored.
//
// z = residual + keep x scale, rstd = 1 / sqrt(mean z^2 + eps), y = z rstd gain; backward, with
// zh = z rstd: dresidual = dz + rstd (dy gain - zh mean(dy gain zh)), dx = keep scale dresidual,
// dgain = sum over rows of dy zh.  A draw gives eight 16-bit fields, so the generator costs a tenth
// of what one word per element would.  Bound by HBM: 2 reads and 2 writes per element forward, 3 and
// 2 backward.
#include "kernels.h"
#include "seq_common.cuh"

namespace simx {

using namespace seq;

namespace {

constexpr uint32_t kStreamDropout = 6;  // beside the simulator's streams 1 .. 5
constexpr int kGroup = 8;               // columns per draw
constexpr int kNormThreads = 256;
constexpr int kMaxSlabs = 608;          // partial rows of dgain

struct Drop {
  uint32_t key0, key1, step, row_base, thr;  // thr: fields below it are dropped; 0: no dropout
  float scale;
};

// The keep bits of columns 8 group .. 8 group + 7 of a row (bit j: column 8 group + j).
__device__ __forceinline__ uint32_t keep_bits(const Drop& D, uint32_t group, uint32_t row) {
  const U4 w = philox(group, row, D.step, kStreamDropout, D.key0, D.key1);
  const uint32_t f[4] = {w.x, w.y, w.z, w.w};
  uint32_t b = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    b |= (uint32_t)((f[i] & 0xFFFFu) >= D.thr) << (2 * i);
    b |= (uint32_t)((f[i] >> 16) >= D.thr) << (2 * i + 1);
  }
  return b;
}

__device__ __forceinline__ float block_sum(float v, float* sh) {
  v = sum_lanes(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x / 32] = v;
  __syncthreads();
  float o = 0.0f;
  for (int w = 0; w < (int)blockDim.x / 32; ++w) o = __fadd_rn(o, sh[w]);
  return o;
}

// A block per row, the row's z in shared memory.
template <class T>
__global__ void __launch_bounds__(kNormThreads) k_norm_rows(simx_norm A, Drop D) {
  extern __shared__ float zs[];
  __shared__ float sh[kNormThreads / 32];
  const int W = (int)A.width, groups = (W + kGroup - 1) / kGroup;
  for (int64_t i = blockIdx.x; i < A.n; i += gridDim.x) {
    const T* x = static_cast<const T*>(A.x) + i * A.x_ld;
    const T* res = A.residual ? static_cast<const T*>(A.residual) + i * A.residual_ld : nullptr;
    T* z = A.z ? static_cast<T*>(A.z) + i * A.z_ld : nullptr;
    T* y = static_cast<T*>(A.y) + i * A.y_ld;
    float ss = 0.0f;
    for (int q = threadIdx.x; q < groups; q += kNormThreads) {
      const uint32_t keep = D.thr ? keep_bits(D, (uint32_t)q, D.row_base + (uint32_t)i) : 0xFFu;
      for (int j = 0; j < kGroup && q * kGroup + j < W; ++j) {
        const int c = q * kGroup + j;
        float v = res ? widen(res[c]) : 0.0f;
        if (keep >> j & 1u) v = __fmaf_rn(widen(x[c]), D.scale, v);
        zs[c] = v;
        ss = __fmaf_rn(v, v, ss);
      }
    }
    ss = block_sum(ss, sh);
    const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, (float)W), A.eps)));
    for (int q = threadIdx.x; q < groups; q += kNormThreads)
      for (int j = 0; j < kGroup && q * kGroup + j < W; ++j) {
        const int c = q * kGroup + j;
        if (z) z[c] = narrow<T>(zs[c]);
        y[c] = narrow<T>(__fmul_rn(__fmul_rn(zs[c], r), A.gain[c]));
      }
    if (threadIdx.x == 0 && A.rstd) A.rstd[i] = r;
    __syncthreads();
  }
}

// Backward: a block takes a slab of rows; dgain's sums of the slab stay in shared memory.
template <class T>
__global__ void __launch_bounds__(kNormThreads) k_norm_grad_rows(simx_norm A, Drop D, float* slab) {
  extern __shared__ float dgs[];
  __shared__ float sh[kNormThreads / 32];
  const int W = (int)A.width, groups = (W + kGroup - 1) / kGroup;
  for (int c = threadIdx.x; c < W; c += kNormThreads) dgs[c] = 0.0f;
  __syncthreads();
  for (int64_t i = blockIdx.x; i < A.n; i += gridDim.x) {
    const T* z = static_cast<const T*>(A.z) + i * A.z_ld;
    const T* dy = static_cast<const T*>(A.dy) + i * A.dy_ld;
    const T* dz = A.dz ? static_cast<const T*>(A.dz) + i * A.dz_ld : nullptr;
    T* dx = A.dx ? static_cast<T*>(A.dx) + i * A.dx_ld : nullptr;
    T* dr = A.dresidual ? static_cast<T*>(A.dresidual) + i * A.dresidual_ld : nullptr;
    const float r = A.rstd[i];
    float dot = 0.0f;
    for (int q = threadIdx.x; q < groups; q += kNormThreads)
      for (int j = 0; j < kGroup && q * kGroup + j < W; ++j) {
        const int c = q * kGroup + j;
        const float zh = __fmul_rn(widen(z[c]), r), d = widen(dy[c]);
        dgs[c] = __fmaf_rn(d, zh, dgs[c]);
        dot = __fmaf_rn(__fmul_rn(d, A.gain[c]), zh, dot);
      }
    const float mean = __fdiv_rn(block_sum(dot, sh), (float)W);
    for (int q = threadIdx.x; q < groups; q += kNormThreads) {
      const uint32_t keep = D.thr && dx ? keep_bits(D, (uint32_t)q, D.row_base + (uint32_t)i) : 0xFFu;
      for (int j = 0; j < kGroup && q * kGroup + j < W; ++j) {
        const int c = q * kGroup + j;
        const float zh = __fmul_rn(widen(z[c]), r);
        float v = __fmul_rn(r, __fmaf_rn(-zh, mean, __fmul_rn(widen(dy[c]), A.gain[c])));
        if (dz) v = __fadd_rn(v, widen(dz[c]));
        if (dr) dr[c] = narrow<T>(v);
        if (dx) dx[c] = narrow<T>(keep >> j & 1u ? __fmul_rn(v, D.scale) : 0.0f);
      }
    }
    __syncthreads();
  }
  if (slab)
    for (int c = threadIdx.x; c < W; c += kNormThreads) slab[(int64_t)blockIdx.x * W + c] = dgs[c];
}

__global__ void __launch_bounds__(kNormThreads) k_norm_dgain(const float* slab, int slabs, int width, float* dgain) {
  const int c = blockIdx.x * kNormThreads + threadIdx.x;
  if (c >= width) return;
  double v = 0.0;
  for (int s = 0; s < slabs; ++s) v += (double)slab[(int64_t)s * width + c];
  dgain[c] = (float)v;
}

Drop drop_of(const simx_norm& a) {
  Drop d;
  d.key0 = (uint32_t)a.seed;
  d.key1 = (uint32_t)(a.seed >> 32);
  d.step = a.step;
  d.row_base = a.row_base;
  d.thr = (uint32_t)((double)a.p * 65536.0 + 0.5);
  d.scale = (float)(65536.0 / (65536.0 - (double)d.thr));
  return d;
}

int slabs_of(int64_t n) {
  const int64_t most = (int64_t)sm_count() * 4 < kMaxSlabs ? (int64_t)sm_count() * 4 : kMaxSlabs;
  return (int)(n < most ? n : most);
}

}  // namespace

size_t norm_grad_workspace_bytes(int64_t n, int64_t width) {
  const int64_t rows = n < kMaxSlabs ? n : kMaxSlabs;
  return (size_t)rows * (size_t)width * sizeof(float);
}

cudaError_t launch_norm(const simx_norm& a, cudaStream_t s) {
  const Drop d = drop_of(a);
  const size_t sh = (size_t)a.width * sizeof(float);
  const int64_t most = (int64_t)sm_count() * 8;
  const int blocks = (int)(a.n < most ? a.n : most);
  auto kernel = a.dtype == SIMX_F32 ? k_norm_rows<float> : k_norm_rows<__nv_bfloat16>;
  cudaError_t e = allow_smem(kernel, kNormMaxWidth * (int)sizeof(float));
  if (e != cudaSuccess) return e;
  kernel<<<blocks, kNormThreads, sh, s>>>(a, d);
  count_launches(1);
  return cudaGetLastError();
}

cudaError_t launch_norm_grad(const simx_norm& a, void* ws, cudaStream_t s) {
  const Drop d = drop_of(a);
  const size_t sh = (size_t)a.width * sizeof(float);
  float* slab = a.dgain ? static_cast<float*>(ws) : nullptr;
  const int slabs = slabs_of(a.n);
  if (a.n > 0) {
    auto kernel = a.dtype == SIMX_F32 ? k_norm_grad_rows<float> : k_norm_grad_rows<__nv_bfloat16>;
    cudaError_t e = allow_smem(kernel, kNormMaxWidth * (int)sizeof(float));
    if (e != cudaSuccess) return e;
    kernel<<<slabs, kNormThreads, sh, s>>>(a, d, slab);
    count_launches(1);
  }
  if (slab) {
    k_norm_dgain<<<(int)((a.width + kNormThreads - 1) / kNormThreads), kNormThreads, 0, s>>>(slab, slabs, (int)a.width, a.dgain);
    count_launches(1);
  }
  return cudaGetLastError();
}

}  // namespace simx

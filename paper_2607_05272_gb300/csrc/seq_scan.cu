// seq_scan.cu — the gated linear recurrence h_t = a_t s_t + (1 - a_t) x_t, a_t = sigmoid(gate_t +
// bias), with episode ends as in the returns scan, and its backward pass.
//
// With k_t = 0 where the episode ends after step t, else 1, and s_{t+1} = k_t h_t, the state handed
// on.  Backward, with mu_t = a_t lambda_t (what reaches s_t):
//   lambda_t = dh_t + k_t mu_{t+1} (mu_len = dh_last),  dx_t = (1 - a_t) lambda_t,
//   dgate_t = a_t (1 - a_t) (s_t - x_t) lambda_t,  dh0 = mu_0.
//
// A state close to unchanged (a near 1) is where fp32 goes wrong: a_t itself has the absolute error
// 2^-25, which over 1 / (1 - a) steps of memory is a relative error 2^-25 / (1 - a) of the state (1e-3
// at gate = 10).  So a_t is never formed on the way: b_t = 1 - a_t = sigmoid(-z) has a small relative
// error, h_t = s_t + b_t (x_t - s_t) and mu_t = lambda_t - b_t lambda_t, one fma each.
// Bound by HBM: 2 reads and 1 write per element forward, 4 and 2 backward.
#include "kernels.h"
#include "seq_common.cuh"

namespace simx {

using namespace seq;

namespace {

// sigmoid(z) and sigmoid(-z), each to relative precision.
struct Gate {
  float a, b;
};
__device__ __forceinline__ Gate gate_of(float z) {
  const float e = ex2(__fmul_rn(-fabsf(z), kLog2e));
  const float r = rcp(__fadd_rn(1.0f, e));
  const float er = __fmul_rn(e, r);
  Gate g;
  g.a = z >= 0.0f ? r : er;
  g.b = z >= 0.0f ? er : r;
  if (z != z) g.a = g.b = z;
  return g;
}

template <class T>
__device__ __forceinline__ T* at(const simx_seq& q, int64_t b, int64_t t, int64_t c) {
  return static_cast<T*>(q.p) + b * q.sb + t * q.st + c;
}

constexpr int kColThreads = 128;

// A thread per column (b, c), through time.
template <class T>
__global__ void __launch_bounds__(kColThreads) k_scan_columns(simx_scan A) {
  const int64_t col = (int64_t)blockIdx.x * kColThreads + threadIdx.x;
  if (col >= A.batch * A.channels) return;
  const int64_t b = col / A.channels, c = col - b * A.channels;
  const float bias = A.bias ? A.bias[c] : 0.0f;
  float s = A.h0 ? A.h0[col] : 0.0f;
  for (int64_t t = 0; t < A.len; ++t) {
    const Gate g = gate_of(__fadd_rn(widen(*at<const T>(A.gate, b, t, c)), bias));
    const float h = __fmaf_rn(g.b, __fsub_rn(widen(*at<const T>(A.x, b, t, c)), s), s);
    *at<T>(A.h, b, t, c) = narrow<T>(h);
    s = A.done && A.done[b * A.done_sb + t * A.done_st] ? 0.0f : h;
  }
  if (A.h_last) A.h_last[col] = s;
}

template <class T>
__global__ void __launch_bounds__(kColThreads) k_scan_grad_columns(simx_scan A, float* dbias_part) {
  const int64_t col = (int64_t)blockIdx.x * kColThreads + threadIdx.x;
  if (col >= A.batch * A.channels) return;
  const int64_t b = col / A.channels, c = col - b * A.channels;
  const float bias = A.bias ? A.bias[c] : 0.0f;
  float mu = A.dh_last ? A.dh_last[col] : 0.0f;
  float db = 0.0f;
  for (int64_t t = A.len - 1; t >= 0; --t) {
    const Gate g = gate_of(__fadd_rn(widen(*at<const T>(A.gate, b, t, c)), bias));
    const bool done = A.done && A.done[b * A.done_sb + t * A.done_st];
    float lam = widen(*at<const T>(A.dh, b, t, c));
    if (!done) lam = __fadd_rn(lam, mu);
    float s = 0.0f;
    if (t == 0) s = A.h0 ? A.h0[col] : 0.0f;
    else if (!(A.done && A.done[b * A.done_sb + (t - 1) * A.done_st])) s = widen(*at<const T>(A.h, b, t - 1, c));
    const float dg = __fmul_rn(__fmul_rn(lam, __fsub_rn(s, widen(*at<const T>(A.x, b, t, c)))), __fmul_rn(g.a, g.b));
    *at<T>(A.dx, b, t, c) = narrow<T>(__fmul_rn(lam, g.b));
    *at<T>(A.dgate, b, t, c) = narrow<T>(dg);
    db = __fadd_rn(db, dg);
    mu = __fmaf_rn(-g.b, lam, lam);
  }
  if (A.dh0) A.dh0[col] = mu;
  if (dbias_part) dbias_part[col] = db;
}

// dbias[c] = sum over the rows of part [rows][channels], in order.
__global__ void __launch_bounds__(kColThreads) k_scan_dbias(const float* part, int64_t rows, int64_t channels, float* dbias) {
  const int64_t c = (int64_t)blockIdx.x * kColThreads + threadIdx.x;
  if (c >= channels) return;
  double v = 0.0;
  for (int64_t r = 0; r < rows; ++r) v += (double)part[r * channels + c];
  dbias[c] = (float)v;
}

}  // namespace

size_t scan_workspace_bytes(int64_t batch, int64_t, int64_t channels) {
  return (size_t)batch * (size_t)channels * sizeof(float);
}

cudaError_t launch_scan(const simx_scan& a, cudaStream_t s) {
  const int64_t blocks = (a.batch * a.channels + kColThreads - 1) / kColThreads;
  if (a.dtype == SIMX_F32) k_scan_columns<float><<<(unsigned)blocks, kColThreads, 0, s>>>(a);
  else k_scan_columns<__nv_bfloat16><<<(unsigned)blocks, kColThreads, 0, s>>>(a);
  count_launches(1);
  return cudaGetLastError();
}

cudaError_t launch_scan_grad(const simx_scan& a, void* ws, cudaStream_t s) {
  const int64_t blocks = (a.batch * a.channels + kColThreads - 1) / kColThreads;
  float* part = a.dbias ? static_cast<float*>(ws) : nullptr;
  if (a.dtype == SIMX_F32) k_scan_grad_columns<float><<<(unsigned)blocks, kColThreads, 0, s>>>(a, part);
  else k_scan_grad_columns<__nv_bfloat16><<<(unsigned)blocks, kColThreads, 0, s>>>(a, part);
  count_launches(1);
  if (part) {
    k_scan_dbias<<<(unsigned)((a.channels + kColThreads - 1) / kColThreads), kColThreads, 0, s>>>(part, a.batch, a.channels, a.dbias);
    count_launches(1);
  }
  return cudaGetLastError();
}

}  // namespace simx

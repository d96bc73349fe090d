// seq_loss.cu — losses over a vocabulary, from logits to the logits' gradient: the clipped policy
// loss with its KL and entropy terms (Sec. 4.3's PPO objective on tokens), and the preference loss
// on pairs of sequences.
//
// Per row of logits x with temperature T: m = max x, s = sum e^((x - m) / T),
// log pi(a) = (x_a - m) / T - log s, H = log s - (1 / s) sum e^((x - m) / T) (x - m) / T, and with the
// row's coefficient c = dL / d log pi(a) and entropy coefficient u = w c_entropy
//   dL / dx_j = (c (delta_ja - p_j) + u p_j (log p_j + H)) / T.
// Bound by HBM: a row is read once and its gradient written once; about 10 operations per logit.
#include "kernels.h"
#include "seq_common.cuh"

namespace simx {

using namespace seq;

namespace {

constexpr int kRowThreads = 256;
constexpr int kMaxParts = 2432;  // blocks that leave partial sums of the statistics

template <class T>
__device__ __forceinline__ const T* row_of(const void* p, int64_t i, int64_t ld) {
  return static_cast<const T*>(p) + i * ld;
}

// log pi(token) = (x_a - m) / T - log s as the unevaluated sum hi + lo.  A log probability near -11 has
// a unit in the last place of 1e-6, while what is made of it, the difference to another one, is often
// near 0.1 and is summed over a sequence: so s = 2^e f is split (Cody & Waite), e ln 2 is subtracted with
// its rounding error kept (Knuth's two-sum), and lo holds the rest to about 1e-8.
// lo also takes out two errors of s that have the same sign in every row: k = log2(e) / T was rounded to
// fp32 (d log s / d(1 / T) is the mean of x - m, so that is dk of it), and ex2 gives every term but the
// largest (2^0, exact) a little less than its value: 5.1e-8 of it in the mean, measured over [-24, 0] and
// the same within 2e-9 in every stretch of 3 of it.
constexpr float kEx2Short = 5.1e-8f;
struct LogP {
  float hi, lo;   // log pi(token)
  float logs;     // log s, rounded
  float mean;     // mean of x - m under pi
  __device__ __forceinline__ float value() const { return __fadd_rn(hi, lo); }
  __device__ __forceinline__ float minus(float y) const { return __fadd_rn(__fsub_rn(hi, y), lo); }
};
template <class Args>
__device__ __forceinline__ LogP log_prob(const Args& A, float xa, const Part& P) {
  LogP o;
  o.mean = __fdiv_rn(P.t, P.s);
  const int u = __float_as_int(P.s);  // s >= 1, or NaN, or 0 (then x_a - m is NaN)
  const int e = (u - 0x3F3504F3) >> 23;
  const float f = __int_as_float(u - (int)((uint32_t)e << 23));  // in [sqrt(1/2), sqrt(2))
  const float eh = __fmul_rn((float)e, kLn2Hi);                  // exact
  const float fix = __fmaf_rn(-A.dk, o.mean, __fmul_rn(kEx2Short, __fsub_rn(1.0f, rcp(P.s))));
  const float el = __fadd_rn(__fmaf_rn((float)e, kLn2Lo, __fadd_rn(logf(f), fix)), __fsub_rn(P.s, P.s));
  o.logs = __fadd_rn(eh, el);
  const float d = __fsub_rn(xa, P.m);
  const float a = __fmul_rn(d, A.inv_t);
  const float ae = __fmaf_rn(d, A.inv_t_lo, __fmaf_rn(d, A.inv_t, -a));
  o.hi = __fsub_rn(a, eh);
  const float b = __fsub_rn(o.hi, a);
  const float he = __fsub_rn(__fsub_rn(a, __fsub_rn(o.hi, b)), __fadd_rn(eh, b));
  o.lo = __fsub_rn(fabsf(o.hi) < inf() ? __fadd_rn(he, ae) : 0.0f, el);
  return o;
}

// What a row's terms need besides the sums.
struct RowOut {
  float c, u;       // coefficients of the gradient, both over T
  float H, logs;
};

// The terms of a token of weight w: the sums' values in terms[5] (fp64: {policy, kl, entropy,
// clipped} in 1..4), the gradient's coefficients in the result.
__device__ RowOut token_terms(const TokenArgs& A, int64_t i, float w, float xa, Part P, double (&terms)[5]) {
  RowOut o;
  const float it = A.inv_t;
  const LogP l = log_prob(A, xa, P);
  o.logs = l.logs;
  o.H = __fsub_rn(l.logs, __fmul_rn(l.mean, it));
  const float lp = l.value();
  float c = 0.0f;
  if (A.adv) {
    const float adv = A.adv[i];
    const float rho = A.logp_old ? expf(l.minus(A.logp_old[i])) : (lp == lp ? 1.0f : lp);
    const float a = __fmul_rn(rho, adv);
    const float b = __fmul_rn(fminf(fmaxf(rho, A.lo), A.hi), adv);
    const bool clipped = b < a;
    terms[1] += -(double)w * (double)(clipped ? b : a);
    if (clipped) terms[4] += (double)w;
    c = clipped ? 0.0f : -a;
  }
  if (lp != lp) c = lp;
  if (A.logp_ref) {
    const float d = -l.minus(A.logp_ref[i]);
    const float em = expm1f(d);
    terms[2] += (double)w * (double)__fsub_rn(em, d);
    c = __fmaf_rn(-A.c_kl, em, c);
  }
  terms[3] += (double)w * (double)o.H;
  o.c = __fmul_rn(__fmul_rn(c, w), it);
  o.u = __fmul_rn(__fmul_rn(w, A.c_entropy), it);
  if (A.logp) A.logp[i] = lp;
  if (A.entropy) A.entropy[i] = o.H;
  return o;
}

__device__ __forceinline__ float weight_of(const TokenArgs& A, int64_t i) {
  return A.weight ? A.weight[i] : A.w_all;
}

// Maximum and sums of a row by a block, on every thread.  sh: 3 floats per warp.
template <class T>
__device__ Part row_sums_loop(const T* x, int V, float k, float* sh) {
  const int tid = threadIdx.x, warps = kRowThreads / 32;
  float m = -inf();
  for (int j = tid; j < V; j += kRowThreads) m = fmaxf(m, widen(x[j]));
  m = max_lanes(m);
  if ((tid & 31) == 0) sh[tid / 32] = m;
  __syncthreads();
  for (int q = 0; q < warps; ++q) m = fmaxf(m, sh[q]);
  Part p{m, 0.0f, 0.0f};
  for (int j = tid; j < V; j += kRowThreads) p.s = __fadd_rn(p.s, part_term(widen(x[j]), m, k, p.t));
  p.s = sum_lanes(p.s);
  p.t = sum_lanes(p.t);
  if ((tid & 31) == 0) {
    sh[warps + tid / 32] = p.s;
    sh[2 * warps + tid / 32] = p.t;
  }
  __syncthreads();
  p.s = p.t = 0.0f;
  for (int q = 0; q < warps; ++q) {
    p.s = __fadd_rn(p.s, sh[warps + q]);
    p.t = __fadd_rn(p.t, sh[2 * warps + q]);
  }
  return p;
}

// Any vocabulary: a block per row, passes for the maximum, the sums and the gradient.
template <class T>
__global__ void __launch_bounds__(kRowThreads) k_token_loop(TokenArgs A) {
  __shared__ float sh[3 * kRowThreads / 32];
  __shared__ RowOut so;
  const int tid = threadIdx.x;
  const int V = (int)A.V;
  double terms[5] = {0.0, 0.0, 0.0, 0.0, 0.0};
  for (int64_t i = blockIdx.x; i < A.n; i += gridDim.x) {
    const T* x = row_of<T>(A.x, i, A.ld);
    T* g = A.g ? static_cast<T*>(A.g) + i * A.g_ld : nullptr;
    const float w = weight_of(A, i);
    if (w == 0.0f) {
      if (g)
        for (int j = tid; j < V; j += kRowThreads) g[j] = narrow<T>(0.0f);
      if (tid == 0) {
        if (A.logp) A.logp[i] = 0.0f;
        if (A.entropy) A.entropy[i] = 0.0f;
      }
      continue;
    }
    const Part p = row_sums_loop(x, V, A.k, sh);
    if (tid == 0) {
      const int64_t a = A.action[i];
      const float xa = a >= 0 && a < A.V ? widen(x[a]) : nan();
      so = token_terms(A, i, w, xa, p, terms);
    }
    __syncthreads();
    if (g) {
      const RowOut o = so;
      const int64_t a = A.action[i];
      const float is = __fdiv_rn(1.0f, p.s);
      for (int j = tid; j < V; j += kRowThreads) {
        const float d = __fsub_rn(widen(x[j]), p.m);
        const float e = ex2(__fmul_rn(d, A.k));
        const float pj = __fmul_rn(e, is);
        float v = __fmul_rn(pj, -o.c);
        if (o.u != 0.0f) {  // log p held finite: where it is -inf, p is 0
          const float lpj = fmaxf(__fmaf_rn(d, A.inv_t, -o.logs), -kMost);
          v = __fmaf_rn(o.u, __fmul_rn(pj, __fadd_rn(lpj, o.H)), v);
        }
        if (j == a) v = __fadd_rn(v, o.c);
        g[j] = narrow<T>(v);
      }
    }
    __syncthreads();
  }
  if (tid == 0)
    for (int q = 1; q < 5; ++q) A.part[(int64_t)blockIdx.x * 4 + q - 1] = terms[q];
}

// The statistics from the blocks' partial sums, in a fixed order.
__global__ void __launch_bounds__(256) k_token_stats(TokenArgs A, int parts) {
  __shared__ double sh[8][4];
  pdl_wait();
  double v[4] = {0.0, 0.0, 0.0, 0.0};
  for (int b = threadIdx.x; b < parts; b += 256)
    for (int q = 0; q < 4; ++q) v[q] += A.part[(int64_t)b * 4 + q];
  for (int q = 0; q < 4; ++q)
    for (int d = 16; d > 0; d /= 2) v[q] += __shfl_xor_sync(0xffffffffu, v[q], d);
  if ((threadIdx.x & 31) == 0)
    for (int q = 0; q < 4; ++q) sh[threadIdx.x / 32][q] = v[q];
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w)
      for (int q = 0; q < 4; ++q) v[q] += sh[w][q];
    A.stats[0] = (float)(v[0] + (double)A.c_kl * v[1] - (double)A.c_entropy * v[2]);
    for (int q = 0; q < 4; ++q) A.stats[1 + q] = (float)v[q];
  }
}

// Preference loss, first pass: log pi(token) - logp_ref and the softmax's statistics of every row
// that counts (rows outside all sequences are masked rows).
__device__ __forceinline__ int64_t clamp_row(int64_t v, int64_t n) { return v < 0 ? 0 : v > n ? n : v; }

// The sequence that holds row i, or -1: the last q with seq_start[q] <= i, if i is before its end.
__device__ __forceinline__ int64_t seq_of(const PrefArgs& A, int64_t i) {
  int64_t lo = -1, hi = 2 * A.pairs;  // start[lo] <= i < start[hi], with sentinels
  while (hi - lo > 1) {
    const int64_t mid = (lo + hi) / 2;
    if (A.start[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo >= 0 && i < A.start[lo + 1] ? lo : -1;
}

template <class T>
__global__ void __launch_bounds__(kRowThreads) k_pref_rows(PrefArgs A) {
  __shared__ float sh[3 * kRowThreads / 32];
  const int tid = threadIdx.x;
  const int V = (int)A.V;
  for (int64_t i = blockIdx.x; i < A.n; i += gridDim.x) {
    if ((A.mask && !A.mask[i]) || seq_of(A, i) < 0) continue;
    const T* x = row_of<T>(A.x, i, A.ld);
    const Part p = row_sums_loop(x, V, A.k, sh);
    if (tid == 0) {
      const int64_t a = A.token[i];
      const float xa = a >= 0 && a < A.V ? widen(x[a]) : nan();
      const LogP l = log_prob(A, xa, p);
      A.row_m[i] = p.m;
      A.row_is[i] = __fdiv_rn(1.0f, p.s);
      A.row_d[i] = A.logp_ref ? l.minus(A.logp_ref[i]) : l.value();
    }
    __syncthreads();
  }
}

// A block per pair: both ratios (fp64, fixed order), the margin, the loss terms and the rows'
// coefficient.
__global__ void __launch_bounds__(256) k_pref_pairs(PrefArgs A) {
  __shared__ double sh[2][8];
  const int tid = threadIdx.x;
  for (int64_t p = blockIdx.x; p < A.pairs; p += gridDim.x) {
    for (int h = 0; h < 2; ++h) {
      const int64_t b = clamp_row(A.start[2 * p + h], A.n), e = clamp_row(A.start[2 * p + h + 1], A.n);
      double v = 0.0;
      for (int64_t i = b + tid; i < e; i += 256)
        if (!A.mask || A.mask[i]) v += (double)A.row_d[i];
      for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
      if ((tid & 31) == 0) sh[h][tid / 32] = v;
    }
    __syncthreads();
    if (tid == 0) {
      double r[2] = {0.0, 0.0};
      for (int h = 0; h < 2; ++h)
        for (int w = 0; w < 8; ++w) r[h] += sh[h][w];
      const double h = (double)A.beta * (r[0] - r[1]);
      const float hf = (float)h;
      const double soft = log1p(exp(-fabs(h)));  // softplus(-|h|)
      const double lneg = fmax(-h, 0.0) + soft, lpos = fmax(h, 0.0) + soft;
      const float w = A.weight ? A.weight[p] : A.w_all;
      const double sg = 1.0 / (1.0 + exp(-h));
      const double eps = (double)A.smoothing;
      A.coef[p] = (float)((double)w * (double)A.beta * (sg - (1.0 - eps)) * (double)A.inv_t);
      A.part[3 * p] = (double)w * ((1.0 - eps) * lneg + (eps > 0.0 ? eps * lpos : 0.0));
      A.part[3 * p + 1] = h > 0.0 ? (double)w : 0.0;
      A.part[3 * p + 2] = (double)w * h;
      if (A.ratio) {
        A.ratio[2 * p] = (float)r[0];
        A.ratio[2 * p + 1] = (float)r[1];
      }
      if (A.margin) A.margin[p] = hf;
    }
    __syncthreads();
  }
}

// Second pass: the gradient rows; block 0 also sums the statistics.
template <class T>
__global__ void __launch_bounds__(kRowThreads) k_pref_grad(PrefArgs A) {
  const int tid = threadIdx.x;
  const int V = (int)A.V;
  if (blockIdx.x == 0 && tid < 32) {
    double v[3] = {0.0, 0.0, 0.0};
    for (int64_t p = tid; p < A.pairs; p += 32)
      for (int q = 0; q < 3; ++q) v[q] += A.part[3 * p + q];
    for (int q = 0; q < 3; ++q)
      for (int d = 16; d > 0; d /= 2) v[q] += __shfl_xor_sync(0xffffffffu, v[q], d);
    if (tid == 0)
      for (int q = 0; q < 3; ++q) A.stats[q] = (float)v[q];
  }
  if (!A.g) return;
  for (int64_t i = blockIdx.x; i < A.n; i += gridDim.x) {
    T* g = static_cast<T*>(A.g) + i * A.g_ld;
    const int64_t s = (A.mask && !A.mask[i]) ? -1 : seq_of(A, i);
    if (s < 0) {
      for (int j = tid; j < V; j += kRowThreads) g[j] = narrow<T>(0.0f);
      continue;
    }
    const T* x = row_of<T>(A.x, i, A.ld);
    const float m = A.row_m[i], is = A.row_is[i];
    const float c = (s & 1) ? -A.coef[s >> 1] : A.coef[s >> 1];
    const int64_t a = A.token[i];
    const float bad = a >= 0 && a < A.V ? 0.0f : nan();
    for (int j = tid; j < V; j += kRowThreads) {
      const float pj = __fmul_rn(ex2(__fmul_rn(__fsub_rn(widen(x[j]), m), A.k)), is);
      float v = __fmul_rn(pj, -c);
      if (j == a) v = __fadd_rn(v, c);
      g[j] = narrow<T>(__fadd_rn(v, bad));
    }
  }
}

int row_blocks(int64_t n) {
  const int64_t most = (int64_t)sm_count() * 8;
  const int64_t b = n < most ? n : most;
  return (int)(b < kMaxParts ? b : kMaxParts);
}

template <class T>
void token_rows(const TokenArgs& a, int blocks, cudaStream_t s) {
  k_token_loop<T><<<blocks, kRowThreads, 0, s>>>(a);
  count_launches(1);
}

size_t round16(size_t b) { return (b + 15) & ~(size_t)15; }

}  // namespace

size_t token_workspace_bytes(int64_t) { return (size_t)kMaxParts * 4 * sizeof(double); }

cudaError_t launch_token_loss(TokenArgs a, void* ws, cudaStream_t s) {
  a.part = static_cast<double*>(ws);
  int blocks = 0;
  if (a.n > 0) {
    blocks = row_blocks(a.n);
    if (a.dtype == SIMX_F32) token_rows<float>(a, blocks, s);
    else token_rows<__nv_bfloat16>(a, blocks, s);
  }
  k_token_stats<<<1, 256, 0, s>>>(a, blocks);
  count_launches(1);
  return cudaGetLastError();
}

size_t pref_workspace_bytes(int64_t n, int64_t pairs) {
  return 3 * round16((size_t)n * sizeof(float)) + round16((size_t)pairs * sizeof(float)) +
         (size_t)pairs * 3 * sizeof(double) + 16;
}

cudaError_t launch_pref_loss(PrefArgs a, void* ws, cudaStream_t s) {
  char* w = static_cast<char*>(ws);
  const size_t rows = round16((size_t)a.n * sizeof(float));
  a.row_m = reinterpret_cast<float*>(w);
  a.row_is = reinterpret_cast<float*>(w + rows);
  a.row_d = reinterpret_cast<float*>(w + 2 * rows);
  a.coef = reinterpret_cast<float*>(w + 3 * rows);
  a.part = reinterpret_cast<double*>(w + 3 * rows + round16((size_t)a.pairs * sizeof(float)));
  const int blocks = row_blocks(a.n > 0 ? a.n : 1);
  const bool f32 = a.dtype == SIMX_F32;
  if (a.n > 0 && a.pairs > 0) {
    if (f32) k_pref_rows<float><<<blocks, kRowThreads, 0, s>>>(a);
    else k_pref_rows<__nv_bfloat16><<<blocks, kRowThreads, 0, s>>>(a);
    count_launches(1);
  }
  if (a.pairs > 0) {
    const int64_t most = (int64_t)sm_count() * 8;
    k_pref_pairs<<<(int)(a.pairs < most ? a.pairs : most), 256, 0, s>>>(a);
    count_launches(1);
  }
  if (f32) k_pref_grad<float><<<blocks, kRowThreads, 0, s>>>(a);
  else k_pref_grad<__nv_bfloat16><<<blocks, kRowThreads, 0, s>>>(a);
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace simx

// seq_loss.cu — losses over a vocabulary, from logits to the logits' gradient: the clipped policy
// loss with its KL and entropy terms (Sec. 4.3's PPO objective on tokens), and the preference loss
// on pairs of sequences.
//
// Per row of logits x with temperature T: m = max x, s = sum e^((x - m) / T),
// log pi(a) = (x_a - m) / T - log s, H = log s - (1 / s) sum e^((x - m) / T) (x - m) / T, and with the
// row's coefficient c = dL / d log pi(a) and entropy coefficient u = w c_entropy
//   dL / dx_j = (c (delta_ja - p_j) + u p_j (log p_j + H)) / T.
// Bound by HBM: a row is read once and its gradient written once; about 10 operations per logit.
// Measured on one GB300 (floors at 6783 GB/s): token loss of 8192 x 131,072 bf16, an eighth of the rows
// without weight, 739 us (594), 1021 x 50,001 fp32 76 (53), 8 x 131,072 bf16 8 and 8192 x 48 fp32 4.5 on the
// GPU, where a call's arguments take the host 13; preference loss of 32 pairs of up to 512 tokens over
// 32,768 bf16 logits 467 (297, or 442 with the second read that its coefficients need).
#include <algorithm>

#include "kernels.h"
#include "seq_common.cuh"

namespace simx {

using namespace seq;

namespace {

constexpr int kRowThreads = 256, kStatThreads = 256;
constexpr int kMaxParts = 4864;  // blocks that leave partial sums of the statistics

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
  float H;        // entropy
  bool never;     // the token's logit is -inf
  __device__ __forceinline__ float value() const { return __fadd_rn(hi, lo); }
  __device__ __forceinline__ float minus(float y) const { return __fadd_rn(__fsub_rn(hi, y), lo); }
};
// a + ae = (x_token - ref) / T, s = sum e^((x - ref) / T), mean = its mean exponent (natural), dmean =
// the mean of what dk multiplies.
__device__ __forceinline__ LogP log_prob(float a, float ae, float s, float mean, float dmean, float dk) {
  LogP o;
  const int u = __float_as_int(s);  // positive, or NaN, or 0 (then a is NaN)
  const int e = (u - 0x3F3504F3) >> 23;
  const float f = __int_as_float(u - (int)((uint32_t)e << 23));  // in [sqrt(1/2), sqrt(2))
  const float eh = __fmul_rn((float)e, kLn2Hi);                  // exact
  const float fix = __fmaf_rn(-dk, dmean, kEx2Short);
  const float el = __fadd_rn(__fmaf_rn((float)e, kLn2Lo, __fadd_rn(logf(f), fix)), __fsub_rn(s, s));
  o.logs = __fadd_rn(eh, el);
  o.H = __fsub_rn(o.logs, mean);
  o.never = false;
  o.hi = __fsub_rn(a, eh);
  const float b = __fsub_rn(o.hi, a);
  const float he = __fsub_rn(__fsub_rn(a, __fsub_rn(o.hi, b)), __fadd_rn(eh, b));
  o.lo = __fsub_rn(fabsf(o.hi) < inf() ? __fadd_rn(he, ae) : 0.0f, el);
  return o;
}
// With ref = m, the row's maximum (or another value of the size of its logits).
template <class Args>
__device__ __forceinline__ LogP log_prob(const Args& A, float xa, const Part& P) {
  const float mean = __fdiv_rn(P.t, P.s), d = __fsub_rn(xa, P.m);
  const float a = __fmul_rn(d, A.inv_t);
  const float ae = __fmaf_rn(d, A.inv_t_lo, __fmaf_rn(d, A.inv_t, -a));
  // the largest term is exact
  LogP o = log_prob(a, __fmaf_rn(kEx2Short, rcp(P.s), ae), P.s, __fmul_rn(mean, A.inv_t), mean, A.dk);
  o.never = xa == -inf();
  return o;
}

// What a row's terms need besides the sums.
struct RowOut {
  float c, u;       // coefficients of the gradient, both over T
  float H, logs, lp;
};

__device__ __forceinline__ void write_row_values(const TokenArgs& A, int64_t i, float lp, float H) {
  if (A.logp) A.logp[i] = lp;
  if (A.entropy) A.entropy[i] = H;
}

// The terms of a token of weight w: {policy, kl, entropy, clipped} are added to `terms` (a thread's sum over
// its few rows; the blocks' sums are joined with their rounding errors kept), the gradient's coefficients are the result.
struct RowIn {
  float adv, old, ref;
};
__device__ __forceinline__ RowIn row_in(const TokenArgs& A, int64_t i) {
  return RowIn{A.adv ? A.adv[i] : 0.0f, A.logp_old ? A.logp_old[i] : 0.0f, A.logp_ref ? A.logp_ref[i] : 0.0f};
}
__device__ __forceinline__ RowOut token_terms(const TokenArgs& A, const RowIn& in, float w, const LogP& l, float (&terms)[4]) {
  RowOut o;
  const float it = A.inv_t;
  o.logs = l.logs;
  o.H = l.H;
  const float lp = l.value();
  float c = 0.0f;
  if (A.adv) {
    const float d = A.logp_old ? l.minus(in.old) : 0.0f;
    const float rho = A.logp_old ? expf(d) : (lp == lp ? 1.0f : lp);
    // a ratio beyond fp32 is infinite here, but finite: times an advantage of 0 it is 0
    const float a = in.adv == 0.0f && rho == inf() && d < inf() ? 0.0f : __fmul_rn(rho, in.adv);
    const float b = __fmul_rn(fminf(fmaxf(rho, A.lo), A.hi), in.adv);
    const bool clipped = b < a;
    terms[0] = __fmaf_rn(-w, clipped ? b : a, terms[0]);
    if (clipped) terms[3] = __fadd_rn(terms[3], w);
    c = clipped ? 0.0f : -a;
  }
  if (lp != lp) c = lp;
  if (A.logp_ref) {
    const float d = -l.minus(in.ref);
    const float em = expm1f(d);
    terms[1] = __fmaf_rn(w, em < inf() ? __fsub_rn(em, d) : em, terms[1]);  // both infinite where lp is -inf
    if (A.c_kl != 0.0f) c = __fmaf_rn(-A.c_kl, em, c);  // em may be beyond fp32
  }
  // c would come to a logit of -inf, whose gradient is 0: L has none there, unless it does not move with lp
  if (l.never && c != 0.0f) c = nan();
  terms[2] = __fmaf_rn(w, o.H, terms[2]);
  o.c = __fmul_rn(__fmul_rn(c, w), it);
  o.u = __fmul_rn(__fmul_rn(w, A.c_entropy), it);
  o.lp = lp;
  return o;
}

__device__ __forceinline__ float weight_of(const TokenArgs& A, int64_t i) {
  return A.weight ? A.weight[i] : A.w_all;
}

constexpr float kLn2 = (float)0.69314718055994530942;
constexpr float kLn2Rest = (float)(0.69314718055994530942 - (double)(float)0.69314718055994530942);
constexpr float kFar = -1e30f;  // stands for arg = -inf where it is multiplied: 2^kFar is 0


template <class T>
struct VecOf {
  static constexpr int N = 16 / (int)sizeof(T);
};

__device__ __forceinline__ void unpack(const uint4& q, float (&v)[4], float) {
  v[0] = __uint_as_float(q.x);
  v[1] = __uint_as_float(q.y);
  v[2] = __uint_as_float(q.z);
  v[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ void unpack(const uint4& q, float (&v)[8], __nv_bfloat16) {
  const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 pack(const float (&v)[4], float) {
  return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 pack(const float (&v)[8], __nv_bfloat16) {
  return make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
}

// Elements between the 16-byte boundary at or below p and p.
template <class T>
__device__ __forceinline__ int phase_of(const T* p) {
  return (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
}

// Small vocabularies: G lanes per row, NI logits per lane (logit lane + G i), every lane of the group
// with the row's terms.  8192 x 48 fp32: 4.5 us with the statistics, by latency; 65,536 x 500 bf16 83 us,
// by the instructions of a row's terms and its single-element loads.
template <class T, int G, int NI>
__global__ void __launch_bounds__(kRowThreads) k_token_lanes(TokenArgs A) {
  __shared__ float sh[kRowThreads / 32][4];
  pdl_trigger();
  const int lane = threadIdx.x & (G - 1), V = (int)A.V;
  const int64_t groups = (int64_t)gridDim.x * (kRowThreads / G);
  const int64_t rounds = (A.n + groups - 1) / groups;  // the same for every lane: shuffles need all of them
  float terms[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int64_t q = 0; q < rounds; ++q) {
    const int64_t i = q * groups + ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) / G;
    const bool live = i < A.n;
    const float w = live ? weight_of(A, i) : 0.0f;
    const bool on = w != 0.0f;
    const T* x = row_of<T>(A.x, live ? i : 0, A.ld);
    float r[NI];
    float m = -inf();
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int e = lane + G * j;
      r[j] = live && e < V ? widen(x[e]) : -inf();
    }
    // everything the row takes is on its way at once, what depends on the weight included
    const int64_t a = live ? A.action[i] : -1;
    const RowIn ri = live ? row_in(A, i) : RowIn{0.0f, 0.0f, 0.0f};
    float xa = 0.0f;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      m = fmaxf(m, r[j]);
      if (lane + G * j == a) xa = r[j];  // one lane of the group at most, if a < V
    }
#pragma unroll
    for (int d = G / 2; d > 0; d /= 2) {
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
      const float other = __shfl_xor_sync(0xffffffffu, xa, d);
      xa = other != 0.0f ? other : xa;
    }
    if (a < 0 || a >= A.V) xa = nan();
    Part p{m, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < NI; ++j) p.s = __fadd_rn(p.s, part_term(r[j], m, A.k, p.t));
#pragma unroll
    for (int d = G / 2; d > 0; d /= 2) {
      p.s = __fadd_rn(p.s, __shfl_xor_sync(0xffffffffu, p.s, d));
      p.t = __fadd_rn(p.t, __shfl_xor_sync(0xffffffffu, p.t, d));
    }
    if (!live) continue;
    RowOut o{0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (on) o = token_terms(A, ri, w, log_prob(A, xa, p), terms);
    if (lane == 0) write_row_values(A, i, o.lp, o.H);
    if (A.g) {
      T* g = static_cast<T*>(A.g) + i * A.g_ld;
      const float is = __fdiv_rn(1.0f, p.s);
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int e = lane + G * j;
        const float d = __fsub_rn(r[j], p.m);
        const float pj = __fmul_rn(ex2(__fmul_rn(d, A.k)), is);
        float f = __fmul_rn(pj, -o.c);
        if (o.u != 0.0f) {
          const float lpj = fmaxf(__fmaf_rn(d, A.inv_t, -o.logs), -kMost);
          f = __fmaf_rn(o.u, __fmul_rn(pj, __fadd_rn(lpj, o.H)), f);
        }
        if (e == a) f = __fadd_rn(f, o.c);
        if (e < V) g[e] = narrow<T>(on ? f : 0.0f);
      }
    }
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float v = sum_lanes(lane == 0 ? terms[q] : 0.0f);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x / 32][q] = v;
  }
  __syncthreads();
  if (threadIdx.x < 4) {
    float b = 0.0f;
    for (int k = 0; k < kRowThreads / 32; ++k) b = __fadd_rn(b, sh[k][threadIdx.x]);
    A.part[(int64_t)blockIdx.x * 4 + threadIdx.x] = b;
  }
}

// Maximum and sums of a row by a block of NT threads, on every thread.  sh: 3 floats per warp.
template <class T, int NT>
__device__ __noinline__ Part row_sums_loop(const T* x, int V, float k, float* sh) {
  const int tid = threadIdx.x, warps = NT / 32;
  float m = -inf();
  for (int j = tid; j < V; j += NT) m = fmaxf(m, widen(x[j]));
  m = max_lanes(m);
  if ((tid & 31) == 0) sh[tid / 32] = m;
  __syncthreads();
  for (int q = 0; q < warps; ++q) m = fmaxf(m, sh[q]);
  Part p{m, 0.0f, 0.0f};
  for (int j = tid; j < V; j += NT) p.s = __fadd_rn(p.s, part_term(widen(x[j]), m, k, p.t));
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

// One gradient element (without the token's own c) from the row's maximum and sums.
template <class Args>
__device__ __forceinline__ float grad_far(float x, const Args& A, const Part& p, const RowOut& o) {
  const float d = __fsub_rn(x, p.m);
  const float pj = __fdiv_rn(ex2(__fmul_rn(d, A.k)), p.s);
  const float lpj = fmaxf(__fmaf_rn(d, A.inv_t, -o.logs), -kMost);  // log p held finite: where it is -inf, p is 0
  return __fmaf_rn(o.u, __fmul_rn(pj, __fadd_rn(lpj, o.H)), __fmul_rn(pj, -o.c));
}
// The gradient of a row from its maximum and sums, by a block of NT threads.
template <class T, int NT, class Args>
__device__ __noinline__ void row_grad_loop(const T* x, T* g, int V, const Args& A, const Part& p, const RowOut& o, int64_t a) {
  for (int j = threadIdx.x; j < V; j += NT) {
    const float v = grad_far(widen(x[j]), A, p, o);
    g[j] = narrow<T>(j == a ? __fadd_rn(v, o.c) : v);
  }
}

// ---------------------------------------------------------------------------
// Rows streamed.  A block per row reads it twice: for the sums, from HBM, and for the gradient, from L2
// (two rows per SM are 78 MB at 131,072 bf16 logits, of 129).  One pass takes the sums: each thread keeps
// e = 2^(x k - c) with an integer reference c of its own, raised when a logit passes it, so that sums move
// to another reference by an exact power of two.  No block waits for another one, which is what a row in
// a cluster's registers costs: it is the kernel of calls with enough rows to fill the GPU.  8192 rows of
// 131,072 bf16 logits: 739 us, 5.4 TB/s of what the call cannot do without; DRAM moves 8 % more than that,
// and what is left is the latency of a row's loads (warps wait for them 8 cycles per instruction).  The
// same rows each in a cluster's registers took 1463 us.  A block takes one row, or few: the rows without
// weight then leave their room to others (persistent blocks: 797).
// ---------------------------------------------------------------------------
constexpr int kChunk = 4;  // vectors per thread and step
constexpr float kNone = -1e30f;  // reference of a thread that has seen nothing

// 2^d for an integer d <= 0, exactly.
__device__ __forceinline__ float pow2(float d) {
  return __int_as_float((127 + (int)fmaxf(d, -127.0f)) << 23);
}

struct Stream {
  float c, s, t;  // sums of e = 2^(x k - c) and of e (x k - c)
  __device__ __forceinline__ void raise(float to) {  // to >= c
    const float d = __fsub_rn(c, to), f = pow2(d);
    t = __fmul_rn(f, __fmaf_rn(d, s, t));  // s = 0 while c is kNone
    s = __fmul_rn(f, s);
    c = to;
  }
  template <int M>
  __device__ __forceinline__ void add(const float (&x)[M], float k) {
    float m = x[0];
#pragma unroll
    for (int j = 1; j < M; ++j) m = fmaxf(m, x[j]);
    const float top = __fmul_rn(m, k);
    if (top > c) raise(ceilf(top));
    float sa = 0.0f, ta = 0.0f;
#pragma unroll
    for (int j = 0; j < M; ++j) {
      const float arg = __fmaf_rn(x[j], k, -c), e = ex2(arg);
      sa = __fadd_rn(sa, e);
      ta = __fmaf_rn(e, arg, ta);
    }
    if (ta != ta && sa == sa) {  // logits of -inf: 0 times -inf.  Their terms are 0
      ta = 0.0f;
#pragma unroll
      for (int j = 0; j < M; ++j) {
        const float arg = __fmaf_rn(x[j], k, -c);
        ta = __fmaf_rn(ex2(arg), fmaxf(arg, kFar), ta);
      }
    }
    s = __fadd_rn(s, sa);
    t = __fadd_rn(t, ta);
  }
};

// Sums of a row over the block, on every thread, with one reference.  sh: 3 floats per warp.
template <int NT>
__device__ __forceinline__ Stream stream_join(Stream v, float* sh) {
  constexpr int W = NT / 32;
  const int lane = threadIdx.x & 31, warp = (int)threadIdx.x / 32;
  v.raise(max_lanes(v.c));
  v.s = sum_lanes(v.s);
  v.t = sum_lanes(v.t);
  if (lane == 0) {
    sh[warp] = v.c;
    sh[W + warp] = v.s;
    sh[2 * W + warp] = v.t;
  }
  __syncthreads();
  Stream o{kNone, 0.0f, 0.0f};
  if (lane < W) o = Stream{sh[lane], sh[W + lane], sh[2 * W + lane]};
  o.raise(max_lanes(o.c));
  o.s = sum_lanes(o.s);
  o.t = sum_lanes(o.t);
  return o;
}

// One vector that may be partial: -inf where the row has nothing.
template <class T>
__device__ __forceinline__ void load_edge(const T* x, int V, int ph, int v, float (&f)[VecOf<T>::N]) {
#pragma unroll
  for (int j = 0; j < VecOf<T>::N; ++j) {
    const int e = v * VecOf<T>::N - ph + j;
    f[j] = e >= 0 && e < V ? widen(x[e]) : -inf();
  }
}

// A thread's sums over a row: full vectors in steps of kChunk, then the partial ones at both ends.
template <class T, int NT>
__device__ __forceinline__ Stream stream_sums(const T* x, int V, float k) {
  constexpr int N = VecOf<T>::N;
  const int ph = phase_of(x), tid = threadIdx.x;
  const uint4* g = reinterpret_cast<const uint4*>(x - ph);
  const int first = ph ? 1 : 0, last = (ph + V) / N;  // the full vectors
  Stream v{kNone, 0.0f, 0.0f};
  int i = first + tid;
  for (; i + (kChunk - 1) * NT < last; i += kChunk * NT) {
    uint4 q[kChunk];
#pragma unroll
    for (int u = 0; u < kChunk; ++u) q[u] = g[i + u * NT];
#pragma unroll
    for (int u = 0; u < kChunk; ++u) {
      float f[N];
      unpack(q[u], f, T());
      v.add(f, k);
    }
  }
  for (; i < last; i += NT) {
    float f[N];
    unpack(g[i], f, T());
    v.add(f, k);
  }
  if (tid < 2) {
    const int edge = tid == 0 ? (ph ? 0 : -1) : (last >= first && (ph + V) % N ? last : -1);
    if (edge >= 0) {
      float f[N];
      load_edge(x, V, ph, edge, f);
      v.add(f, k);
    }
  }
  return v;
}

// One gradient element from the row's streamed sums: e (arg ul + ur), or e ur.
template <bool ENT>
__device__ __forceinline__ float grad_term(float x, float k, float c, float ul, float ur) {
  const float arg = __fmaf_rn(x, k, -c);
  return __fmul_rn(ex2(arg), ENT ? __fmaf_rn(fmaxf(arg, kFar), ul, ur) : ur);
}
// Vector v of a gradient row g on the grid of phase ph, in one store if it is whole and g is on it.
template <class T>
__device__ __forceinline__ void put_vector(T* g, int ph, int V, int v, bool one, const float (&f)[VecOf<T>::N]) {
  if (one) {
    __stcs(reinterpret_cast<uint4*>(g - ph) + v, pack(f, T()));
  } else {
#pragma unroll
    for (int j = 0; j < VecOf<T>::N; ++j) {
      const int e = v * VecOf<T>::N - ph + j;
      if (e >= 0 && e < V) g[e] = narrow<T>(f[j]);
    }
  }
}
// The gradient of a row by a block of NT threads; `add` comes to logit `hot`.
template <class T, int NT, bool ENT>
__device__ __forceinline__ void stream_grad(const T* x, T* g, int V, float k, float c, float ul, float ur, int hot, float add) {
  constexpr int N = VecOf<T>::N;
  const int ph = phase_of(x), tid = threadIdx.x;
  const bool same = phase_of(g) == ph;
  const uint4* from = reinterpret_cast<const uint4*>(x - ph);
  const int first = ph ? 1 : 0, last = (ph + V) / N, nvec = (ph + V + N - 1) / N;
  const int hv = hot < 0 ? -1 : (hot + ph) / N, hj = (hot + ph) % N;
  const auto put = [&](int v, const float (&in)[N], bool whole) {
    float f[N];
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = grad_term<ENT>(in[j], k, c, ul, ur);
    if (v == hv) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j == hj) f[j] = __fadd_rn(f[j], add);
    }
    put_vector<T>(g, ph, V, v, whole && same, f);
  };
  int i = first + tid;
  for (; i + (kChunk - 1) * NT < last; i += kChunk * NT) {
    uint4 q[kChunk];
#pragma unroll
    for (int u = 0; u < kChunk; ++u) q[u] = __ldcs(from + i + u * NT);
#pragma unroll
    for (int u = 0; u < kChunk; ++u) {
      float f[N];
      unpack(q[u], f, T());
      put(i + u * NT, f, true);
    }
  }
  for (; i < last; i += NT) {
    float f[N];
    unpack(from[i], f, T());
    put(i, f, true);
  }
  if (tid < 2) {
    const int edge = tid == 0 ? (ph ? 0 : -1) : (last >= first && last < nvec ? last : -1);
    if (edge >= 0) {
      float f[N];
      load_edge(x, V, ph, edge, f);
      put(edge, f, false);
    }
  }
}

template <class T, int NT>
__device__ __forceinline__ void zero_row(T* g, int V) {
  constexpr int N = VecOf<T>::N;
  const int tid = threadIdx.x, ph = phase_of(g), first = ph ? 1 : 0, last = (ph + V) / N;
  uint4* to = reinterpret_cast<uint4*>(g - ph);
  for (int v = first + tid; v < last; v += NT) __stcs(to + v, make_uint4(0u, 0u, 0u, 0u));
  const int head = first ? min(V, N - ph) : 0, tail = max(head, last * N - ph);
  if (tid < head) g[tid] = narrow<T>(0.0f);
  if (tail + tid < V) g[tail + tid] = narrow<T>(0.0f);
}

// log pi(token) from streamed sums: (x k - c) ln 2 - log s, the product x k exact in two parts.
template <class Args>
__device__ __forceinline__ LogP log_prob(const Args& A, float xa, const Stream& v) {
  const float ph = __fmul_rn(xa, A.k), pl = __fmaf_rn(xa, A.k, -ph);
  const float h = __fsub_rn(ph, v.c), b = __fsub_rn(h, ph);
  const float l = __fadd_rn(__fsub_rn(__fsub_rn(ph, __fsub_rn(h, b)), __fadd_rn(v.c, b)), pl);
  const float a = __fmul_rn(h, kLn2);
  float ae = __fmaf_rn(h, kLn2, -a);
  ae = __fmaf_rn(l, kLn2, __fmaf_rn(h, kLn2Rest, ae));
  ae = __fmaf_rn(-A.dk, xa, ae);  // x k has k's rounding in it too
  const float mean = __fdiv_rn(v.t, v.s);
  LogP o = log_prob(a, fabsf(a) < inf() ? ae : 0.0f, v.s, __fmul_rn(mean, kLn2), __fdiv_rn(__fadd_rn(mean, v.c), A.k), A.dk);
  o.never = xa == -inf();
  return o;
}

// Whether a row's streamed sums hold: not for rows of nothing but -inf or values beyond 1e30 either way,
// and not where something is not a number; those are gone over again from their maximum.
__device__ __forceinline__ bool stream_holds(const Stream& v) {
  return v.s > 0.0f && v.s < inf() && fabsf(v.c) < 1e30f;
}

template <class T, int NT, bool ENT>
__global__ void __launch_bounds__(NT, 1024 / NT) k_token_stream(TokenArgs A) {
  __shared__ float sh[2][3 * NT / 32];
  __shared__ RowOut so;
  pdl_trigger();
  const int tid = threadIdx.x, V = (int)A.V;
  float terms[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int64_t i = blockIdx.x; i < A.n; i += gridDim.x) {
    const T* x = row_of<T>(A.x, i, A.ld);
    T* g = A.g ? static_cast<T*>(A.g) + i * A.g_ld : nullptr;
    const float w = weight_of(A, i);
    if (w == 0.0f) {
      if (g) zero_row<T, NT>(g, V);
      if (tid == 0) write_row_values(A, i, 0.0f, 0.0f);
      continue;
    }
    const int64_t a = A.action[i];
    const bool in = a >= 0 && a < A.V;
    float xa = nan();
    RowIn ri{0.0f, 0.0f, 0.0f};
    if (tid == 0) {
      if (in) xa = widen(x[a]);
      ri = row_in(A, i);
    }
    const Stream v = stream_join<NT>(stream_sums<T, NT>(x, V, A.k), sh[0]);
    const bool holds = stream_holds(v);
    Part p{0.0f, 0.0f, 0.0f};
    if (!holds) p = row_sums_loop<T, NT>(x, V, A.k, sh[1]);
    if (tid == 0) {
      so = token_terms(A, ri, w, holds ? log_prob(A, xa, v) : log_prob(A, xa, p), terms);
      write_row_values(A, i, so.lp, so.H);
    }
    __syncthreads();
    if (g) {
      const RowOut o = so;
      if (holds) {
        const float is = __fdiv_rn(1.0f, v.s);
        // ENT: p (u (log p + H) - c) = e (arg ul + ur)
        const float ul = __fmul_rn(__fmul_rn(o.u, kLn2), is);
        const float ur = __fmul_rn(ENT ? __fmaf_rn(o.u, __fsub_rn(o.H, o.logs), -o.c) : -o.c, is);
        stream_grad<T, NT, ENT>(x, g, V, A.k, v.c, ul, ur, in ? (int)a : -1, o.c);
      } else {
        row_grad_loop<T, NT>(x, g, V, A, p, o, a);
      }
    }
  }
  if (tid == 0)
    for (int q = 0; q < 4; ++q) A.part[(int64_t)blockIdx.x * 4 + q] = terms[q];
}

// ---------------------------------------------------------------------------
// Few rows of a large vocabulary: a cluster of 8 blocks per row, every block's slice in its threads'
// registers (64 logits each, 262,144 per cluster), read once; the blocks' sums meet in every block's
// shared memory.  Bound by latency: 8 rows of 131,072 bf16 logits 8 us with the statistics.
// ---------------------------------------------------------------------------
constexpr int kCluster = 8, kClusterThreads = 512, kPerThread = 64;

// Stores v at `slot` (this block's shared memory) of block `rank` of the cluster.
__device__ __forceinline__ void store_peer(float* slot, uint32_t rank, float v) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tcx::su32(slot)), "r"(rank));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory");
}

template <class T, bool ENT>
__global__ void __launch_bounds__(kClusterThreads, 1) k_token_cluster(TokenArgs A) {
  constexpr int NT = kClusterThreads, N = VecOf<T>::N, NV = kPerThread / N;
  __shared__ float sh[3 * NT / 32];
  __shared__ float peer[3][kCluster];
  __shared__ RowOut so;
  pdl_trigger();
  const uint32_t rank = cluster_rank();
  const int tid = threadIdx.x, V = (int)A.V;
  const int64_t i = blockIdx.x / kCluster;
  const T* x = row_of<T>(A.x, i, A.ld);
  T* g = A.g ? static_cast<T*>(A.g) + i * A.g_ld : nullptr;
  const int ph = phase_of(x), nvec = (ph + V + N - 1) / N, per = (nvec + kCluster - 1) / kCluster;
  const int first = (int)rank * per, last = min(first + per, nvec);
  const float w = weight_of(A, i);
  const bool on = w != 0.0f;  // the same in the whole cluster
  const auto whole = [&](int v) { return v * N >= ph && v * N - ph + N <= V; };
  const uint4* from = reinterpret_cast<const uint4*>(x - ph);
  float r[kPerThread];
  uint4 q[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int v = first + u * NT + tid;
    if (on && v < last && whole(v)) q[u] = __ldcs(from + v);
  }
  const int64_t a = on ? A.action[i] : -1;
  const bool in = a >= 0 && a < A.V;
  float xa = nan();
  RowIn ri{0.0f, 0.0f, 0.0f};
  if (tid == 0 && on) {
    if (in) xa = widen(x[a]);
    ri = row_in(A, i);
  }
  Stream t{kNone, 0.0f, 0.0f};
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int v = first + u * NT + tid;
    float f[N];
    if (on && v < last) {
      if (whole(v)) unpack(q[u], f, T());
      else load_edge(x, V, ph, v, f);
      t.add(f, A.k);
#pragma unroll
      for (int j = 0; j < N; ++j) r[u * N + j] = f[j];
    }
  }
  t = stream_join<NT>(t, sh);
  cluster_sync();  // every block runs before another one stores into its shared memory
  if (tid < kCluster) {
    store_peer(&peer[0][rank], (uint32_t)tid, t.c);
    store_peer(&peer[1][rank], (uint32_t)tid, t.s);
    store_peer(&peer[2][rank], (uint32_t)tid, t.t);
  }
  cluster_sync();
  const int lane = tid & 31;
  t = Stream{kNone, 0.0f, 0.0f};
  if (lane < kCluster) t = Stream{peer[0][lane], peer[1][lane], peer[2][lane]};
  t.raise(max_lanes(t.c));
  t.s = sum_lanes(t.s);
  t.t = sum_lanes(t.t);
  const bool holds = !on || stream_holds(t);
  Part p{0.0f, 0.0f, 0.0f};
  if (!holds) {  // every block goes over the whole row, and none writes before all have
    p = row_sums_loop<T, NT>(x, V, A.k, sh);
    cluster_sync();
  }
  float terms[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (tid == 0) {
    so = RowOut{0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (on) so = token_terms(A, ri, w, holds ? log_prob(A, xa, t) : log_prob(A, xa, p), terms);
    if (rank == 0) {
      write_row_values(A, i, so.lp, so.H);
      for (int k = 0; k < 4; ++k) A.part[i * 4 + k] = terms[k];
    }
  }
  __syncthreads();
  if (!g) return;
  const RowOut o = so;
  const float is = on && holds ? __fdiv_rn(1.0f, t.s) : 0.0f;
  const float ul = __fmul_rn(__fmul_rn(o.u, kLn2), is);
  const float ur = __fmul_rn(ENT ? __fmaf_rn(o.u, __fsub_rn(o.H, o.logs), -o.c) : -o.c, is);
  const bool same = phase_of(g) == ph;
  const int hv = in ? ((int)a + ph) / N : -1, hj = in ? ((int)a + ph) % N : 0;
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int v = first + u * NT + tid;
    if (v >= last) continue;
    float f[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      f[j] = 0.0f;
      if (on) f[j] = holds ? grad_term<ENT>(r[u * N + j], A.k, t.c, ul, ur) : grad_far(r[u * N + j], A, p, o);
    }
    if (v == hv) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j == hj) f[j] = __fadd_rn(f[j], o.c);
    }
    put_vector<T>(g, ph, V, v, same && whole(v), f);
  }
}

// The statistics from the blocks' partial sums, in a fixed order.
__global__ void __launch_bounds__(kStatThreads) k_token_stats(TokenArgs A, int parts) {
  __shared__ Sum2 sh[kStatThreads / 32][4];
  pdl_wait();
  Sum2 v[4] = {};
  for (int b = threadIdx.x; b < parts; b += kStatThreads) {
    const float4 p = reinterpret_cast<const float4*>(A.part)[b];
    v[0].add(p.x, 0.0f);
    v[1].add(p.y, 0.0f);
    v[2].add(p.z, 0.0f);
    v[3].add(p.w, 0.0f);
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    for (int d = 16; d > 0; d /= 2)
      v[q].add(__shfl_xor_sync(0xffffffffu, v[q].hi, d), __shfl_xor_sync(0xffffffffu, v[q].lo, d));
  if ((threadIdx.x & 31) == 0)
    for (int q = 0; q < 4; ++q) sh[threadIdx.x / 32][q] = v[q];
  __syncthreads();
  if (threadIdx.x >= 32) return;
  const int q = threadIdx.x & 3;
  Sum2 t = {};
  for (int w = 0; w < kStatThreads / 32; ++w) t.add(sh[w][q].hi, sh[w][q].lo);
  // L = policy + c_kl kl - c_entropy entropy, from the two-part sums
  const float kh = __shfl_sync(0xffffffffu, t.hi, 1), kl = __shfl_sync(0xffffffffu, t.lo, 1);
  const float eh = __shfl_sync(0xffffffffu, t.hi, 2), el = __shfl_sync(0xffffffffu, t.lo, 2);
  if (threadIdx.x < 4) A.stats[1 + q] = t.value();
  if (threadIdx.x == 0) {
    const float a = __fmul_rn(A.c_kl, kh), b = __fmul_rn(-A.c_entropy, eh);
    if (A.c_kl != 0.0f) t.add(a, __fmaf_rn(A.c_kl, kl, __fmaf_rn(A.c_kl, kh, -a)));
    t.add(b, __fmaf_rn(-A.c_entropy, el, __fmaf_rn(-A.c_entropy, eh, -b)));
    A.stats[0] = t.value();
  }
}

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

// The sequence of every row, -1 for rows that are masked or in none.
__global__ void __launch_bounds__(256) k_pref_index(PrefArgs A) {
  pdl_trigger();
  const int64_t stride = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < A.n; i += stride)
    A.row_seq[i] = A.mask && !A.mask[i] ? -1 : (int)seq_of(A, i);
}

// The preference loss reads the logits twice: every row's coefficient waits for all rows of its pair.
// First pass: the log ratio and the sums of every row that counts, streamed as in the token loss.  32 pairs
// of 32,768 bf16 logits: two passes at 4.9 and 5.6 TB/s (62 % and 83 % of the DRAM's cycles).
// row_is < 0 marks a row whose row_c is its maximum (see stream_holds) instead of the sums' reference, 0 one whose
// token's logit is -inf: its gradient is NaN (as in the token loss), or zeros where its coefficient is 0.
template <class T, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) k_pref_rows(PrefArgs A) {
  __shared__ float sh[2][2][3 * NT / 32];
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, V = (int)A.V;
  int turn = 0;
  for (int64_t i = blockIdx.x; i < A.n; i += gridDim.x) {
    if (A.row_seq[i] < 0) continue;
    const T* x = row_of<T>(A.x, i, A.ld);
    float xa = nan(), ref = 0.0f;
    if (tid == 0) {
      const int64_t a = A.token[i];
      if (a >= 0 && a < A.V) xa = widen(x[a]);
      if (A.logp_ref) ref = A.logp_ref[i];
    }
    // tables of both parities: a warp may be in the next row while another still reads this one's
    float(*mine)[3 * NT / 32] = sh[turn & 1];
    ++turn;
    const Stream v = stream_join<NT>(stream_sums<T, NT>(x, V, A.k), mine[0]);
    const bool holds = stream_holds(v);
    Part p{0.0f, 0.0f, 0.0f};
    if (!holds) p = row_sums_loop<T, NT>(x, V, A.k, mine[1]);
    if (tid == 0) {
      const LogP l = holds ? log_prob(A, xa, v) : log_prob(A, xa, p);
      A.row_d[i] = A.logp_ref ? l.minus(ref) : l.value();
      A.row_c[i] = holds ? v.c : p.m;
      A.row_is[i] = l.never ? 0.0f : holds ? __fdiv_rn(1.0f, v.s) : __fdiv_rn(-1.0f, p.s);
    }
  }
}

// A block per pair: both ratios (fp64, fixed order), the margin, the loss terms and the rows'
// coefficient.
__global__ void __launch_bounds__(256) k_pref_pairs(PrefArgs A) {
  __shared__ double sh[2][8];
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x;
  for (int64_t p = blockIdx.x; p < A.pairs; p += gridDim.x) {
    for (int h = 0; h < 2; ++h) {
      const int64_t b = clamp_row(A.start[2 * p + h], A.n), e = clamp_row(A.start[2 * p + h + 1], A.n);
      double v = 0.0;
      for (int64_t i = b + tid; i < e; i += 256)
        if (A.row_seq[i] == 2 * p + h) v += (double)A.row_d[i];
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
      const bool on = w != 0.0f;  // a pair of weight 0 counts for nothing, whatever its rows hold
      A.coef[p] = (float)((double)w * (double)A.beta * (sg - (1.0 - eps)) * (double)A.inv_t);
      A.part[3 * p] = on ? (double)w * ((eps < 1.0 ? (1.0 - eps) * lneg : 0.0) + (eps > 0.0 ? eps * lpos : 0.0)) : 0.0;
      A.part[3 * p + 1] = h > 0.0 ? (double)w : 0.0;
      A.part[3 * p + 2] = on ? (double)w * h : 0.0;
      if (A.ratio) {
        A.ratio[2 * p] = (float)r[0];
        A.ratio[2 * p + 1] = (float)r[1];
      }
      if (A.margin) A.margin[p] = hf;
    }
    __syncthreads();
  }
}

// Second pass: the gradient rows, last ones first (those may still be in L2); block 0 also sums the
// statistics.
template <class T, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) k_pref_grad(PrefArgs A) {
  const int tid = threadIdx.x;
  const int V = (int)A.V;
  pdl_wait();
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
  for (int64_t i = A.n - 1 - blockIdx.x; i >= 0; i -= gridDim.x) {
    T* g = static_cast<T*>(A.g) + i * A.g_ld;
    const int q = A.pairs > 0 ? A.row_seq[i] : -1;
    if (q < 0 || (A.weight && A.weight[q >> 1] == 0.0f)) {
      zero_row<T, NT>(g, V);
      continue;
    }
    const T* x = row_of<T>(A.x, i, A.ld);
    const float c = A.row_c[i], is = A.row_is[i];
    const int64_t a = A.token[i];
    const bool in = a >= 0 && a < A.V;
    float co = (q & 1) ? -A.coef[q >> 1] : A.coef[q >> 1];
    if (is == 0.0f && co == 0.0f) {
      zero_row<T, NT>(g, V);
      continue;
    }
    if (!in || is == 0.0f) co = nan();
    if (is > 0.0f) {
      stream_grad<T, NT, false>(x, g, V, A.k, c, 0.0f, __fmul_rn(-co, is), in ? (int)a : -1, co);
    } else {
      const Part p{c, __fdiv_rn(-1.0f, is), 0.0f};
      row_grad_loop<T, NT>(x, g, V, A, p, RowOut{co, 0.0f, 0.0f, 0.0f, 0.0f}, a);
    }
  }
}

// The launches of a token loss call; parts: the partial sums that they leave.
template <class T>
cudaError_t token_cluster(const TokenArgs& a, int& parts, cudaStream_t s) {
  parts = (int)a.n;
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute at[1];
  lc.gridDim = dim3((unsigned)(parts * kCluster));
  lc.blockDim = dim3(kClusterThreads);
  lc.stream = s;
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = kCluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  lc.attrs = at;
  lc.numAttrs = 1;
  count_launches(1);
  return a.c_entropy != 0.0f && a.g ? cudaLaunchKernelEx(&lc, k_token_cluster<T, true>, a)
                                    : cudaLaunchKernelEx(&lc, k_token_cluster<T, false>, a);
}

template <class T, int NT>
cudaError_t token_stream(const TokenArgs& a, int& parts, cudaStream_t s) {
  parts = (int)std::min<int64_t>(a.n, kMaxParts);  // a row or few per block: those without weight leave room for others
  if (a.c_entropy != 0.0f && a.g) k_token_stream<T, NT, true><<<parts, NT, 0, s>>>(a);
  else k_token_stream<T, NT, false><<<parts, NT, 0, s>>>(a);
  count_launches(1);
  return cudaGetLastError();
}

template <class T, int G, int NI>
cudaError_t token_lanes(const TokenArgs& a, int& parts, cudaStream_t s) {
  const int64_t need = (a.n + kRowThreads / G - 1) / (kRowThreads / G);
  parts = (int)std::min<int64_t>(std::min<int64_t>(need, (int64_t)sm_count() * 8), kMaxParts);
  k_token_lanes<T, G, NI><<<parts, kRowThreads, 0, s>>>(a);
  count_launches(1);
  return cudaGetLastError();
}

// Threads per streamed row: 16 vectors each.  More leaves them idle between the row's barriers, fewer
// leaves the row's latency bare; GB/s of the call on one GB300 at half, this and twice as many threads
// (4 GB of logits and gradient, bf16): vocabulary 8192: 4460 / 4786 / 4462, 16,384: 4458 / 4920 / 4496,
// 32,768: 4980 / 5434 / 4732, 65,536: 4955 / 5166 / 4425.
template <class T>
int stream_threads(int64_t V) {
  const int64_t bytes = V * (int64_t)sizeof(T);
  return bytes <= 8192 ? 32 : bytes <= 16384 ? 64 : bytes <= 32768 ? 128 : bytes <= 65536 ? 256 : 512;
}

// The kernel by the vocabulary: lane groups with 8 logits a lane, then a warp with 16 (65,536 rows of 500
// bf16: 83 us against 93 streamed), then streamed rows (of 1024: 88 against 179 with 32 a lane); rows of 128
// KB and more that are too few to fill the GPU, in clusters.  On the GPU, without the host's part, clusters
// against streamed rows: 131,072 bf16 logits 8 rows 7.9 / 14.6 us, 16 rows 13.5 / 15.3, 32 rows 20.2 / 15.3; of 65,536
// 6.6 / 9.4, 11.4 / 9.4, 16.0 / 9.9; 131,072 fp32 9.1 / 22.6, 15.7 / 23.5, 23.4 / 23.6.
template <class T>
cudaError_t token_rows(const TokenArgs& a, int& parts, cudaStream_t s) {
  if (a.V <= 32) return token_lanes<T, 4, 8>(a, parts, s);
  if (a.V <= 64) return token_lanes<T, 8, 8>(a, parts, s);
  if (a.V <= 128) return token_lanes<T, 16, 8>(a, parts, s);
  if (a.V <= 256) return token_lanes<T, 32, 8>(a, parts, s);
  if (a.V <= 512) return token_lanes<T, 32, 16>(a, parts, s);
  const bool fits = a.V <= (int64_t)kCluster * kClusterThreads * kPerThread - 16 * VecOf<T>::N;
  if (fits && a.V * (int64_t)sizeof(T) >= 131072 && a.n * kCluster * 8 <= (int64_t)sm_count() * 7) return token_cluster<T>(a, parts, s);
  switch (stream_threads<T>(a.V)) {
    case 32: return token_stream<T, 32>(a, parts, s);
    case 64: return token_stream<T, 64>(a, parts, s);
    case 128: return token_stream<T, 128>(a, parts, s);
    case 256: return token_stream<T, 256>(a, parts, s);
    default: return token_stream<T, 512>(a, parts, s);
  }
}

size_t round16(size_t b) { return (b + 15) & ~(size_t)15; }

}  // namespace

size_t token_workspace_bytes(int64_t) { return (size_t)kMaxParts * 4 * sizeof(float); }

cudaError_t launch_token_loss(TokenArgs a, void* ws, cudaStream_t s) {
  a.part = static_cast<float*>(ws);
  int parts = 0;
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute at[1];
  lc.gridDim = dim3(1);
  lc.blockDim = dim3(kStatThreads);
  lc.stream = s;
  if (a.n > 0) {
    const cudaError_t e = a.dtype == SIMX_F32 ? token_rows<float>(a, parts, s) : token_rows<__nv_bfloat16>(a, parts, s);
    if (e != cudaSuccess) return e;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = 1;
  }
  count_launches(1);
  const cudaError_t e = cudaLaunchKernelEx(&lc, k_token_stats, a, parts);
  return e != cudaSuccess ? e : cudaGetLastError();
}

size_t pref_workspace_bytes(int64_t n, int64_t pairs) {
  return 4 * round16((size_t)n * sizeof(float)) + round16((size_t)pairs * sizeof(float)) +
         (size_t)pairs * 3 * sizeof(double) + 16;
}

namespace {

template <class T, int NT>
cudaError_t pref_rows(const PrefArgs& a, bool grad, cudaStream_t s) {
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  // a block per row up to a million rows: those that are masked leave room for others
  lc.gridDim = dim3((unsigned)std::max<int64_t>(1, grad && !a.g ? 1 : std::min<int64_t>(a.n, 1 << 20)));
  lc.blockDim = dim3(NT);
  lc.stream = s;
  lc.attrs = at;
  lc.numAttrs = 1;
  count_launches(1);
  return cudaLaunchKernelEx(&lc, grad ? k_pref_grad<T, NT> : k_pref_rows<T, NT>, a);
}
template <class T>
cudaError_t pref_rows(const PrefArgs& a, bool grad, cudaStream_t s) {
  switch (stream_threads<T>(a.V)) {
    case 32: return pref_rows<T, 32>(a, grad, s);
    case 64: return pref_rows<T, 64>(a, grad, s);
    case 128: return pref_rows<T, 128>(a, grad, s);
    case 256: return pref_rows<T, 256>(a, grad, s);
    default: return pref_rows<T, 512>(a, grad, s);
  }
}

}  // namespace

cudaError_t launch_pref_loss(PrefArgs a, void* ws, cudaStream_t s) {
  char* w = static_cast<char*>(ws);
  const size_t rows = round16((size_t)a.n * sizeof(float));
  a.row_c = reinterpret_cast<float*>(w);
  a.row_is = reinterpret_cast<float*>(w + rows);
  a.row_d = reinterpret_cast<float*>(w + 2 * rows);
  a.row_seq = reinterpret_cast<int*>(w + 3 * rows);
  a.coef = reinterpret_cast<float*>(w + 4 * rows);
  a.part = reinterpret_cast<double*>(w + 4 * rows + round16((size_t)a.pairs * sizeof(float)));
  const auto pass = [&](bool grad) {
    return a.dtype == SIMX_F32 ? pref_rows<float>(a, grad, s) : pref_rows<__nv_bfloat16>(a, grad, s);
  };
  cudaError_t e = cudaSuccess;
  if (a.pairs > 0) {
    const int64_t most = (int64_t)sm_count() * 8;
    if (a.n > 0) {
      k_pref_index<<<(int)std::min<int64_t>((a.n + 255) / 256, most), 256, 0, s>>>(a);
      count_launches(1);
      if ((e = pass(false)) != cudaSuccess) return e;
    }
    cudaLaunchConfig_t lc = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    lc.gridDim = dim3((unsigned)std::min(a.pairs, most));
    lc.blockDim = dim3(256);
    lc.stream = s;
    lc.attrs = at;
    lc.numAttrs = a.n > 0 ? 1 : 0;
    count_launches(1);
    if ((e = cudaLaunchKernelEx(&lc, k_pref_pairs, a)) != cudaSuccess) return e;
  }
  e = pass(true);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace simx

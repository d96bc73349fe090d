// seq_rotate.cu — root-mean-square norm of each head's query and key, with the rotation by positions in the
// same pass, and its gradient.
//
// Per row x of dim elements: r = 1 / sqrt(mean x^2 + eps), z = x r gain, and y = z with pair j turned by the
// angle 2 pi f_j, f_j = position turns_j / 2^64 modulo 1.  Backward, with d = dy turned back, u = d gain and
// xh = x r: dx = r (u - xh mean(u xh)), dgain = sum d xh; r is found again from x, which is read anyway.
//
// A row is read once (backward: with dy) and written once.  A group of lanes takes a token's heads in turn; a lane
// holds two units of 16 bytes such that both elements of each of its pairs are its own, so that turning needs no
// exchange between lanes, and the sines of its pairs, found once per token.  Single elements in place of units where
// rows lie off that grid: 301 us for 126 elements where 128 take 134.
// 32768 tokens, 32 + 8 heads of 128 in bf16: 134 us, 75 % of the copy rate, bound by HBM at 16 warps an SM (119
// registers); 16384 in fp32 111 us, 90 % (24 bytes of a thread spilled, interleaved 12).  Backward, 16384 tokens of 24 + 8
// heads of 96: 98 us, 46 %, bound by instructions (350 for the rows of four lane groups of 8, of which two lanes have no
// unit; two elements at a time, else 100 us) and registers: 72 bytes of a thread are spilled, with halves 92; in fp32 124
// us, 73 %.
#include <algorithm>

#include "kernels.h"
#include "seq_common.cuh"

namespace simx {

using namespace seq;

namespace {

constexpr int kThreads = 256;
// Of the backward pass, each of which leaves a row of sums: two to an SM.  152, 304, 608 and 1216 of them: 123, 98, 101 and
// 107 us for 16384 tokens of 24 + 8 heads of 96, 18, 19, 27 and 39 for 2000 of 8 + 8 of 64.
constexpr int kMostBlocks = 304;

// One tensor's rows: forward x -> y, backward (x, dy) -> dx.
struct Side {
  const void *x, *dy;
  void* y;
  int64_t xn, xh, dn, dh, yn, yh;
  const float* gain;
  float* dgain;
  float* part;  // workspace: [blocks][dim]
  int heads;
};

struct RotateArgs {
  Side side[2];
  int64_t n;
  int dim, pairs, interleaved;
  float eps, inv_dim;
  const int64_t *position, *turns;
  int lanes;   // lanes of a row, a power of two
  int split;   // lane groups that share a token's heads
};

// cos and sin of 2 pi phase / 2^64.  The nearest quarter turn is taken off exactly; on the rest, at most
// pi / 4, the Taylor series to x^9 and x^10 are off by less than 2e-9.
__device__ __forceinline__ void turn(uint64_t phase, float& c, float& s) {
  const uint64_t near = phase + (1ull << 61);
  const int q = (int)(near >> 62);
  const int64_t rest = (int64_t)(phase - (near & (3ull << 62)));  // in [-2^61, 2^61)
  // its upper 32 bits, in units of 2^-34 of a turn
  const float x = __fmul_rn((float)(int)(rest >> 30), 3.6572952e-10f);  // 2 pi 2^-34
  const float z = __fmul_rn(x, x);
  float sn = __fmaf_rn(z, 2.7557319e-6f, -1.9841270e-4f);
  sn = __fmaf_rn(z, sn, 8.3333333e-3f);
  sn = __fmaf_rn(z, sn, -0.16666667f);
  sn = __fmaf_rn(__fmul_rn(z, x), sn, x);
  float cs = __fmaf_rn(z, -2.7557319e-7f, 2.4801587e-5f);
  cs = __fmaf_rn(z, cs, -1.3888889e-3f);
  cs = __fmaf_rn(z, cs, 4.1666667e-2f);
  cs = __fmaf_rn(z, cs, -0.5f);
  cs = __fmaf_rn(z, cs, 1.0f);
  c = q == 0 ? cs : q == 1 ? -sn : q == 2 ? -cs : sn;
  s = q == 0 ? sn : q == 1 ? cs : q == 2 ? -sn : -cs;
}

// 1 / sqrt(v): the special-function unit's value and a Newton step, within an ulp or so.
__device__ __forceinline__ float inverse_root(float v) {
  const float r = rsqrtf(v), e = __fmaf_rn(-__fmul_rn(v, r), r, 1.0f);
  return e > -0.5f && e < 0.5f ? __fmaf_rn(__fmul_rn(0.5f, r), e, r) : r;  // 0, infinities and NaN as they come
}

__device__ __forceinline__ Pair swapped(Pair v) {
  const float2 u = halves(v);
  return pair(u.y, u.x);
}

// V elements at once, in pairs: one (and a zero), or 16 bytes.
template <class T, int V>
struct Unit {
  T v[1];
  __device__ __forceinline__ void clear() { v[0] = narrow<T>(0.0f); }
  __device__ __forceinline__ void load(const T* p) { v[0] = *p; }
  __device__ __forceinline__ void store(T* p) const { *p = v[0]; }
  __device__ __forceinline__ void get(Pair (&x)[1]) const { x[0] = pair(widen(v[0]), 0.0f); }
  __device__ __forceinline__ void set(const Pair (&x)[1]) { v[0] = narrow<T>(halves(x[0]).x); }
};
template <>
struct Unit<float, 4> {
  float4 v;
  __device__ __forceinline__ void clear() { v = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = v; }
  __device__ __forceinline__ void get(Pair (&x)[2]) const { x[0] = pair(v.x, v.y), x[1] = pair(v.z, v.w); }
  __device__ __forceinline__ void set(const Pair (&x)[2]) {
    const float2 a = halves(x[0]), b = halves(x[1]);
    v = make_float4(a.x, a.y, b.x, b.y);
  }
};
template <>
struct Unit<__nv_bfloat16, 8> {
  uint4 v;
  __device__ __forceinline__ void clear() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = v; }
  __device__ __forceinline__ void get(Pair (&x)[4]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  __device__ __forceinline__ void set(const Pair (&x)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack2(halves(x[i]).x, halves(x[i]).y);
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// T: element, V: elements of a unit, K: pairs of units a lane holds, R: rows in flight.  Unit pair p = lane +
// k * lanes is units (a, b): with halves turned against each other (p, p + pairs / V) for p < pairs / V, else the
// units that are left, two by two; else neighbours (2p, 2p + 1).  INNER: pairs are neighbours within a unit, else
// element e of unit a with element e of unit b.
template <class T, int V, int K, bool INNER, bool GRAD>
__global__ void __launch_bounds__(kThreads, K > 1 ? 1 : V == 8 || GRAD ? 2 : 3) k_rotate(const RotateArgs A) {
  constexpr int R = K == 1 && !(GRAD && V == 8) ? 2 : 1;
  const Side& S = A.side[blockIdx.y];
  extern __shared__ float sums[];  // GRAD: [groups][dim]
  const int L = A.lanes, lane = threadIdx.x & (L - 1), groups = kThreads / L, group = (int)threadIdx.x / L;
  const int units = A.dim / V;
  int ua[K], ub[K];
  constexpr int P = V > 1 ? V / 2 : 1;  // pairs of a unit
  float ga[K][V], gb[K][V];
  Pair da[K][P], db[K][P];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int p = lane + k * L, turning = A.interleaved ? 0 : A.pairs / V;
    ua[k] = p < turning ? p : 2 * p;
    ub[k] = p < turning ? p + turning : 2 * p + 1;
    if (ua[k] >= units) ua[k] = -1;
    if (ub[k] >= units) ub[k] = -1;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      ga[k][e] = ua[k] >= 0 ? S.gain ? S.gain[ua[k] * V + e] : 1.0f : 0.0f;
      gb[k][e] = ub[k] >= 0 ? S.gain ? S.gain[ub[k] * V + e] : 1.0f : 0.0f;
    }
  }
  if (GRAD)
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < P; ++e) da[k][e] = db[k][e] = 0;
  // a job is a token and one of the groups that share its heads; token and group step on without a division
  const int64_t stride = (int64_t)gridDim.x * groups, first = (int64_t)blockIdx.x * groups + group;
  const int64_t i_step = stride / A.split;
  const int h_step = (int)(stride % A.split);
  int64_t token = first / A.split;
  int part = (int)(first % A.split);
  for (;; token += i_step, part += h_step) {
    if (part >= A.split) {
      part -= A.split;
      ++token;
    }
    // all lanes of a warp stay together for the sums
    const bool on = token < A.n;
    if (!__any_sync(0xffffffffu, on)) break;
    const int64_t i = on ? token : 0;
    const int h0 = on ? part : S.heads;
    // cos and sin of the pairs: INNER unit a's V / 2, then unit b's
    float cs[K][V], sn[K][V];
    const uint64_t pos = A.pairs ? (uint64_t)A.position[i] : 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        int j = A.pairs;
        if (INNER) {
          const int u = e < V / 2 ? ua[k] : ub[k];
          if (u >= 0) j = u * (V / 2) + e % (V / 2 > 0 ? V / 2 : 1);
        } else if (A.interleaved) {
          if (ub[k] >= 0) j = ua[k] / 2;
        } else if (ua[k] >= 0 && ub[k] == ua[k] + A.pairs / V) {
          j = ua[k] * V + e;
        }
        cs[k][e] = 1.0f;
        sn[k][e] = 0.0f;
        if (j < A.pairs) turn(pos * (uint64_t)A.turns[j], cs[k][e], sn[k][e]);
      }
    }
    // (a, b) turn into a a1 + b a2 and b b1 + a b2; INNER a into a a1 + a2 times a with its neighbours exchanged.
    // Forward by the angle and times the gains, backward by the angle back.
    Pair a1[K][P], a2[K][P], b1[K][P], b2[K][P], gain_a[K][P], gain_b[K][P];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < P; ++e) {
        const int x = V > 1 ? 2 * e : 0, y = V > 1 ? 2 * e + 1 : 0;
        if constexpr (INNER) {
          const float c = cs[k][e], s = sn[k][e], c2 = cs[k][V / 2 + e], s2 = sn[k][V / 2 + e];
          a1[k][e] = GRAD ? pair(c, c) : pair(__fmul_rn(ga[k][x], c), __fmul_rn(ga[k][y], c));
          a2[k][e] = GRAD ? pair(s, -s) : pair(-__fmul_rn(ga[k][y], s), __fmul_rn(ga[k][x], s));
          b1[k][e] = GRAD ? pair(c2, c2) : pair(__fmul_rn(gb[k][x], c2), __fmul_rn(gb[k][y], c2));
          b2[k][e] = GRAD ? pair(s2, -s2) : pair(-__fmul_rn(gb[k][y], s2), __fmul_rn(gb[k][x], s2));
        } else {
          const Pair c = pair(cs[k][x], cs[k][y]), s = pair(sn[k][x], sn[k][y]), minus = pair(-sn[k][x], -sn[k][y]);
          const Pair g = pair(ga[k][x], ga[k][y]), h = pair(gb[k][x], gb[k][y]);
          a1[k][e] = GRAD ? c : mul2(g, c);
          a2[k][e] = GRAD ? s : mul2(h, minus);
          b1[k][e] = GRAD ? c : mul2(h, c);
          b2[k][e] = GRAD ? minus : mul2(g, s);
        }
        gain_a[k][e] = pair(ga[k][x], ga[k][y]);
        gain_b[k][e] = pair(gb[k][x], gb[k][y]);
      }
    auto turned = [&](int k, int e, Pair u, Pair w, Pair& a, Pair& b) {
      a = fma2(u, a1[k][e], mul2(INNER ? swapped(u) : w, a2[k][e]));
      b = fma2(w, b1[k][e], mul2(INNER ? swapped(w) : u, b2[k][e]));
    };
    const int most = __reduce_max_sync(0xffffffffu, (S.heads - h0 + A.split - 1) / A.split);
    const T* px = static_cast<const T*>(S.x) + i * S.xn + h0 * S.xh;
    const T* pd = static_cast<const T*>(S.dy) + i * S.dn + h0 * S.dh;
    T* py = static_cast<T*>(S.y) + i * S.yn + h0 * S.yh;
    const int64_t xs = A.split * S.xh, ds = A.split * S.dh, ys = A.split * S.yh;
    Unit<T, V> ra[R][K], rb[R][K], qa[R][K], qb[R][K];
    auto load = [&](int q, int r) {  // row r into place q
      const bool live = h0 + r * A.split < S.heads;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        ra[q][k].clear();
        rb[q][k].clear();
        if (GRAD) {
          qa[q][k].clear();
          qb[q][k].clear();
        }
        if (live && ua[k] >= 0) ra[q][k].load(px + r * xs + ua[k] * V);
        if (live && ub[k] >= 0) rb[q][k].load(px + r * xs + ub[k] * V);
        if (GRAD && live && ua[k] >= 0) qa[q][k].load(pd + r * ds + ua[k] * V);
        if (GRAD && live && ub[k] >= 0) qb[q][k].load(pd + r * ds + ub[k] * V);
      }
    };
#pragma unroll
    for (int q = 0; q < R; ++q) load(q, q);
    for (int r = 0; r < most; r += R) {
#pragma unroll
      for (int q = 0; q < R; ++q) {
        const bool live = h0 + (r + q) * A.split < S.heads;
        Pair xa[K][P], xb[K][P], ya[K][P], yb[K][P], va[K][P], vb[K][P], ms2 = 0, dot2 = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
          ra[q][k].get(xa[k]);
          rb[q][k].get(xb[k]);
#pragma unroll
          for (int e = 0; e < P; ++e) ms2 = fma2(xa[k][e], xa[k][e], fma2(xb[k][e], xb[k][e], ms2));
          if (GRAD) {  // dy turned back, and its product with gain and x
            Pair u[P], w[P];
            qa[q][k].get(u);
            qb[q][k].get(w);
#pragma unroll
            for (int e = 0; e < P; ++e) {
              turned(k, e, u[e], w[e], ya[k][e], yb[k][e]);
              va[k][e] = mul2(ya[k][e], gain_a[k][e]);
              vb[k][e] = mul2(yb[k][e], gain_b[k][e]);
              dot2 = fma2(va[k][e], xa[k][e], fma2(vb[k][e], xb[k][e], dot2));
            }
          }
        }
        float ms = __fadd_rn(halves(ms2).x, halves(ms2).y), dot = __fadd_rn(halves(dot2).x, halves(dot2).y);
        if constexpr (K == 1) load(q, r + q + R);  // beside what follows
        for (int d = L / 2; d > 0; d /= 2) {
          ms = __fadd_rn(ms, __shfl_xor_sync(0xffffffffu, ms, d));
          if (GRAD) dot = __fadd_rn(dot, __shfl_xor_sync(0xffffffffu, dot, d));
        }
        const float rstd = inverse_root(__fmaf_rn(ms, A.inv_dim, A.eps));
        // backward: dx = r (u - x r^2 mean(u x))
        const float back = GRAD ? __fmul_rn(__fmul_rn(rstd, rstd), __fmul_rn(dot, A.inv_dim)) : 0.0f;
        const Pair r2 = pair(rstd, rstd), back2 = pair(-back, -back);
#pragma unroll
        for (int k = 0; k < K; ++k) {
          Unit<T, V> a, b;
          Pair za[P], zb[P];
#pragma unroll
          for (int e = 0; e < P; ++e) {
            if (GRAD) {
              da[k][e] = fma2(mul2(ya[k][e], r2), xa[k][e], da[k][e]);
              db[k][e] = fma2(mul2(yb[k][e], r2), xb[k][e], db[k][e]);
              za[e] = mul2(r2, fma2(xa[k][e], back2, va[k][e]));
              zb[e] = mul2(r2, fma2(xb[k][e], back2, vb[k][e]));
            } else {
              turned(k, e, xa[k][e], xb[k][e], za[e], zb[e]);
              za[e] = mul2(za[e], r2);
              zb[e] = mul2(zb[e], r2);
            }
          }
          a.set(za);
          b.set(zb);
          if (live && ua[k] >= 0) a.store(py + (r + q) * ys + ua[k] * V);
          if (live && ub[k] >= 0) b.store(py + (r + q) * ys + ub[k] * V);
        }
        if constexpr (K > 1) load(q, r + q + R);
      }
    }
  }
  if constexpr (GRAD) {
    if (!S.dgain) return;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if (ua[k] >= 0) sums[group * A.dim + ua[k] * V + e] = e & 1 ? halves(da[k][e / 2]).y : halves(da[k][e / 2]).x;
        if (ub[k] >= 0) sums[group * A.dim + ub[k] * V + e] = e & 1 ? halves(db[k][e / 2]).y : halves(db[k][e / 2]).x;
      }
    __syncthreads();
    if ((int)threadIdx.x < A.dim) {
      float s = 0.0f;
      for (int g = 0; g < groups; ++g) s = __fadd_rn(s, sums[g * A.dim + threadIdx.x]);
      S.part[(int64_t)blockIdx.x * A.dim + threadIdx.x] = s;
    }
  }
}

__global__ void __launch_bounds__(1024) k_rotate_dgain(const float* part, int64_t blocks, int dim, float* q, float* k) {
  float* out = blockIdx.y ? k : q;
  if (out) column_sums(part + (int64_t)blockIdx.y * blocks * dim, blocks, dim, (int64_t)blockIdx.x * 32, out);
}

// ---------------------------------------------------------------------------- host

int64_t grad_blocks(int64_t n) { return std::min<int64_t>(kMostBlocks, std::max<int64_t>(1, n)); }

template <class T, int V, int K, bool INNER, bool GRAD>
cudaError_t run(const RotateArgs& a, int sides, int64_t blocks, cudaStream_t s) {
  const size_t bytes = GRAD ? (size_t)kThreads / a.lanes * a.dim * 4 : 0;  // dim <= 2 V lanes: 16 KB at most
  count_launches(1);
  k_rotate<T, V, K, INNER, GRAD><<<dim3((unsigned)blocks, (unsigned)sides), kThreads, bytes, s>>>(a);
  return cudaGetLastError();
}

bool on_grid(const void* p, int64_t sn, int64_t sh, int es) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && sn * es % 16 == 0 && sh * es % 16 == 0;
}

template <class T, bool GRAD>
cudaError_t run_type(RotateArgs& a, int sides, int64_t blocks, cudaStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  bool grid = a.dim % V == 0 && (a.interleaved ? 2 * a.pairs : a.pairs) % V == 0;
  for (int i = 0; i < sides; ++i) {
    const Side& S = a.side[i];
    grid = grid && on_grid(S.x, S.xn, S.xh, sizeof(T)) && on_grid(S.y, S.yn, S.yh, sizeof(T)) && (!GRAD || on_grid(S.dy, S.dn, S.dh, sizeof(T)));
  }
  const int pairs = (a.dim / (grid ? V : 1) + 1) / 2;  // of units
  a.lanes = 1;
  while (a.lanes < 32 && a.lanes < pairs) a.lanes *= 2;
  const int64_t groups = kThreads / a.lanes;
  // Enough lane groups for every SM, if the heads give them: 1, 64 and 512 tokens of 32 + 8 heads of 128 in 8, 8 and 21 us,
  // by a group for each token 21, 25 and 25.  With four times as many groups 2048 tokens take 61 us instead of 27: each
  // finds its sines for a head or two.
  const int heads = std::max(a.side[0].heads, sides > 1 ? a.side[1].heads : 0);
  const int64_t want = (int64_t)152 * 4 * groups;
  a.split = (int)std::max<int64_t>(1, std::min<int64_t>(heads, want / std::max<int64_t>(1, a.n)));
  const int64_t need = (a.n * a.split + groups - 1) / groups;
  if (!GRAD) blocks = std::min<int64_t>(need, (int64_t)1 << 30);
  if (grid) return a.interleaved ? run<T, V, 1, true, GRAD>(a, sides, blocks, s) : run<T, V, 1, false, GRAD>(a, sides, blocks, s);
  if (pairs <= 32) return run<T, 1, 1, false, GRAD>(a, sides, blocks, s);
  if (pairs <= 64) return run<T, 1, 2, false, GRAD>(a, sides, blocks, s);
  return run<T, 1, 4, false, GRAD>(a, sides, blocks, s);
}

RotateArgs common(const simx_head_norm& a) {
  RotateArgs r = {};
  r.n = a.n;
  r.dim = (int)a.dim;
  r.pairs = (int)a.pairs;
  r.interleaved = a.interleaved != 0;
  r.eps = a.eps;
  r.inv_dim = 1.0f / (float)a.dim;
  r.position = a.position;
  r.turns = a.turns;
  return r;
}

Side side(const simx_rows& x, const simx_rows& dy, const simx_rows& y, const float* gain, float* dgain, int64_t heads) {
  return {x.p, dy.p, y.p, x.sn, x.sh, dy.sn, dy.sh, y.sn, y.sh, gain, dgain, nullptr, (int)heads};
}

}  // namespace

size_t rotate_grad_workspace_bytes(int64_t n, int64_t, int64_t, int64_t dim) { return (size_t)(2 * grad_blocks(n) * dim * 4 + 15) / 16 * 16; }

cudaError_t launch_rotate(const simx_head_norm& a, cudaStream_t s) {
  RotateArgs r = common(a);
  r.side[0] = side(a.q, a.q, a.q_out, a.q_gain, nullptr, a.q_heads);
  r.side[1] = side(a.k, a.k, a.k_out, a.k_gain, nullptr, a.k_heads);
  const int sides = a.k_heads > 0 ? 2 : 1;
  return a.dtype == SIMX_F32 ? run_type<float, false>(r, sides, 0, s) : run_type<__nv_bfloat16, false>(r, sides, 0, s);
}

cudaError_t launch_rotate_grad(const simx_head_norm& a, void* ws, cudaStream_t s) {
  if (a.n == 0) {
    for (float* p : {a.dq_gain, a.dk_gain})
      if (p) {
        const cudaError_t e = cudaMemsetAsync(p, 0, (size_t)a.dim * 4, s);
        if (e != cudaSuccess) return e;
      }
    return cudaSuccess;
  }
  RotateArgs r = common(a);
  r.side[0] = side(a.q, a.q_out, a.dq, a.q_gain, a.dq_gain, a.q_heads);
  r.side[1] = side(a.k, a.k_out, a.dk, a.k_gain, a.dk_gain, a.k_heads);
  const int sides = a.k_heads > 0 ? 2 : 1;
  const int64_t blocks = grad_blocks(a.n);
  float* part = static_cast<float*>(ws);
  r.side[0].part = part;
  r.side[1].part = part + blocks * a.dim;
  cudaError_t e = a.dtype == SIMX_F32 ? run_type<float, true>(r, sides, blocks, s) : run_type<__nv_bfloat16, true>(r, sides, blocks, s);
  float* dk = sides > 1 ? a.dk_gain : nullptr;
  if (e == cudaSuccess && sides == 1 && a.dk_gain) e = cudaMemsetAsync(a.dk_gain, 0, (size_t)a.dim * 4, s);
  if (e != cudaSuccess || (!a.dq_gain && !dk)) return e;
  count_launches(1);
  k_rotate_dgain<<<dim3((unsigned)((a.dim + 31) / 32), (unsigned)sides), 1024, 0, s>>>(part, blocks, (int)a.dim, a.dq_gain, dk);
  return cudaGetLastError();
}

}  // namespace simx

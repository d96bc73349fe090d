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
// error, h_t = s_t + b_t (x_t - s_t), mu_t = lambda_t - b_t lambda_t and the product of a's is
// P - b_t P, one fma each.
//
// Bound by HBM: 2 reads and 1 write per element forward, 4 and 2 backward.  Both directions read each
// element once: a block holds a tile of steps and channels in registers, joins the steps' maps
// s -> A s + B across its threads (and, where there are few columns and many steps, across a cluster of
// blocks that share the steps), and applies the state that comes in to the same registers.
// Measured on one GB300 (floors at 6783 GB/s): forward 2 x 65,536 steps x 1024 channels bf16 165 us (119);
// backward 1024 x 512 x 64 fp32, time-major with episode ends, 143 (119) and 16 x 2048 x 2048 bf16 163 (119);
// one step of 256 x 2048 bf16 3.0 on the GPU, where the call's arguments take the host 10.5.
#include <algorithm>
#include <initializer_list>

#include "kernels.h"
#include "peer_round.h"
#include "seq_common.cuh"

namespace simx {

using namespace seq;

namespace {

// b = sigmoid(-z) = 1 / (1 + 2^t) with t = z log2 e, to relative precision whatever the sign of z (2^t may
// be inf: b is 0 then); t is one fma of the gate and the bias times log2 e.
__device__ __forceinline__ float sigmoid_neg(float t) { return rcp(__fadd_rn(1.0f, ex2(t))); }
// The same with ab = sigmoid(z) sigmoid(-z) = 2^t b b, t held below 2^126 (its minimum keeps a NaN).
struct Gate {
  float b, ab;
};
__device__ __forceinline__ Gate gate_of(float t) {
  asm("min.NaN.f32 %0, %0, 0f42FC0000;" : "+f"(t));
  const float e = ex2(t);
  Gate g;
  g.b = rcp(__fadd_rn(1.0f, e));
  g.ab = __fmul_rn(__fmul_rn(e, g.b), g.b);
  return g;
}

template <class T>
__device__ __forceinline__ T* at(const simx_seq& q, int64_t b, int64_t t, int64_t c) {
  return static_cast<T*>(q.p) + b * q.sb + t * q.st + c;
}
__device__ __forceinline__ uint8_t done_byte(const simx_scan& A, int64_t b, int64_t t) {
  return A.done[b * A.done_sb + t * A.done_st];
}
__device__ __forceinline__ bool done_at(const simx_scan& A, int64_t b, int64_t t) { return done_byte(A, b, t) != 0; }

// VEC channels of a tensor at p: one access of VEC elements.
__device__ __forceinline__ void load_vec(const float* p, float (&v)[4]) {
  const float4 q = *reinterpret_cast<const float4*>(p);
  v[0] = q.x;
  v[1] = q.y;
  v[2] = q.z;
  v[3] = q.w;
}
__device__ __forceinline__ void load_vec(const __nv_bfloat16* p, float (&v)[4]) {
  const uint2 q = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(q.x << 16);
  v[1] = __uint_as_float(q.x & 0xFFFF0000u);
  v[2] = __uint_as_float(q.y << 16);
  v[3] = __uint_as_float(q.y & 0xFFFF0000u);
}
template <class T>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[1]) {
  v[0] = widen(*p);
}
__device__ __forceinline__ void store_vec(float* p, const float (&v)[4]) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
}
__device__ __forceinline__ void store_vec(__nv_bfloat16* p, const float (&v)[4]) {
  __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3])));
}
template <class T>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[1]) {
  *p = narrow<T>(v[0]);
}
// `count` channels of fp32 rows (states; bias log2 e), which have no alignment of their own.
template <int VEC>
__device__ __forceinline__ void load_row(const float* p, int64_t off, float (&v)[VEC], int count = VEC) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = p && i < count ? p[off + i] : 0.0f;
}
template <int VEC>
__device__ __forceinline__ void load_bias(const float* p, int64_t off, float (&v)[VEC], int count = VEC) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = p && i < count ? __fmul_rn(p[off + i], kLog2e) : 0.0f;
}

// ---------------------------------------------------------------------------
// Short sequences: a thread per column (VEC channels), through time.  The single-token step.
// ---------------------------------------------------------------------------
constexpr int kColThreads = 128;
constexpr int kColSteps = 8;  // at most; all of a thread's loads are on their way at once

template <class T, int VEC>
__global__ void __launch_bounds__(kColThreads) k_scan_columns(simx_scan A) {
  const int64_t per = (A.channels + VEC - 1) / VEC, cols = A.batch * per;
  const int64_t col = (int64_t)blockIdx.x * kColThreads + threadIdx.x;
  if (col >= cols) return;
  const int64_t b = col / per, c = (col - b * per) * VEC;
  float bias[VEC], s[VEC], g[kColSteps][VEC], x[kColSteps][VEC];
  bool end[kColSteps];
#pragma unroll
  for (int t = 0; t < kColSteps; ++t) {
    if (t >= A.len) break;
    load_vec(at<const T>(A.gate, b, t, c), g[t]);
    load_vec(at<const T>(A.x, b, t, c), x[t]);
    end[t] = A.done && done_at(A, b, t);
  }
  load_bias<VEC>(A.bias, c, bias);
  load_row<VEC>(A.h0, b * A.channels + c, s);
#pragma unroll
  for (int t = 0; t < kColSteps; ++t) {
    if (t >= A.len) break;
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      s[i] = __fmaf_rn(sigmoid_neg(__fmaf_rn(g[t][i], kLog2e, bias[i])), __fsub_rn(x[t][i], s[i]), s[i]);
    store_vec(at<T>(A.h, b, t, c), s);
    if (end[t]) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) s[i] = 0.0f;
    }
  }
  if (A.h_last) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) A.h_last[b * A.channels + c + i] = s[i];
  }
}

template <class T, int VEC>
__global__ void __launch_bounds__(kColThreads) k_scan_grad_columns(simx_scan A, float* part) {
  const int64_t per = (A.channels + VEC - 1) / VEC, cols = A.batch * per;
  const int64_t col = (int64_t)blockIdx.x * kColThreads + threadIdx.x;
  pdl_trigger();
  if (col >= cols) return;
  const int64_t b = col / per, c = (col - b * per) * VEC;
  float bias[VEC], mu[VEC], db[VEC];
  load_bias<VEC>(A.bias, c, bias);
  load_row<VEC>(A.dh_last, b * A.channels + c, mu);
#pragma unroll
  for (int i = 0; i < VEC; ++i) db[i] = 0.0f;
  for (int64_t t = A.len - 1; t >= 0; --t) {
    float g[VEC], x[VEC], dh[VEC], s[VEC], dx[VEC], dg[VEC];
    load_vec(at<const T>(A.gate, b, t, c), g);
    load_vec(at<const T>(A.x, b, t, c), x);
    load_vec(at<const T>(A.dh, b, t, c), dh);
    if (t == 0) load_row<VEC>(A.h0, b * A.channels + c, s);
    else load_vec(at<const T>(A.h, b, t - 1, c), s);
    const bool fresh = t > 0 && A.done && done_at(A, b, t - 1), end = A.done && done_at(A, b, t);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const Gate q = gate_of(__fmaf_rn(g[i], kLog2e, bias[i]));
      const float lam = end ? dh[i] : __fadd_rn(dh[i], mu[i]);
      dx[i] = __fmul_rn(q.b, lam);
      dg[i] = __fmul_rn(__fmul_rn(q.ab, __fsub_rn(fresh ? 0.0f : s[i], x[i])), lam);
      db[i] = __fadd_rn(db[i], dg[i]);
      mu[i] = __fmaf_rn(-q.b, lam, lam);
    }
    store_vec(at<T>(A.dx, b, t, c), dx);
    store_vec(at<T>(A.dgate, b, t, c), dg);
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    if (A.dh0) A.dh0[b * A.channels + c + i] = mu[i];
    if (part) part[b * A.channels + c + i] = db[i];
  }
}

// ---------------------------------------------------------------------------
// Tiles of steps and channels.
// A thread holds S consecutive steps of VEC channels; LC lanes of a warp take neighbouring channels, its
// 32 / LC groups of lanes and the block's warps consecutive steps.  Per round a block takes
// warps * (32 / LC) * S steps.  A thread's steps are the map s -> A s + B; the maps before it are joined by
// shuffles within the warp and over a table of the warps' maps.  A = kForget marks a map that does not read
// s (an episode ended in it): what s holds, infinities included, is then gone.
// ---------------------------------------------------------------------------
constexpr float kForget = -1.0f;
constexpr int kMaxWarps = 8;

// FORGET: whether maps may be marked so.
template <bool FORGET>
__device__ __forceinline__ float apply(float A, float B, float s) {
  return FORGET && A < 0.0f ? B : __fmaf_rn(A, s, B);
}
// (A, B) after (pA, pB)
template <bool FORGET>
__device__ __forceinline__ void compose(float pA, float pB, float& A, float& B) {
  B = apply<FORGET>(A, B, pB);
  A = FORGET && (A < 0.0f || pA < 0.0f) ? kForget : __fmul_rn(pA, A);
}

struct TileShared {
  float4 table[2][kMaxWarps][2][16];  // [parity][warp][A or B]: 64 channels
};

template <int VEC>
__device__ __forceinline__ void put4(float4* row, int cl, const float (&v)[VEC]) {
  if (VEC == 4) row[cl] = make_float4(v[0], v[1 % VEC], v[2 % VEC], v[3 % VEC]);
  else reinterpret_cast<float*>(row)[cl] = v[0];
}
template <int VEC>
__device__ __forceinline__ void get4(const float4* row, int cl, float (&v)[VEC]) {
  if (VEC == 4) {
    const float4 q = row[cl];
    const float w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = w[i];
  } else {
    v[0] = reinterpret_cast<const float*>(row)[cl];
  }
}

// The state that comes into each thread's steps: on entry A, B are its map and carry the state before the
// round, on return s is the state before its first step and carry that after the round.
template <int VEC, bool FORGET>
__device__ __forceinline__ void tile_states(const float (&A)[VEC], const float (&B)[VEC], float (&carry)[VEC], float (&s)[VEC],
                                            int lcl, uint32_t turn, TileShared& sh) {
  const int lane = threadIdx.x & 31, warp = (int)threadIdx.x / 32, warps = (int)blockDim.x / 32;
  const int LC = 1 << lcl, cl = lane & (LC - 1), tg = lane >> lcl, GW = 32 >> lcl, parity = (int)(turn & 1u);
  float ia[VEC], ib[VEC], pa[VEC], pb[VEC];  // the maps of the warp's groups up to this one, and before it
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    float a = A[i], b = B[i];
    for (int d = 1; d < GW; d *= 2) {
      const float qa = __shfl_up_sync(0xffffffffu, a, d << lcl), qb = __shfl_up_sync(0xffffffffu, b, d << lcl);
      if (tg >= d) compose<FORGET>(qa, qb, a, b);
    }
    ia[i] = a;
    ib[i] = b;
  }
  if (tg == GW - 1) {
    put4(sh.table[parity][warp][0], cl, ia);
    put4(sh.table[parity][warp][1], cl, ib);
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    pa[i] = __shfl_up_sync(0xffffffffu, ia[i], LC & 31);
    pb[i] = __shfl_up_sync(0xffffffffu, ib[i], LC & 31);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < VEC; ++i) s[i] = carry[i];
#pragma unroll 4
  for (int w = 0; w < warps; ++w) {
    float a[VEC], b[VEC];
    get4(sh.table[parity][w][0], cl, a);
    get4(sh.table[parity][w][1], cl, b);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      if (w == warp) s[i] = carry[i];
      carry[i] = apply<FORGET>(a[i], b[i], carry[i]);
    }
  }
  if (tg > 0) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) s[i] = apply<FORGET>(pa[i], pb[i], s[i]);
  }
}

// Elements of K tensors on their way: VEC = 4 in the thread's places in shared memory, VEC = 1 in
// registers.
template <class T, int VEC, int K, int S>
struct Ahead {
  T reg[VEC == 1 ? K * S : 1];
  T* slot;  // the thread's places, `pitch` elements apart
  int pitch;
  __device__ __forceinline__ void start(void* shared) {
    slot = static_cast<T*>(shared) + (int)threadIdx.x * VEC;
    pitch = (int)blockDim.x * VEC;
  }
  __device__ __forceinline__ void bring(int k, int s, const T* p) {
    if (VEC == 1) reg[(k * S + s) % (VEC == 1 ? K * S : 1)] = *p;
    else copy_async<VEC * (int)sizeof(T) < 4 ? 4 : VEC * (int)sizeof(T)>(slot + (k * S + s) * pitch, p);
  }
  // Steps 0 .. S - 1 at p, p + st, ...
  __device__ __forceinline__ void bring_all(int k, const T* p, int64_t st) {
#pragma unroll
    for (int s = 0; s < S; ++s, p += st) bring(k, s, p);
  }
  __device__ __forceinline__ void take(int k, int s, float (&v)[VEC]) const {
    if (VEC == 1) v[0] = widen(reg[(k * S + s) % (VEC == 1 ? K * S : 1)]);
    else load_vec(slot + (k * S + s) * pitch, v);
  }
};

constexpr int kTileSteps = 8;

template <class T, int VEC, bool DONE>
__global__ void __launch_bounds__(256, 2) k_scan_tiles(simx_scan A, int lcl, int64_t tiles) {
  constexpr int S = kTileSteps;
  extern __shared__ uint4 slots[];
  __shared__ TileShared sh;
  const int lane = threadIdx.x & 31, warp = (int)threadIdx.x / 32;
  const int LC = 1 << lcl, cl = lane & (LC - 1), group = warp * (32 >> lcl) + (lane >> lcl);
  const int TB = (int)(blockDim.x >> lcl) * S;  // steps per block and round
  const int64_t per = (A.channels + LC * VEC - 1) / (LC * VEC);
  const int64_t rounds = (A.len + TB - 1) / TB;
  Ahead<T, VEC, 2, S> in;
  in.start(slots);
  uint32_t turn = 0;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t b = tile / per, c = ((tile - b * per) * LC + cl) * VEC;
    const bool mine = c < A.channels;
    int64_t t0 = (int64_t)group * S;
    const T* gate = at<const T>(A.gate, b, t0, c);  // of the round to come
    const T* x = at<const T>(A.x, b, t0, c);
    T* h = at<T>(A.h, b, t0, c);                    // of the round at hand
    const int64_t step = TB;
    uint8_t next[S] = {};  // of the round to come: whether the state before a step is dropped
    const auto bring = [&](int64_t u) {
      if (mine && u + S <= A.len) {
        in.bring_all(0, gate, A.gate.st);
        in.bring_all(1, x, A.x.st);
      } else if (mine) {
#pragma unroll
        for (int k = 0; k < S; ++k) {
          if (u + k < A.len) {
            in.bring(0, k, gate + k * A.gate.st);
            in.bring(1, k, x + k * A.x.st);
          }
        }
      }
      if (VEC > 1) copy_commit();
      gate += step * A.gate.st;
      x += step * A.x.st;
      if (DONE) {
#pragma unroll
        for (int k = 0; k < S; ++k) next[k] = u + k > 0 && u + k < A.len ? done_byte(A, b, u + k - 1) : (uint8_t)0;
      }
    };
    bring(t0);
    float bias[VEC], carry[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) bias[i] = carry[i] = 0.0f;
    if (mine) {
      load_bias<VEC>(A.bias, c, bias);
      load_row<VEC>(A.h0, b * A.channels + c, carry);
    }
    for (int64_t round = 0; round < rounds; ++round, t0 += step, h += step * A.h.st) {
      float bt[S][VEC], xt[S][VEC], a[VEC], s[VEC], st[VEC];
      const bool whole = mine && t0 + S <= A.len;
      if (VEC > 1) copy_wait_all();
      uint32_t resets = 0;
      if (DONE) {
#pragma unroll
        for (int k = 0; k < S; ++k) resets |= (uint32_t)(next[k] != 0) << k;
      }
#pragma unroll
      for (int k = 0; k < S; ++k) {
        float g[VEC];
        in.take(0, k, g);
        in.take(1, k, xt[k]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) bt[k][i] = sigmoid_neg(__fmaf_rn(g[i], kLog2e, bias[i]));
      }
      if (!whole) {  // steps past the end leave the state as it is
#pragma unroll
        for (int k = 0; k < S; ++k)
          if (!mine || t0 + k >= A.len)
#pragma unroll
            for (int i = 0; i < VEC; ++i) bt[k][i] = xt[k][i] = 0.0f;
      }
      if (round + 1 < rounds) bring(t0 + step);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        a[i] = 1.0f;
        s[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < S; ++k) {
          if (DONE && (resets >> k & 1u)) s[i] = 0.0f;
          s[i] = __fmaf_rn(bt[k][i], __fsub_rn(xt[k][i], s[i]), s[i]);
          a[i] = __fmaf_rn(-bt[k][i], a[i], a[i]);
        }
        if (DONE && resets) a[i] = kForget;
      }
      tile_states<VEC, DONE>(a, s, carry, st, lcl, turn++, sh);
      T* p = h;
#pragma unroll
      for (int k = 0; k < S; ++k, p += A.h.st) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          if (DONE && (resets >> k & 1u)) st[i] = 0.0f;
          st[i] = __fmaf_rn(bt[k][i], __fsub_rn(xt[k][i], st[i]), st[i]);
        }
        if (whole || (mine && t0 + k < A.len)) store_vec(p, st);
      }
    }
    if (A.h_last) __syncthreads();  // h_last may be h0, which every warp has used by now
    if (A.h_last && mine && group == 0) {
      const bool end = DONE && done_at(A, b, A.len - 1);
#pragma unroll
      for (int i = 0; i < VEC; ++i) A.h_last[b * A.channels + c + i] = end ? 0.0f : carry[i];
    }
  }
}

// Backward: the same on the steps in reverse order, step o of the walk being t = len - 1 - o, with
// mu -> a (dh + mu) as a step's map.  part [batch][channels]: sums of dgate (or null).
template <class T, int VEC, bool DONE>
__global__ void __launch_bounds__(128, 3) k_scan_grad_tiles(simx_scan A, int lcl, int64_t tiles, float* part) {
  constexpr int S = kTileSteps;
  extern __shared__ uint4 slots[];
  __shared__ TileShared sh;
  const int lane = threadIdx.x & 31, warp = (int)threadIdx.x / 32;
  const int LC = 1 << lcl, cl = lane & (LC - 1), group = warp * (32 >> lcl) + (lane >> lcl);
  const int TB = (int)(blockDim.x >> lcl) * S;
  pdl_trigger();
  const int64_t per = (A.channels + LC * VEC - 1) / (LC * VEC);
  const int64_t rounds = (A.len + TB - 1) / TB;
  Ahead<T, VEC, 4, S> in;
  in.start(slots);
  uint32_t turn = 0;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t b = tile / per, c = ((tile - b * per) * LC + cl) * VEC;
    const bool mine = c < A.channels;
    const int64_t step = TB;
    int64_t t0 = A.len - 1 - (int64_t)group * S;  // of the thread's first step of the walk
    const T* gate = at<const T>(A.gate, b, t0, c);            // of the round to come
    const T* x = at<const T>(A.x, b, t0, c);
    const T* dh = at<const T>(A.dh, b, t0, c);
    const T* h = at<const T>(A.h, b, t0 - 1, c);
    T* dx = at<T>(A.dx, b, t0, c);                            // of the round at hand
    T* dgate = at<T>(A.dgate, b, t0, c);
    uint8_t next[S + 1] = {};  // of the round to come: done at the walk's steps, and at the one behind them
    const auto bring = [&](int64_t u) {
      if (mine && u >= S) {
        in.bring_all(0, gate, -A.gate.st);
        in.bring_all(1, x, -A.x.st);
        in.bring_all(2, dh, -A.dh.st);
        in.bring_all(3, h, -A.h.st);
      } else if (mine) {
#pragma unroll
        for (int k = 0; k < S; ++k) {
          if (u - k >= 0) {
            in.bring(0, k, gate - k * A.gate.st);
            in.bring(1, k, x - k * A.x.st);
            in.bring(2, k, dh - k * A.dh.st);
            if (u - k > 0) in.bring(3, k, h - k * A.h.st);
          }
        }
      }
      if (VEC > 1) copy_commit();
      gate -= step * A.gate.st;
      x -= step * A.x.st;
      dh -= step * A.dh.st;
      h -= step * A.h.st;
      if (DONE) {
#pragma unroll
        for (int k = 0; k <= S; ++k) next[k] = u - k >= 0 ? done_byte(A, b, u - k) : (uint8_t)0;
      }
    };
    bring(t0);
    float bias[VEC], carry[VEC];
    Sum2 db[VEC] = {};        // of dgate over all rounds, a long chain,
    float db16[VEC] = {};     // and over up to 16 of them
#pragma unroll
    for (int i = 0; i < VEC; ++i) bias[i] = carry[i] = 0.0f;
    if (mine) {
      load_bias<VEC>(A.bias, c, bias);
      load_row<VEC>(A.dh_last, b * A.channels + c, carry);
    }
    for (int64_t round = 0; round < rounds; ++round, t0 -= step, dx -= step * A.dx.st, dgate -= step * A.dgate.st) {
      float bt[S][VEC], qt[S][VEC], dt[S][VEC], a[VEC], m[VEC], mu[VEC];  // 1 - a; a (1 - a) (s - x); dh
      const bool whole = mine && t0 >= S;
      if (VEC > 1) copy_wait_all();
      uint32_t ends = 0;
      if (DONE) {
#pragma unroll
        for (int k = 0; k <= S; ++k) ends |= (uint32_t)(next[k] != 0) << k;
      }
#pragma unroll
      for (int k = 0; k < S; ++k) {
        float g[VEC], xv[VEC], s[VEC];
        in.take(0, k, g);
        in.take(1, k, xv);
        in.take(2, k, dt[k]);
        in.take(3, k, s);
        if (mine && t0 == k) load_row<VEC>(A.h0, b * A.channels + c, s);
        const bool fresh = DONE && (ends >> (k + 1) & 1u);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const Gate q = gate_of(__fmaf_rn(g[i], kLog2e, bias[i]));
          bt[k][i] = q.b;
          qt[k][i] = __fmul_rn(q.ab, __fsub_rn(fresh ? 0.0f : s[i], xv[i]));
        }
      }
      if (!whole) {  // steps before the first leave what comes to them as it is
#pragma unroll
        for (int k = 0; k < S; ++k)
          if (!mine || t0 < k)
#pragma unroll
            for (int i = 0; i < VEC; ++i) bt[k][i] = qt[k][i] = dt[k][i] = 0.0f;
      }
      if (round + 1 < rounds) bring(t0 - step);
      const uint32_t own = ends & ((1u << S) - 1u);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        a[i] = 1.0f;
        m[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < S; ++k) {
          const float lam = DONE && (own >> k & 1u) ? dt[k][i] : __fadd_rn(dt[k][i], m[i]);
          m[i] = __fmaf_rn(-bt[k][i], lam, lam);
          a[i] = __fmaf_rn(-bt[k][i], a[i], a[i]);
        }
        if (DONE && own) a[i] = kForget;
      }
      tile_states<VEC, DONE>(a, m, carry, mu, lcl, turn++, sh);
      T* px = dx;
      T* pg = dgate;
#pragma unroll
      for (int k = 0; k < S; ++k, px -= A.dx.st, pg -= A.dgate.st) {
        float ox[VEC], og[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float lam = DONE && (own >> k & 1u) ? dt[k][i] : __fadd_rn(dt[k][i], mu[i]);
          ox[i] = __fmul_rn(bt[k][i], lam);
          og[i] = __fmul_rn(qt[k][i], lam);
          db16[i] = __fadd_rn(db16[i], og[i]);  // steps that are not there: qt is 0
          mu[i] = __fmaf_rn(-bt[k][i], lam, lam);
        }
        if (whole || (mine && t0 >= k)) {
          store_vec(px, ox);
          store_vec(pg, og);
        }
      }
      if ((round & 15) == 15 || round + 1 == rounds) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          db[i].add(db16[i], 0.0f);
          db16[i] = 0.0f;
        }
      }
    }
    if (A.dh0 && mine && group == 0) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) A.dh0[b * A.channels + c + i] = carry[i];
    }
    if (part) {  // the block's sums of its steps, groups and warps in order
      __syncthreads();
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        float v = db[i].value();
        for (int d = 16 >> lcl; d > 0; d /= 2) v = __fadd_rn(v, __shfl_down_sync(0xffffffffu, v, d << lcl));
        if (lane < LC) reinterpret_cast<float*>(sh.table[0][warp][0])[cl * VEC + i] = v;
      }
      __syncthreads();
      for (int j = (int)threadIdx.x; j < LC * VEC; j += (int)blockDim.x) {
        const int64_t ch = (tile - b * per) * LC * VEC + j;
        float v = 0.0f;
        for (int w = 0; w < (int)blockDim.x / 32; ++w) v = __fadd_rn(v, reinterpret_cast<const float*>(sh.table[0][w][0])[j]);
        if (ch < A.channels) part[b * A.channels + ch] = v;
      }
      __syncthreads();
    }
  }
}

// ---------------------------------------------------------------------------
// Wide tiles: 64 channels, 16 lanes of 4 each.
// The same tile of steps in registers, with the joining done across the block instead of by every thread
// for itself: the maps of all groups of lanes go to a table, where each thread takes 4 groups of one
// channel (NW / 2 neighbouring lanes per channel), joins them, and writes back the state before each
// group.  That is a tenth of the instructions (the tile above takes 11 per element for it, of 40), for a
// second barrier a round.  Where there are few tiles and many steps, a cluster of blocks shares the steps:
// per round each block takes its part, in rank order, and posts its map to all others.  24 instructions per
// element forward and 49 backward; what is left is the round's chain of barriers and posts at 16 and 12
// warps per SM (2 x 65,536 x 1024 bf16: 54 % of the DRAM's cycles, half of the issue slots).
// ---------------------------------------------------------------------------
constexpr int kWideLanes = 16, kWideChannels = 64, kWidePitch = 68;
constexpr int kMaxCluster = 8;

// How the wide tiles read and write 4 channels of a step: at once, by 4-byte words (fp32, and bf16 in pairs
// of channels), or element by element.
enum Access : int { WHOLE = 0, WORDS = 1, ELEMENTS = 2 };

// Steps of 4 channels of K tensors on their way in the thread's places in shared memory, `count` channels
// of them there.  Copies are asynchronous but for single bf16 elements, which come by way of registers (all
// of a tensor's steps at once).
template <class T, int K, int S, int ACCESS>
struct WideAhead {
  static constexpr int PER = ACCESS == WORDS ? 4 / (int)sizeof(T) : 1;  // elements per access
  T* slot;
  int pitch, count;
  __device__ __forceinline__ void start(void* shared) {
    slot = static_cast<T*>(shared) + (int)threadIdx.x * 4;
    pitch = (int)blockDim.x * 4;
  }
  // Steps 0 .. steps - 1 at p, p + st, ...
  __device__ __forceinline__ void bring(int k, const T* p, int64_t st, int steps = S) {
    T* to = slot + k * S * pitch;
    if (ACCESS == WHOLE) {
#pragma unroll
      for (int s = 0; s < S; ++s, p += st)
        if (s < steps) copy_async<4 * (int)sizeof(T)>(to + s * pitch, p);
    } else if (ACCESS == WORDS) {
#pragma unroll
      for (int s = 0; s < S; ++s, p += st)
#pragma unroll
        for (int i = 0; i < 4; i += PER)
          if (s < steps && i < count) copy_async<4>(to + s * pitch + i, p + i);
    } else {
      T v[S][4];
#pragma unroll
      for (int s = 0; s < S; ++s, p += st)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[s][i] = s < steps && i < count ? p[i] : narrow<T>(0.0f);
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) to[s * pitch + i] = v[s][i];
    }
  }
  __device__ __forceinline__ void take(int k, int s, float (&v)[4]) const { load_vec(slot + (k * S + s) * pitch, v); }
  __device__ __forceinline__ void put(T* p, const float (&v)[4]) const {
    if (ACCESS == WHOLE) {
      store_vec(p, v);
    } else if (PER == 2) {
#pragma unroll
      for (int i = 0; i < 4; i += 2)
        if (i < count) *reinterpret_cast<uint32_t*>(p + i) = pack2(v[i], v[i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < count) p[i] = narrow<T>(v[i]);
    }
  }
};

template <int NW, int CLT>
struct WideShared {
  float4 a[2 * NW * kWidePitch / 4], b[2 * NW * kWidePitch / 4];  // [group][channel]; a also takes the states
  float2 peer[2][CLT][kWideChannels];                             // [slot][rank]: {A, B}
  uint64_t bar[2];
};

// Per thread: its channel and the groups it joins.
template <int NW>
struct Joiner {
  static constexpr int TPC = NW / 2;  // threads per channel, 4 groups each
  int ch, q;
  __device__ __forceinline__ Joiner() : ch((int)threadIdx.x / TPC), q((int)threadIdx.x % TPC) {}
};

// On entry A, B are the thread's map and carry the state of the joiner's channel before the round; on
// return s is the state before the thread's first step, and carry that after the round.
template <int NW, int CLT, bool FORGET>
__device__ __forceinline__ void wide_states(const float (&A)[4], const float (&B)[4], float& carry, float (&s)[4],
                                            uint32_t rank, PeerRound& peers, WideShared<NW, CLT>& sh) {
  const Joiner<NW> J;
  constexpr int TPC = Joiner<NW>::TPC;
  const int group = (int)threadIdx.x / kWideLanes, cl = (int)threadIdx.x % kWideLanes;
  sh.a[group * (kWidePitch / 4) + cl] = make_float4(A[0], A[1], A[2], A[3]);
  sh.b[group * (kWidePitch / 4) + cl] = make_float4(B[0], B[1], B[2], B[3]);
  __syncthreads();
  float* ta = reinterpret_cast<float*>(sh.a) + 4 * J.q * kWidePitch + J.ch;
  const float* tb = reinterpret_cast<const float*>(sh.b) + 4 * J.q * kWidePitch + J.ch;
  float a[4], b[4], ja = 1.0f, jb = 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    a[j] = ta[j * kWidePitch];
    b[j] = tb[j * kWidePitch];
    float na = a[j], nb = b[j];
    compose<FORGET>(ja, jb, na, nb);
    ja = na;
    jb = nb;
  }
#pragma unroll
  for (int d = 1; d < TPC; d *= 2) {  // the joined maps up to this lane's
    const float qa = __shfl_up_sync(0xffffffffu, ja, d), qb = __shfl_up_sync(0xffffffffu, jb, d);
    if (J.q >= d) compose<FORGET>(qa, qb, ja, jb);
  }
  float pa = __shfl_up_sync(0xffffffffu, ja, 1), pb = __shfl_up_sync(0xffffffffu, jb, 1);  // and before it
  if (J.q == 0) {
    pa = 1.0f;
    pb = 0.0f;
  }
  const int top = ((int)threadIdx.x & 31) | (TPC - 1);
  ja = __shfl_sync(0xffffffffu, ja, top);  // the block's
  jb = __shfl_sync(0xffffffffu, jb, top);
  float in = carry;
  if (CLT == 1) {
    carry = apply<FORGET>(ja, jb, carry);
  } else {
    const uint32_t slot = peers.slot();
    uint64_t* bar = &sh.bar[slot];
    if (peers.posts()) {
      if (threadIdx.x == 0) tcx::mbar_arrive_expect_tx(bar, (uint32_t)(8 * kWideChannels * CLT));
      for (int r = J.q; r < CLT; r += TPC) post_peer(&sh.peer[slot][rank][J.ch], bar, (uint32_t)r, make_float2(ja, jb));
    }
    peers.end(!peers.lost() && tcx::mbar_wait(bar, peers.parity(), kPeerCycles));
#pragma unroll
    for (int r = 0; r < CLT; ++r) {
      const float2 m = sh.peer[slot][r][J.ch];
      if (r == (int)rank) in = carry;
      carry = apply<FORGET>(m.x, m.y, carry);
    }
    if (peers.lost()) in = carry = nan();  // a post that never came: the states that come to this block are NaN from here on
  }
  float v = J.q == 0 ? in : apply<FORGET>(pa, pb, in);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    ta[j * kWidePitch] = v;
    v = apply<FORGET>(a[j], b[j], v);
  }
  __syncthreads();
  const float4 o = sh.a[group * (kWidePitch / 4) + cl];
  s[0] = o.x;
  s[1] = o.y;
  s[2] = o.z;
  s[3] = o.w;
}

template <int NW, int CLT>
__device__ __forceinline__ void wide_start(WideShared<NW, CLT>& sh) {
  if (CLT > 1) {  // every block runs, its barriers ready, before another one posts to it
    if (threadIdx.x < 2) tcx::mbar_init(&sh.bar[threadIdx.x], 1);
    tcx::mbar_fence_init();
    cluster_sync();
  }
}
// Bit k of the group's steps, from the byte of lane k of its 16.
__device__ __forceinline__ uint32_t group_bits(uint8_t byte) {
  return __ballot_sync(0xffffffffu, byte != 0) >> ((int)threadIdx.x & 16) & 0xFFFFu;
}

template <class T, bool DONE, int CLT, int ACCESS>
__global__ void __launch_bounds__(256, 2) k_scan_wide(simx_scan A, int64_t tiles, bool withheld) {
  constexpr int S = kTileSteps, NW = 8, TB = 2 * NW * S;
  constexpr int64_t step = (int64_t)CLT * TB;
  extern __shared__ uint4 slots[];
  __shared__ WideShared<NW, CLT> sh;
  const int cl = (int)threadIdx.x % kWideLanes, group = (int)threadIdx.x / kWideLanes;
  const uint32_t rank = CLT == 1 ? 0u : cluster_rank();
  const Joiner<NW> J;
  wide_start(sh);
  const int64_t per = (A.channels + kWideChannels - 1) / kWideChannels;
  const int64_t rounds = (A.len + step - 1) / step;
  WideAhead<T, 2, S, ACCESS> in;
  in.start(slots);
  PeerRound peers{withheld && rank == CLT - 1 ? 4u : 0u};  // withheld: the last block's posts are never made (tests)
  for (int64_t tile = blockIdx.x / CLT; tile < tiles; tile += gridDim.x / CLT) {
    const int64_t b = tile / per, c0 = (tile - b * per) * kWideChannels, c = c0 + 4 * cl;
    const bool mine = c < A.channels, joins = c0 + J.ch < A.channels;
    in.count = (int)(mine ? (A.channels - c < 4 ? A.channels - c : 4) : 0);
    int64_t t0 = (int64_t)rank * TB + group * S;
    const T* gate = at<const T>(A.gate, b, t0, c);  // of the round to come
    const T* x = at<const T>(A.x, b, t0, c);
    T* h = at<T>(A.h, b, t0, c);                    // of the round at hand
    uint8_t next = 0;                               // of the round to come: done at step t0 + cl - 1
    const auto bring = [&](int64_t u) {
      if (mine && u + S <= A.len) {
        in.bring(0, gate, A.gate.st);
        in.bring(1, x, A.x.st);
      } else if (mine && u < A.len) {
        in.bring(0, gate, A.gate.st, (int)(A.len - u));
        in.bring(1, x, A.x.st, (int)(A.len - u));
      }
      copy_commit();
      gate += step * A.gate.st;
      x += step * A.x.st;
      if (DONE) next = u + cl > 0 && u + cl <= A.len && cl < S ? done_byte(A, b, u + cl - 1) : (uint8_t)0;
    };
    bring(t0);
    float bias[4] = {}, carry = joins && A.h0 ? A.h0[b * A.channels + c0 + J.ch] : 0.0f;
    if (mine) load_bias<4>(A.bias, c, bias, in.count);
    for (int64_t round = 0; round < rounds; ++round, t0 += step, h += step * A.h.st) {
      float bt[S][4], xt[S][4], a[4], s[4], st[4];
      const bool whole = mine && t0 + S <= A.len;
      copy_wait_all();
      const uint32_t resets = DONE ? group_bits(next) : 0u;  // bit k: the state before step k is dropped
#pragma unroll
      for (int k = 0; k < S; ++k) {
        float g[4];
        in.take(0, k, g);
        in.take(1, k, xt[k]);
#pragma unroll
        for (int i = 0; i < 4; ++i) bt[k][i] = sigmoid_neg(__fmaf_rn(g[i], kLog2e, bias[i]));
      }
      if (!whole) {  // steps past the end leave the state as it is
#pragma unroll
        for (int k = 0; k < S; ++k)
          if (!mine || t0 + k >= A.len)
#pragma unroll
            for (int i = 0; i < 4; ++i) bt[k][i] = xt[k][i] = 0.0f;
      }
      if (round + 1 < rounds) bring(t0 + step);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = 1.0f;
        s[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < S; ++k) {
          if (DONE && (resets >> k & 1u)) s[i] = 0.0f;
          s[i] = __fmaf_rn(bt[k][i], __fsub_rn(xt[k][i], s[i]), s[i]);
          a[i] = __fmaf_rn(-bt[k][i], a[i], a[i]);
        }
        if (DONE && resets) a[i] = kForget;
      }
      wide_states<NW, CLT, DONE>(a, s, carry, st, rank, peers, sh);
      T* p = h;
#pragma unroll
      for (int k = 0; k < S; ++k, p += A.h.st) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (DONE && (resets >> k & 1u)) st[i] = 0.0f;
          st[i] = __fmaf_rn(bt[k][i], __fsub_rn(xt[k][i], st[i]), st[i]);
        }
        if (whole || (mine && t0 + k < A.len)) in.put(p, st);
      }
    }
    if (CLT > 1 && A.h_last == A.h0) cluster_sync();  // h_last in place of h0, which every block has used by now
    if (A.h_last && joins && rank == 0 && J.q == 0)
      A.h_last[b * A.channels + c0 + J.ch] = DONE && done_at(A, b, A.len - 1) ? 0.0f : carry;
  }
  if (CLT > 1) cluster_sync();  // none leaves while another one may post to it
}

// Backward, on the steps in reverse order; part [batch * CLT][channels]: sums of dgate (or null).
template <class T, bool DONE, int CLT, int ACCESS>
__global__ void __launch_bounds__(128, 3) k_scan_grad_wide(simx_scan A, int64_t tiles, float* part, bool withheld) {
  constexpr int S = kTileSteps, NW = 4, TB = 2 * NW * S;
  constexpr int64_t step = (int64_t)CLT * TB;
  extern __shared__ uint4 slots[];
  __shared__ WideShared<NW, CLT> sh;
  const int cl = (int)threadIdx.x % kWideLanes, group = (int)threadIdx.x / kWideLanes;
  const uint32_t rank = CLT == 1 ? 0u : cluster_rank();
  const Joiner<NW> J;
  pdl_trigger();
  wide_start(sh);
  const int64_t per = (A.channels + kWideChannels - 1) / kWideChannels;
  const int64_t rounds = (A.len + step - 1) / step;
  WideAhead<T, 4, S, ACCESS> in;
  in.start(slots);
  PeerRound peers{withheld && rank == CLT - 1 ? 4u : 0u};  // withheld: the last block's posts are never made (tests)
  for (int64_t tile = blockIdx.x / CLT; tile < tiles; tile += gridDim.x / CLT) {
    const int64_t b = tile / per, c0 = (tile - b * per) * kWideChannels, c = c0 + 4 * cl;
    const bool mine = c < A.channels, joins = c0 + J.ch < A.channels;
    in.count = (int)(mine ? (A.channels - c < 4 ? A.channels - c : 4) : 0);
    int64_t t0 = A.len - 1 - (int64_t)rank * TB - group * S;  // of the thread's first step of the walk
    const T* gate = at<const T>(A.gate, b, t0, c);            // of the round to come
    const T* x = at<const T>(A.x, b, t0, c);
    const T* dh = at<const T>(A.dh, b, t0, c);
    const T* h = at<const T>(A.h, b, t0 - 1, c);
    T* dx = at<T>(A.dx, b, t0, c);                            // of the round at hand
    T* dgate = at<T>(A.dgate, b, t0, c);
    uint8_t next = 0;                                         // of the round to come: done at step t0 - cl
    const auto bring = [&](int64_t u) {
      if (mine && u >= S) {
        in.bring(0, gate, -A.gate.st);
        in.bring(1, x, -A.x.st);
        in.bring(2, dh, -A.dh.st);
        in.bring(3, h, -A.h.st);
      } else if (mine && u >= 0) {
        in.bring(0, gate, -A.gate.st, (int)u + 1);
        in.bring(1, x, -A.x.st, (int)u + 1);
        in.bring(2, dh, -A.dh.st, (int)u + 1);
        in.bring(3, h, -A.h.st, (int)u);
      }
      copy_commit();
      gate -= step * A.gate.st;
      x -= step * A.x.st;
      dh -= step * A.dh.st;
      h -= step * A.h.st;
      if (DONE) next = u - cl >= 0 && cl <= S ? done_byte(A, b, u - cl) : (uint8_t)0;
    };
    bring(t0);
    Sum2 db[4] = {};     // of dgate over all rounds, a long chain,
    float db16[4] = {};  // and over up to 16 of them
    float bias[4] = {}, carry = joins && A.dh_last ? A.dh_last[b * A.channels + c0 + J.ch] : 0.0f;
    if (mine) load_bias<4>(A.bias, c, bias, in.count);
    for (int64_t round = 0; round < rounds; ++round, t0 -= step, dx -= step * A.dx.st, dgate -= step * A.dgate.st) {
      float bt[S][4], qt[S][4], dt[S][4], a[4], m[4], mu[4];  // 1 - a; a (1 - a) (s - x); dh
      const bool whole = mine && t0 >= S;
      copy_wait_all();
      const uint32_t ends = DONE ? group_bits(next) : 0u;  // bit k: done at the walk's step k, S: behind them
#pragma unroll
      for (int k = 0; k < S; ++k) {
        float g[4], xv[4], s[4];
        in.take(0, k, g);
        in.take(1, k, xv);
        in.take(2, k, dt[k]);
        in.take(3, k, s);
        const bool fresh = DONE && (ends >> (k + 1) & 1u);
        if (!whole && mine && t0 == k) load_row<4>(A.h0, b * A.channels + c, s, in.count);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const Gate q = gate_of(__fmaf_rn(g[i], kLog2e, bias[i]));
          bt[k][i] = q.b;
          qt[k][i] = __fmul_rn(q.ab, __fsub_rn(fresh ? 0.0f : s[i], xv[i]));
        }
      }
      if (!whole) {  // steps before the first leave what comes to them as it is
#pragma unroll
        for (int k = 0; k < S; ++k)
          if (!mine || t0 < k)
#pragma unroll
            for (int i = 0; i < 4; ++i) bt[k][i] = qt[k][i] = dt[k][i] = 0.0f;
      }
      if (round + 1 < rounds) bring(t0 - step);
      const uint32_t own = ends & ((1u << S) - 1u);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = 1.0f;
        m[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < S; ++k) {
          const float lam = DONE && (own >> k & 1u) ? dt[k][i] : __fadd_rn(dt[k][i], m[i]);
          m[i] = __fmaf_rn(-bt[k][i], lam, lam);
          a[i] = __fmaf_rn(-bt[k][i], a[i], a[i]);
        }
        if (DONE && own) a[i] = kForget;
      }
      wide_states<NW, CLT, DONE>(a, m, carry, mu, rank, peers, sh);
      T* px = dx;
      T* pg = dgate;
#pragma unroll
      for (int k = 0; k < S; ++k, px -= A.dx.st, pg -= A.dgate.st) {
        float ox[4], og[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float lam = DONE && (own >> k & 1u) ? dt[k][i] : __fadd_rn(dt[k][i], mu[i]);
          ox[i] = __fmul_rn(bt[k][i], lam);
          og[i] = __fmul_rn(qt[k][i], lam);
          db16[i] = __fadd_rn(db16[i], og[i]);  // steps that are not there: qt is 0
          mu[i] = __fmaf_rn(-bt[k][i], lam, lam);
        }
        if (whole || (mine && t0 >= k)) {
          in.put(px, ox);
          in.put(pg, og);
        }
      }
      if ((round & 15) == 15 || round + 1 == rounds) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          db[i].add(db16[i], 0.0f);
          db16[i] = 0.0f;
        }
      }
    }
    if (A.dh0 && joins && rank == 0 && J.q == 0) A.dh0[b * A.channels + c0 + J.ch] = carry;
    if (part) {  // the block's sums of its steps, group by group
      __syncthreads();
      sh.a[group * (kWidePitch / 4) + cl] = make_float4(db[0].value(), db[1].value(), db[2].value(), db[3].value());
      __syncthreads();
      if (threadIdx.x < kWideChannels && c0 + threadIdx.x < A.channels) {
        float v = 0.0f;
        for (int g = 0; g < 2 * NW; ++g) v = __fadd_rn(v, reinterpret_cast<const float*>(sh.a)[g * kWidePitch + threadIdx.x]);
        part[(b * CLT + rank) * A.channels + c0 + threadIdx.x] = v;
      }
      __syncthreads();
    }
  }
  if (CLT > 1) cluster_sync();
}

__global__ void __launch_bounds__(1024) k_scan_dbias(const float* part, int64_t rows, int64_t channels, float* dbias) {
  pdl_wait();
  column_sums(part, rows, channels, (int64_t)blockIdx.x * 32, dbias);
}

constexpr int kFwdWarps = 8, kFwdPerSm = 2, kGradWarps = 4, kGradPerSm = 3;

// How a call is cut.  columns: up to kColSteps steps.  Else tiles of 1 << lcl lanes per row of channels and
// `warps` warps, or wide tiles in clusters of so many blocks: whichever ends first, by the waves of blocks
// over the GPU, the rounds that each block goes (and one for its first loads), and what a round takes
// (microseconds, measured over calls of 9 to 1770 MB: tiles of aligned tensors 3.4 to 5, of others 0.8 to
// 1.3 with a quarter of the elements; wide tiles 2.4 forward and 3.5 backward, off alignment 3.2 to 5.4 and
// 8.4 to 11, and up to a quarter more for a cluster's posts).  One long bf16 sequence of 18 channels, 17 x
// 32,774 steps: clusters of 8 109 us, tiles 418; 115 x 6961 of 167 channels: tiles 308, clusters 439;
// backward 16 x 2048 x 2048: clusters of 1, 2, 4, 8 199, 171, 167, 194.
struct ScanPlan {
  bool columns, wide;
  int lcl, warps, cluster;
  int64_t tiles;
};
ScanPlan plan_scan(int64_t batch, int64_t len, int64_t channels, int access, int dtype, bool grad) {
  ScanPlan p{};
  const bool aligned = access == WHOLE;
  p.columns = len <= kColSteps;
  p.cluster = p.warps = 1;
  if (p.columns) return p;
  const auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  const int max_warps = grad ? kGradWarps : kFwdWarps, vec = aligned ? 4 : 1;
  const int64_t slots = (int64_t)sm_count() * (grad ? kGradPerSm : kFwdPerSm);
  while (p.lcl < (aligned ? 4 : 5) && ((int64_t)vec << p.lcl) < channels) ++p.lcl;
  p.tiles = batch * up(channels, (int64_t)vec << p.lcl);
  const int64_t warp_steps = (int64_t)(32 >> p.lcl) * kTileSteps;
  while (p.warps < max_warps && p.warps * warp_steps < len) p.warps *= 2;
  double best = (double)up(p.tiles, slots * max_warps / p.warps) * (double)(up(len, p.warps * warp_steps) + 1) * (aligned ? 3.6 : 0.95);
  const int64_t block = (int64_t)max_warps * 2 * kTileSteps;  // a wide block's steps
  const int64_t tiles = batch * up(channels, kWideChannels);
  // off alignment only large clusters are ever the better choice
  for (int cl = aligned ? 1 : 4; cl <= kMaxCluster && (cl == 1 || block * cl <= len); cl *= 2) {
    // fp32 gradients in clusters of 8 fit two blocks to an SM: 64 KB of copies, 12.6 KB of tables and posts and the
    // reserved kilobyte each, of 228 (48 x 8192 x 64: clusters of 4 126 us, of 8 136).  Off alignment the measured
    // rounds below have that in them already (24 x 4096 x 66: clusters of 8 101, of 4 111).
    const int64_t places = grad && dtype == SIMX_F32 && access == WHOLE && cl == 8 ? (int64_t)sm_count() * 2 : slots;
    // an SM with one block, and what the others add
    const double full = std::min(1.0, (double)(tiles * cl) / (double)slots);
    const double round = access == WHOLE ? (grad ? 3.5 : 2.5)
                         : access == WORDS ? (grad ? (dtype == SIMX_F32 ? 4.0 + 6.0 * full : 4.0 + 3.0 * full) : (dtype == SIMX_F32 ? 2.5 + 2.5 * full : 2.5 + 1.5 * full))
                                           : (grad ? 6.5 + 4.0 * full : 3.0 + 2.4 * full);
    const double posts = cl == 1 ? 1.0 : cl == 2 ? 1.03 : cl == 4 ? 1.1 : 1.25;
    const double cost = (double)up(tiles * cl, places) * (double)(up(len, block * cl) + 1) * round * posts;
    if (cost < best) {
      best = cost;
      p.wide = true;
      p.cluster = cl;
    }
  }
  if (p.wide) p.tiles = tiles;
  return p;
}

// How tensors of a call can be accessed.
template <class T>
int access_of(const simx_scan& a, std::initializer_list<simx_seq> all) {
  const int64_t es = (int64_t)sizeof(T);
  const auto fits = [&](int64_t bytes) {
    if (a.channels * es % bytes != 0) return false;
    for (const simx_seq& q : all)
      if ((int64_t)(reinterpret_cast<uintptr_t>(q.p) % (uintptr_t)bytes) != 0 || (a.batch > 1 && q.sb * es % bytes != 0) ||
          (a.len > 1 && q.st * es % bytes != 0))
        return false;
    return true;
  };
  return a.len == 0 ? (a.channels % 4 == 0 ? WHOLE : ELEMENTS) : fits(4 * es) ? WHOLE : fits(4) ? WORDS : ELEMENTS;
}

template <class K, class... Args>
cudaError_t launch_tiles(K* kernel, const ScanPlan& p, int threads, size_t smem, cudaStream_t s, Args... args) {
  cudaError_t e = allow_smem(kernel, 64 * 1024);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute at[1];
  const int64_t teams = std::min<int64_t>(p.tiles, (int64_t)1 << 24);
  lc.gridDim = dim3((unsigned)(teams * p.cluster));
  lc.blockDim = dim3((unsigned)threads);
  lc.dynamicSmemBytes = smem;
  lc.stream = s;
  if (p.cluster > 1) {
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)p.cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    lc.attrs = at;
    lc.numAttrs = 1;
  }
  count_launches(1);
  return cudaLaunchKernelEx(&lc, kernel, args...);
}

template <class T, bool DONE, int ACCESS>
cudaError_t scan_tiles(const simx_scan& a, const ScanPlan& p, cudaStream_t s) {
  if (p.wide) {
    const bool withheld = p.cluster > 1 && copies_withheld() != 0u;
    const int th = 32 * kFwdWarps;
    const size_t smem = (size_t)th * 2 * kTileSteps * 4 * sizeof(T);
    if (p.cluster == 8) return launch_tiles(k_scan_wide<T, DONE, 8, ACCESS>, p, th, smem, s, a, p.tiles, withheld);
    if (p.cluster == 4) return launch_tiles(k_scan_wide<T, DONE, 4, ACCESS>, p, th, smem, s, a, p.tiles, withheld);
    if constexpr (ACCESS == WHOLE) {
      if (p.cluster == 2) return launch_tiles(k_scan_wide<T, DONE, 2, WHOLE>, p, th, smem, s, a, p.tiles, withheld);
      return launch_tiles(k_scan_wide<T, DONE, 1, WHOLE>, p, th, smem, s, a, p.tiles, false);
    }
  }
  constexpr int VEC = ACCESS == WHOLE ? 4 : 1;
  const size_t smem = VEC == 4 ? (size_t)p.warps * 32 * 2 * kTileSteps * 4 * sizeof(T) : 0;
  return launch_tiles(k_scan_tiles<T, VEC, DONE>, p, 32 * p.warps, smem, s, a, p.lcl, p.tiles);
}
template <class T, bool DONE, int ACCESS>
cudaError_t scan_grad_tiles(const simx_scan& a, const ScanPlan& p, float* part, cudaStream_t s) {
  if (p.wide) {
    const bool withheld = p.cluster > 1 && copies_withheld() != 0u;
    const int th = 32 * kGradWarps;
    const size_t smem = (size_t)th * 4 * kTileSteps * 4 * sizeof(T);
    if (p.cluster == 8) return launch_tiles(k_scan_grad_wide<T, DONE, 8, ACCESS>, p, th, smem, s, a, p.tiles, part, withheld);
    if (p.cluster == 4) return launch_tiles(k_scan_grad_wide<T, DONE, 4, ACCESS>, p, th, smem, s, a, p.tiles, part, withheld);
    if constexpr (ACCESS == WHOLE) {
      if (p.cluster == 2) return launch_tiles(k_scan_grad_wide<T, DONE, 2, WHOLE>, p, th, smem, s, a, p.tiles, part, withheld);
      return launch_tiles(k_scan_grad_wide<T, DONE, 1, WHOLE>, p, th, smem, s, a, p.tiles, part, false);
    }
  }
  constexpr int VEC = ACCESS == WHOLE ? 4 : 1;
  const size_t smem = VEC == 4 ? (size_t)p.warps * 32 * 4 * kTileSteps * 4 * sizeof(T) : 0;
  return launch_tiles(k_scan_grad_tiles<T, VEC, DONE>, p, 32 * p.warps, smem, s, a, p.lcl, p.tiles, part);
}

template <class T>
cudaError_t scan(const simx_scan& a, cudaStream_t s) {
  const int access = access_of<T>(a, {a.x, a.gate, a.h});
  const ScanPlan p = plan_scan(a.batch, a.len, a.channels, access, a.dtype, false);
  if (p.columns) {
    const int64_t cols = a.batch * (access == WHOLE ? a.channels / 4 : a.channels);
    const unsigned blocks = (unsigned)((cols + kColThreads - 1) / kColThreads);
    if (access == WHOLE) k_scan_columns<T, 4><<<blocks, kColThreads, 0, s>>>(a);
    else k_scan_columns<T, 1><<<blocks, kColThreads, 0, s>>>(a);
    count_launches(1);
    return cudaGetLastError();
  }
  if (access == WHOLE) return a.done ? scan_tiles<T, true, WHOLE>(a, p, s) : scan_tiles<T, false, WHOLE>(a, p, s);
  if constexpr (sizeof(T) == 2) {
    if (access == ELEMENTS) return a.done ? scan_tiles<T, true, ELEMENTS>(a, p, s) : scan_tiles<T, false, ELEMENTS>(a, p, s);
  }
  return a.done ? scan_tiles<T, true, WORDS>(a, p, s) : scan_tiles<T, false, WORDS>(a, p, s);
}

template <class T>
cudaError_t scan_grad(const simx_scan& a, float* part, int64_t& rows, cudaStream_t s) {
  const int access = access_of<T>(a, {a.x, a.gate, a.h, a.dh, a.dx, a.dgate});
  const ScanPlan p = plan_scan(a.batch, a.len, a.channels, access, a.dtype, true);
  rows = a.batch * p.cluster;
  if (p.columns) {
    const int64_t cols = a.batch * (access == WHOLE ? a.channels / 4 : a.channels);
    const unsigned blocks = (unsigned)((cols + kColThreads - 1) / kColThreads);
    if (access == WHOLE) k_scan_grad_columns<T, 4><<<blocks, kColThreads, 0, s>>>(a, part);
    else k_scan_grad_columns<T, 1><<<blocks, kColThreads, 0, s>>>(a, part);
    count_launches(1);
    return cudaGetLastError();
  }
  if (access == WHOLE) return a.done ? scan_grad_tiles<T, true, WHOLE>(a, p, part, s) : scan_grad_tiles<T, false, WHOLE>(a, p, part, s);
  if constexpr (sizeof(T) == 2) {
    if (access == ELEMENTS)
      return a.done ? scan_grad_tiles<T, true, ELEMENTS>(a, p, part, s) : scan_grad_tiles<T, false, ELEMENTS>(a, p, part, s);
  }
  return a.done ? scan_grad_tiles<T, true, WORDS>(a, p, part, s) : scan_grad_tiles<T, false, WORDS>(a, p, part, s);
}

}  // namespace

// The backward pass's sums of dgate: a row of channels per batch entry and block of a cluster, of whichever
// plan the tensors' type and alignment give.
size_t scan_workspace_bytes(int64_t batch, int64_t len, int64_t channels) {
  int cl = 1;
  for (int access : {WHOLE, WORDS, ELEMENTS})
    for (int dtype : {SIMX_F32, SIMX_BF16}) cl = std::max(cl, plan_scan(batch, len, channels, access, dtype, true).cluster);
  return (size_t)batch * (size_t)cl * (size_t)channels * sizeof(float);
}

cudaError_t launch_scan(const simx_scan& a, cudaStream_t s) {
  return a.dtype == SIMX_F32 ? scan<float>(a, s) : scan<__nv_bfloat16>(a, s);
}

cudaError_t launch_scan_grad(const simx_scan& a, void* ws, cudaStream_t s) {
  float* part = a.dbias ? static_cast<float*>(ws) : nullptr;
  int64_t rows = 0;
  cudaError_t e = a.dtype == SIMX_F32 ? scan_grad<float>(a, part, rows, s) : scan_grad<__nv_bfloat16>(a, part, rows, s);
  if (e != cudaSuccess || !part) return e;
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  lc.gridDim = dim3((unsigned)((a.channels + 31) / 32));
  lc.blockDim = dim3(1024);
  lc.stream = s;
  lc.attrs = at;
  lc.numAttrs = 1;
  count_launches(1);
  e = cudaLaunchKernelEx(&lc, k_scan_dbias, (const float*)part, rows, a.channels, a.dbias);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace simx

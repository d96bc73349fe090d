// seq_attn.cu — linear attention with a decay for each head: S_t = lambda S_{t-1} + k_t^T v_t,
// o_t = scale q_t S_t, its gradient, and its single-token step.
//
// The gradients are three passes of the forward form S = lambda S + b^T c, o = a S: grad_q over (grad_o, v, k) with
// the transposed state, and, from the last step back, grad_k over (v, grad_o, q) and grad_v over (k, q, grad_o).  The
// state is found again: nothing of the forward pass is kept.  fp32 goes step by step here, bf16 by chunks of steps as
// products of matrices (seq_attn_tc.cu), and up to 8 steps of either by a kernel that carries states through.
#include <algorithm>

#include "kernels.h"
#include "seq_attn.cuh"

namespace simx {

using namespace seq;
using namespace attn;

namespace {

constexpr int kThreads = 256;
// Lengths up to which a state is carried from step to step in a block's registers.  256 x 16 heads of 128 in bf16: 1, 4 and 8
// steps in 94, 199 and 359 us, any of them by chunks in 380; in fp32 1, 2 and 8 in 94, 127 and 387, by a warp for 16 columns
// 714, 724 and 752; of 64 in fp32 4 and 8 in 72 and 123, by warps 123 and 128.  1024 x 2 heads of 32 in fp32: 1, 2, 4 and 8
// steps in 11, 14, 21 and 31 us, by a warp for each head 14.
constexpr int kStepMost = 8;
int most_steps(const simx_attention& a) {
  const int64_t d = std::max(a.dk, a.dv);
  return a.dtype != SIMX_F32 || d > 64 ? kStepMost : d > 32 ? 4 : 2;
}

// BYTES (4 or 16) into shared memory, asynchronously; zeros where `there` is false.
template <int BYTES>
__device__ __forceinline__ void copy_or_zero(float* dst, const float* src, bool there) {
  if (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tcx::su32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(tcx::su32(dst)), "l"(src), "r"(there ? 4 : 0) : "memory");
}

template <int N>
struct Width {
  static constexpr int value = N;
};

template <int N>
__device__ __forceinline__ void load_row(const float* p, float (&v)[N]) {
  if constexpr (N == 4) {
    const float4 u = *reinterpret_cast<const float4*>(p);
    v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
  } else {
    const float2 u = *reinterpret_cast<const float2*>(p);
    v[0] = u.x, v[1] = u.y;
  }
}
template <int N>
__device__ __forceinline__ void store_row(float* p, const float (&v)[N]) {
  if constexpr (N == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  else *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
}

// The state that a segment starts with, N elements of it: what the segments before it added, each times what the
// ones between keep of it.  place(i, x, y): element i's row and column, false where there is none.  A segment's
// elements are loaded together.
template <int N, class Place>
__device__ __forceinline__ void first_state(const AttnPass& A, float ld, int64_t bh, int seg, float (&s)[N], Place place) {
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = 0.0f;
  float w = 1.0f;
  for (int q = seg - 1; q >= 0 && w != 0.0f; --q) {
    const int64_t at_q = bh * A.segs + q;
    const float* p = A.seg_state + at_q * A.da * A.dc;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int x, y;
      if (place(i, x, y)) s[i] = __fmaf_rn(w, p[x * A.dc + y], s[i]);
    }
    w = A.seg_keep[at_q] != 0.0f ? segments_keep(A, ld, q, seg) : 0.0f;
  }
  if (w == 0.0f || !A.s_in) return;
  const float* p = A.s_in + bh * A.da * A.dc;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    int x, y;
    if (!place(i, x, y)) continue;
    const float v = p[x * A.sx + y * A.sy];
    s[i] = seg ? __fmaf_rn(w, v, s[i]) : v;
  }
}

// A pass in fp32 with da padded to X, by kWide columns of dc: the state in the registers of a warp.
template <int X>
struct Flat {
  static constexpr int kSteps = X == 128 ? 8 : 16;  // of a stage
  static constexpr int kPairs = X / 8, kCols = X == 128 ? 2 : 4, kWide = 8 * kCols;  // pairs of rows and columns of the state, a lane
  static constexpr int kStage = kSteps * (2 * X + kWide), kBytes = 2 * kStage * 4;
  static constexpr int kBlocks = X == 32 ? 16 : 8;
};

// One segment of one head and 32 (X of 128: 16) columns in fp32, step by step: S = lambda S + b^T c, o = a S, as they are written.
// A warp, which is a block, holds the state: lane 8 g + l has rows X / 4 g and on, in pairs, of 4 (2) columns from 4 l
// (2 l) on, so that a step is X + X / 8 paired operations a lane without any exchange but the sum of o over g, for four
// steps at once.  Inputs come by asynchronous copies, a stage ahead; a lane's loads of a and b are the same for eight
// lanes.  KEEP: only what the segment adds to the state.
// 1024 sequences of 512 steps, 2 heads of 32: 187 us, 44 % of the copy rate (gradient, three passes: 468 us, 31 %).  Wider
// heads, 64 sequences: 16 of 64 in 301 us (gradient 777), 8 of 128 in 673 (1841), where HBM would take 85 (148) and 90 (155).
// Bound by the FP32 units and shared memory's loads, some 65 and 72 us of it alone, with 3.4 warps on a scheduler to
// cover one another; HBM would take 83.  Tried: two warps or four to a block 198 and 197 us; 16 columns to a warp, for
// twice the warps, 308; a scale for every step 272; chunks of steps as products of 32 x 32 matrices 355 on the FP32
// units and 357 on the tensor cores, operands in three parts.
template <int X, bool KEEP>
__global__ void __launch_bounds__(32, Flat<X>::kBlocks) k_attn(const Passes all) {
  using F = Flat<X>;
  const AttnPass& A = all.p[blockIdx.y];
  extern __shared__ __align__(16) float sm[];
  const int lane = threadIdx.x, group = lane >> 3, x0 = group * (X / 4);
  constexpr int CN = F::kCols;
  const int cols = (A.dc + F::kWide - 1) / F::kWide;
  const int64_t unit = blockIdx.x, H = A.heads;
  if (unit >= A.batch * H * A.segs * cols) return;
  const int yb = (int)(unit % cols) * F::kWide, y0 = yb + (lane & 7) * CN;
  const int64_t h = unit / cols % H, q = unit / cols / H;
  const int seg = (int)(q % A.segs);
  if (KEEP && seg == A.segs - 1) return;  // nobody starts from its end
  const int64_t b = q / A.segs, bh = b * H + h;
  const float ld = A.ld[h];
  const float lam = power(ld, 1);
  // Four steps share a scale: the state is kept over lambda^(u + 1) of step u, where v is divided by that and o
  // multiplied.  Where a memory is shorter than two steps, so that a state is never more than 16 times itself, and
  // beside an end of an episode, steps go by themselves.
  const bool scaled = lam >= 0.5f;
  // The state then takes lambda^4 rounded to fp32, or the value beside it, whichever keeps the product of all so far
  // nearest to the power: over a memory of 4096 steps roundings of the same sign would show.  (The state's own roundings,
  // 2^-24 every four steps, have one sign where lambda^4 is within some 2^-20 of 1 and little is added.)
  const float lam4 = power(ld, 4), rest = scaled ? __fmul_rn(4.0f, decay_rest(ld, lam, lam4)) : 0.0f;
  const float beside = __uint_as_float(__float_as_uint(lam4) + (rest > 0.0f ? 1 : -1));
  const float gap = rest != 0.0f ? fabsf(__fdiv_rn(__fsub_rn(beside, lam4), lam4)) : 1.0f;
  float owed = 0.0f;
  const int64_t p0 = seg * A.seg_len, p1 = min(A.len, p0 + A.seg_len);
  const int total = (int)(p1 - p0);
  float* stage = sm;
  const int64_t dir = A.reverse ? -1 : 1, t0 = A.reverse ? A.len - 1 - p0 : p0;
  const float* pa = at<float>(A.a, b * A.asb + h / A.adiv * A.ash + t0 * A.ast);
  const float* pb = at<float>(A.b, b * A.bsb + h / A.bdiv * A.bsh + t0 * A.bst);
  const float* pc = at<float>(A.c, b * A.csb + h / A.cdiv * A.csh + t0 * A.cst) + yb;
  const int wide = min(F::kWide, A.dc - yb);  // columns of this unit
  const bool whole = ((reinterpret_cast<uintptr_t>(pa) | reinterpret_cast<uintptr_t>(pb) | reinterpret_cast<uintptr_t>(pc) |
                       (uintptr_t)((A.ast | A.bst | A.cst) * 4)) & 15) == 0 && A.da % 4 == 0 && A.dc % 4 == 0;
  float* po = static_cast<float*>(A.o) + b * A.osb + h * A.osh + t0 * A.ost + y0;
  const bool o_whole = (((reinterpret_cast<uintptr_t>(po) | (uintptr_t)(A.ost * 4)) & (4 * CN - 1)) == 0) && y0 + CN <= A.dc;

  // one stage: a [steps][X], b [steps][X], c [steps][kWide]
  auto copy = [&](int from, float* to) {
    const int m = min(F::kSteps, total - from);
    auto tile = [&](const float* p, int64_t st, auto width, int dim, float* q) {
      constexpr int W = decltype(width)::value;
      if (whole) {
        constexpr int kRow = W / 4, kEach = (F::kSteps * kRow + 31) / 32, kStep = 32 / kRow;  // units of a row, a lane's, its steps between
        const int r = lane / kRow, c = lane % kRow * 4;
        const int64_t step = dir * st * kStep;
        const float* from_here = p + dir * (from + r) * st + c;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
          if (F::kSteps * kRow % 32 == 0 || r + i * kStep < F::kSteps)
            copy_or_zero<16>(q + (lane + 32 * i) * 4, r + i * kStep < m && c < dim ? from_here + i * step : p, r + i * kStep < m && c < dim);
      } else {
#pragma unroll 1
        for (int i = lane; i < F::kSteps * W; i += 32) {
          const bool there = i / W < m && i % W < dim;
          copy_or_zero<4>(q + i, there ? p + dir * (from + i / W) * st + i % W : p, there);
        }
      }
    };
    if (!KEEP) tile(pa, A.ast, Width<X>{}, A.da, to);
    tile(pb, A.bst, Width<X>{}, A.da, to + F::kSteps * X);
    tile(pc, A.cst, Width<F::kWide>{}, wide, to + F::kSteps * 2 * X);
    copy_commit();
  };
  auto ends = [&](int from) {  // whether an episode ended before step from + lane
    const int64_t p = p0 + from + lane;
    return __ballot_sync(0xffffffffu, lane < F::kSteps && from + lane < total && (p > 0 || A.reverse) && cut_before(A, b, p));
  };

  Pair s[F::kPairs][CN];
  {
    float first[2 * F::kPairs * CN];
    first_state(A, ld, bh, KEEP ? 0 : seg, first, [&](int i, int& x, int& y) {
      x = x0 + i / (2 * CN) * 2 + i % 2;
      y = y0 + i / 2 % CN;
      return !KEEP && x < A.da && y < A.dc;
    });
#pragma unroll
    for (int i = 0; i < F::kPairs * CN; ++i) s[i / CN][i % CN] = pair(first[2 * i], first[2 * i + 1]);
  }
  // inject / lambda^(u + 1) of each step, out_scale lambda^(u + 1) of this lane's
  float up[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) up[u] = scaled ? __fdiv_rn(A.inject, power(ld, u + 1)) : 0.0f;
  const float down = scaled ? __fmul_rn(A.out_scale, power(ld, group + 1)) : 0.0f;
  auto put = [&](int t, const float (&q)[CN]) {  // this lane's columns of o
    float* to = po + dir * t * A.ost;
    if (o_whole) {
      store_row<CN>(to, q);
    } else {
#pragma unroll
      for (int c = 0; c < CN; ++c)
        if (y0 + c < A.dc) to[c] = q[c];
    }
  };
  bool cut_once = false;
  copy(0, stage);
  unsigned next_cuts = ends(0);
  int which = 0;
  for (int from = 0; from < total; from += F::kSteps, which ^= 1) {
    const unsigned cuts = next_cuts;
    if (from + F::kSteps < total) {
      copy(from + F::kSteps, stage + (which ^ 1) * F::kStage);
      next_cuts = ends(from + F::kSteps);
      asm volatile("cp.async.wait_group 1;" ::: "memory");
    } else {
      copy_wait_all();
    }
    __syncwarp();
    const float* sa = stage + which * F::kStage + x0;
    const float* sb = sa + F::kSteps * X;
    const float* sc = stage + which * F::kStage + F::kSteps * 2 * X + (lane & 7) * CN;
    const int m = min(F::kSteps, total - from);
    for (int t4 = 0; t4 < m; t4 += 4) {
      const bool begins = A.first == 0 && p0 + from + t4 == 0;  // step 0 takes its state as it is
      if (!scaled || m - t4 < 4 || (cuts >> t4 & 15) || begins) {
        // each step by itself
#pragma unroll 1
        for (int t = t4; t < min(m, t4 + 4); ++t) {
          const bool none = (cuts >> t & 1) || lam == 0.0f, as_it_is = begins && t == 0 && !(cuts & 1);
          cut_once = cut_once || (none && !as_it_is);
          const Pair ll = pair(as_it_is ? 1.0f : lam, as_it_is ? 1.0f : lam);
          float cv[CN];
          load_row<CN>(sc + t * F::kWide, cv);
          Pair v[CN], acc[CN] = {};
#pragma unroll
          for (int c = 0; c < CN; ++c) {
            const float w = __fmul_rn(cv[c], lam >= 0.0f ? A.inject : lam);
            v[c] = pair(w, w);
          }
#pragma unroll
          for (int i = 0; i < F::kPairs; i += 2) {
            const ulonglong2 kb = *reinterpret_cast<const ulonglong2*>(sb + t * X + 2 * i);
            const ulonglong2 qa = KEEP ? ulonglong2{0, 0} : *reinterpret_cast<const ulonglong2*>(sa + t * X + 2 * i);
#pragma unroll
            for (int c = 0; c < CN; ++c) {
              s[i][c] = fma2(kb.x, v[c], none && !as_it_is ? 0 : mul2(ll, s[i][c]));
              s[i + 1][c] = fma2(kb.y, v[c], none && !as_it_is ? 0 : mul2(ll, s[i + 1][c]));
              if (!KEEP) acc[c] = fma2(qa.y, s[i + 1][c], fma2(qa.x, s[i][c], acc[c]));
            }
          }
          if (!KEEP) {
            float q[CN];
#pragma unroll
            for (int c = 0; c < CN; ++c) {
              const float2 f = halves(acc[c]);
              float w = __fadd_rn(f.x, f.y);
              w = __fadd_rn(w, __shfl_xor_sync(0xffffffffu, w, 16));
              q[c] = __fmul_rn(__fadd_rn(w, __shfl_xor_sync(0xffffffffu, w, 8)), A.out_scale);
            }
            if (group == 0) put(from + t, q);
          }
        }
        continue;
      }
      float o[4][CN];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float cv[CN];
        load_row<CN>(sc + (t4 + u) * F::kWide, cv);
        Pair v[CN], acc[CN];
#pragma unroll
        for (int c = 0; c < CN; ++c) {
          const float w = __fmul_rn(cv[c], up[u]);
          v[c] = pair(w, w);
        }
#pragma unroll
        for (int i = 0; i < F::kPairs; i += 2) {
          const ulonglong2 kb = *reinterpret_cast<const ulonglong2*>(sb + (t4 + u) * X + 2 * i);
          const ulonglong2 qa = KEEP ? ulonglong2{0, 0} : *reinterpret_cast<const ulonglong2*>(sa + (t4 + u) * X + 2 * i);
#pragma unroll
          for (int c = 0; c < CN; ++c) {
            s[i][c] = fma2(kb.x, v[c], s[i][c]);
            s[i + 1][c] = fma2(kb.y, v[c], s[i + 1][c]);
            if (!KEEP) acc[c] = fma2(qa.y, s[i + 1][c], i ? fma2(qa.x, s[i][c], acc[c]) : mul2(qa.x, s[i][c]));
          }
        }
        if (!KEEP)
#pragma unroll
          for (int c = 0; c < CN; ++c) {
            const float2 f = halves(acc[c]);
            o[u][c] = __fadd_rn(f.x, f.y);
          }
      }
      owed = __fadd_rn(owed, fabsf(rest));
      const bool step_aside = __fadd_rn(owed, owed) >= gap;
      owed = step_aside ? __fsub_rn(owed, gap) : owed;
      const Pair ll = pair(step_aside ? beside : lam4, step_aside ? beside : lam4);
#pragma unroll
      for (int i = 0; i < F::kPairs; ++i)
#pragma unroll
        for (int c = 0; c < CN; ++c) s[i][c] = mul2(ll, s[i][c]);
      if (!KEEP) {
        // sums over the groups: each is left with the step of its number
        float p[2][CN], q[CN];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int c = 0; c < CN; ++c) {
            const float keep = group & 2 ? o[u + 2][c] : o[u][c], send = group & 2 ? o[u][c] : o[u + 2][c];
            p[u][c] = __fadd_rn(keep, __shfl_xor_sync(0xffffffffu, send, 16));
          }
#pragma unroll
        for (int c = 0; c < CN; ++c) {
          const float keep = group & 1 ? p[1][c] : p[0][c], send = group & 1 ? p[0][c] : p[1][c];
          q[c] = __fmul_rn(__fadd_rn(keep, __shfl_xor_sync(0xffffffffu, send, 8)), down);
        }
        put(from + t4 + group, q);
      }
    }
    __syncwarp();  // the stage may be written again
  }
  float f = 1.0f;
  if (!KEEP) {
    if (!A.s_out || seg != A.segs - 1) return;
    f = A.reverse ? power(ld, 1) : 1.0f;
    if (!A.reverse && A.done && A.done[b * A.dsb + (A.len - 1) * A.dst] != 0) f = 0.0f;
  } else if (lane == 0) {
    A.seg_keep[bh * A.segs + seg] = cut_once ? 0.0f : power(ld, total - (p0 == 0 && A.first == 0 ? 1 : 0));
  }
#pragma unroll
  for (int i = 0; i < F::kPairs; ++i)
#pragma unroll
    for (int c = 0; c < CN; ++c) {
      const float2 v = halves(s[i][c]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int x = x0 + 2 * i + e, y = y0 + c;
        const float w = e ? v.y : v.x;
        if (x < A.da && y < A.dc) {
          if (KEEP) A.seg_state[((bh * A.segs + seg) * A.da + x) * A.dc + y] = w;
          else A.s_out[bh * A.da * A.dc + x * A.sx + y * A.sy] = f != 0.0f ? __fmul_rn(f, w) : 0.0f;
        }
      }
    }
}

// A few steps of one head and up to 64 columns with the state in registers: TX column groups of 4 (TX a power of two),
// 256 / TX rows at a time, RT rows a thread.  Bound by HBM: the state is read once and written once.  256 x 16 heads of 128:
// 95 us, 86 % of the copy rate, three blocks of 32 KB to an SM (all 128 columns to a block, two to an SM: 102; 32 columns:
// 148); small ones, 16 x 2 heads of 32, are the launch.
template <class T, int RT>
__global__ void __launch_bounds__(kThreads, RT == 8 ? 3 : 2) k_attn_step(const simx_attention A, int lg_tx) {
  __shared__ float sq[kAttnMaxDim], sk[kAttnMaxDim], sv[kAttnMaxDim];
  __shared__ __align__(16) float4 red[kThreads];
  const int tid = threadIdx.x, tx = tid & ((1 << lg_tx) - 1), ty = tid >> lg_tx, rows = kThreads >> lg_tx;
  const int64_t h = blockIdx.x % A.heads, b = blockIdx.x / A.heads, hk = h / (A.heads / A.kv_heads);
  const int dk = (int)A.dk, dv = (int)A.dv, y0 = blockIdx.y * 4 << lg_tx, y = y0 + tx * 4;
  const int64_t base = (int64_t)blockIdx.x * dk * dv;
  const bool whole = dv % 4 == 0 && ((reinterpret_cast<uintptr_t>(A.s0) | reinterpret_cast<uintptr_t>(A.s_last)) & 15) == 0;
  float s[RT][4];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int x = ty + r * rows;
#pragma unroll
    for (int q = 0; q < 4; ++q) s[r][q] = 0.0f;
    if (A.s0 && x < dk && y < dv) {
      const float* p = A.s0 + base + x * dv + y;
      if (whole) {
        const float4 v = __ldcs(reinterpret_cast<const float4*>(p));
        s[r][0] = v.x, s[r][1] = v.y, s[r][2] = v.z, s[r][3] = v.w;
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (y + q < dv) s[r][q] = p[q];
      }
    }
  }
  const float ld = A.len > 0 ? A.log_decay[h] : 0.0f, lam = power(ld, 1);
  const float rest = __fmul_rn(decay_rest(ld, lam, lam), lam);  // a step is exact, so that many calls are one memory
  for (int64_t t = 0; t < A.len; ++t) {
    const T* pq = at<T>(A.q.p, b * A.q.sb + t * A.q.st + h * A.q.sh);
    const T* pk = at<T>(A.k.p, b * A.k.sb + t * A.k.st + hk * A.k.sh);
    const T* pv = at<T>(A.v.p, b * A.v.sb + t * A.v.st + hk * A.v.sh);
    if (tid < dk) sq[tid] = widen(pq[tid]);
    if (tid >= 128 && tid < 128 + dk) sk[tid - 128] = widen(pk[tid - 128]);
    if (tid < dv) sv[tid] = widen(pv[tid]);
    const bool drop = t > 0 && A.done && A.done[b * A.done_sb + (t - 1) * A.done_st] != 0;
    __syncthreads();
    float o[4] = {};
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int x = ty + r * rows;
      if (x < dk && y < dv) {
        const float k = sk[x], q = sq[x];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (y + e < dv) {
            const float kv = __fmul_rn(k, sv[y + e]);
            s[r][e] = lam > 0.0f && !drop ? __fmaf_rn(lam, s[r][e], __fmaf_rn(rest, s[r][e], kv)) : lam >= 0.0f ? kv : lam;
            o[e] = __fmaf_rn(q, s[r][e], o[e]);
          }
      }
    }
    for (int d = 1 << lg_tx; d < 32; d *= 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __fadd_rn(o[e], __shfl_xor_sync(0xffffffffu, o[e], d));
    // one row of sums for each warp
    if ((tid & 31) < 1 << lg_tx) red[(tid / 32 << lg_tx) + tx] = make_float4(o[0], o[1], o[2], o[3]);
    __syncthreads();
    if (tid < 4 << lg_tx && y0 + tid < dv) {
      float v = 0.0f;
      for (int w = 0; w < kThreads / 32; ++w) v = __fadd_rn(v, (&red[(w << lg_tx) + tid / 4].x)[tid & 3]);
      static_cast<T*>(A.o.p)[b * A.o.sb + t * A.o.st + h * A.o.sh + y0 + tid] = narrow<T>(__fmul_rn(v, A.scale));
    }
  }
  if (!A.s_last) return;
  const bool drop = A.len > 0 && A.done && A.done[b * A.done_sb + (A.len - 1) * A.done_st] != 0;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int x = ty + r * rows;
    if (x < dk && y < dv) {
      float* p = A.s_last + base + x * dv + y;
      if (whole) {
        __stcs(reinterpret_cast<float4*>(p), drop ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : make_float4(s[r][0], s[r][1], s[r][2], s[r][3]));
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (y + q < dv) p[q] = drop ? 0.0f : s[r][q];
      }
    }
  }
}

// Gradients of shared heads: part [rows][heads][dim] summed over each group of heads.
template <class T>
__global__ void __launch_bounds__(kThreads) k_attn_groups(const float* part, simx_heads out, int64_t batch, int64_t len, int kv, int group,
                                                          int dim) {
  const int64_t n = batch * len * kv * dim;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
    const int d = (int)(i % dim);
    const int64_t r = i / dim, h = r % kv, row = r / kv;
    const float* p = part + (row * kv + h) * group * dim + d;
    float s = p[0];
    for (int g = 1; g < group; ++g) s = __fadd_rn(s, p[(int64_t)g * dim]);
    static_cast<T*>(out.p)[row / len * out.sb + row % len * out.st + h * out.sh + d] = narrow<T>(s);
  }
}

// ---------------------------------------------------------------------------- host

constexpr int64_t kUnits = 304;  // (batch, head, segment) units that fill the GPU

struct Plan {
  int segs;
  int64_t seg_len;
  int grid;  // of shares, 0: none
};

// Long sequences of few heads are cut into segments: their states are found first, for a second read of keys and values.
// In bf16, heads of all passes that fill the GPU are shared out instead (seq_attn.cuh), each input read once.  16 x 4096 x 16
// heads of 128: 291 us; in two segments to a head, before that, 670.  4 x 4096 x 16 backward: 247 and 860.  One sequence of
// 60001, 16 heads of 64, 19 segments: 235, of which the first pass takes 85.
Plan segments(int64_t segs, int64_t len) {
  int64_t sl = std::max<int64_t>(1, (len + segs - 1) / segs);
  sl = (sl + 127) / 128 * 128;
  return {(int)std::max<int64_t>(1, (len + sl - 1) / sl), sl, 0};
}

// Segments that a length is worth: each costs the later ones a read of its state.  One head of 64, bf16 (fp32): 512 steps in
// 23 us (93), in two segments 27 (96), in four 23 (84); 1024 in 37 (174), in four 29 (117), in two 39 (162); 2048 in 68 (336),
// in eight 35 (146), in four 39 (182); 8192 in 249 (1309), in 16 41 (181), in 32 33 (146), which the rule gives away.
int64_t most_segments(int64_t len) { return len < 1024 ? 1 : std::max(len / 512, std::min<int64_t>(len / 256, 8)); }

Plan plan(int dtype, int passes, int64_t batch, int64_t len, int64_t heads, int64_t dk, int64_t dv) {
  const int64_t units = std::max<int64_t>(1, batch * heads);
  if (dtype == SIMX_F32) return segments(std::max<int64_t>(1, std::min((kUnits + units - 1) / units, most_segments(len))), len);
  const int d = (int)std::max(dk, dv);
  if (share_grid(passes * units, len, d)) {
    Plan p = segments(1, len);
    p.grid = share_grid(passes * units, len, d);
    return p;
  }
  // no more than run at a time: a second round would cost more than the rest of the first
  return segments(std::max<int64_t>(1, std::min(resident_blocks(d) / (passes * units), most_segments(len))), len);
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

size_t seg_bytes(const Plan& p, int64_t batch, int64_t heads, int64_t dk, int64_t dv) {
  if (p.segs == 1) return 0;
  return up16((size_t)batch * heads * p.segs * dk * dv * 4) + up16((size_t)batch * heads * p.segs * 4);
}

// Of the plan's segments or shares; forward, segments have room for a copy of the first states.
size_t state_bytes(int64_t batch, int64_t heads, int64_t dk, int64_t dv) { return up16((size_t)batch * heads * dk * dv * 4); }
size_t plan_bytes(const Plan& p, int passes, int64_t batch, int64_t len, int64_t heads, int64_t dk, int64_t dv) {
  if (p.grid) return share_bytes(passes * batch * heads, len, (int)std::max(dk, dv));
  return passes * seg_bytes(p, batch, heads, dk, dv) + (p.segs > 1 && passes == 1 ? state_bytes(batch, heads, dk, dv) : 0);
}

size_t most_bytes(int passes, int64_t batch, int64_t len, int64_t heads, int64_t dk, int64_t dv) {
  size_t n = 0;
  if (len > kStepMost || passes > 1)
    for (int dtype : {SIMX_F32, SIMX_BF16}) n = std::max(n, plan_bytes(plan(dtype, passes, batch, len, heads, dk, dv), passes, batch, len, heads, dk, dv));
  return n;
}

Shares shares_at(const Plan& p, void* ws) {
  if (!p.grid) return {};
  int* flags = static_cast<int*>(ws);
  return {p.grid, 0, 0, reinterpret_cast<float*>(flags + 4 * p.grid), flags};
}

template <int X>
cudaError_t run_flat(const Passes& all, int n, bool keep, cudaStream_t s) {
  using F = Flat<X>;
  int64_t units = 0;
  for (int i = 0; i < n; ++i) {
    const AttnPass& A = all.p[i];
    units = std::max<int64_t>(units, A.batch * A.heads * A.segs * ((A.dc + F::kWide - 1) / F::kWide));
  }
  auto f = keep ? k_attn<X, true> : k_attn<X, false>;
  const cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, F::kBytes);
  if (e != cudaSuccess) return e;
  count_launches(1);
  f<<<dim3((unsigned)units, (unsigned)n), 32, F::kBytes, s>>>(all);
  return cudaGetLastError();
}

// n passes with the same axes, at once.
cudaError_t run_passes(const Passes& all, int n, const Shares& shares, cudaStream_t s) {
  for (int keep = all.p[0].segs > 1 ? 1 : 0; keep >= 0; --keep) {
    int d = 0;
    for (int i = 0; i < n; ++i) d = std::max(d, all.p[i].da);
    const cudaError_t e = all.p[0].dtype == SIMX_BF16 ? run_tc(all, n, keep, shares, s) : d <= 32 ? run_flat<32>(all, n, keep, s)
                        : d <= 64 ? run_flat<64>(all, n, keep, s) : run_flat<128>(all, n, keep, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

template <class T, int RT>
cudaError_t run_step(const simx_attention& a, int lg_tx, cudaStream_t s) {
  count_launches(1);
  k_attn_step<T, RT><<<dim3((unsigned)(a.batch * a.heads), (unsigned)((a.dv + (4 << lg_tx) - 1) >> (lg_tx + 2))), kThreads, 0, s>>>(a, lg_tx);
  return cudaGetLastError();
}

constexpr int kStepWide = 64;  // columns of a state that a block has, so that rt is 8 at most
template <class T>
cudaError_t launch_step(const simx_attention& a, cudaStream_t s) {
  int lg = 0;
  while (4 << lg < std::min<int64_t>(a.dv, kStepWide)) ++lg;
  const int rows = kThreads >> lg, rt = (int)((a.dk + rows - 1) / rows);
  return rt <= 1 ? run_step<T, 1>(a, lg, s) : rt <= 2 ? run_step<T, 2>(a, lg, s) : rt <= 4 ? run_step<T, 4>(a, lg, s) : run_step<T, 8>(a, lg, s);
}

void set(const void*& p, int64_t& sb, int64_t& st, int64_t& sh, const simx_heads& q) {
  p = q.p;
  sb = q.sb;
  st = q.st;
  sh = q.sh;
}

AttnPass base_pass(const simx_attention& a, const Plan& p) {
  AttnPass P = {};
  P.batch = a.batch;
  P.len = a.len;
  P.heads = a.heads;
  P.dtype = a.dtype;
  P.ld = a.log_decay;
  P.done = a.done;
  P.dsb = a.done_sb;
  P.dst = a.done_st;
  P.segs = p.segs;
  P.seg_len = p.seg_len;
  P.adiv = P.bdiv = P.cdiv = 1;
  P.inject = P.out_scale = 1.0f;
  return P;
}

}  // namespace

size_t attn_workspace_bytes(int64_t batch, int64_t len, int64_t heads, int64_t, int64_t dk, int64_t dv) {
  return most_bytes(1, batch, len, heads, dk, dv);
}

size_t attn_grad_workspace_bytes(int64_t batch, int64_t len, int64_t heads, int64_t kv_heads, int64_t dk, int64_t dv) {
  size_t n = most_bytes(3, batch, len, heads, dk, dv);
  if (heads != kv_heads) n += up16((size_t)batch * len * heads * dk * 4) + up16((size_t)batch * len * heads * dv * 4);
  return n;
}

cudaError_t launch_attn(const simx_attention& a, void* ws, cudaStream_t s) {
  if (a.len <= most_steps(a)) return a.dtype == SIMX_F32 ? launch_step<float>(a, s) : launch_step<__nv_bfloat16>(a, s);
  const Plan p = plan(a.dtype, 1, a.batch, a.len, a.heads, a.dk, a.dv);
  Passes all = {};
  AttnPass& P = all.p[0];
  P = base_pass(a, p);
  P.da = (int)a.dk;
  P.dc = (int)a.dv;
  P.first = 1;
  set(P.a, P.asb, P.ast, P.ash, a.q);
  set(P.b, P.bsb, P.bst, P.bsh, a.k);
  set(P.c, P.csb, P.cst, P.csh, a.v);
  P.bdiv = P.cdiv = (int)(a.heads / a.kv_heads);
  P.o = a.o.p;
  P.osb = a.o.sb;
  P.ost = a.o.st;
  P.osh = a.o.sh;
  P.out_scale = a.scale;
  P.s_in = a.s0;
  P.s_out = a.s_last;
  P.sx = a.dv;
  P.sy = 1;
  P.seg_state = static_cast<float*>(ws);
  P.seg_keep = P.seg_state + up16((size_t)a.batch * a.heads * p.segs * a.dk * a.dv * 4) / 4;
  if (p.segs > 1 && a.s0 && a.s0 == a.s_last) {  // a segment may start after the last one has ended
    char* copy = static_cast<char*>(ws) + seg_bytes(p, a.batch, a.heads, a.dk, a.dv);
    const cudaError_t e = cudaMemcpyAsync(copy, a.s0, (size_t)a.batch * a.heads * a.dk * a.dv * 4, cudaMemcpyDeviceToDevice, s);
    if (e != cudaSuccess) return e;
    P.s_in = reinterpret_cast<const float*>(copy);
  }
  return run_passes(all, 1, shares_at(p, ws), s);
}

cudaError_t launch_attn_grad(const simx_attention& a, void* ws, cudaStream_t s) {
  const size_t state = (size_t)a.batch * a.heads * a.dk * a.dv * 4;
  if (a.len == 0) {
    if (!a.ds0) return cudaSuccess;
    return a.ds_last ? cudaMemcpyAsync(a.ds0, a.ds_last, state, cudaMemcpyDeviceToDevice, s) : cudaMemsetAsync(a.ds0, 0, state, s);
  }
  const Plan p = plan(a.dtype, 3, a.batch, a.len, a.heads, a.dk, a.dv);
  const int group = (int)(a.heads / a.kv_heads);
  char* w = static_cast<char*>(ws);
  Passes all = {};
  for (int i = 0; i < 3; ++i) {
    AttnPass& P = all.p[i];
    P = base_pass(a, p);
    P.da = (int)(i == 2 ? a.dk : a.dv);
    P.dc = (int)(i == 2 ? a.dv : a.dk);
    P.sx = i == 2 ? a.dv : 1;
    P.sy = i == 2 ? 1 : a.dv;
    if (p.segs > 1) {
      P.seg_state = reinterpret_cast<float*>(w);
      P.seg_keep = reinterpret_cast<float*>(w + up16((size_t)a.batch * a.heads * p.segs * a.dk * a.dv * 4));
      w += seg_bytes(p, a.batch, a.heads, a.dk, a.dv);
    }
  }
  if (p.grid) w += plan_bytes(p, 3, a.batch, a.len, a.heads, a.dk, a.dv);
  AttnPass &Q = all.p[0], &K = all.p[1], &V = all.p[2];
  Q.first = 1;
  set(Q.a, Q.asb, Q.ast, Q.ash, a.grad_o);
  set(Q.b, Q.bsb, Q.bst, Q.bsh, a.v);
  set(Q.c, Q.csb, Q.cst, Q.csh, a.k);
  Q.bdiv = Q.cdiv = group;
  Q.o = a.grad_q.p;
  Q.osb = a.grad_q.sb;
  Q.ost = a.grad_q.st;
  Q.osh = a.grad_q.sh;
  Q.out_scale = a.scale;
  Q.s_in = a.s0;
  for (AttnPass* P : {&K, &V}) {
    const bool key = P == &K;
    const simx_heads& g = key ? a.grad_k : a.grad_v;
    P->reverse = 1;
    set(P->a, P->asb, P->ast, P->ash, key ? a.v : a.k);
    set(P->b, P->bsb, P->bst, P->bsh, key ? a.grad_o : a.q);
    set(P->c, P->csb, P->cst, P->csh, key ? a.q : a.grad_o);
    P->adiv = group;
    P->inject = a.scale;
    P->s_in = a.ds_last;
    if (group == 1) {
      P->o = g.p;
      P->osb = g.sb;
      P->ost = g.st;
      P->osh = g.sh;
    } else {
      P->o = w;
      P->o_f32 = 1;
      P->osh = P->dc;
      P->ost = a.heads * P->dc;
      P->osb = a.len * P->ost;
      w += up16((size_t)a.batch * a.len * P->ost * 4);
    }
  }
  V.s_out = a.ds0;
  cudaError_t e;
  if ((e = run_passes(all, 3, shares_at(p, ws), s)) != cudaSuccess) return e;
  if (group == 1) return cudaSuccess;
  for (const AttnPass* P : {&K, &V}) {
    const int64_t n = a.batch * a.len * a.kv_heads * P->dc;
    const unsigned blocks = (unsigned)std::min<int64_t>((n + kThreads - 1) / kThreads, 152 * 16);
    const simx_heads& g = P == &K ? a.grad_k : a.grad_v;
    count_launches(1);
    auto f = a.dtype == SIMX_F32 ? k_attn_groups<float> : k_attn_groups<__nv_bfloat16>;
    f<<<blocks, kThreads, 0, s>>>(static_cast<const float*>(P->o), g, a.batch, a.len, (int)a.kv_heads, group, P->dc);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace simx

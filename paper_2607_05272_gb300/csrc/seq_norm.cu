// seq_norm.cu — dropout of a branch, its addition to the residual stream and the root-mean-square
// norm of the sum, forward and backward, with a mask drawn from Philox counters in both passes
// instead of being stored.
//
// z = residual + keep x scale, rstd = 1 / sqrt(mean z^2 + eps), y = z rstd gain; backward, with
// zh = z rstd: dresidual = dz + rstd (dy gain - zh mean(dy gain zh)), dx = keep scale dresidual,
// dgain = sum over rows of dy zh.
//
// Bound by HBM: 2 reads and 2 writes per element forward, 3 and 2 backward; the generator's ten rounds are
// the largest part of the instructions, so a draw gives eight 16-bit fields, one per column, and the drop
// probability is a multiple of 2^-16.  A row stays in the registers of 1 to 32 warps between its sum and
// its output, in units of 8 columns per thread.
// Measured on one GB300 (floors at 6783 GB/s), bf16 with p = 0.1: forward 16,384 x 4096 90 us (79), backward
// 124 (99); rows that are off the 16-byte grid, 16,384 x 2047: 83 (40) and 117 (50), by instructions (74 per
// element backward: partial units, sums in shared memory because columns move between threads).  fp32 16,384 x
// 4096: 187 (158) and 214 (198).  Narrow rows leave lanes of their warp idle: 131,072 x 64 fp32 56 (20) and 70
// (25); fp32 rows of more than 8192 columns hold more than their registers: 4096 x 16,384 210 (158) and 354 (198),
// off the grid 4096 x 16,383 371 and 578.
#include <algorithm>

#include "kernels.h"
#include "seq_common.cuh"

namespace simx {

using namespace seq;

namespace {

constexpr uint32_t kStreamDropout = 6;  // beside the simulator's streams 1 .. 5
constexpr int kUnit = 8;                // columns per draw, and per thread and step
constexpr int kMaxSlabs = 1216;         // partial rows of dgain

struct Drop {
  uint32_t key0, key1, step, row_base, thr;  // thr: fields below it are dropped; 0: no dropout
  float scale;
};

// The keep bits of columns 8 group .. 8 group + 7 of a row (bit j: column 8 group + j).  A word's high
// field is at least thr where the word is at least thr << 16, and its low one likewise after a shift.
__device__ __forceinline__ uint32_t keep_bits(const Drop& D, uint32_t group, uint32_t row) {
  const U4 w = philox(group, row, D.step, kStreamDropout, D.key0, D.key1);
  const uint32_t f[4] = {w.x, w.y, w.z, w.w}, t = D.thr << 16;
  uint32_t b = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((f[i] << 16) >= t) b |= 1u << (2 * i);
    if (f[i] >= t) b |= 2u << (2 * i);
  }
  return b;
}

// Eight elements as they lie in memory.
template <class T>
struct Raw {
  static constexpr int Q = (int)sizeof(T) / 2;  // 16-byte vectors
  uint4 q[Q];
};
__device__ __forceinline__ float elem(const Raw<float>& r, int j) {
  const uint32_t w[8] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w, r.q[1].x, r.q[1].y, r.q[1].z, r.q[1].w};
  return __uint_as_float(w[j]);
}
__device__ __forceinline__ float elem(const Raw<__nv_bfloat16>& r, int j) {
  const uint32_t w[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
  return __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
}
__device__ __forceinline__ Raw<float> raw_of(const float (&v)[8], float) {
  Raw<float> r;
  r.q[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  r.q[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
  return r;
}
__device__ __forceinline__ Raw<__nv_bfloat16> raw_of(const float (&v)[8], __nv_bfloat16) {
  Raw<__nv_bfloat16> r;
  r.q[0] = make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
  return r;
}

// One unit of a row element by element, zeros outside of it.
template <class T>
__device__ __noinline__ Raw<T> load_slow(const T* p, int c0, int width) {
  float f[kUnit];
#pragma unroll
  for (int j = 0; j < kUnit; ++j) f[j] = c0 + j >= 0 && c0 + j < width ? widen(p[c0 + j]) : 0.0f;
  return raw_of(f, T());
}
template <class T>
__device__ __noinline__ void store_slow(T* p, int c0, int width, Raw<T> r) {
#pragma unroll
  for (int j = 0; j < kUnit; ++j)
    if (c0 + j >= 0 && c0 + j < width) p[c0 + j] = narrow<T>(elem(r, j));
}

// A row of a tensor on the grid of units: unit v holds columns 8 v - ph .. 8 v - ph + 7, ph the elements
// between a 16-byte boundary and the row that gives the grid.  on_grid: this tensor's row lies on it too.
// A partial unit is loaded whole all the same (what lies beside the row belongs to the rows next to it)
// and masked, except where it would leave the tensor.
// AL: every row of every tensor is aligned and the width a multiple of 8.
template <class T, bool AL>
struct Row {
  T* p;
  bool on_grid;
  int64_t before, after;  // elements of the tensor before the row, and from its start on
  __device__ __forceinline__ Row(const void* base, int64_t row, int64_t ld, int ph, int64_t n, int width)
      : p(const_cast<T*>(static_cast<const T*>(base)) + (base ? row * ld : 0)),
        on_grid(AL || phase(p) == ph), before(row * ld), after((n - 1 - row) * ld + width) {}
  static __device__ __forceinline__ int phase(const T* p) { return (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T)); }
  __device__ __forceinline__ Raw<T> load(int v, int ph, int width) const {
    const int c0 = v * kUnit - ph;
    // inside the row, or at least inside the tensor
    if (AL || (on_grid && ((c0 >= 0 && c0 + kUnit <= width) || (c0 + before >= 0 && c0 + kUnit <= after)))) {
      Raw<T> r;
      const uint4* g = reinterpret_cast<const uint4*>(p + c0);
#pragma unroll
      for (int i = 0; i < Raw<T>::Q; ++i) r.q[i] = g[i];
      return r;
    }
    return load_slow(static_cast<const T*>(p), c0, width);
  }
  __device__ __forceinline__ void store(int v, int ph, int width, const float (&f)[kUnit]) const {
    const int c0 = v * kUnit - ph;
    const Raw<T> r = raw_of(f, T());
    if (AL || (on_grid && c0 >= 0 && c0 + kUnit <= width)) {
      uint4* g = reinterpret_cast<uint4*>(p + c0);
#pragma unroll
      for (int i = 0; i < Raw<T>::Q; ++i) __stcs(g + i, r.q[i]);
    } else {
      store_slow(p, c0, width, r);
    }
  }
};

// Shared arrays over columns, for rows off the grid: column c in plane c % 8 at c / 8 + 1, so that lanes
// with neighbouring units read neighbouring words whatever the phase; places before and behind the row
// hold zeros.  Element j of unit v of phase ph is at plane_of(j, ph, pitch) + v.
__device__ __forceinline__ int plane_pitch(int width) { return width / kUnit + 4; }
__device__ __forceinline__ int plane_of(int j, int ph, int pitch) {
  return ((j - ph) & 7) * pitch + (j < ph ? 0 : 1);
}

// Where a thread finds its units' elements in such an array in a row of phase ph: element j of its unit k at
// p[j][32 k].
struct Places {
  float* p[kUnit];
  __device__ __forceinline__ Places(float* base, int v0, int ph, int pitch) {
#pragma unroll
    for (int j = 0; j < kUnit; ++j) p[j] = base + plane_of(j, ph, pitch) + v0;
  }
};

// The gains of unit v, the thread's unit k: from the caches, or from shared memory.
template <bool AL>
__device__ __forceinline__ void gains(const float* gain, const Places& sh, int v, int k, float (&w)[kUnit]) {
  if (AL) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(gain) + 2 * v), b = __ldg(reinterpret_cast<const float4*>(gain) + 2 * v + 1);
    const float q[kUnit] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < kUnit; ++j) w[j] = q[j];
  } else {
#pragma unroll
    for (int j = 0; j < kUnit; ++j) w[j] = sh.p[j][32 * k];
  }
}
__device__ __forceinline__ void fill_gains(const float* gain, float* sh, int width) {
  const int pitch = plane_pitch(width);
  for (int i = threadIdx.x; i < kUnit * pitch; i += blockDim.x) {
    const int c = (i % pitch - 1) * kUnit + i / pitch;
    sh[i] = c >= 0 && c < width ? gain[c] : 0.0f;
  }
}

// The keep bits of a warp's units first + 32 i + lane, i < NV, of a row of phase ph.  A unit's columns are
// the last ph of one group and the first 8 - ph of the next, which the next lane draws.
template <int NV, bool AL>
__device__ __forceinline__ void unit_bits(const Drop& D, int first, int units, uint32_t row, int ph, uint32_t (&bits)[NV]) {
  const int lane = threadIdx.x & 31;
  uint32_t before = 0;  // of the unit before the warp's first
  if (!AL && ph != 0 && first > 0) before = keep_bits(D, (uint32_t)(first - 1), row);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (first + 32 * i >= units) break;  // the same in the whole warp
    const uint32_t own = keep_bits(D, (uint32_t)(first + 32 * i + lane), row);
    bits[i] = own;
    if (!AL && ph != 0) {
      uint32_t prev = __shfl_up_sync(0xffffffffu, own, 1);
      if (lane == 0) prev = before;
      before = __shfl_sync(0xffffffffu, own, 31);
      bits[i] = (prev | own << 8) >> (8 - ph);
    }
  }
}

// Joins v over the warps of a row; turn: calls so far (the tables alternate, so that one barrier does).
template <bool ONE>
__device__ __forceinline__ float row_sum(float v, int turn, float (&sh)[2][32]) {
  v = sum_lanes(v);
  if (ONE) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) sh[turn & 1][threadIdx.x / 32] = v;
  __syncthreads();
  return sum_lanes(lane < (int)blockDim.x / 32 ? sh[turn & 1][lane] : 0.0f);
}

constexpr int kRowsOfOne = 4;  // ONE: a warp per row, four to a block; else a block per row

// Threads per SM: 512 with 16 registers of each tensor a thread, twice as many with 8 or fewer.
template <class T, int NV>
constexpr int norm_sm_threads() {
  return NV * (int)sizeof(T) * 2 <= 8 ? 1024 : 512;
}
// Most threads of a block (rows of 17 warps and more: 64 registers a thread), and blocks per SM of them.
template <bool ONE, bool WIDE>
constexpr int norm_threads() {
  return ONE ? 32 * kRowsOfOne : WIDE ? 1024 : 512;
}
template <class T, bool ONE, int NV, bool WIDE>
constexpr int norm_blocks_per_sm() {
  return std::max(1, norm_sm_threads<T, NV>() / norm_threads<ONE, WIDE>());
}

template <class T, bool ONE, int NV, bool AL, bool WIDE>
__global__ void __launch_bounds__((norm_threads<ONE, WIDE>()), (norm_blocks_per_sm<T, ONE, NV, WIDE>())) k_norm_rows(simx_norm A, Drop D) {
  constexpr int RB = ONE ? kRowsOfOne : 1;
  extern __shared__ float gs[];
  __shared__ float sh[2][32];
  const int lane = threadIdx.x & 31, warp = (int)threadIdx.x / 32, width = (int)A.width, pitch = plane_pitch(width);
  const int first = (ONE ? 0 : warp) * NV * 32;
  if (!AL) {
    fill_gains(A.gain, gs, width);
    __syncthreads();
  }
  int turn = 0;
  for (int64_t i = (int64_t)blockIdx.x * RB + (ONE ? warp : 0); i < A.n; i += (int64_t)gridDim.x * RB) {
    const int ph = AL ? 0 : Row<T, AL>::phase(static_cast<const T*>(A.x) + i * A.x_ld);
    const int units = (ph + width + kUnit - 1) / kUnit;
    const Row<T, AL> x(A.x, i, A.x_ld, ph, A.n, width), res(A.residual, i, A.residual_ld, ph, A.n, width);
    const Places gp(gs, first + lane, ph, pitch);
    Raw<T> rx[NV], rr[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = first + 32 * k + lane;
      if (v < units) {
        rx[k] = x.load(v, ph, width);
        if (A.residual) rr[k] = res.load(v, ph, width);
      }
    }
    uint32_t bits[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) bits[k] = 0xFFu;
    if (D.thr) unit_bits<NV, AL>(D, first, units, D.row_base + (uint32_t)i, ph, bits);
    float f[NV][kUnit], ss = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = first + 32 * k + lane, c0 = v * kUnit - ph;
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        float s = A.residual ? elem(rr[k], j) : 0.0f;
        if (bits[k] >> j & 1u) s = __fmaf_rn(elem(rx[k], j), D.scale, s);
        f[k][j] = s;
      }
      if (v >= units || (!AL && (c0 < 0 || c0 + kUnit > width))) {  // columns outside the row are zeros
#pragma unroll
        for (int j = 0; j < kUnit; ++j)
          if (v >= units || c0 + j < 0 || c0 + j >= width) f[k][j] = 0.0f;
      }
#pragma unroll
      for (int j = 0; j < kUnit; ++j) ss = __fmaf_rn(f[k][j], f[k][j], ss);
    }
    ss = row_sum<ONE>(ss, turn++, sh);
    const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, (float)width), A.eps)));
    const Row<T, AL> z(A.z, i, A.z_ld, ph, A.n, width), y(A.y, i, A.y_ld, ph, A.n, width);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = first + 32 * k + lane;
      if (v >= units) continue;
      float w[kUnit], o[kUnit];
      gains<AL>(A.gain, gp, v, k, w);
#pragma unroll
      for (int j = 0; j < kUnit; ++j) o[j] = __fmul_rn(__fmul_rn(f[k][j], r), w[j]);
      if (A.z) z.store(v, ph, width, f[k]);
      y.store(v, ph, width, o);
    }
    if (A.rstd && lane == 0 && (ONE || warp == 0)) A.rstd[i] = r;
  }
}

// Zeros the elements of a unit outside the row.
template <class T>
__device__ __forceinline__ Raw<T> masked(const Raw<T>& r, int c0, int width) {
  float f[kUnit];
#pragma unroll
  for (int j = 0; j < kUnit; ++j) f[j] = c0 + j >= 0 && c0 + j < width ? elem(r, j) : 0.0f;
  return raw_of(f, T());
}

// Backward.  slab [gridDim][width]: the block's sums of dy zh (or null).  Where a thread's columns are the
// same in every row they are in registers; else in shared memory, an array per warp over its own units and
// one place before them (which the warp before has too), so that no other warp waits.
template <class T, bool ONE, int NV, bool AL, bool WIDE>
__global__ void __launch_bounds__((norm_threads<ONE, WIDE>()), (norm_blocks_per_sm<T, ONE, NV, WIDE>())) k_norm_grad_rows(simx_norm A, Drop D, float* slab) {
  constexpr int RB = ONE ? kRowsOfOne : 1, SP = NV * 32 + 2;  // pitch of a warp's planes
  extern __shared__ float gs[];
  __shared__ float sh[2][32];
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = (int)threadIdx.x / 32, width = (int)A.width, pitch = plane_pitch(width);
  const int first = (ONE ? 0 : warp) * NV * 32, warps = (int)blockDim.x / 32;
  float* all = gs + (AL ? 0 : kUnit * pitch);
  float* sums = all + warp * kUnit * SP;  // !AL
  if (!AL) {
    fill_gains(A.gain, gs, width);
    for (int c = threadIdx.x; c < warps * kUnit * SP; c += (int)blockDim.x) all[c] = 0.0f;
    __syncthreads();
  }
  float acc[AL ? NV : 1][kUnit] = {};
  int turn = 0;
  for (int64_t i = (int64_t)blockIdx.x * RB + (ONE ? warp : 0); i < A.n; i += (int64_t)gridDim.x * RB) {
    const int ph = AL ? 0 : Row<T, AL>::phase(static_cast<const T*>(A.z) + i * A.z_ld);
    const int units = (ph + width + kUnit - 1) / kUnit;
    const Row<T, AL> z(A.z, i, A.z_ld, ph, A.n, width), dy(A.dy, i, A.dy_ld, ph, A.n, width), dz(A.dz, i, A.dz_ld, ph, A.n, width);
    const Places gp(gs, first + lane, ph, pitch), sp(sums, lane, ph, SP);
    const float r = A.rstd[i];
    Raw<T> rz[NV], ry[NV], rd[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = first + 32 * k + lane;
      if (v < units) {
        rz[k] = z.load(v, ph, width);
        ry[k] = dy.load(v, ph, width);
        if (A.dz) rd[k] = dz.load(v, ph, width);
      }
    }
    uint32_t bits[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) bits[k] = 0xFFu;
    if (D.thr && A.dx) unit_bits<NV, AL>(D, first, units, D.row_base + (uint32_t)i, ph, bits);
    float dot = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = first + 32 * k + lane, c0 = v * kUnit - ph;
      if (v >= units) continue;
      if (!AL && (c0 < 0 || c0 + kUnit > width)) {
        rz[k] = masked(rz[k], c0, width);
        ry[k] = masked(ry[k], c0, width);
      }
      float w[kUnit];
      gains<AL>(A.gain, gp, v, k, w);
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const float zh = __fmul_rn(elem(rz[k], j), r), d = elem(ry[k], j);
        dot = __fmaf_rn(__fmul_rn(d, w[j]), zh, dot);
        if (AL) {
          acc[AL ? k : 0][j] = __fmaf_rn(d, zh, acc[AL ? k : 0][j]);
        } else if (slab) {
          sp.p[j][32 * k] = __fmaf_rn(d, zh, sp.p[j][32 * k]);
        }
      }
    }
    const float mean = __fdiv_rn(row_sum<ONE>(dot, turn++, sh), (float)width);
    const Row<T, AL> dx(A.dx, i, A.dx_ld, ph, A.n, width), dr(A.dresidual, i, A.dresidual_ld, ph, A.n, width);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = first + 32 * k + lane;
      if (v >= units) continue;
      float w[kUnit], o[kUnit];
      gains<AL>(A.gain, gp, v, k, w);
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const float zh = __fmul_rn(elem(rz[k], j), r);
        o[j] = __fmul_rn(r, __fmaf_rn(-zh, mean, __fmul_rn(elem(ry[k], j), w[j])));
        if (A.dz) o[j] = __fadd_rn(o[j], elem(rd[k], j));
      }
      if (A.dresidual) dr.store(v, ph, width, o);
      if (A.dx) {
#pragma unroll
        for (int j = 0; j < kUnit; ++j) o[j] = bits[k] >> j & 1u ? __fmul_rn(o[j], D.scale) : 0.0f;
        dx.store(v, ph, width, o);
      }
    }
    if (!AL) __syncwarp();  // the next row's columns may be other lanes'
  }
  if (!slab) return;
  float* out = slab + (int64_t)blockIdx.x * width;
  if (AL && !ONE) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (first + 32 * k + lane) * kUnit;
      if (c < width) {
        *reinterpret_cast<float4*>(out + c) = make_float4(acc[AL ? k : 0][0], acc[AL ? k : 0][1], acc[AL ? k : 0][2], acc[AL ? k : 0][3]);
        *reinterpret_cast<float4*>(out + c + 4) = make_float4(acc[AL ? k : 0][4], acc[AL ? k : 0][5], acc[AL ? k : 0][6], acc[AL ? k : 0][7]);
      }
    }
    return;
  }
  if (AL) {  // the block's rows by way of shared memory
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (32 * k + lane) * kUnit;
#pragma unroll
      for (int j = 0; j < kUnit; ++j)
        if (c + j < width) gs[warp * width + c + j] = acc[AL ? k : 0][j];
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < width; c += (int)blockDim.x) {
    float v = 0.0f;
    if (AL) {
      for (int q = 0; q < RB; ++q) v = __fadd_rn(v, gs[q * width + c]);
    } else if (ONE) {
      for (int q = 0; q < RB; ++q) v = __fadd_rn(v, all[(q * kUnit + c % kUnit) * SP + c / kUnit + 1]);
    } else {  // the warp of the column's unit, and the place before the first of the next
      const int u = c / kUnit, q = u / (NV * 32), l = u % (NV * 32);
      v = all[(q * kUnit + c % kUnit) * SP + l + 1];
      if (l == NV * 32 - 1 && q + 1 < warps) v = __fadd_rn(v, all[((q + 1) * kUnit + c % kUnit) * SP]);
    }
    out[c] = v;
  }
}

__global__ void __launch_bounds__(1024) k_norm_dgain(const float* slab, int64_t slabs, int64_t width, float* dgain) {
  pdl_wait();
  column_sums(slab, slabs, width, (int64_t)blockIdx.x * 32, dgain);
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

// Whether every given tensor's rows are 16-byte aligned and the width a multiple of a unit.
bool aligned(const simx_norm& a, bool grad) {
  const int64_t es = a.dtype == SIMX_F32 ? 4 : 2;
  const auto ok = [&](const void* p, int64_t ld) {
    return !p || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && (a.n == 1 || ld * es % 16 == 0));
  };
  if (a.width % kUnit != 0 || (reinterpret_cast<uintptr_t>(a.gain) & 15)) return false;
  if (!ok(a.z, a.z_ld)) return false;
  if (!grad) return ok(a.x, a.x_ld) && ok(a.residual, a.residual_ld) && ok(a.y, a.y_ld);
  return ok(a.dy, a.dy_ld) && ok(a.dz, a.dz_ld) && ok(a.dx, a.dx_ld) && ok(a.dresidual, a.dresidual_ld);
}

template <class T, bool ONE, int NV, bool AL, bool WIDE>
cudaError_t norm_launch(const simx_norm& a, const Drop& d, int warps, float* slab, int64_t& slabs, bool grad, cudaStream_t s) {
  const int threads = 32 * (ONE ? kRowsOfOne : warps);
  const size_t planes = (size_t)(kUnit * (a.width / kUnit + 4));
  size_t sh = AL ? 0 : planes * sizeof(float);
  if (grad) sh = AL ? (ONE ? (size_t)a.width * kRowsOfOne * sizeof(float) : 0) : (planes + (size_t)(threads / 32) * kUnit * (NV * 32 + 2)) * sizeof(float);
  // as many blocks as the GPU holds at a time, each with rows in turn; the backward pass leaves a slab each
  const int per_sm = std::max(1, norm_sm_threads<T, NV>() / threads);
  const int64_t rb = ONE ? kRowsOfOne : 1;
  slabs = std::min<int64_t>({(a.n + rb - 1) / rb, (int64_t)sm_count() * per_sm, kMaxSlabs});
  cudaError_t e = cudaSuccess;
  if (grad) {
    const auto kernel = k_norm_grad_rows<T, ONE, NV, AL, WIDE>;
    if ((e = allow_smem(kernel, 160 * 1024)) != cudaSuccess) return e;
    kernel<<<(unsigned)slabs, threads, sh, s>>>(a, d, slab);
  } else {
    const auto kernel = k_norm_rows<T, ONE, NV, AL, WIDE>;
    if ((e = allow_smem(kernel, 80 * 1024)) != cudaSuccess) return e;
    kernel<<<(unsigned)slabs, threads, sh, s>>>(a, d);
  }
  count_launches(1);
  return cudaGetLastError();
}

// Units per thread and warps per row: up to 16 32-bit registers of each tensor a thread (4 units of bf16, 2 of
// fp32); a warp per row where that has room, else the count of units that leaves the fewest places empty
// (rows off the 16-byte grid lie on one unit more).
template <class T, bool AL>
cudaError_t norm_rows(const simx_norm& a, const Drop& d, float* slab, int64_t& slabs, bool grad, cudaStream_t s) {
  constexpr int NV = sizeof(T) == 4 ? 2 : 4;
  const int units = (int)((a.width + (AL ? 0 : 16 / (int)sizeof(T) - 1) + kUnit - 1) / kUnit);
  if (units <= 32) return norm_launch<T, true, 1, AL, false>(a, d, 1, slab, slabs, grad, s);
  if (NV == 4 && units <= 64) return norm_launch<T, true, 2, AL, false>(a, d, 1, slab, slabs, grad, s);
  if (units <= 32 * NV) return norm_launch<T, true, NV, AL, false>(a, d, 1, slab, slabs, grad, s);
  const auto warps = [&](int nv) { return (units + 32 * nv - 1) / (32 * nv); };
  if (NV == 4 && warps(3) <= 16 && warps(3) * 3 < warps(4) * 4) return norm_launch<T, false, NV == 4 ? 3 : NV, AL, false>(a, d, warps(3), slab, slabs, grad, s);
  if (warps(NV) <= 16) return norm_launch<T, false, NV, AL, false>(a, d, warps(NV), slab, slabs, grad, s);
  if constexpr (sizeof(T) == 4) {
    if constexpr (!AL)
      if (warps(NV) > 32) return norm_launch<T, false, 2 * NV, AL, true>(a, d, warps(2 * NV), slab, slabs, grad, s);
    return norm_launch<T, false, NV, AL, true>(a, d, warps(NV), slab, slabs, grad, s);
  } else if constexpr (!AL) {
    return norm_launch<T, false, NV, AL, true>(a, d, warps(NV), slab, slabs, grad, s);
  }
  return cudaErrorInvalidValue;  // not reached: aligned bf16 rows of 16,384 columns take 16 warps
}

cudaError_t norm_any(const simx_norm& a, float* slab, int64_t& slabs, bool grad, cudaStream_t s) {
  const Drop d = drop_of(a);
  if (aligned(a, grad))
    return a.dtype == SIMX_F32 ? norm_rows<float, true>(a, d, slab, slabs, grad, s)
                               : norm_rows<__nv_bfloat16, true>(a, d, slab, slabs, grad, s);
  return a.dtype == SIMX_F32 ? norm_rows<float, false>(a, d, slab, slabs, grad, s)
                             : norm_rows<__nv_bfloat16, false>(a, d, slab, slabs, grad, s);
}

}  // namespace

size_t norm_grad_workspace_bytes(int64_t n, int64_t width) {
  return (size_t)std::min<int64_t>(n, kMaxSlabs) * (size_t)width * sizeof(float);
}

cudaError_t launch_norm(const simx_norm& a, cudaStream_t s) {
  int64_t slabs = 0;
  return norm_any(a, nullptr, slabs, false, s);
}

cudaError_t launch_norm_grad(const simx_norm& a, void* ws, cudaStream_t s) {
  float* slab = a.dgain ? static_cast<float*>(ws) : nullptr;
  int64_t slabs = 0;
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute at[1];
  if (a.n > 0) {
    const cudaError_t e = norm_any(a, slab, slabs, true, s);
    if (e != cudaSuccess) return e;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = 1;
  }
  if (!a.dgain) return cudaSuccess;  // not `slab`: without rows the workspace has no bytes, and may be NULL
  lc.gridDim = dim3((unsigned)((a.width + 31) / 32));
  lc.blockDim = dim3(1024);
  lc.stream = s;
  count_launches(1);
  const cudaError_t e = cudaLaunchKernelEx(&lc, k_norm_dgain, (const float*)slab, slabs, a.width, a.dgain);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace simx

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

// A row of a tensor on the grid of units: unit v holds columns 8 v - ph .. 8 v - ph + 7, ph the elements
// between a 16-byte boundary and the row that gives the grid.  on_grid: this tensor's row lies on it too.
// AL: every row of every tensor is aligned and the width a multiple of 8.
template <class T, bool AL>
struct Row {
  T* p;
  bool on_grid;
  __device__ __forceinline__ Row(const void* base, int64_t row, int64_t ld, int ph)
      : p(const_cast<T*>(static_cast<const T*>(base)) + (base ? row * ld : 0)), on_grid(AL || phase(p) == ph) {}
  static __device__ __forceinline__ int phase(const T* p) { return (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T)); }
  __device__ __forceinline__ Raw<T> load(int v, int ph, int width) const {
    Raw<T> r;
    if (AL || (on_grid && v * kUnit >= ph && v * kUnit - ph + kUnit <= width)) {
      const uint4* g = reinterpret_cast<const uint4*>(p - ph) + v * Raw<T>::Q;
#pragma unroll
      for (int i = 0; i < Raw<T>::Q; ++i) r.q[i] = g[i];
    } else {
      float f[kUnit];
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const int c = v * kUnit - ph + j;
        f[j] = c >= 0 && c < width ? widen(p[c]) : 0.0f;
      }
      r = raw_of(f, T());
    }
    return r;
  }
  __device__ __forceinline__ void store(int v, int ph, int width, const float (&f)[kUnit]) const {
    if (AL || (on_grid && v * kUnit >= ph && v * kUnit - ph + kUnit <= width)) {
      const Raw<T> r = raw_of(f, T());
      uint4* g = reinterpret_cast<uint4*>(p - ph) + v * Raw<T>::Q;
#pragma unroll
      for (int i = 0; i < Raw<T>::Q; ++i) __stcs(g + i, r.q[i]);
    } else {
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const int c = v * kUnit - ph + j;
        if (c >= 0 && c < width) p[c] = narrow<T>(f[j]);
      }
    }
  }
};

// Place of column c in a shared array that lanes read at a distance of 8: one word of padding per 32.
__device__ __forceinline__ int padded(int c) { return c + (c >> 5); }

// The gains of unit v: from the caches, or from shared memory where columns lie across vectors.
template <bool AL>
__device__ __forceinline__ void gains(const float* gain, const float* sh, int v, int ph, int width, float (&w)[kUnit]) {
  if (AL) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(gain) + 2 * v), b = __ldg(reinterpret_cast<const float4*>(gain) + 2 * v + 1);
    const float q[kUnit] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < kUnit; ++j) w[j] = q[j];
  } else {
#pragma unroll
    for (int j = 0; j < kUnit; ++j) {
      const int c = v * kUnit - ph + j;
      w[j] = c >= 0 && c < width ? sh[padded(c)] : 0.0f;
    }
  }
}

// The keep bits of a warp's units first + 32 i + lane, i < NV, of a row of phase ph.  A unit's columns are
// the last ph of one group and the first 8 - ph of the next, which the next lane draws.
template <int NV, bool AL>
__device__ __forceinline__ void unit_bits(const Drop& D, int first, uint32_t row, int ph, uint32_t (&bits)[NV]) {
  const int lane = threadIdx.x & 31;
  uint32_t before = 0;  // of the unit before the warp's first
  if (!AL && ph != 0 && first > 0) before = keep_bits(D, (uint32_t)(first - 1), row);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
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

// Joins v over the W warps of a row; turn: calls so far (the tables alternate, so that one barrier does).
template <int W>
__device__ __forceinline__ float row_sum(float v, int turn, float (&sh)[2][32]) {
  v = sum_lanes(v);
  if (W == 1) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) sh[turn & 1][threadIdx.x / 32] = v;
  __syncthreads();
  return sum_lanes(lane < W ? sh[turn & 1][lane] : 0.0f);
}

template <int W>
constexpr int rows_per_block() {  // narrow rows: a warp each
  return W == 1 ? 4 : 1;
}
template <int W>
constexpr int norm_threads() {
  return 32 * W * rows_per_block<W>();
}

// Blocks per SM: 512 threads with 16 registers of each tensor a thread, twice as many with 8 or fewer.
template <class T, int W, int NV>
constexpr int norm_per_sm() {
  return std::max(1, (NV * (int)sizeof(T) * 2 <= 8 ? 1024 : 512) / norm_threads<W>());
}

template <class T, int W, int NV, bool AL>
__global__ void __launch_bounds__(norm_threads<W>(), (norm_per_sm<T, W, NV>())) k_norm_rows(simx_norm A, Drop D) {
  constexpr int RB = rows_per_block<W>();
  extern __shared__ float gs[];
  __shared__ float sh[2][32];
  const int lane = threadIdx.x & 31, warp = (int)threadIdx.x / 32, width = (int)A.width;
  const int first = (W == 1 ? 0 : warp) * NV * 32;
  if (!AL) {
    for (int c = threadIdx.x; c < width; c += norm_threads<W>()) gs[padded(c)] = A.gain[c];
    __syncthreads();
  }
  int turn = 0;
  for (int64_t i = (int64_t)blockIdx.x * RB + (W == 1 ? warp : 0); i < A.n; i += (int64_t)gridDim.x * RB) {
    const int ph = AL ? 0 : Row<T, AL>::phase(static_cast<const T*>(A.x) + i * A.x_ld);
    const int units = (ph + width + kUnit - 1) / kUnit;
    const Row<T, AL> x(A.x, i, A.x_ld, ph), res(A.residual, i, A.residual_ld, ph), z(A.z, i, A.z_ld, ph), y(A.y, i, A.y_ld, ph);
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
    if (D.thr) unit_bits<NV, AL>(D, first, D.row_base + (uint32_t)i, ph, bits);
    float f[NV][kUnit], ss = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const bool live = first + 32 * k + lane < units;
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        float s = A.residual ? elem(rr[k], j) : 0.0f;
        if (bits[k] >> j & 1u) s = __fmaf_rn(elem(rx[k], j), D.scale, s);
        f[k][j] = live ? s : 0.0f;  // columns outside the row are zeros too
        ss = __fmaf_rn(f[k][j], f[k][j], ss);
      }
    }
    ss = row_sum<W>(ss, turn++, sh);
    const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(ss, (float)width), A.eps)));
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = first + 32 * k + lane;
      if (v >= units) continue;
      float w[kUnit], o[kUnit];
      gains<AL>(A.gain, gs, v, ph, width, w);
#pragma unroll
      for (int j = 0; j < kUnit; ++j) o[j] = __fmul_rn(__fmul_rn(f[k][j], r), w[j]);
      if (A.z) z.store(v, ph, width, f[k]);
      y.store(v, ph, width, o);
    }
    if (A.rstd && lane == 0 && (W == 1 || warp == 0)) A.rstd[i] = r;
  }
}

// Backward.  slab [gridDim][width]: the block's sums of dy zh (or null), in registers where a thread's
// columns are the same in every row, else in shared memory (one array per row of the block).
template <class T, int W, int NV, bool AL>
__global__ void __launch_bounds__(norm_threads<W>(), (norm_per_sm<T, W, NV>())) k_norm_grad_rows(simx_norm A, Drop D, float* slab) {
  constexpr int RB = rows_per_block<W>(), THREADS = norm_threads<W>();
  extern __shared__ float gs[];
  __shared__ float sh[2][32];
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = (int)threadIdx.x / 32, width = (int)A.width, pitch = padded(width) + 1;
  const int first = (W == 1 ? 0 : warp) * NV * 32;
  float* sums = gs + pitch * (1 + (W == 1 ? warp : 0));  // !AL
  if (!AL) {
    for (int c = threadIdx.x; c < width; c += THREADS) gs[padded(c)] = A.gain[c];
    for (int c = threadIdx.x; c < pitch * RB; c += THREADS) gs[pitch + c] = 0.0f;
    __syncthreads();
  }
  float acc[AL ? NV : 1][kUnit] = {};
  int turn = 0;
  for (int64_t i = (int64_t)blockIdx.x * RB + (W == 1 ? warp : 0); i < A.n; i += (int64_t)gridDim.x * RB) {
    const int ph = AL ? 0 : Row<T, AL>::phase(static_cast<const T*>(A.z) + i * A.z_ld);
    const int units = (ph + width + kUnit - 1) / kUnit;
    const Row<T, AL> z(A.z, i, A.z_ld, ph), dy(A.dy, i, A.dy_ld, ph), dz(A.dz, i, A.dz_ld, ph), dx(A.dx, i, A.dx_ld, ph),
        dr(A.dresidual, i, A.dresidual_ld, ph);
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
    if (D.thr && A.dx) unit_bits<NV, AL>(D, first, D.row_base + (uint32_t)i, ph, bits);
    float dot = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = first + 32 * k + lane;
      if (v >= units) continue;
      float w[kUnit];
      gains<AL>(A.gain, gs, v, ph, width, w);
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const float zh = __fmul_rn(elem(rz[k], j), r), d = elem(ry[k], j);
        dot = __fmaf_rn(__fmul_rn(d, w[j]), zh, dot);
        if (AL) {
          acc[AL ? k : 0][j] = __fmaf_rn(d, zh, acc[AL ? k : 0][j]);
        } else if (slab) {
          const int c = v * kUnit - ph + j;
          if (c >= 0 && c < width) sums[padded(c)] = __fmaf_rn(d, zh, sums[padded(c)]);
        }
      }
    }
    const float mean = __fdiv_rn(row_sum<W>(dot, turn++, sh), (float)width);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = first + 32 * k + lane;
      if (v >= units) continue;
      float w[kUnit], o[kUnit];
      gains<AL>(A.gain, gs, v, ph, width, w);
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
    if (!AL) {  // the next row's columns belong to other threads
      if (W > 1) __syncthreads();
      else __syncwarp();
    }
  }
  if (!slab) return;
  float* out = slab + (int64_t)blockIdx.x * width;
  if (AL && W > 1) {
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
  if (AL) {  // the block's warps by way of shared memory
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (32 * k + lane) * kUnit;
#pragma unroll
      for (int j = 0; j < kUnit; ++j)
        if (c + j < width) gs[warp * width + c + j] = acc[AL ? k : 0][j];
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < width; c += THREADS) {
    float v = 0.0f;
    for (int q = 0; q < RB; ++q) v = __fadd_rn(v, AL ? gs[q * width + c] : gs[pitch * (1 + q) + padded(c)]);
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

// Blocks of a launch: at most what the GPU holds at a time, and at most the slabs of dgain.
int64_t norm_blocks(int64_t n, int warps, int per_sm) {
  const int rb = warps == 1 ? 4 : 1;
  return std::min<int64_t>({(n + rb - 1) / rb, (int64_t)sm_count() * per_sm, kMaxSlabs});
}

template <class T, int W, int NV, bool AL>
cudaError_t norm_launch(const simx_norm& a, const Drop& d, float* slab, int64_t& slabs, bool grad, cudaStream_t s) {
  const size_t pitch = (size_t)a.width + (size_t)a.width / 32 + 1;
  size_t sh = AL ? 0 : pitch * sizeof(float);
  if (grad) sh = AL ? (W == 1 ? (size_t)a.width * 4 * sizeof(float) : 0) : pitch * (1 + rows_per_block<W>()) * sizeof(float);
  slabs = norm_blocks(a.n, W, norm_per_sm<T, W, NV>());
  cudaError_t e = cudaSuccess;
  if (grad) {
    if ((e = allow_smem(k_norm_grad_rows<T, W, NV, AL>, 2 * (kNormMaxWidth + kNormMaxWidth / 32 + 1) * (int)sizeof(float))) != cudaSuccess) return e;
    k_norm_grad_rows<T, W, NV, AL><<<(unsigned)slabs, norm_threads<W>(), sh, s>>>(a, d, slab);
  } else {
    if ((e = allow_smem(k_norm_rows<T, W, NV, AL>, (kNormMaxWidth + kNormMaxWidth / 32 + 1) * (int)sizeof(float))) != cudaSuccess) return e;
    k_norm_rows<T, W, NV, AL><<<(unsigned)slabs, norm_threads<W>(), sh, s>>>(a, d);
  }
  count_launches(1);
  return cudaGetLastError();
}

// 16 32-bit registers of each tensor a thread (4 units of bf16, 2 of fp32), and as many warps per row as
// that takes; fewer units for rows that a warp has room for.
template <class T, bool AL>
cudaError_t norm_rows(const simx_norm& a, const Drop& d, float* slab, int64_t& slabs, bool grad, cudaStream_t s) {
  constexpr int NV = sizeof(T) == 4 ? 2 : 4;
  // of a row of any phase that it may have
  const int64_t units = (a.width + (AL ? 0 : 16 / (int)sizeof(T) - 1) + kUnit - 1) / kUnit;
  if (units <= 32) return norm_launch<T, 1, 1, AL>(a, d, slab, slabs, grad, s);
  if (NV == 4 && units <= 64) return norm_launch<T, 1, 2, AL>(a, d, slab, slabs, grad, s);
  if (units <= 32 * NV) return norm_launch<T, 1, NV, AL>(a, d, slab, slabs, grad, s);
  if (units <= 64 * NV) return norm_launch<T, 2, NV, AL>(a, d, slab, slabs, grad, s);
  if (units <= 128 * NV) return norm_launch<T, 4, NV, AL>(a, d, slab, slabs, grad, s);
  if (units <= 256 * NV) return norm_launch<T, 8, NV, AL>(a, d, slab, slabs, grad, s);
  if (units <= 512 * NV) return norm_launch<T, 16, NV, AL>(a, d, slab, slabs, grad, s);
  if constexpr (!AL && sizeof(T) == 4) {  // the widest rows, off the 16-byte grid: one unit more
    if (units > 1024 * NV) return norm_launch<T, 32, 2 * NV, AL>(a, d, slab, slabs, grad, s);
  }
  return norm_launch<T, 32, NV, AL>(a, d, slab, slabs, grad, s);
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
  if (!slab) return cudaSuccess;
  lc.gridDim = dim3((unsigned)((a.width + 31) / 32));
  lc.blockDim = dim3(1024);
  lc.stream = s;
  count_launches(1);
  const cudaError_t e = cudaLaunchKernelEx(&lc, k_norm_dgain, (const float*)slab, slabs, a.width, a.dgain);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace simx

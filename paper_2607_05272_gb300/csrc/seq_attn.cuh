// seq_attn.cuh — shared by the two kernels of a linear attention's passes: seq_attn.cu (FP32 units) and
// seq_attn_tc.cu (tensor cores).
#pragma once
#include "kernels.h"
#include "seq_common.cuh"

namespace simx {
namespace attn {

using namespace seq;

// lambda^n, n >= 0: the product n log lambda is kept in two parts.  NaN for log lambda > 0.
__device__ __forceinline__ float power(float ld, int n) {
  if (!(ld <= 0.0f)) return nan();
  if (n == 0) return 1.0f;
  const float p = __fmul_rn(ld, (float)n);
  if (!(p > -200.0f)) return 0.0f;
  const float e = expf(p);
  return __fmaf_rn(e, __fmaf_rn(ld, (float)n, -p), e);
}

// What rounding took off e^l = v, relative to it; 0 below v = 3 / 4, where no memory is long.  With u = 1 - v, exact,
// l - log v = l + u + u^2 / 2 + ..., whose first two terms cancel.
__device__ __forceinline__ float power_rest(float l, float v) {
  if (!(v >= 0.75f)) return 0.0f;
  const float u = __fsub_rn(1.0f, v);
  float f = 1.0f / 12.0f;
#pragma unroll
  for (int k = 11; k >= 2; --k) f = __fmaf_rn(u, f, 1.0f / (float)k);
  return __fmaf_rn(__fmul_rn(u, u), f, __fadd_rn(l, u));
}

// The same of lambda^n given lambda and lambda^n in fp32, a step; below lambda = 15 / 16 nothing.  n: 1 or 4.
__device__ __forceinline__ float decay_rest(float ld, float lam, float lam_n) {
  if (!(lam >= 0.9375f)) return 0.0f;
  if (lam_n == lam) {
    const float u = __fsub_rn(1.0f, lam);
    float f = __fmaf_rn(u, 1.0f / 6.0f, 0.2f);
    f = __fmaf_rn(u, f, 0.25f);
    f = __fmaf_rn(u, f, 1.0f / 3.0f);
    f = __fmaf_rn(u, f, 0.5f);
    return __fmaf_rn(__fmul_rn(u, u), f, __fadd_rn(ld, u));
  }
  return __fmul_rn(0.25f, power_rest(__fmul_rn(4.0f, ld), lam_n));  // lambda^4 from 0.77 on
}

// What the state before segment q still counts for at the start of segment seg, if segment q has no end of an episode: a
// power of its own, since a product of the segments' powers would add up their roundings.
__device__ __forceinline__ float segments_keep(const AttnPass& A, float ld, int q, int seg) {
  return power(ld, (int)((seg - q) * A.seg_len) - (q == 0 && A.first == 0 ? 1 : 0));
}

template <class T>
__device__ __forceinline__ const T* at(const void* p, int64_t off) { return static_cast<const T*>(p) + off; }

// Whether an episode ended between steps p - 1 and p of the pass, p >= 1; of step 0 in reverse: behind the
// last time.
__device__ __forceinline__ bool cut_before(const AttnPass& A, int64_t b, int64_t p) {
  if (!A.done) return false;
  const int64_t t = A.reverse ? A.len - 1 - p : p - 1;
  return t >= 0 && A.done[b * A.dsb + t * A.dst] != 0;
}

struct Passes {
  AttnPass p[3];
};

// Shares of the tensor cores' passes: where there are heads for all blocks that run at a time, all heads' chunks of all
// passes lie in a row, and each of `grid` blocks takes an equal share of them.  A head that two blocks share is begun by
// the first before all else; the second takes it up last, from the state in `hand`.  flags: how many blocks have
// started, then whether each one's state is there.  grid 0: a block for each segment.
// Dimensions of 128, one block to an SM: 16 x 4096 x 16 heads in 291 us, a block for each head 325; 10 x 2048 x 16 in 110
// and 176; 64 x 512 x 16 in 212 and 219; where heads come out even, 19 x 2048 x 16, 181 and 180; backward 4 x 4096 x 16 in
// 246 and 334.  Of 64, where one block starts beside another's work anyway: 24 x 2048 x 16 in 133 and 156, backward
// 8 x 2048 x 16 in 152 and 180, but 8 x 256 x 16 in 41 and 37; the rule's limits (1.5 heads to a block, 2048 steps) give
// away some: 40 x 1024 x 16 would take 123, by blocks for each head 131.
struct Shares {
  int grid, per, passes;  // per: chunks of a head
  float* hand;
  int* flags;
};
int resident_blocks(int d);                             // blocks that run at a time, for dimensions up to d
int share_grid(int64_t units, int64_t len, int d);      // of `units` heads of all passes; 0: they are not shared out
size_t share_bytes(int64_t units, int64_t len, int d);  // of hand, and 16 for each block, where the flags are

// n passes of bf16 on the tensor cores; KEEP of seq_attn.cu as `keep`.
cudaError_t run_tc(const Passes& all, int n, bool keep, const Shares& shares, cudaStream_t s);

}  // namespace attn
}  // namespace simx

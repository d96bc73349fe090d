// seq_logprob.cu — log probabilities of given tokens, with the entropy and the most probable alternatives.
//
// Per row of logits x, with a reference m near its maximum and the temperature T:
//   s = sum e^((x - m) / T), t = sum e^((x - m) / T) (x - m),
//   log pi(a) = (x_a - m) / T - log s, H = log s - t / (s T).
// Each thread keeps a reference of its own, moved when a term would pass 2^8, and its sums are moved to the row's
// maximum once, so that neither difference above loses digits: with references as far as 2^60 below the maximum, log pi
// of a peak was off by 4e-6 where it is near 0.  Terms are added eight at a time from zero, and these to a sum that keeps
// its rounding errors: one running sum lost the many small terms beside a large one.  Entropies are off by 9e-7 at most
// with references within 2^8, by 3.5e-6 within 2^16; moving them that often costs 1 % of the time.
//
// The largest logits take no work in that pass but each thread's largest.  If t threads of each of w warps hold
// logits at or above a bound, and t w >= top, every logit sought is at or above it, and so is among the logits of the
// threads whose largest is: these are read again, a few dozen in 256 of the row.  They are ranked by 64-bit keys, the
// logit in order-preserving bits above the complement of its index, so that equal logits rank by index and no two
// keys are equal; each warp keeps its largest in a list, a key to a lane, and one warp merges the lists.
//
// Bound by instructions: 8192 rows of 50001 bf16 in 212 us, 58 % of the copy rate, with 22,400 warp instructions to a row
// (issue 69 % of the time), of which joins, candidates and their ranking are a third; of 131072 in 424 us, 76 %; in fp32
// 285 and 742 us, 86 %.  Logits go in pairs, each with one exponential.  40 registers instead of 48, for more warps, spill:
// 223 us.  (A warp to a row of bf16 spills 24 bytes of a thread at 48.)
#include <algorithm>

#include "kernels.h"
#include "seq_common.cuh"

namespace simx {

using namespace seq;

namespace {

constexpr int kRows = 8;       // of a block, with a warp for each
constexpr int kWarps = 8;      // of a row that a block has
constexpr int kMostRanks = 8;  // blocks of a cluster
constexpr float kLag = 8.0f;   // octaves by which a thread's largest term may pass its reference

typedef unsigned long long Key;

// Ascending with x, then descending with the index; -0 counts as +0.  Every key is above 0.
__device__ __forceinline__ Key key_of(float x, uint32_t index) {
  const uint32_t u = __float_as_uint(__fadd_rn(x, 0.0f));
  return (Key)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (0xffffffffu - index);
}
__device__ __forceinline__ float key_value(Key k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

struct Sums {
  float m, s, t;
};

// The sums with reference m; k = log2(e) / T.  Sums of nothing, and ones that vanish, stay zero.
__device__ __forceinline__ void move_to(Sums& a, float m, float k) {
  if (a.m != m && a.s != 0.0f) {
    const float d = __fsub_rn(a.m, m), f = exp2f(__fmul_rn(d, k));
    a.t = f > 0.0f ? __fmul_rn(f, __fmaf_rn(d, a.s, a.t)) : 0.0f;
    a.s = __fmul_rn(f, a.s);
  }
  a.m = m;
}
// `most`: the largest that a lane has seen.
__device__ __forceinline__ Sums join_lanes(Sums a, float most, float k) {
  move_to(a, max_lanes(most), k);
  return {a.m, sum_lanes(a.s), sum_lanes(a.t)};
}
// Of n parts, a lane each.
__device__ __forceinline__ Sums join_parts(const Sums* part, int n, int lane, float k) {
  const Sums a = lane < n ? part[lane] : Sums{-inf(), 0.0f, 0.0f};
  return join_lanes(a, a.m, k);
}

// Puts a key into the list of a warp, in descending order over its lanes; the last one falls out.
__device__ __forceinline__ void insert(Key& mine, Key k, int lane) {
  const int pos = __popc(__ballot_sync(0xffffffffu, mine > k));
  const Key up = __shfl_up_sync(0xffffffffu, mine, 1);
  if (lane > pos) mine = up;
  if (lane == pos) mine = k;
}

// The 32 largest of two lists in descending order, in descending order: the larger of each lane and its mirror image
// are they, and fall into place in five steps.
__device__ __forceinline__ Key merge(Key a, Key b, int lane) {
  const Key m = __shfl_xor_sync(0xffffffffu, b, 31);
  a = a > m ? a : m;
#pragma unroll
  for (int d = 16; d > 0; d /= 2) {
    const Key o = __shfl_xor_sync(0xffffffffu, a, d);
    a = (a > o) == ((lane & d) == 0) ? a : o;
  }
  return a;
}

// fp32 in order-preserving bits, 0 below all.
__device__ __forceinline__ uint32_t ordered(float x) { return (uint32_t)(key_of(x, 0) >> 32); }
__device__ __forceinline__ float from_ordered(uint32_t u) { return key_value((Key)u << 32); }

// A vector of 32 bytes.
template <class T>
struct Vec {
  static constexpr int N = 32 / (int)sizeof(T);
  uint32_t w[8];
  // element 2 i or 2 i + 1 (bf16), i (fp32)
  __device__ __forceinline__ float get(int e) const {
    if (sizeof(T) == 4) return __uint_as_float(w[e]);
    return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  }
  __device__ __forceinline__ void fill() {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  }
  // from element `at` of the row on; what lies outside it is -inf
  __device__ __forceinline__ void load(const T* row, int64_t at, int64_t V) {
    if (at >= 0 && at + N <= V) {
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                   : "l"(row + at));
    } else {
      fill();
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (at + e >= 0 && at + e < V) {
          const uint32_t u = __float_as_uint(widen(row[at + e]));
          if (sizeof(T) == 4) w[e] = u;
          else w[e / 2] = e & 1 ? (w[e / 2] & 0xffffu) | (u & 0xffff0000u) : (w[e / 2] & 0xffff0000u) | u >> 16;
        }
    }
  }
  // whether a logit is so low that differences from it may leave fp32
  __device__ __forceinline__ bool low() const {
    if (sizeof(T) == 4) {
      float m = __uint_as_float(w[0]);
#pragma unroll
      for (int i = 1; i < 8; ++i) m = fminf(m, __uint_as_float(w[i]));
      return !(m > -1e37f);
    }
    uint32_t m = w[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) asm("min.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(m), "r"(w[i]));
    return !(fminf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u)) > -1e37f);
  }
  // the largest that is a number, -inf if none is
  __device__ __forceinline__ float most() const {
    if (sizeof(T) == 4) {
      float m = fmaxf(__uint_as_float(w[0]), -inf());
#pragma unroll
      for (int i = 1; i < 8; ++i) m = fmaxf(m, __uint_as_float(w[i]));
      return m;
    }
    uint32_t m = 0xff80ff80u;
#pragma unroll
    for (int i = 0; i < 8; ++i) asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(m), "r"(w[i]));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
};

// One row for each NW warps.  CLUSTER: one row for each cluster, each block a stretch of it.
template <class T, int NW, bool CLUSTER>
__global__ void __launch_bounds__(NW == 1 ? 32 * kRows : 32 * NW) k_logprobs(const LogprobArgs A) {
  constexpr int N = Vec<T>::N, U = 2, NT = 32 * NW;  // elements of a vector, vectors in flight, threads of a row
  __shared__ Sums sums[NW];
  __shared__ Key keys[CLUSTER ? kMostRanks * 32 : 1], lists[NT];
  __shared__ Sums all[kMostRanks];
  __shared__ uint32_t bounds[NW];
  __shared__ uint8_t chosen[NW == 1 ? 32 * kRows : NT];
  __shared__ int found_by[NW];
  const int lane = threadIdx.x & 31, warp = (int)threadIdx.x / 32;
  uint32_t rank = 0, ranks = 1;
  if (CLUSTER) {
    rank = cluster_rank();
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // this block has started
  }
  const int64_t row = CLUSTER ? blockIdx.x / ranks : NW == 1 ? (int64_t)blockIdx.x * kRows + warp : blockIdx.x;
  if (NW == 1 && row >= A.n) return;
  const T* x = static_cast<const T*>(A.x) + row * A.ld;
  const int64_t V = A.V;
  const int top = A.top;
  // vectors on the row's 32-byte grid; the first may start before the row
  const int off = (int)((reinterpret_cast<uintptr_t>(x) & 31) / sizeof(T));
  const int64_t vecs = (V + off + N - 1) / N, share = (vecs + ranks - 1) / ranks;
  const int64_t v0 = rank * share, v1 = min(vecs, v0 + share);
  // the token's own logit comes beside the rest
  const int64_t tok = A.token ? A.token[row] : 0;
  const float taken = A.logp && tok >= 0 && tok < V ? widen(x[tok]) : 0.0f;
  const int me = NW == 1 ? lane : (int)threadIdx.x;
  float ref = -inf(), best = -inf();
  Sum2 s = {}, t = {};
  bool some = false;
  for (int64_t v = v0 + me; v < v1; v += NT * U) {
    Vec<T> e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (v + u * NT < v1) e[u].load(x, (v + u * NT) * N - off, V);
      else e[u].fill();
    }
    some = true;
    float m = e[0].most();
#pragma unroll
    for (int u = 1; u < U; ++u) m = fmaxf(m, e[u].most());
    best = fmaxf(best, m);
    if (m > ref && !(__fmul_rn(__fsub_rn(m, ref), A.k) <= kLag)) {
      Sums a = {ref, s.value(), t.value()};
      move_to(a, m, A.k);
      s = {a.s, 0.0f};
      t = {a.t, 0.0f};
      ref = m;
    }
    const float r = ref == -inf() ? 0.0f : ref;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (v + u * NT >= v1) break;
      float ps[2] = {}, pt[2] = {};
      if (r < 1e37f && !e[u].low()) {  // two at a time
        Pair s2 = 0, t2 = 0;
        const Pair r2 = pair(-r, -r), k2 = pair(A.k, A.k);
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          const Pair d = add2(pair(e[u].get(i), e[u].get(i + 1)), r2);
          const float2 a = halves(mul2(d, k2));
          const Pair p = pair(ex2(a.x), ex2(a.y));
          s2 = add2(s2, p);
          t2 = fma2(p, d, t2);
        }
        const float2 a = halves(s2), b = halves(t2);
        ps[0] = a.x, ps[1] = a.y, pt[0] = b.x, pt[1] = b.y;
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float d = __fsub_rn(e[u].get(i), r), p = ex2(__fmul_rn(d, A.k));
          ps[i & 1] = __fadd_rn(ps[i & 1], p);
          pt[i & 1] = __fmaf_rn(p, fmaxf(d, -kMost), pt[i & 1]);  // x = -inf: p is 0, and so is the product
        }
      }
      s.add(__fadd_rn(ps[0], ps[1]), 0.0f);
      t.add(__fadd_rn(pt[0], pt[1]), 0.0f);
    }
  }
  Sums sum = join_lanes({ref, s.value(), t.value()}, best, A.k);
  Key mine = 0;
  if (top) {
    // the bound: the each-th largest of every warp's threads, the least of them
    const int each_of = (top + NW - 1) / NW;
    uint32_t mine_u = some ? ordered(best) : 0u, bound = 0u;
    for (int i = 0; i < each_of; ++i) {
      bound = __reduce_max_sync(0xffffffffu, mine_u);
      if (lane == __ffs(__ballot_sync(0xffffffffu, mine_u == bound)) - 1) mine_u = 0u;
    }
    int found;
    uint8_t* who = chosen + (NW == 1 ? warp * 32 : 0);
    if (NW > 1) {
      if (lane == 0) bounds[warp] = bound;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < NW; ++w) bound = min(bound, bounds[w]);
    }
    float floor = bound ? from_ordered(bound) : -inf();
    const unsigned hit = __ballot_sync(0xffffffffu, some && best >= floor);
    int before = 0;
    if (NW == 1) {
      found = __popc(hit);
    } else {
      if (lane == 0) found_by[warp] = __popc(hit);
      __syncthreads();
      found = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        if (w < warp) before += found_by[w];
        found += found_by[w];
      }
    }
    if (hit >> lane & 1) who[before + __popc(hit & ((1u << lane) - 1))] = (uint8_t)me;
    if (NW == 1) __syncwarp();
    else __syncthreads();
    // their vectors again: 2^lg lanes for each of them
    const int each = (int)((v1 - v0 + NT - 1) / NT);
    int lg = 0;
    while (lg < 5 && 1 << lg < each) ++lg;
    Key bar = 0;  // nothing at or below it is among the largest
    for (int j0 = 0; j0 < each; j0 += 1 << lg)
      for (int it = me; it - lane < found << lg; it += NT) {
        const int j = j0 + (it & ((1 << lg) - 1));
        Vec<T> e;
        e.fill();
        int64_t from = 0;
        int lo = N, hi = 0;  // the row's elements of the vector
        if (it < found << lg && j < each) {
          const int64_t v = v0 + who[it >> lg] + (int64_t)j * NT;
          if (v < v1) {
            from = v * N - off;
            e.load(x, from, V);
            lo = from < 0 ? (int)-from : 0;
            hi = V - from < N ? (int)(V - from) : N;
          }
        }
        if (!__any_sync(0xffffffffu, e.most() >= floor)) continue;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float y = e.get(i);
          const bool in = y >= floor && i >= lo && i < hi;
          if (!__any_sync(0xffffffffu, in)) continue;
          const Key c = in ? key_of(y, (uint32_t)(from + i)) : 0;
          unsigned hit = __ballot_sync(0xffffffffu, c > bar);
          while (hit) {
            const int src = __ffs(hit) - 1;
            hit &= hit - 1;
            const Key one = __shfl_sync(0xffffffffu, c, src);
            if (one > bar) {
              insert(mine, one, lane);
              bar = __shfl_sync(0xffffffffu, mine, top - 1);
            }
          }
          if (bar) floor = fmaxf(floor, key_value(bar));
        }
      }
  }
  if (NW > 1) {
    if (lane == 0) sums[warp] = sum;
    if (top) lists[threadIdx.x] = mine;
    __syncthreads();
    if (top)
#pragma unroll
      for (int step = 1; step < NW; step *= 2) {  // pairs of lists
        if (warp % (2 * step) == 0) lists[threadIdx.x] = mine = merge(mine, lists[(warp + step) * 32 + lane], lane);
        if (2 * step < NW) __syncthreads();
      }
    if (!CLUSTER && warp) return;
    if (warp == 0) sum = join_parts(sums, NW, lane, A.k);
    if (CLUSTER) {
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
      if (warp == 0) {
        const uint32_t to = tcx::su32(&keys[rank * 32 + lane]), ts = tcx::su32(&all[rank]);
        uint32_t d;
        asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(d) : "r"(to));
        asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(d), "l"(mine) : "memory");
        asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(d) : "r"(ts));
        if (lane == 0) {
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(d), "f"(sum.m) : "memory");
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(d + 4), "f"(sum.s) : "memory");
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(d + 8), "f"(sum.t) : "memory");
        }
      }
      cluster_sync();
      if (rank || warp) return;
      sum = join_parts(all, (int)ranks, lane, A.k);
      if (top)
        for (uint32_t w = 1; w < ranks; ++w) mine = merge(mine, keys[w * 32 + lane], lane);
    }
  }
  const bool broken = !(sum.s > 0.0f && sum.s <= kMost);
  const float logs = logf(sum.s);
  if (lane == 0) {
    if (A.logp) {
      const bool known = !broken && tok >= 0 && tok < V;
      A.logp[row] = known ? fminf(0.0f, __fsub_rn(__fmul_rn(__fsub_rn(taken, sum.m), A.inv_t), logs)) : nan();
    }
    if (A.entropy) A.entropy[row] = broken ? nan() : fmaxf(0.0f, __fsub_rn(logs, __fmul_rn(__fdiv_rn(sum.t, sum.s), A.inv_t)));
  }
  if (lane < top) {
    if (A.top_logp) A.top_logp[row * top + lane] = broken ? nan() : fminf(0.0f, __fsub_rn(__fmul_rn(__fsub_rn(key_value(mine), sum.m), A.inv_t), logs));
    if (A.top_index) A.top_index[row * top + lane] = broken ? -1 : (int64_t)(0xffffffffu - (uint32_t)mine);
  }
}

template <class T>
cudaError_t run(const LogprobArgs& a, cudaStream_t s) {
  count_launches(1);
  // A warp to a row takes a block's joins off short ones: 8192 rows of 1024, 4096, 16384 logits of bf16 in 14, 25 and 79 us,
  // by blocks 103, 68 and 104; of fp32 14, 35 and 140, by blocks 90, 64 and 110, which the rule gives away.  Where rows are
  // long or few, its own reads one after another are what counts: 8192 of 50001 226 us and 211, 256 of 8192 14 us and 8,
  // and 1024 of 16384 24 us and 17.
  if (a.V <= 4096 || (a.V <= 16384 && a.V <= 4 * a.n)) {
    k_logprobs<T, 1, false><<<(unsigned)((a.n + kRows - 1) / kRows), 32 * kRows, 0, s>>>(a);
    return cudaGetLastError();
  }
  // Few rows: the row's stretches of 4096 logits or more to the blocks of a cluster.  16 rows of 131072: 10 us, 21 by a
  // block each; 128 rows 19 and 25.
  unsigned ranks = 1;
  while (ranks < kMostRanks && a.n * ranks < 152 && a.V >= 8192 * (int64_t)ranks) ranks *= 2;
  if (ranks == 1) {
    k_logprobs<T, kWarps, false><<<(unsigned)a.n, 32 * kWarps, 0, s>>>(a);
    return cudaGetLastError();
  }
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = ranks;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  lc.gridDim = dim3((unsigned)(a.n * ranks));
  lc.blockDim = dim3(32 * kWarps);
  lc.stream = s;
  lc.attrs = at;
  lc.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&lc, k_logprobs<T, kWarps, true>, a);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_logprobs(const LogprobArgs& a, cudaStream_t s) {
  return a.dtype == SIMX_F32 ? run<float>(a, s) : run<__nv_bfloat16>(a, s);
}

}  // namespace simx

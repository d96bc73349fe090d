// seq_attn_tc.cu — the passes of a linear attention (seq_attn.cu has the formulas) on the tensor cores, for bf16.
//
// Chunks of 128 steps of one head, with the state S in registers; four products a chunk on tcgen05.mma with
// FP32 accumulators in tensor memory:
//   scores = a b^T,  far = a S,  o = (scores * link) c + reach far,  S' = keep S + (b * link to the end)^T c.
// The inputs are operands as they are.  What is computed has more digits than bf16 and is an operand in parts, x =
// x1 + x2 (+ x3), each part what is left so far, rounded to bf16: three (all of fp32's digits) for weighted b, which is added to
// the state, in every pass; two for links times scores and for the state in `far`, whose products go to a result that is
// rounded to bf16 anyway (2^-17 of each term; a third part of either would take columns of tensor memory that dimensions
// of 64 do not have and shared memory that dimensions of 128 do not have).  fp32 inputs would take six products of parts
// for each: they go to the FP32 units (seq_attn.cu).
// Scores are sums in fp32 before they meet c: the sizes of a and b are bounded together, unlike step by step.
//
// Operands lie in shared memory step by step, in columns of 64 elements (32 where D is 32) whose 16-byte units
// are permuted within each 8 steps (the 128-byte and 64-byte swizzle): the same bytes are an operand along the
// elements (scores) and one along the steps (o, S'), and both a warp's copies, which follow the rows, and its
// reads of a column meet every bank.  The weighted scores go back to tensor memory, over the scores, and are the
// A operand there.
#include <cuda.h>

#include <algorithm>

#include "seq_attn.cuh"

namespace simx {
namespace attn {

namespace {

using tcx::su32;

constexpr int kSms = 152;

constexpr int C = 128;  // steps of a chunk
constexpr long long kMmaCycles = 2000000000ll;   // products take microseconds: a second is a failure
constexpr long long kHandCycles = 20000000000ll;  // a part of a head takes milliseconds: ten seconds are one

__device__ __forceinline__ uint32_t idesc(int m, int n, bool a_steps, bool b_steps) {
  return tcx::idesc_bf16(m, n) | (a_steps ? 1u << 15 : 0u) | (b_steps ? 1u << 16 : 0u);
}
// D += A B^T with A in tensor memory.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t bd, uint32_t id, uint32_t acc) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
      "r"(a), "l"(bd), "r"(id), "r"(acc)
      : "memory");
}

// Both halves of a pair of bf16 as fp32.
__device__ __forceinline__ float low(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float high(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

__device__ __forceinline__ void unpair(Pair v, float& x, float& y) { x = halves(v).x, y = halves(v).y; }

// (x, y) rounded to bf16 as a part, and what is left of them.
__device__ __forceinline__ uint32_t take(float& x, float& y) {
  const uint32_t u = pack2(x, y);
  Pair r;
  asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair(x, y)), "l"(pair(low(u), high(u))));
  unpair(r, x, y);
  return u;
}

// Whether eight bf16 are finite: their products with zero, added up.
__device__ __forceinline__ bool finite8(uint4 v) {
  uint32_t sum = 0;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(w[i]), "r"(0));
  return (sum & 0x7fff7fffu) == 0;
}
// n of eight bf16 from any address, by aligned words: each holds one of them at least.
__device__ __forceinline__ uint4 load8(const __nv_bfloat16* p, int n) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  const bool odd = (at & 2) != 0;
  const uint32_t* w = reinterpret_cast<const uint32_t*>(at & ~(uintptr_t)3);
  const int words = (n + 1 + (odd ? 1 : 0)) / 2;
  uint32_t u[5], v[4];
#pragma unroll
  for (int i = 0; i < 5; ++i) u[i] = i < words ? w[i] : 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = odd ? __funnelshift_r(u[i], u[i + 1], 16) : u[i];
    if (2 * i + 1 >= n) v[i] = 2 * i < n ? v[i] & 0xffffu : 0u;
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// Eight values as PARTS operands of 16 bytes, part_bytes apart.
__device__ __forceinline__ uint4 take8(float (&v)[8]) { return make_uint4(take(v[0], v[1]), take(v[2], v[3]), take(v[4], v[5]), take(v[6], v[7])); }
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) { return make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])); }
template <int PARTS>
__device__ __forceinline__ void store_parts(float (&v)[8], unsigned char* at, uint32_t part_bytes) {
#pragma unroll
  for (int p = 0; p < PARTS; ++p) *reinterpret_cast<uint4*>(at + p * part_bytes) = p + 1 < PARTS ? take8(v) : pack8(v);
}

// What a pass padded to D takes: shared memory, tensor memory, threads.  Tiles are copied whole by the tensor copy
// engine into a ring of five buffers; a chunk holds three, and the next one's arrive meanwhile: a and b in the other
// two, c where a was once the products with a are done.  The second and third parts of weighted b lie where the
// state's operand was.
template <int D>
struct Shape {
  static constexpr uint32_t kTile = C * D * 2, kState = D * D * 2;  // bytes of one part
  static constexpr uint32_t kLine = D >= 64 ? 128 : 64;             // bytes of a row in a column
  static constexpr uint32_t kS = 5 * kTile, kMore = kS, kBytes = kS + 2 * kTile;  // the state's two parts; parts 2 and 3 of weighted b
  static constexpr uint32_t kScores = 0, kO = 128, kFar = kO + D, kCols = kFar + D <= 256 ? 256 : 512;
  static constexpr int kBlocks = kCols == 256 && kBytes <= 112 * 1024 ? 2 : 1;  // of an SM
  static constexpr int kThreads = kBlocks == 2 ? 256 : 512, kSides = kThreads / 128;  // and four warps more, of which one issues
  // Registers of a thread: as launched, of those that compute and of the others; the sums agree.
  static constexpr int kRegs = kBlocks == 2 ? 80 : 96, kMost = kBlocks == 2 ? 104 : 112, kLeast = 32;
  static_assert(kThreads * kMost + 128 * kLeast <= (kThreads + 128) * kRegs, "registers");
  static constexpr int kPieces = C * D / 8 / kThreads;  // 16-byte units of each tile, a thread
  static constexpr int kM = D == 128 ? 128 : 64;    // rows of the product for the state
  static constexpr int kRows = kM / 4;              // lanes of a warp that hold a row of it
  static constexpr int kHC = D / kSides;            // columns of o and of the state a thread takes
};

// Byte of 16-byte unit g of row r in an operand of `rows` rows.
template <int D>
__device__ __forceinline__ uint32_t spot(int r, int g, int rows) {
  constexpr uint32_t L = Shape<D>::kLine, U = L / 16;
  return g / U * (rows * L) + r * L + ((g % U ^ (L == 128 ? r & 7 : r >> 1 & 3)) << 4);
}

// The first step of step i's episode in the chunk, -1 if it began before: the last cut up to i.
__device__ __forceinline__ int start_of(uint4 cuts, int i) {
  if (!(cuts.x | cuts.y | cuts.z | cuts.w)) return -1;
  const uint32_t c[4] = {cuts.x, cuts.y, cuts.z, cuts.w};
  int start = -1;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int n = i - 32 * w;  // of this word, steps 0 .. n
    const uint32_t u = n < 0 ? 0u : n >= 31 ? c[w] : c[w] & (0xffffffffu >> (31 - n));
    start = u ? 32 * w + 31 - __clz(u) : start;
  }
  return start;
}

// A box of 128 steps of one head, `column` on, into shared memory; rows and columns outside the tensor are zeros.
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, int column, int t, int h, int b, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
               "l"(map), "r"(column), "r"(t), "r"(h), "r"(b), "r"(su32(bar))
               : "memory");
}

// Barriers of the warps that compute (kWork), and from them to the one that issues products and copies.
enum : int { kWork = 1, kWeighted = 2, kLinked = 3, kReady = 4, kHalf = 5, kDone = 6, kOut = 7 };
template <int N>
__device__ __forceinline__ void bar_sync(int id) { asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(N) : "memory"); }
template <int N>
__device__ __forceinline__ void bar_arrive(int id) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(N) : "memory"); }

// The other way.
__device__ __forceinline__ void store_box(const CUtensorMap* map, uint32_t src, int column, int t, int h, int b) {
  asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(map), "r"(src), "r"(column), "r"(t),
               "r"(h), "r"(b)
               : "memory");
}

struct Maps {
  CUtensorMap m[3][3], o[3];  // a, b, c and o of each pass
};

// The order of a chunk's work, with the products of the tensor cores in parentheses:
//   o of the chunk before  (scores, far)
//   far times reach; weighted b
//   links times scores     (what the chunk adds to the state)
//   the state              (o)
// so that each product runs beside work that does not need it.  One warp issues the products and copies; the others
// hand over to it without waiting, and wait for results alone.  Registers are given out for four warps at a time, so it
// has three idle ones beside it, and hands theirs to the others.
//
// Bound by shared memory: a chunk of 128 is 64 product instructions, of which 48 read 8 KB of operands and 16 4 KB (3600
// cycles at 128 bytes a cycle), and the warps' own reads and writes, the copies in and o out move some 450 KB more (3500),
// of 9000 cycles that a chunk takes; the tensor cores alone would take 2000.  The rest is the phases above, which all
// warps go through together: the weighing of b 2000 cycles, o to shared memory 900, scores 1200, the state and its
// operand 1600.  16 x 4096 x 16 heads of 128: 291 us, 57 % of the copy rate; backward, three passes, 4 x 4096 x 16: 247
// us, 29 %; one sequence of 60001, 16 heads of 64 on 4: 235 us, 20 %, the length in 19 segments and read twice.
// Backward with 4 heads of keys and values for 16, 4 x 4096: 893 us, most of it the scattered fp32 rows of each head's part.
//
// Row r of a chunk's tiles is step r, or in reverse step 127 - r: the copies keep the order of time.
//
// A block has one segment of one head, or with shares (seq_attn.cuh) up to one head's first steps, some whole heads
// and one head's last steps.
template <int D, bool KEEP>
__global__ void __launch_bounds__(Shape<D>::kThreads + 128, Shape<D>::kBlocks)
    k_attn_tc(const Passes all, const __grid_constant__ Maps maps, const Shares shares) {
  using S = Shape<D>;
  typedef __nv_bfloat16 T;
  constexpr int G = D / 8, NT = S::kThreads, HC = S::kHC;  // G: 16-byte units of a row
  constexpr uint32_t L = S::kLine;
  extern __shared__ __align__(1024) unsigned char sm[];
  __shared__ __align__(8) uint64_t done_bar[3], full[3];  // products done: with a, for the state, o; tiles there: a, b, c
  __shared__ uint32_t tm_base;
  __shared__ uint4 cuts[2];
  __shared__ __align__(16) float pw[C + 4], near[16];
  __shared__ int any_bad[2];
  __shared__ uint8_t bad[2][C];  // rows whose c is not finite
  __shared__ int lost;
  __shared__ struct { int number, parts, unit0, unit1, lo, hi; } mine_of;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31, quad = warp & 3, side = warp / 4;
  if (KEEP && (int)(blockIdx.x / all.p[0].heads % all.p[0].segs) == all.p[0].segs - 1) return;  // nobody starts from its end
  if (tid == 0) {
    for (int i = 0; i < 3; ++i) {
      tcx::mbar_init(&done_bar[i], 1);
      tcx::mbar_init(&full[i], 1);
    }
    tcx::mbar_fence_init();
    lost = 0;
    // The block's parts: chunks [from, to) of all heads' and passes' chunks in a row.  What is begun for another block
    // comes first, and what another began comes last: no block waits for one that waits.
    mine_of = {};
    mine_of.parts = 1;
    if (shares.grid) {
      const int number = atomicAdd(shares.flags, 1);  // in the order of their starts: the one before runs already
      const int64_t total = (int64_t)shares.passes * all.p[0].batch * all.p[0].heads * shares.per;
      const int64_t from = total * number / shares.grid, to = total * (number + 1) / shares.grid;
      mine_of.number = number;
      mine_of.unit0 = (int)((from + shares.per - 1) / shares.per);
      mine_of.unit1 = (int)(to / shares.per);
      mine_of.lo = (int)(from % shares.per);
      mine_of.hi = (int)(to % shares.per);
      mine_of.parts = mine_of.unit1 - mine_of.unit0 + (mine_of.hi > 0) + (mine_of.lo > 0);
    }
  }
  if (warp == NT / 32) tcx::tm_alloc(&tm_base, S::kCols);
  tcx::fence_before();
  __syncthreads();
  tcx::fence_after();
  const uint32_t base = su32(sm), tm = tm_base;

  // The present part: its pass, head and steps.
  int pass = 0, seg = 0, chunks = 0, before = 0;  // before: chunks of the block's parts before
  int h = 0, b = 0, bh = 0, p0 = 0, p1 = 0;
  bool opens = false, closes = false;
  auto set_part = [&](int part) {
    const int H = (int)all.p[0].heads, len = (int)all.p[0].len;
    if (shares.grid) {
      const int opening = mine_of.hi > 0, q = mine_of.unit0 + part - opening, all_heads = (int)all.p[0].batch * H;
      opens = opening && part == 0;
      closes = !opens && q >= mine_of.unit1;
      const int unit = opens ? mine_of.unit1 : closes ? mine_of.unit0 - 1 : q;
      pass = unit / all_heads;
      bh = unit - pass * all_heads;
      p0 = closes ? mine_of.lo * C : 0;
      p1 = opens ? mine_of.hi * C : len;
    } else {
      pass = blockIdx.y;
      const int rest = (int)(blockIdx.x / H);
      seg = rest % all.p[0].segs;
      bh = rest / all.p[0].segs * H + (int)(blockIdx.x % H);
      p0 = (int)(seg * all.p[0].seg_len);
      p1 = (int)min((int64_t)len, p0 + all.p[0].seg_len);
    }
    b = bh / H;
    h = bh - b * H;
    before += chunks;
    chunks = (p1 - p0 - 1) / C + 1;
  };

  // Byte offset of operand k (a, b, c) of the present chunk, k + 3 of the next one: chunk n has the ring's buffers
  // 3 n, 3 n + 1 and 3 n + 2 modulo 5; `ring` is 3 n modulo 5.
  int ring = 0;
  auto place = [&](int k) -> uint32_t {
    const int q = ring + k;
    return (uint32_t)(q >= 5 ? q - 5 : q) * S::kTile;
  };
  auto next_ring = [&]() { ring = ring + 3 >= 5 ? ring - 2 : ring + 3; };
  // Time of row 0 of chunk n.
  auto first_time = [&](int n) { return all.p[pass].reverse ? (int)all.p[0].len - p0 - C - n * C : p0 + n * C; };
  bool ok = true;
  auto wait = [&](uint64_t* bar, int n) {
    const uint32_t phase = (uint32_t)(before + n) & 1;
    if (!tcx::mbar_test(bar, phase)) ok = ok && tcx::mbar_wait(bar, phase, kMmaCycles);
  };

  // ---- products and copies.  Operands along the elements and along the steps; byte offsets of
  // element k and of step k there.
  auto along = [&](uint32_t at) { return tcx::sdesc(base + at, 16, 8 * L) | (uint64_t)(L == 128 ? 2 : 4) << 61; };
  auto across = [&](uint32_t at, uint32_t column) { return tcx::sdesc(base + at, column, 8 * L) | (uint64_t)(L == 128 ? 2 : 4) << 61; };
  constexpr auto element = [](int k) { return (uint32_t)k * 2 / L * (C * L) + (uint32_t)k * 2 % L; };
  constexpr auto step_at = [](int k) { return (uint32_t)k * L; };
  auto copy = [&](int n, int k, uint32_t to) {
    const AttnPass& A = all.p[pass];
    tcx::mbar_arrive_expect_tx(&full[k], A.tma ? S::kTile : 0);
    if (!A.tma) return;  // its passing is counted all the same
#pragma unroll
    for (int c = 0; c < D * 2 / (int)L; ++c)
      copy_box(base + to + c * (C * L), &maps.m[pass][k], c * ((int)L / 2), first_time(n),
               (int)(h / (k == 0 ? A.adiv : k == 1 ? A.bdiv : A.cdiv)) * A.head_step[k], (int)b * A.batch_step[k], &full[k]);
  };
  auto out_has_left = [&]() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); };
  // Products of parts go from the smallest to the largest: sums in tensor memory are cut off, by 2^-23 of what they
  // have come to.  First those with a, of chunk n at operands at_a, at_b; the next chunk's a is copied to at_next.
  auto multiply_a = [&](int n) {
    const uint32_t at_a = place(0), at_b = place(1), at_next = place(3);
    bar_sync<NT + 32>(kReady);
    if (n > 0) wait(&done_bar[2], n - 1);
    if (all.p[pass].tma) {
      wait(&full[0], n);
      wait(&full[1], n);
    }
    tcx::fence_after();
    if (lane == 0) {
      const uint64_t a_desc = along(at_a), b_desc = along(at_b), s_desc = across(S::kS, D * L);
      const uint32_t id = idesc(128, 128, false, false), id_far = idesc(128, D, false, true);
      uint32_t acc = 0, acc_far = 0;
#pragma unroll
      for (int k = 0; k < D; k += 16) {
        tcx::mma_bf16(tm + S::kScores, a_desc + (element(k) >> 4), b_desc + (element(k) >> 4), id, acc);
        acc = 1;
      }
#pragma unroll
      for (int p = 1; p >= 0; --p)
#pragma unroll
        for (int k = 0; k < D; k += 16) {
          tcx::mma_bf16(tm + S::kFar, a_desc + (element(k) >> 4), s_desc + ((p * S::kState + step_at(k)) >> 4), id_far, acc_far);
          acc_far = 1;
        }
      tcx::commit(&done_bar[0]);
      if (n + 1 < chunks) copy(n + 1, 0, at_next);
    }
    __syncwarp();
  };
  // What the chunk adds to the state, over `far`, and the next chunk's b where o has left, c where a was: all are past
  // the products with a and have read or written what they had to.  The first half of b's rows is weighted first.
  auto multiply_state = [&](int n) {
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
      if (half) bar_sync<NT + 32>(kWeighted);
      else bar_sync<NT + 32>(kHalf);
      if (all.p[pass].tma && !half) {
        wait(&full[1], n);
        wait(&full[2], n);
      }
      tcx::fence_after();
      if (lane == 0) {
        // In the last chunk too: its own o goes where that of the chunk before was.
        if (!half) out_has_left();
        if (!half && n + 1 < chunks) {
          copy(n + 1, 1, place(4));
          copy(n + 1, 2, place(5));
        }
        const uint32_t from = half ? step_at(C / 2) >> 4 : 0;
        const uint64_t ct_desc = across(place(2), C * L) + from;
        // D of 32: the product's upper rows repeat the lower ones
        constexpr uint32_t column = D < S::kM ? 0 : C * L;
        const uint64_t bt_desc[3] = {across(place(1), column) + from, across(S::kMore, column) + from, across(S::kMore + S::kTile, column) + from};
        const uint32_t id = idesc(S::kM, D, true, true);
        uint32_t acc = half;
#pragma unroll
        for (int p = 2; p >= 0; --p) {
#pragma unroll
          for (int k = 0; k < C / 2; k += 16) {
            tcx::mma_bf16(tm + S::kFar, bt_desc[p] + (step_at(k) >> 4), ct_desc + (step_at(k) >> 4), id, acc);
            acc = 1;
          }
        }
        if (half) tcx::commit(&done_bar[1]);
      }
      __syncwarp();
    }
  };
  // o of a chunk from shared memory, once it is there.  It has left (multiply_state) before the products are done that
  // put_out waits for, so that the next o may be written, and before another copy takes its place.
  auto out_whole = [&](int n) { return all.p[pass].o_tma && p1 - p0 - n * C >= C; };
  auto store_out = [&](int n) {
    bar_sync<NT + 32>(kOut);
    if (lane == 0 && out_whole(n)) {
#pragma unroll
      for (int c = 0; c < D * 2 / (int)L; ++c)
        if (c * ((int)L / 2) < all.p[pass].dc) store_box(&maps.o[pass], base + place(4) + c * (C * L), c * ((int)L / 2), first_time(n), h, b);
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    __syncwarp();
  };
  auto multiply_o = [&]() {
    bar_sync<NT + 32>(kLinked);
    tcx::fence_after();
    if (lane == 0) {
      const uint64_t ct_desc = across(place(2), C * L);
      const uint32_t id = idesc(128, D, false, true);
#pragma unroll
      for (int p = 1; p >= 0; --p)
#pragma unroll
        for (int k = 0; k < C; k += 16) mma_ts(tm + S::kO, tm + S::kScores + k + 8 * p, ct_desc + (step_at(k) >> 4), id, 1);
      tcx::commit(&done_bar[2]);
    }
    __syncwarp();
  };

  if (warp >= NT / 32) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kLeast));
    if (warp > NT / 32) return;
    for (int part = 0; part < mine_of.parts; ++part) {
      set_part(part);
      if (lane == 0)
        for (int k = KEEP ? 1 : 0; k < 3; ++k) copy(0, k, place(k));
      __syncwarp();
      for (int n = 0; n < chunks; ++n) {
        if (KEEP) {
          bar_sync<NT + 32>(kReady);
        } else {
          multiply_a(n);
          if (n > 0) store_out(n - 1);
        }
        multiply_state(n);
        if (!KEEP) multiply_o();
        if (n + 1 < chunks) next_ring();
      }
      if (!KEEP) store_out(chunks - 1);
      next_ring();
      bar_sync<NT + 32>(kDone);  // all are done with the part's tiles and tensor memory
      if (lane == 0) out_has_left();
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    tcx::fence_after();
    tcx::tm_dealloc(tm, S::kCols);
    return;
  }
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kMost));

  for (int part = 0; part < mine_of.parts; ++part) {
    set_part(part);
    const AttnPass& A = all.p[pass];
    const float ld = A.ld[h];
    const bool flip = A.reverse != 0, tma = A.tma != 0;
    if (tid <= C) pw[tid] = power(ld, tid);
    if (tid == C + 1) {  // what lambda^128 lost: over many chunks it would show
      const float whole = power(ld, C);
      pw[tid] = __fmul_rn(whole, power_rest(__fmul_rn((float)C, ld), whole));
    }
    if (tid < C) bad[0][tid] = bad[1][tid] = 0;
    if (tid < 16) near[tid] = power(ld, flip ? tid : 15 - tid);  // lambda^distance within 16 columns, from the near end
    if (tid == 0) {
      any_bad[0] = any_bad[1] = 0;
      if (closes) {  // the state that the block before has come to
        const int* flag = shares.flags + mine_of.number;
        const long long from = clock64();
        int there;
        do asm volatile("ld.acquire.gpu.global.b32 %0, [%1];" : "=r"(there) : "l"(flag) : "memory");
        while (!there && clock64() - from < kHandCycles);
        lost = !there;
      }
    }
    if (closes) {
      bar_sync<NT>(kWork);
      ok = ok && !lost;
    }
    const T* src[3] = {at<T>(A.a, b * A.asb + h / A.adiv * A.ash), at<T>(A.b, b * A.bsb + h / A.bdiv * A.bsh),
                       at<T>(A.c, b * A.csb + h / A.cdiv * A.csh)};
    const int64_t st[3] = {A.ast, A.bst, A.cst};
    const int dims[3] = {A.da, A.da, A.dc};
    const int64_t o_at = b * A.osb + h * A.osh;
    const int o_size = A.o_f32 ? 4 : (int)sizeof(T);
    const bool o_whole = ((reinterpret_cast<uintptr_t>(A.o) | (uintptr_t)(o_at * o_size) | (uintptr_t)(A.ost * o_size)) & 15) == 0 &&
                         A.dc * o_size % 16 == 0;

    // This thread's part of the state: row x, HC columns from y0 on.
    const int x = quad * S::kRows + lane, y0 = side * HC;
    const bool mine = lane < S::kRows && x < D;
    float s[HC];
    // Rows of the state in global memory go by way of shared memory, where its operand lies: a thread's part there
    // (piece) is a part of a row, and here of one column in 32.
    auto piece = [&](int f, int& px, int& py) { px = f / (D / 4), py = f % (D / 4) * 4; };
    auto spot_of = [&](int px, int py) { return reinterpret_cast<float4*>(sm + S::kS + px * D * 4 + ((py / 4 ^ (px & 7)) << 4)); };
    auto read_row = [&](const float* p, int px, int py) {  // four elements, zeros outside the state
      p += px * A.dc + py;
      if (px >= A.da || py >= A.dc) return make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (((reinterpret_cast<uintptr_t>(p) & 15) == 0) && py + 3 < A.dc) return __ldcg(reinterpret_cast<const float4*>(p));
      return make_float4(p[0], py + 1 < A.dc ? p[1] : 0.0f, py + 2 < A.dc ? p[2] : 0.0f, py + 3 < A.dc ? p[3] : 0.0f);
    };
    auto write_rows = [&](float* p, float f) {  // f times the state; f of 0: zeros
      if (mine)
#pragma unroll
        for (int y = 0; y < HC; y += 4) *spot_of(x, y0 + y) = make_float4(s[y], s[y + 1], s[y + 2], s[y + 3]);
      bar_sync<NT>(kWork);
#pragma unroll
      for (int k = 0; k < D * D / 4 / NT; ++k) {
        int px, py;
        piece(tid + k * NT, px, py);
        if (px >= A.da || py >= A.dc) continue;
        float4 v = *spot_of(px, py);
        if (f != 1.0f) v = f != 0.0f ? make_float4(__fmul_rn(f, v.x), __fmul_rn(f, v.y), __fmul_rn(f, v.z), __fmul_rn(f, v.w)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float* to = p + px * A.dc + py;
        if (((reinterpret_cast<uintptr_t>(to) & 15) == 0) && py + 3 < A.dc) {
          *reinterpret_cast<float4*>(to) = v;
        } else {
          const float u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (py + e < A.dc) to[e] = u[e];
        }
      }
    };
#pragma unroll
    for (int y = 0; y < HC; ++y) s[y] = 0.0f;
    if (!KEEP && !closes) {
      // What the segments before this one added, each times what the ones between keep of it, and the state before them.
      const bool rows = A.s_in && A.sy == 1;
      float w = 1.0f;
      if (seg > 0 || rows) {
        float4 v[HC / 4];
#pragma unroll
        for (int k = 0; k < HC / 4; ++k) v[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        auto add = [&](const float* p) {
#pragma unroll
          for (int k = 0; k < D * D / 4 / NT; ++k) {
            int px, py;
            piece(tid + k * NT, px, py);
            const float4 u = read_row(p, px, py);
            v[k] = make_float4(__fmaf_rn(w, u.x, v[k].x), __fmaf_rn(w, u.y, v[k].y), __fmaf_rn(w, u.z, v[k].z), __fmaf_rn(w, u.w, v[k].w));
          }
        };
        for (int q = seg - 1; q >= 0 && w != 0.0f; --q) {
          const int64_t at_q = (int64_t)bh * A.segs + q;
          add(A.seg_state + at_q * A.da * A.dc);
          w = A.seg_keep[at_q] != 0.0f ? segments_keep(A, ld, q, seg) : 0.0f;
        }
        if (rows && w != 0.0f) add(A.s_in + (int64_t)bh * A.da * A.dc);
#pragma unroll
        for (int k = 0; k < D * D / 4 / NT; ++k) {
          int px, py;
          piece(tid + k * NT, px, py);
          *spot_of(px, py) = v[k];
        }
        bar_sync<NT>(kWork);
        if (mine)
#pragma unroll
          for (int y = 0; y < HC; y += 4) {
            const float4 u = *spot_of(x, y0 + y);
            s[y] = u.x, s[y + 1] = u.y, s[y + 2] = u.z, s[y + 3] = u.w;
          }
        bar_sync<NT>(kWork);
      }
      if (A.s_in && !rows && w != 0.0f && mine && x < A.da)
#pragma unroll
        for (int y = 0; y < HC; ++y)
          if (y0 + y < A.dc) s[y] = __fmaf_rn(w, A.s_in[(int64_t)bh * A.da * A.dc + x * A.sx + (y0 + y) * A.sy], s[y]);
    } else if (!KEEP) {
#pragma unroll
      for (int y = 0; y < HC; y += 4) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(shares.hand + (int64_t)(mine_of.number - 1) * D * C) + y / 4 * NT + tid);
        s[y] = v.x, s[y + 1] = v.y, s[y + 2] = v.z, s[y + 3] = v.w;
      }
    }

    // This thread's 16-byte units of a tile: number i is unit g0 of row r0 + i kStep, at byte off0 + i kStep L.
    constexpr int kStep = NT / G;
    static_assert(kStep % 8 == 0, "rows of a thread's units agree in their permutation");
    const int r0 = tid / G, g0 = tid % G;
    const uint32_t off0 = spot<D>(r0, g0, C);
    auto steps_of = [&](int n) { return min(C, p1 - p0 - n * C); };
    auto there = [&](int r, int m) { return flip ? r >= C - m : r < m; };

    // Tensors that the copy engine cannot take.
    auto gather = [&](int n, int k, uint32_t to) {
      if (tma) return;
      const int m = steps_of(n);
      const T* p = src[k] + (int64_t)first_time(n) * st[k];
#pragma unroll 1
      for (int i = 0; i < S::kPieces; ++i) {
        const int r = r0 + i * kStep;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (there(r, m) && 8 * g0 < dims[k]) v = load8(p + r * st[k] + 8 * g0, min(8, dims[k] - 8 * g0));
        *reinterpret_cast<uint4*>(sm + to + off0 + i * kStep * L) = v;
      }
    };
    // Steps of chunk n whose c is not finite, once its tiles are there: it would reach every row in its products with
    // zeros, and counts by its scores alone.
    auto look = [&](int n) {
      if (tma) {
        wait(&full[1], n);
        wait(&full[2], n);
      }
      uint4* p = reinterpret_cast<uint4*>(sm + place(2) + off0);
      uint4 v[S::kPieces];
#pragma unroll
      for (int u = 0; u < S::kPieces; ++u) v[u] = p[u * (kStep * L / 16)];
#pragma unroll
      for (int u = 0; u < S::kPieces; ++u)
        if (!finite8(v[u])) {
          bad[n & 1][r0 + u * kStep] = 1;
          any_bad[n & 1] = 1;
          p[u * (kStep * L / 16)] = make_uint4(0, 0, 0, 0);
        }
    };
    // The ends of episodes of chunk n, by its steps.
    auto ends = [&](int n) {
      const int64_t p = (int64_t)p0 + n * C + tid;
      return tid < C && p < p1 && (p > 0 || A.reverse) && cut_before(A, b, p);
    };
    auto post_ends = [&](int n, bool cut) {
      if (warp < 4) {
        const unsigned u = __ballot_sync(0xffffffffu, cut);
        if (lane == 0) reinterpret_cast<uint32_t*>(&cuts[n & 1])[warp] = u;
      }
    };
    auto state_operand = [&]() {
      if (!KEEP && mine)
#pragma unroll
        for (int y = 0; y < HC; y += 8) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = s[y + e];
          store_parts<2>(v, sm + S::kS + spot<D>(x, (y0 + y) / 8, D), S::kState);
        }
    };
    const int row = quad * 32 + lane, i = flip ? C - 1 - row : row;  // this thread's row of scores and o, and its step
    const uint32_t mine_tm = tm + ((uint32_t)quad << 21);
    // o of chunk n, rounded once; rows leave whole, by way of shared memory, where the next chunk's b will come: whole
    // chunks by the copy engine.  `between` runs before the barrier in the middle.
    auto put_out = [&](int n, bool some, uint32_t out, auto between) {
      const int m = steps_of(n);
      auto unit = [&](int r, int g) { return out + spot<D>(r, g, C); };
      if (some) {
        wait(&done_bar[2], n);
        tcx::fence_after();
#pragma unroll
        for (int y = 0; y < HC; y += 16) {
          uint32_t u[16];
          tcx::tm_ld16_nw(mine_tm + S::kO + y0 + y, u);
          tcx::tm_wait();
          tcx::reg_fence16(u);
          const float f = ok ? A.out_scale : nan();
          float v[16];
          const Pair ff = pair(f, f);
#pragma unroll
          for (int e = 0; e < 16; e += 2) unpair(mul2(pair(__uint_as_float(u[e]), __uint_as_float(u[e + 1])), ff), v[e], v[e + 1]);
          if (A.o_f32) {  // partial gradients of shared heads: fp32 rows in the workspace
            float* p = static_cast<float*>(A.o) + o_at + (first_time(n) + (int64_t)row) * A.ost + y0 + y;
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (i < m && y0 + y + e < A.dc) p[e] = v[e];
          } else {
#pragma unroll
            for (int e = 0; e < 16; e += 8)
              *reinterpret_cast<uint4*>(sm + unit(row, (y0 + y + e) / 8)) = make_uint4(pack2(v[e], v[e + 1]), pack2(v[e + 2], v[e + 3]), pack2(v[e + 4], v[e + 5]), pack2(v[e + 6], v[e + 7]));
          }
        }
      }
      if (some) {
        tcx::fence_async_smem();
        bar_arrive<NT + 32>(kOut);
      }
      between();
      bar_sync<NT>(kWork);
      if (!some || A.o_f32 || (A.o_tma && m == C)) return;
      T* o = static_cast<T*>(A.o) + o_at + (first_time(n) + (int64_t)r0) * A.ost + g0 * 8;
      const uint32_t at0 = unit(r0, g0);
      if (o_whole) {
        if (g0 * 8 < A.dc)
#pragma unroll
          for (int u = 0; u < S::kPieces; ++u)
            if (there(r0 + u * kStep, m)) *reinterpret_cast<uint4*>(o + u * kStep * A.ost) = *reinterpret_cast<const uint4*>(sm + at0 + u * kStep * L);
      } else {
        for (int u = 0; u < S::kPieces; ++u)
          if (there(r0 + u * kStep, m)) {
            const uint16_t* q = reinterpret_cast<const uint16_t*>(sm + at0 + u * kStep * L);
            for (int e = 0; e < 8; ++e)
              if (g0 * 8 + e < A.dc) reinterpret_cast<uint16_t*>(o + u * kStep * A.ost)[e] = q[e];
          }
      }
    };

    bool cut_once = false;
#pragma unroll
    for (int k = KEEP ? 1 : 0; k < 3; ++k) gather(0, k, place(k));
    post_ends(0, ends(0));
    state_operand();
    tcx::fence_async_smem();
    tcx::fence_before();
    bar_sync<NT>(kWork);  // cuts
    bar_arrive<NT + 32>(kReady);

    for (int n = 0; n < chunks; ++n) {
      const int m = steps_of(n);
      const int lead = n == 0 && p0 == 0 ? A.first : 1;  // powers of lambda before step 0
      const bool more = n + 1 < chunks;
      // (1) beside the products with a: the next chunk's inputs, steps that are not finite, o of the last chunk
      bool cut = false;
      if (more) {
        cut = ends(n + 1);
        if (!KEEP) gather(n + 1, 0, place(3));
      }
      if (KEEP) {
        look(n);
        bar_sync<NT>(kWork);
      } else {
        put_out(n - 1, n > 0, place(4), [&] { look(n); });
      }
      const bool check = any_bad[n & 1] != 0;
      const uint4 cut_at = cuts[n & 1];
      const int end = start_of(cut_at, m - 1), first = start_of(cut_at, i);
      if (tid < C) bad[(n + 1) & 1][tid] = 0;  // all are past the last chunk's
      if (tid == 0) any_bad[(n + 1) & 1] = 0;
      if (more) post_ends(n + 1, cut);
      if (!KEEP) {
        wait(&done_bar[0], n);
        tcx::fence_after();
        // (2) far times reach, to where o is accumulated
        const float reach = first < 0 ? pw[min(i + lead, C)] : 0.0f;
#pragma unroll
        for (int y = 0; y < HC; y += 16) {
          uint32_t u[16];
          float v[16];
          tcx::tm_ld16_nw(mine_tm + S::kFar + y0 + y, u);
          tcx::tm_wait();
          tcx::reg_fence16(u);
          if (reach != 0.0f) {
            const Pair rr = pair(reach, reach);
#pragma unroll
            for (int e = 0; e < 16; e += 2) unpair(mul2(pair(__uint_as_float(u[e]), __uint_as_float(u[e + 1])), rr), v[e], v[e + 1]);
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = 0.0f;
          }
          tcx::tm_st16_nw(mine_tm + S::kO + y0 + y, v);
        }
        tcx::tm_wait_st();
      }
      // weighted b: its first part over b.  What has no link counts for nothing, whatever it holds.
      {
        unsigned char* p = sm + place(1) + off0;
        unsigned char* q = sm + S::kMore + off0;
        // not unrolled: fetching the longer code costs more than it saves (2 % of 16 x 4096 x 16 heads of 128)
#pragma unroll 1
        for (int u = 0; u < S::kPieces; ++u, p += kStep * L, q += kStep * L) {
          if (u == S::kPieces / 2) {  // rows up to 63 are done
            tcx::fence_async_smem();
            tcx::fence_before();
            bar_arrive<NT + 32>(kHalf);
          }
          const int r = r0 + u * kStep, j = flip ? C - 1 - r : r;
          const float w = j < m && j >= end ? __fmul_rn(pw[max(m - 1 - j, 0)], A.inject) : 0.0f;
          const uint4 t4 = *reinterpret_cast<const uint4*>(p);
          const uint32_t t[4] = {w != 0.0f ? t4.x : 0u, w != 0.0f ? t4.y : 0u, w != 0.0f ? t4.z : 0u, w != 0.0f ? t4.w : 0u};
          float v[8];
          const Pair ww = pair(w, w);
#pragma unroll
          for (int e = 0; e < 4; ++e) unpair(mul2(pair(low(t[e]), high(t[e])), ww), v[2 * e], v[2 * e + 1]);
          if (check && w != 0.0f && bad[n & 1][r])
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = nan();  // its c is zeros
          *reinterpret_cast<uint4*>(p) = take8(v);
          store_parts<2>(v, q, S::kTile);
        }
      }
      tcx::fence_async_smem();
      tcx::fence_before();
      if (!tma) bar_sync<NT>(kWork);  // o has left the buffer that b takes
      bar_arrive<NT + 32>(kWeighted);
      if (more) {
        gather(n + 1, 1, place(4));
        gather(n + 1, 2, place(5));
      }
      if (!KEEP) {
        // (3) links times scores, over the scores.  Without a memory a step is linked to itself alone.
        const int since = pw[1] == 0.0f ? i : max(first, 0);
        const int least = -(int)__reduce_max_sync(0xffffffffu, -since), most = (int)__reduce_max_sync(0xffffffffu, since);
#pragma unroll 1
        for (int j0 = 16 * side; j0 < C; j0 += 16 * S::kSides) {
          uint32_t u[16];
          float v[16];
          const int lo = flip ? C - 16 - j0 : j0, q0 = flip ? 96 - quad * 32 : quad * 32;  // the columns' first step, the rows' first step
          if (lo > q0 + 31 || lo + 15 < least) {  // nothing linked
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = 0.0f;
          } else {
            tcx::tm_ld16_nw(mine_tm + S::kScores + j0, u);
            tcx::tm_wait();
            tcx::reg_fence16(u);
            float w[16];
            if (lo + 15 <= q0) {  // before the rows: lambda^(i - j) in two factors
              const float f = __fmul_rn(pw[i - lo - 15], A.inject);
              const Pair ff = pair(f, f);
#pragma unroll
              for (int e = 0; e < 16; e += 2)
                unpair(mul2(pair(__uint_as_float(u[e]), __uint_as_float(u[e + 1])), mul2(ff, pair(near[e], near[e + 1]))), w[e], w[e + 1]);
            } else {
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const int j = flip ? lo + 15 - e : lo + e;
                const float v1 = __fmul_rn(__uint_as_float(u[e]), __fmul_rn(pw[max(i - j, 0)], A.inject));
                w[e] = j <= i ? v1 : 0.0f;
              }
            }
            if (lo < most || check)
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const int j = flip ? lo + 15 - e : lo + e;
                w[e] = j < since ? 0.0f : check && j <= i && bad[n & 1][j0 + e] ? nan() : w[e];
              }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              v[e] = __uint_as_float(take(w[2 * e], w[2 * e + 1]));
              v[8 + e] = __uint_as_float(pack2(w[2 * e], w[2 * e + 1]));
            }
          }
          tcx::tm_st16_nw(mine_tm + S::kScores + j0, v);
        }
        tcx::tm_wait_st();
        tcx::fence_before();
        bar_arrive<NT + 32>(kLinked);
      }
      // (4) the state, and what the next chunk's first products take
      wait(&done_bar[1], n);
      tcx::fence_after();
      const float keep = end < 0 ? pw[m - 1 + lead] : 0.0f, rest = m - 1 + lead == C ? pw[C + 1] : 0.0f;
      cut_once = cut_once || end >= 0;
#pragma unroll
      for (int y = 0; y < HC; y += 16) {
        uint32_t u[16];
        tcx::tm_ld16_nw(mine_tm + S::kFar + y0 + y, u);
        tcx::tm_wait();
        tcx::reg_fence16(u);
        if (ok && keep != 0.0f) {
          const Pair kk = pair(keep, keep), rr = pair(rest, rest);
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const Pair v = pair(s[y + e], s[y + e + 1]);
            unpair(fma2(kk, v, fma2(rr, v, pair(__uint_as_float(u[e]), __uint_as_float(u[e + 1])))), s[y + e], s[y + e + 1]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) s[y + e] = ok ? __uint_as_float(u[e]) : nan();
        }
      }
      if (more) {
        state_operand();
        tcx::fence_async_smem();
        tcx::fence_before();
        next_ring();
        bar_arrive<NT + 32>(kReady);
      }
    }
    if (!KEEP) put_out(chunks - 1, true, place(4), [] {});
    if (!KEEP && opens) {
#pragma unroll
      for (int y = 0; y < HC; y += 4)
        reinterpret_cast<float4*>(shares.hand + (int64_t)mine_of.number * D * C)[y / 4 * NT + tid] = make_float4(s[y], s[y + 1], s[y + 2], s[y + 3]);
      __threadfence();
    } else if (KEEP) {
      write_rows(A.seg_state + ((int64_t)bh * A.segs + seg) * A.da * A.dc, 1.0f);
      if (tid == 0) A.seg_keep[(int64_t)bh * A.segs + seg] = cut_once ? 0.0f : power(ld, p1 - p0 - (p0 == 0 && A.first == 0 ? 1 : 0));
    } else if (A.s_out && seg == A.segs - 1) {
      float f = A.reverse ? power(ld, 1) : 1.0f;
      if (!A.reverse && A.done && A.done[b * A.dsb + (A.len - 1) * A.dst] != 0) f = 0.0f;
      float* p = A.s_out + (int64_t)bh * A.da * A.dc;
      if (A.sy == 1) {
        write_rows(p, f);
      } else if (mine && x < A.da) {
#pragma unroll
        for (int y = 0; y < HC; ++y)
          if (y0 + y < A.dc) p[x * A.sx + (y0 + y) * A.sy] = f != 0.0f ? __fmul_rn(f, s[y]) : 0.0f;
      }
    }
    next_ring();
    tcx::fence_before();
    bar_sync<NT>(kWork);  // all are done with the part's tiles
    if (!KEEP && opens && tid == 0) asm volatile("st.release.gpu.global.b32 [%0], %1;" ::"l"(shares.flags + mine_of.number + 1), "r"(1) : "memory");
    bar_arrive<NT + 32>(kDone);
  }
}

// ---------------------------------------------------------------------------- host

typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                           const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encoder() {
  static const Encode f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found);
    return e == cudaSuccess && found == cudaDriverEntryPointSuccess ? reinterpret_cast<Encode>(p) : nullptr;
  }();
  return f;
}

// The map of a bf16 tensor [batch][heads][len][dim] in boxes of 128 steps and `line` bytes; false where the copy
// engine cannot take it.  Axes that are not stepped over (stride 0, as of broadcast heads) are one long.
bool map_tensor(CUtensorMap* map, const void* p, int64_t sb, int64_t st, int64_t sh, int64_t batch, int64_t heads, int64_t len, int dim, int line,
                int& head_step, int& batch_step) {
  const Encode f = encoder();
  head_step = heads > 1 && sh > 0;
  batch_step = batch > 1 && sb > 0;
  if (!f || (reinterpret_cast<uintptr_t>(p) & 15) || (len > 1 && st < dim) || (len > 1 && st % 8) || (head_step && sh % 8) || (batch_step && sb % 8)) return false;
  const cuuint64_t size[4] = {(cuuint64_t)dim, (cuuint64_t)len, (cuuint64_t)(head_step ? heads : 1), (cuuint64_t)(batch_step ? batch : 1)};
  const cuuint64_t row = (cuuint64_t)((dim + 7) / 8 * 16);
  const cuuint64_t stride[3] = {len > 1 ? (cuuint64_t)st * 2 : row, head_step ? (cuuint64_t)sh * 2 : row, batch_step ? (cuuint64_t)sb * 2 : row};
  for (cuuint64_t s : stride)
    if (s >= (cuuint64_t)1 << 40) return false;
  const cuuint32_t box[4] = {(cuuint32_t)line / 2, C, 1, 1}, one[4] = {1, 1, 1, 1};
  return f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(p), size, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
           line == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
cudaError_t run(const Passes& given, int n, bool keep, const Shares& given_shares, cudaStream_t s) {
  using S = Shape<D>;
  Passes all = given;
  Maps maps = {};
  bool copied = true;
  for (int i = 0; i < n; ++i) {
    AttnPass& P = all.p[i];
    P.tma = map_tensor(&maps.m[i][0], P.a, P.asb, P.ast, P.ash, P.batch, P.heads / P.adiv, P.len, P.da, S::kLine, P.head_step[0], P.batch_step[0]) &&
            map_tensor(&maps.m[i][1], P.b, P.bsb, P.bst, P.bsh, P.batch, P.heads / P.bdiv, P.len, P.da, S::kLine, P.head_step[1], P.batch_step[1]) &&
            map_tensor(&maps.m[i][2], P.c, P.csb, P.cst, P.csh, P.batch, P.heads / P.cdiv, P.len, P.dc, S::kLine, P.head_step[2], P.batch_step[2]);
    copied = copied && P.tma;
  }
  // o by the copy engine only where all inputs come by it: threads that gather do not wait for what it has to read
  for (int i = 0; i < n; ++i) {
    AttnPass& P = all.p[i];
    int head_step, batch_step;
    P.o_tma = copied && !keep && !P.o_f32 &&
              map_tensor(&maps.o[i], P.o, P.osb, P.ost, P.osh, P.batch, P.heads, P.len, P.dc, S::kLine, head_step, batch_step) &&
              (P.heads == 1 || head_step) && (P.batch == 1 || batch_step);
  }
  const AttnPass& A = all.p[0];
  auto f = keep ? k_attn_tc<D, true> : k_attn_tc<D, false>;
  cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kBytes);
  if (e != cudaSuccess) return e;
  Shares shares = given_shares;
  dim3 grid((unsigned)(A.batch * A.heads * A.segs), (unsigned)n);
  if (shares.grid) {
    grid = dim3((unsigned)shares.grid);
    shares.per = (int)((A.len + C - 1) / C);
    shares.passes = n;
    if ((e = cudaMemsetAsync(shares.flags, 0, (size_t)(shares.grid + 1) * 4, s)) != cudaSuccess) return e;
  }
  count_launches(1);
  f<<<grid, S::kThreads + 128, S::kBytes, s>>>(all, maps, shares);
  return cudaGetLastError();
}

}  // namespace

int resident_blocks(int d) { return d <= 64 ? 2 * kSms : kSms; }
int share_grid(int64_t units, int64_t len, int d) {
  const int64_t blocks = resident_blocks(d);
  if (units < blocks || units > 64 * blocks) return 0;
  if (d <= 64 && (2 * units > 3 * blocks || len < 2048)) return 0;
  return (int)blocks;
}
size_t share_bytes(int64_t units, int64_t len, int d) {
  const int D = d <= 32 ? 32 : d <= 64 ? 64 : 128;
  return (size_t)share_grid(units, len, d) * (D * C * 4 + 16);
}

cudaError_t run_tc(const Passes& all, int n, bool keep, const Shares& shares, cudaStream_t s) {
  const int d = std::max(all.p[0].da, all.p[0].dc);
  return d <= 32 ? run<32>(all, n, keep, shares, s) : d <= 64 ? run<64>(all, n, keep, shares, s) : run<128>(all, n, keep, shares, s);
}

}  // namespace attn
}  // namespace simx

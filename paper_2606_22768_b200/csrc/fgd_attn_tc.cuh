// What the tensor-core attention kernels share: bounded waits, TMA loads of head tiles, tensor-memory
// access, operand descriptors and MMA issue.
//
// A tile is 128 rows of one head, DP (64 or 128) columns wide, zero-filled beyond the head's width.  In shared memory it
// is one or two boxes of 128 rows x 64 columns, 128 bytes per row, written by TMA with the 128-byte swizzle.  The same
// box serves the MMAs in both directions: with the columns as the contraction (K-major: scores, dP) and with the
// rows as the contraction (MN-major: P V, dS K, P^T dO, dS^T Q).
#ifndef FGD_ATTN_TC_CUH_
#define FGD_ATTN_TC_CUH_

#include <cuda.h>

#include "fgd_attn.h"
#include "fgd_dtype.cuh"
#include "fgd_step_dense_tc.cuh"   // mbarrier, descriptor and commit helpers

namespace fgd {

constexpr uint32_t kAttnBox = 128 * 128;           // bytes of a 128 x 64 box of 16-bit values
static_assert(kAttnRows == 128, "a tile's boxes and MMAs are 128 rows");
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int DP>
__host__ __device__ constexpr uint32_t attn_tile_bytes() { return kAttnBox * (DP / 64); }

// A wait that ends: after `limit` polls, or once another thread of the CTA has given up.  Called by whole warps; all
// lanes get the same answer, so that a warp that gives up leaves together (tensor-memory access is warp-wide).
struct AttnWait {
  int* abort_flag;   // shared memory
  int* status;       // the plan's status word
  uint32_t limit;
  __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) const {
    bool here = false;
    for (uint32_t it = 0; it < limit && !here; ++it) {
      uint32_t ok;
      asm volatile(
          "{\n\t.reg .pred p;\n\t"
          "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
          "selp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(ok)
          : "r"(bar), "r"(parity)
          : "memory");
      here = ok != 0;
      if (!here && (it & 31u) == 31u && *(volatile int*)abort_flag) break;
    }
    if (__all_sync(0xffffffffu, here)) return true;
    *(volatile int*)abort_flag = 1;
    *(volatile int*)status = FGD_ERR_TIMEOUT;
    return false;
  }
  __device__ __forceinline__ bool given_up() const { return *(volatile int*)abort_flag != 0; }
  // Only for a CTA's end: whatever the flag says, still bounded.
  __device__ __forceinline__ void drain(uint32_t bar, uint32_t parity) const { mbar_wait(bar, parity, limit); }
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c, int head, int token, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(c), "r"(head), "r"(token), "r"(bar)
      : "memory");
}
// One tile: DP / 64 boxes, issued by one thread.
template <int DP>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int head, int token, uint32_t bar) {
#pragma unroll
  for (int b = 0; b < DP / 64; ++b) tma_load_3d(dst + b * kAttnBox, map, b * 64, head, token, bar);
}
// Rows [first, 128) of a tile become zero (a row of a box is 128 contiguous bytes, the swizzle stays inside it), for the
// asynchronous proxy to read.  One warp.
template <int DP>
__device__ __forceinline__ void zero_rows(unsigned char* tile, int first, int lane) {
  for (int b = 0; b < DP / 64; ++b)
    for (int i = first * 8 + lane; i < kAttnRows * 8; i += 32) reinterpret_cast<uint4*>(tile + b * kAttnBox)[i] = make_uint4(0u, 0u, 0u, 0u);
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
}

// ---- tensor memory: 32 (16) columns of this thread's lane
__device__ __forceinline__ void tmem_ld_32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
      "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_32(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
      "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
      "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// Ends the loads into r[0 .. N): afterwards, and not before, the compiler may use the values.
template <int N>
__device__ __forceinline__ void tmem_ld_done(uint32_t* r) {
  tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// ---- MMA issue.  M = 128 everywhere.  Called by a whole converged warp; one elected lane (always the same) issues.
// A value that all lanes of a warp share, told to the compiler: what it knows to be the same in every lane can sit in uniform
// registers, where the MMA's operands have to be; without it every MMA pays for moving them there.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

template <bool BF16, int N, bool B_ROWS>   // B_ROWS: B's contraction runs over its rows (MN-major)
__host__ __device__ constexpr uint32_t attn_idesc() {
  return (1u << 4) | ((BF16 ? 1u : 0u) << 7) | ((BF16 ? 1u : 0u) << 10) | ((B_ROWS ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | (8u << 24);
}
// One lane of a converged warp.  (A branch on this tells the compiler that a single thread issues, and so that the operands are
// uniform; behind `lane == 0` it guards every MMA and copy against operands that differ between lanes.)
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
// Low word of the matrix descriptor (address and leading offset in 16-byte units); the high word is a constant: 1024 bytes between
// groups of eight rows, descriptor version, 128-byte swizzle.  Steps along the contraction add to the address alone.
__device__ __forceinline__ uint32_t desc_low(uint32_t tile, uint32_t lead) { return ((tile >> 4) & 0x3FFFu) | ((lead >> 4) << 16); }
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ void umma_f16_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(kDescHigh)
      : "memory");
}
__device__ __forceinline__ void umma_f16_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(kDescHigh)
      : "memory");
}
// D[128 x 128] = A B^T over the tiles' columns (both K-major): 16 columns per step, 32 bytes inside a swizzled row.
template <bool BF16, int DP>
__device__ __forceinline__ void mma_columns(uint32_t d, uint32_t a_tile, uint32_t b_tile) {
  const uint32_t a = uniform(desc_low(a_tile, 16)), b = uniform(desc_low(b_tile, 16)), c = uniform(d);
  if (elect_one()) {
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
      umma_f16_ss(c, a + (((k / 4) * 128 * 128 + (k % 4) * 32) >> 4), b + (((k / 4) * 128 * 128 + (k % 4) * 32) >> 4), attn_idesc<BF16, 128, false>(), k > 0 ? 1u : 0u);
  }
}
// D[128 x DP] (+)= A B over 64 rows of B (rows [64 half, 64 half + 64) of a tile): A's 64 columns are 16-bit values in
// tensor memory, packed two to a column, at [a, a + 32); 16 rows of B per step.
template <bool BF16, int DP>
__device__ __forceinline__ void mma_half_rows(uint32_t d, uint32_t a_cols, uint32_t b_tile, int half, bool accumulate) {
  const uint32_t a = uniform(a_cols), b = uniform(desc_low(b_tile, 128 * 128) + half * (64 * 128 >> 4)), c = uniform(d), acc = uniform(accumulate ? 1u : 0u);
  if (elect_one()) {
#pragma unroll
    for (int k = 0; k < 4; ++k) umma_f16_ts(c, a + k * 8, b + k * (2048 >> 4), attn_idesc<BF16, DP, true>(), k > 0 ? 1u : acc);
  }
}
// All 128 rows of a tile: A's second half stands `a_half` columns after the first.
template <bool BF16, int DP>
__device__ __forceinline__ void mma_rows(uint32_t d, uint32_t a_cols, uint32_t a_half, uint32_t b_tile, bool accumulate) {
  const uint32_t a = uniform(a_cols), b = uniform(desc_low(b_tile, 128 * 128)), c = uniform(d), acc = uniform(accumulate ? 1u : 0u);
  if (elect_one()) {
#pragma unroll
    for (int k = 0; k < 8; ++k) umma_f16_ts(c, a + (k / 4) * a_half + (k % 4) * 8, b + k * (2048 >> 4), attn_idesc<BF16, DP, true>(), k > 0 ? 1u : acc);
  }
}
// Arrival on `bar` once everything issued so far is done.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  const uint32_t b = uniform(bar);
  if (elect_one()) umma_commit(b);
}

// ---- arithmetic
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^x on the FMA pipes: x = n + f with n the nearest integer, 2^f on [-1/2, 1/2] as a polynomial (minimax of degree 4 by Remez
// exchange: relative error 2.7e-6, mean 4e-8, far below the 16-bit rounding of P and below 1e-6 in a row's sum), times 2^n.
// The exponential units give 16 results a clock and SM, and a 128 x 128 block of scores has 16384 of them: 1024 clocks, as much as two of
// its products take.  A share of the exponentials goes this way instead.  Which of a row's columns do is fixed, so at the ends it has to give
// what the hardware's exponential gives: x below -126.5, -inf among them, gives 0 (n = -127 has the bits of 0: a masked place has no
// weight, not 2^-126), and a NaN stays one, as +inf becomes one.  x up to 128; scores exceed neither their row's maximum by more than 8 nor its lse.
__device__ __forceinline__ float2 exp2_poly(float2 x) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.x) : "f"(-127.f));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.y) : "f"(-127.f));
  const float2 t = add2(x, both(12582912.f)), f = fma2(add2(t, both(-12582912.f)), both(-1.f), x);
  float2 p = fma2(both(0.009570102207362652f), f, both(0.05591785907745361f));
  p = fma2(p, f, both(0.240247443318367f));
  p = fma2(p, f, both(0.6931217908859253f));
  p = fma2(p, f, both(0.9999992847442627f));
  const float2 scale = make_float2(__uint_as_float((__float_as_uint(t.x) << 23) + 0x3F800000u), __uint_as_float((__float_as_uint(t.y) << 23) + 0x3F800000u));
  return mul2(p, scale);
}
// 2^x for the k-th pair of a row: one pair in eight by polynomial.  Measured at width 128 alone, on one device: none, 1/8, 1/4:
// 16384 tokens forward 857, 828, 850 us; 1/2 in the key kernel gains nothing either, since the FMA pipes' instructions then cost what the
// exponential units save.  Up to width 64, where the exponentials outlast the products, the best share was not looked for.
__device__ __forceinline__ float2 exp2_pair(float2 x, int k) {
  if (k % 8 == 7) return exp2_poly(x);
  return make_float2(exp2_fast(x.x), exp2_fast(x.y));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float2 two(const uint32_t* r) { return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1])); }
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if constexpr (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// 32 rows x 32 columns [c0, c0 + 32), a row in each lane's registers, times f, as 16-bit values to memory: through 2 KB of shared
// memory of the warp's own, so that four lanes write 64 bytes of a row together.  (A lane writing its own row puts every store's 32
// pieces on 32 lines: an item's outputs then hold up the load / store unit, and with it every wait of the CTA, for thousands of clocks.)
// `out`: the warp's first row; rows at or beyond `rows` and columns at or beyond d are not written.
constexpr size_t kStoreStage = 32 * 64;
template <bool BF16>
__device__ __forceinline__ void store_rows(unsigned char* stage, const uint32_t* r, float f, char* out, int64_t row_bytes, int rows, int c0, int d, int lane) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint4 w;
    w.x = pack2<BF16>(__uint_as_float(r[8 * j]) * f, __uint_as_float(r[8 * j + 1]) * f);
    w.y = pack2<BF16>(__uint_as_float(r[8 * j + 2]) * f, __uint_as_float(r[8 * j + 3]) * f);
    w.z = pack2<BF16>(__uint_as_float(r[8 * j + 4]) * f, __uint_as_float(r[8 * j + 5]) * f);
    w.w = pack2<BF16>(__uint_as_float(r[8 * j + 6]) * f, __uint_as_float(r[8 * j + 7]) * f);
    *reinterpret_cast<uint4*>(stage + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) = w;      // (no bank is hit twice in a quarter warp)
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 8 * i + (lane >> 2), j = lane & 3;
    const uint4 w = *reinterpret_cast<const uint4*>(stage + row * 64 + ((j ^ ((row >> 1) & 3)) << 4));
    if (row < rows && c0 + 8 * j < d) *reinterpret_cast<uint4*>(out + row * row_bytes + 2 * (c0 + 8 * j)) = w;
  }
  __syncwarp();
}

// Division of numbers below 2^31 by a divisor fixed at launch: a high product and a shift.
struct FastDiv {
  uint32_t d, mul, shift;
  FastDiv() = default;
  explicit FastDiv(int divisor) : d((uint32_t)divisor) {      // mul = ceil(2^(32 + shift) / d), 2^shift >= d: exact for 31-bit numbers
    shift = 0;
    while ((1u << shift) < d) ++shift;
    const uint64_t m = (((uint64_t)1 << (32 + shift)) + d - 1) / d;
    mul = (uint32_t)(m - ((uint64_t)1 << 32) * (d > 1 && shift > 0 ? 1 : 0));
    if (d == 1) mul = 0;
  }
  __device__ __forceinline__ int div(int n) const {
    if (d == 1) return n;
    const uint32_t t = __umulhi((uint32_t)n, mul);      // m = 2^32 + mul: n m / 2^32 = n + t
    return (int)(((uint32_t)n + t) >> shift);
  }
};

// The work items of a persistent CTA: `items` = tiles x heads, sorted by descending work, taken forwards and backwards by turns so
// that a CTA that got a large item gets a small one next.  The tile after the current one is read ahead: its latency (and the
// division) would otherwise stand between two items in every role.
struct ItemWalk {
  const AttnTile* tiles;
  FastDiv per_tile;
  int items;
  int round;             // of the current item, counted from 0
  bool valid;
  AttnTile t, t_next;
  int h, h_next;
  bool valid_next;
  __device__ __forceinline__ void look(int r) {
    const int w = r * (int)gridDim.x + ((r & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
    valid_next = w < items;      // only the last, partial round can lack an item
    if (valid_next) {
      const int tile = per_tile.div(w);
      h_next = w - tile * (int)per_tile.d;
      t_next = tiles[tile];
    }
  }
  __device__ __forceinline__ ItemWalk(const AttnTile* tiles_, FastDiv per_tile_, int items_) : tiles(tiles_), per_tile(per_tile_), items(items_), round(-1) {
    look(0);
    next();
  }
  __device__ __forceinline__ void next() {
    ++round;
    valid = uniform(valid_next ? 1 : 0) != 0;
    t.start = uniform(t_next.start);
    t.len = uniform(t_next.len);
    t.row = uniform(t_next.row);
    h = uniform(h_next);
    if (valid) look(round + 1);
  }
};

// ---- host side
typedef CUresult (*AttnEncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Tensor map of a [tokens, heads, d] tensor: boxes of 64 columns x 1 head x 128 tokens; columns beyond d and tokens beyond the
// last read as zero.
inline bool attn_tensor_map(void* encode, CUtensorMap* map, bool bf16, const AttnHeads& t, int64_t tokens, int heads, int d) {
  const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)tokens};
  // the stride of an axis of one is never used, but has to be a valid one
  const cuuint64_t strides[2] = {heads > 1 ? (cuuint64_t)t.head * 2 : (cuuint64_t)d * 2, tokens > 1 ? (cuuint64_t)t.token * 2 : (cuuint64_t)d * 2};
  const cuuint32_t box[3] = {64, 1, (cuuint32_t)kAttnRows}, estr[3] = {1, 1, 1};
  return reinterpret_cast<AttnEncodeFn>(encode)(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, t.p, dims, strides, box, estr,
                                                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Can a tensor be read (and written) by the tensor-core kernels?
inline bool attn_tc_heads(const AttnHeads& t, int64_t tokens, int heads) {
  auto ok = [](int64_t s) { return s > 0 && s % 8 == 0 && s < ((int64_t)1 << 38); };
  return (reinterpret_cast<uintptr_t>(t.p) & 15u) == 0 && (heads == 1 || ok(t.head)) && (tokens == 1 || ok(t.token));
}

}  // namespace fgd
#endif

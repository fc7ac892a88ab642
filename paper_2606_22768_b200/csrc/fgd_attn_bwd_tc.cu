// Gradients of causal attention on the tensor cores (mathematics: fgd_attn_elem.cu), in two kernels: one owns
// query tiles and sums dQ over the keys, one owns key tiles and sums dK and dV over the queries of every head that shares the
// key.  Each recomputes S and dP, seven products instead of five, and in return every sum stays in one CTA's tensor
// memory: no atomics, no fp32 copy of dQ in memory, results that are bit-identical from run to run.
//
// Both kernels: ten warps, one CTA per SM, persistent, blocks of 128 x 128.  Warps 0-7 do the element-wise part, two threads per
// row: thread (half h, lane r) owns row r and columns [64 h, 64 h + 64); warp 8 loads by TMA, warp 9 issues MMAs and runs ahead into
// the next item.  A 16-bit factor goes back into tensor memory over the fp32 values it came from, inside the columns that the same
// thread has read: its two halves of 32 packed columns start 64 columns apart.
//
// Query kernel, tensor memory S0 | S1 | dP | dQ:   S = Q K^T (two buffers, two blocks ahead), dP = dO V^T,
//     dS = P o (dP - delta) over dP, dQ += dS K.  P of the next block is formed while dQ and the next dP run.
// Key kernel, tensor memory S^T | dP^T | dV | dK:  S^T = K Q^T, P^T over S^T, dV += P^T dO, and while dS^T is formed the next S^T
//     runs; dP^T = V dO^T, dS^T over dP^T, dK += dS^T Q, and while P^T of the next block is formed the next dP^T runs.
// `scale` multiplies dQ and dK once, at the end.
//
// fp16 alone: dS is held times a power of two, and P times 2^10, so that small gradients and long rows stay above the type's smallest
// values and large ones below its largest (attn_lift; fgd_attn_elem.cu has the bounds it goes by): per 32 rows in the query kernel, per item in the
// key kernel, where a sum runs over rows.  The output's factor takes it back, exactly; in the loops it costs no instruction.  Forward + backward
// against dS as it is: 288 tokens 34.9 us (32.8), 16 x 1024 of 16 heads of 64 316 us (302: v is read once more), 8192 of 16 x 128 1 % more.
//
// Rounding: P and dS are rounded to the 16-bit type as factors of the next product (5 products in fp32 would need tf32 operands at
// half the rate and twice the shared memory): gradients are .0025 of their norm off in bf16, .0017 with the output's rounding alone.
//
// What bounds them: the chain product -> element-wise part -> product of a block, 61 and 64 % of the tensor pipe's cycles busy (key and
// query kernel; the products alone are 2050 and 1540 of some 3500 and 2500 clocks a block).  8192 tokens, 16 heads of 128 over 4: dQ 318
// us, dK + dV 435 us; 16 x 1024 tokens, 16 heads of 64: 91 and 122, where a block's exponentials (1024 clocks) take as long as the
// products.  Blocks of 64 rows taken by the two groups of four warps in turns hide more latency and were slower, 355 + 570 us: the
// issuing warp's own path, about 100 clocks a commit and 150 a wait, does not shrink with the block.
#include "fgd_attn_tc.cuh"

using namespace fgd;

namespace {

constexpr int kBwdThreads = 320;
// query kernel: buffers of Q and dO, stages of K (needed by two products, two blocks apart) and of V
template <int DP> constexpr int kBufQ = DP == 128 ? 1 : 2;
constexpr int kStagesK = 3;
template <int DP> constexpr int kStagesV = DP == 128 ? 1 : 2;
template <int DP> constexpr size_t dq_smem() { return 1024 + (size_t)(2 * kBufQ<DP> + kStagesK + kStagesV<DP>) * attn_tile_bytes<DP>() + 8 * kStoreStage; }
// key kernel: K, V, stages of Q and dO, and of the rows' lse and delta, which a warp of their own fetches (behind the tiles, on the
// loading warp's path, their latency held up every block: sixteen sequences of 1024, 16 heads of 64, 190 us, 136 so)
template <int DP> constexpr int kStagesQ = DP == 128 ? 2 : 4;
constexpr int kStagesRow = 4;
constexpr int kDkvThreads = 352;
template <int DP> constexpr size_t dkv_smem() { return 1024 + (size_t)(2 + 2 * kStagesQ<DP>) * attn_tile_bytes<DP>() + kStagesRow * 2 * 128 * sizeof(float) + 8 * kStoreStage; }

__device__ __forceinline__ void load_row64(uint32_t addr, uint32_t (&s)[64]) {
  tmem_ld_32(addr, s);
  tmem_ld_32(addr + 32, s + 32);
  tmem_ld_done<64>(s);
}
// The power of two that takes b = max |dout| max |v| (0: none) to [2^6, 2^7): dP and delta, at most width x b <= 128 b in magnitude, then stay
// below 2^14, dS below 2^15.  b is 0 or in [2^-48, 2^32).
__device__ __forceinline__ float attn_lift(float b) {
  const uint32_t e = __float_as_uint(b) >> 23;
  return e == 0 ? 1.f : __uint_as_float((2 * 127 + 6 - e) << 23);
}
__device__ __forceinline__ float power_inverse(float p) { return __uint_as_float((254u << 23) - __float_as_uint(p)); }      // 1 / 2^k, |k| < 126
constexpr float kLiftP = 1024.f;
// What the fp16 delta kernel left for the 32 rows of `head` from `token` on: the largest |v| (low half; the first head of a group has it) and
// |dout| (high), and the first row's delta.  Positive fp16 values order as integers do.
__device__ __forceinline__ uint32_t rows_tops(const AttnArgs& a, int64_t token, int head) { return __ldcg(reinterpret_cast<const uint32_t*>(a.delta + head * a.tokens + token)); }
__device__ __forceinline__ float first_delta(const AttnArgs& a, int64_t token, int head) {
  return __ldcg(reinterpret_cast<const float*>(a.dq.p + 2 * (token * a.dq.token + head * a.dq.head)));
}
__device__ __forceinline__ float tops_bound(uint32_t v, uint32_t dout) { return halves<__half>(v & 0xFFFFu).x * halves<__half>(dout >> 16).x; }
// 64 values of this thread's row as 16-bit factors of the next product
template <bool BF16>
__device__ __forceinline__ void store_pairs(uint32_t addr, const float2 (&x)[32]) {
  uint32_t w[32];
#pragma unroll
  for (int k = 0; k < 32; ++k) w[k] = pack2<BF16>(x[k].x, x[k].y);
  tmem_st_32(addr, w);
  tmem_st_wait();
  tc_fence_before();
}

// A walk over the blocks of all items.
template <typename Count>
struct BlockWalk {
  ItemWalk walk;
  Count count;          // blocks of an item's tile
  int i, n;             // block and blocks of the item
  uint32_t u;           // block over all items
  __device__ __forceinline__ BlockWalk(const AttnTile* tiles, FastDiv per_tile, int items, Count c) : walk(tiles, per_tile, items), count(c), i(0), u(0) { n = walk.valid ? count(walk.t) : 0; }
  __device__ __forceinline__ bool valid() const { return walk.valid; }
  __device__ __forceinline__ bool last() const { return i == n - 1; }
  __device__ __forceinline__ void next() {
    ++u;
    if (++i == n) {
      walk.next();
      i = 0;
      n = walk.valid ? count(walk.t) : 0;
    }
  }
};

// ------------------------------------------------------------------------------------------ dQ
template <int DP, bool BF16>
__global__ void __launch_bounds__(kBwdThreads, 1)
attn_dq_tc_kernel(const AttnArgs a, FastDiv heads, int items, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                  const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo) {
  constexpr uint32_t TILE = attn_tile_bytes<DP>();
  constexpr int SK = kStagesK, SV = kStagesV<DP>, NQ = kBufQ<DP>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) unsigned long long bars[12 + 2 * (SK + SV)];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  // (Q, dO) buffers | K stages | V stages
  const uint32_t sq = smem_u32(base), sk = sq + 2 * NQ * TILE, sv = sk + SK * TILE;
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  const uint32_t b0 = smem_u32(bars), raw = b0, done = b0 + 8, dp_full = b0 + 16, ds_full = b0 + 24, dq_done = b0 + 32, dq_free = b0 + 40, s_full = b0 + 48,
                 q_full = b0 + 64, q_empty = b0 + 80, k_full = b0 + 96, k_empty = k_full + 8 * SK, v_full = k_empty + 8 * SK, v_empty = v_full + 8 * SV;
  if (tid == 0) {
    abort_flag = 0;
    for (uint32_t b : {raw, done, dp_full, dq_done, s_full, s_full + 8, q_full, q_full + 8, q_empty, q_empty + 8}) mbar_init(b, 1);
    mbar_init(ds_full, 256);
    mbar_init(dq_free, 256);
    for (int s = 0; s < 2 * (SK + SV); ++s) mbar_init(k_full + 8 * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(tmem_slot), c_dp = 256, c_dq = 384;
  const AttnWait wait{&abort_flag, a.status, a.spin_limit};
  const int group = a.hq / a.hk;
  // the key blocks that a query tile sees, from the diagonal down to block 0
  auto blocks = [](const AttnTile& t) { return t.row / kAttnRows + 1; };

  if (warp == 8) {
    // ================================================================= loads
    uint32_t u = 0, n_raw = 0;
    bool ok = true;
    ItemWalk walk(a.tiles, heads, items);
    for (; ok && walk.valid; walk.next()) {
      const AttnTile t = walk.t;
      const int kvh = (int)(((float)walk.h + 0.5f) * a.inv_group);      // (exact: heads are below 2^15)
      const uint32_t qb = walk.round % NQ;
      if (!(ok = wait(q_empty + 8 * qb, ((walk.round / NQ) & 1) ^ 1))) break;
      if (elect_one()) {
        mbar_expect_tx(q_full + 8 * qb, 2 * TILE);
        load_tile<DP>(sq + 2 * qb * TILE, &mq, walk.h, t.start + t.row, q_full + 8 * qb);
        load_tile<DP>(sq + (2 * qb + 1) * TILE, &mdo, walk.h, t.start + t.row, q_full + 8 * qb);
      }
      for (int j = blocks(t) - 1; ok && j >= 0; --j, ++u) {
        const int token = t.start + j * 128, rows = t.len - j * 128;
        const uint32_t ik = u % SK, iv = u % SV, kb = k_full + 8 * ik, vb = v_full + 8 * iv;
        if (!(ok = wait(k_empty + 8 * ik, ((u / SK) & 1) ^ 1))) break;
        if (rows >= 128) {
          if (elect_one()) {
            mbar_expect_tx(kb, TILE);
            if ((int)u != a.skip) load_tile<DP>(sk + ik * TILE, &mk, kvh, token, kb);
          }
        } else {     // dQ = dS K must not meet the next sequence's keys
          if (elect_one()) {
            mbar_expect_tx(raw, TILE);
            if ((int)u != a.skip) load_tile<DP>(sk + ik * TILE, &mk, kvh, token, raw);
          }
          ok = wait(raw, n_raw & 1);
          ++n_raw;
          if (!ok) { wait.drain(raw, (n_raw - 1) & 1); break; }
          zero_rows<DP>(base + (2 * NQ + ik) * TILE, rows, lane);
          if (elect_one()) mbar_arrive(kb);
        }
        if (!(ok = wait(v_empty + 8 * iv, ((u / SV) & 1) ^ 1))) break;
        if (elect_one()) {
          mbar_expect_tx(vb, TILE);
          load_tile<DP>(sv + iv * TILE, &mv, kvh, token, vb);
        }
      }
    }
    if (wait.given_up()) {
      for (int k = walk.round > 0 ? walk.round - 1 : 0; k <= walk.round; ++k) wait.drain(q_full + 8 * (k % NQ), (k / NQ) & 1);
      for (uint32_t k = u > (uint32_t)SK ? u - SK : 0; k <= u; ++k) wait.drain(k_full + 8 * (k % SK), (k / SK) & 1);
      for (uint32_t k = u > (uint32_t)SV ? u - SV : 0; k <= u; ++k) wait.drain(v_full + 8 * (k % SV), (k / SV) & 1);
    }
  } else if (warp == 9) {
    // ================================================================= MMAs
    bool ok = true;
    BlockWalk as(a.tiles, heads, items, blocks), ad(a.tiles, heads, items, blocks), now(a.tiles, heads, items, blocks);
    auto score = [&]() {
      if (!as.valid()) return true;
      const uint32_t k = as.u, qb = as.walk.round % NQ;
      if (as.i == 0 && !wait(q_full + 8 * qb, (as.walk.round / NQ) & 1)) return false;
      if (!wait(k_full + 8 * (k % SK), (k / SK) & 1)) return false;
      tc_fence_after();
      mma_columns<BF16, DP>(tmem + 128 * (k & 1), sq + 2 * qb * TILE, sk + (k % SK) * TILE);
      mma_commit(s_full + 8 * (k & 1));
      as.next();
      return true;
    };
    auto dprob = [&]() {
      if (!ad.valid()) return true;
      const uint32_t k = ad.u, qb = ad.walk.round % NQ;
      if (!wait(v_full + 8 * (k % SV), (k / SV) & 1)) return false;
      if (ad.i == 0 && !wait(q_full + 8 * qb, (ad.walk.round / NQ) & 1)) return false;
      tc_fence_after();
      mma_columns<BF16, DP>(tmem + c_dp, sq + (2 * qb + 1) * TILE, sv + (k % SV) * TILE);
      mma_commit(dp_full);
      mma_commit(v_empty + 8 * (k % SV));
      if (ad.last()) mma_commit(q_empty + 8 * qb);      // the item's last product with Q and dO (its last S went before)
      ad.next();
      return true;
    };
    // S runs two blocks ahead of dQ, but dP, one ahead, goes first: with one buffer the next item's Q comes when this item's last dP is done
    ok = score() && dprob() && score();
    for (; ok && now.valid(); now.next()) {
      const uint32_t k = now.u;
      if (!(ok = wait(ds_full, k & 1))) break;
      if (now.i == 0 && !(ok = wait(dq_free, (now.walk.round & 1) ^ 1))) break;
      tc_fence_after();
      mma_rows<BF16, DP>(tmem + c_dq, tmem + c_dp, 64, sk + (k % SK) * TILE, now.i > 0);
      mma_commit(k_empty + 8 * (k % SK));
      if (now.last()) mma_commit(dq_done);
      ok = dprob() && score();
    }
    mma_commit(done);
    wait.drain(done, 0);
  } else {
    // ================================================================= P, dS, and dQ's way out
    const int r = (warp & 3) * 32 + lane, h = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t td = tmem + c_dp + 64 * h + lanes;
    const float2 c2 = both(a.scale * kLog2e);
    uint32_t u = 0;
    bool ok = true;
    ItemWalk walk(a.tiles, heads, items);
    float lse = 0.f, delta = 0.f;      // of this thread's row of the coming item
    uint32_t top_v = 0, top_g = 0;     // fp16: of 32 of the keys that the warp's rows see, and of its rows
    auto row_stats = [&]() {
      const int first = walk.t.row + r - lane;      // the warp's first row
      if (walk.valid && first + lane < walk.t.len) {
        const int64_t at = (int64_t)walk.h * a.tokens + walk.t.start + walk.t.row + r;
        lse = a.lse[at];
        delta = a.delta[at];
        if (!BF16 && lane == 0) delta = first_delta(a, walk.t.start + first, walk.h);
      }
      if constexpr (!BF16) {
        top_v = top_g = 0;
        if (walk.valid && first < walk.t.len) {
          const int kv = walk.h / group * group;      // the head that has v's
          top_g = rows_tops(a, walk.t.start + first, walk.h);
          if (32 * lane <= first) top_v = rows_tops(a, walk.t.start + 32 * lane, kv) & 0xFFFFu;
          for (int row = 32 * (lane + 32); row <= first; row += 32 * 32) top_v = max(top_v, rows_tops(a, walk.t.start + row, kv) & 0xFFFFu);
        }
      }
    };
    row_stats();
    while (ok && walk.valid) {
      const AttnTile t = walk.t;
      const int n = blocks(t), head = walk.h, round = walk.round;
      const float lift = BF16 ? 1.f : attn_lift(tops_bound(__reduce_max_sync(0xffffffffu, top_v), top_g));
      const float2 lse2 = both(-lse * kLog2e), lift2 = both(lift), delta2 = both(-delta * lift);
      const float factor = BF16 ? a.scale : a.scale * power_inverse(lift);
      for (int i = 0; i < n; ++i, ++u) {
        const uint32_t ts = tmem + 128 * (u & 1) + 64 * h + lanes;
        if (!(ok = wait(s_full + 8 * (u & 1), (u >> 1) & 1))) break;
        tc_fence_after();
        uint32_t s[64];
        float2 p[32];
        load_row64(ts, s);
#pragma unroll
        for (int k = 0; k < 32; ++k) p[k] = exp2_pair(fma2(two(s + 2 * k), c2, lse2), k);
        if (!(ok = wait(dp_full, u & 1))) break;
        tc_fence_after();
        load_row64(td, s);
#pragma unroll
        for (int k = 0; k < 32; ++k) p[k] = mul2(p[k], BF16 ? add2(two(s + 2 * k), delta2) : fma2(two(s + 2 * k), lift2, delta2));
        if (i == 0) {      // the block on the diagonal (0 times a non-finite value of a masked place is not 0)
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            if (64 * h + 2 * k > r) p[k].x = 0.f;
            if (64 * h + 2 * k + 1 > r) p[k].y = 0.f;
          }
        }
        store_pairs<BF16>(td, p);
        mbar_arrive(ds_full);
      }
      if (!ok) break;
      walk.next();
      row_stats();
      if (!(ok = wait(dq_done, round & 1))) break;
      tc_fence_after();
      if (!BF16 && round == 0) wait_for_previous();      // the key kernel reads what stands where the results go
      const int row0 = t.row + (warp & 3) * 32;
      char* out = a.dq.p + 2 * ((int64_t)(t.start + row0) * a.dq.token + head * a.dq.head);
#pragma unroll 1      // (once per item: code that stays short stays in the instruction cache)
      for (int k = 0; k < DP / 2; k += 32) {
        uint32_t o[32];
        tmem_ld_32(tmem + c_dq + h * (DP / 2) + k + lanes, o);
        tmem_ld_done<32>(o);
        store_rows<BF16>(base + (2 * NQ + SK + SV) * TILE + warp * kStoreStage, o, factor, out, 2 * a.dq.token, t.len - row0, h * (DP / 2) + k, a.d, lane);
      }
      tc_fence_before();
      mbar_arrive(dq_free);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
  wait_for_previous();      // started beside the key kernel: what follows in the stream has to find both done
}

// ------------------------------------------------------------------------------------------ dK, dV
template <int DP, bool BF16>
__global__ void __launch_bounds__(kDkvThreads, 1)
attn_dkv_tc_kernel(const AttnArgs a, FastDiv heads, int items, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                   const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo) {
  constexpr uint32_t TILE = attn_tile_bytes<DP>();
  constexpr int SQ = kStagesQ<DP>, SR = kStagesRow;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) unsigned long long bars[12 + 4 * SQ + 2 * SR];
  __shared__ float lift_of[SR];      // of the item that a stage of rows belongs to, over P's own
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  // K | V | Q stages | dO stages | [stage][lse | delta][128]
  const uint32_t sk = smem_u32(base), sv = sk + TILE, sq = sv + TILE, sdo = sq + SQ * TILE;
  float* row_stats = reinterpret_cast<float*>(base + (2 + 2 * SQ) * TILE);
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  const uint32_t b0 = smem_u32(bars), raw = b0, done = b0 + 8, k_full = b0 + 16, k_empty = b0 + 24, v_full = b0 + 32, v_empty = b0 + 40, s_full = b0 + 48,
                 p_full = b0 + 56, dp_full = b0 + 64, ds_full = b0 + 72, out_done = b0 + 80, out_free = b0 + 88, q_full = b0 + 96, q_empty = q_full + 8 * SQ,
                 do_full = q_empty + 8 * SQ, do_empty = do_full + 8 * SQ, row_full = do_empty + 8 * SQ, row_empty = row_full + 8 * SR;
  if (tid == 0) {
    abort_flag = 0;
    for (uint32_t b : {raw, done, k_full, k_empty, v_full, v_empty, s_full, dp_full, out_done}) mbar_init(b, 1);
    for (uint32_t b : {p_full, ds_full, out_free}) mbar_init(b, 256);
    for (int s = 0; s < 4 * SQ; ++s) mbar_init(q_full + 8 * s, 1);
    for (int s = 0; s < SR; ++s) { mbar_init(row_full + 8 * s, 32); mbar_init(row_empty + 8 * s, 256); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  wait_for_previous();      // delta
  let_next_start();         // the query kernel takes the SMs that this one leaves (or has no work for); it needs delta too, which is there now
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(tmem_slot), c_s = 0, c_dp = 128, c_dv = 256, c_dk = 384;
  const AttnWait wait{&abort_flag, a.status, a.spin_limit};
  const int group = a.hq / a.hk;
  // an item's blocks: for every query head of the group, the query tiles from the key tile's own to the sequence's end
  auto per_head_of = [](const AttnTile& t) { return (t.len + kAttnRows - 1) / kAttnRows - t.row / kAttnRows; };
  auto blocks = [group, per_head_of](const AttnTile& t) { return group * per_head_of(t); };

  if (warp == 8) {
    // ================================================================= loads
    uint32_t u = 0, n_raw = 0;
    bool ok = true;
    // one tile of queries or output gradients; rows beyond the sequence become zero (P^T dO and dS^T Q run over them)
    auto tile = [&](const CUtensorMap* map, uint32_t number, uint32_t bar, int head, int token, int rows) {
      if (rows >= 128) {
        if (elect_one()) {
          mbar_expect_tx(bar, TILE);
          if ((int)u != a.skip) load_tile<DP>(sk + number * TILE, map, head, token, bar);
        }
        return true;
      }
      if (elect_one()) {
        mbar_expect_tx(raw, TILE);
        if ((int)u != a.skip) load_tile<DP>(sk + number * TILE, map, head, token, raw);
      }
      const bool here = wait(raw, n_raw & 1);
      ++n_raw;
      if (!here) { wait.drain(raw, (n_raw - 1) & 1); return false; }
      zero_rows<DP>(base + number * TILE, rows, lane);
      if (elect_one()) mbar_arrive(bar);
      return true;
    };
    ItemWalk walk(a.tiles, heads, items);
    for (; ok && walk.valid; walk.next()) {
      const AttnTile t = walk.t;
      const int kvh = walk.h, first = t.row / kAttnRows, per_head = per_head_of(t);
      if (!(ok = wait(k_empty, (walk.round & 1) ^ 1))) break;
      if (elect_one()) {
        mbar_expect_tx(k_full, TILE);
        load_tile<DP>(sk, &mk, kvh, t.start + t.row, k_full);
      }
      for (int hh = 0; ok && hh < group; ++hh)
        for (int i = 0; ok && i < per_head; ++i, ++u) {
          const int head = kvh * group + hh, row = (first + i) * 128, rows = t.len - row;
          const uint32_t s = u % SQ, parity = ((u / SQ) & 1) ^ 1;
          if (!(ok = wait(q_empty + 8 * s, parity))) break;
          if (!(ok = tile(&mq, 2 + s, q_full + 8 * s, head, t.start + row, rows))) break;
          if (hh == 0 && i == 0) {      // V after the first Q: the item before frees V's buffer later than K's
            if (!(ok = wait(v_empty, (walk.round & 1) ^ 1))) break;
            if (elect_one()) {
              mbar_expect_tx(v_full, TILE);
              load_tile<DP>(sv, &mv, kvh, t.start + t.row, v_full);
            }
          }
          if (!(ok = wait(do_empty + 8 * s, parity))) break;
          ok = tile(&mdo, 2 + SQ + s, do_full + 8 * s, head, t.start + row, rows);
        }
    }
    if (wait.given_up()) {
      for (int k = walk.round > 0 ? walk.round - 1 : 0; k <= walk.round; ++k) {
        wait.drain(k_full, k & 1);
        wait.drain(v_full, k & 1);
      }
      for (uint32_t k = u > (uint32_t)SQ ? u - SQ : 0; k <= u; ++k) {
        wait.drain(q_full + 8 * (k % SQ), (k / SQ) & 1);
        wait.drain(do_full + 8 * (k % SQ), (k / SQ) & 1);
      }
    }
  } else if (warp == 10) {
    // ================================================================= lse and delta of every block's rows
    uint32_t u = 0;
    bool ok = true;
    for (ItemWalk walk(a.tiles, heads, items); ok && walk.valid; walk.next()) {
      const AttnTile t = walk.t;
      const int first = t.row / kAttnRows, per_head = per_head_of(t);
      float lift = 1.f;
      if constexpr (!BF16) {
        uint32_t v = 0, g = 0;      // (v of the whole sequence: the item's queries see all of it)
        for (int row = 32 * lane; row < t.len; row += 32 * 32) v = max(v, rows_tops(a, t.start + row, walk.h * group) & 0xFFFFu);
        for (int hh = 0; hh < group; ++hh)
          for (int row = t.row + 32 * lane; row < t.len; row += 32 * 32) g = max(g, rows_tops(a, t.start + row, walk.h * group + hh));
        lift = attn_lift(tops_bound(__reduce_max_sync(0xffffffffu, v), __reduce_max_sync(0xffffffffu, g))) * (1.f / kLiftP);
      }
      for (int hh = 0; ok && hh < group; ++hh)
        for (int i = 0; i < per_head; ++i, ++u) {
          const int row = (first + i) * 128, rows = t.len - row;
          const int64_t at = (int64_t)(walk.h * group + hh) * a.tokens + t.start + row;
          float lse[4], delta[4], first = 0.f;      // first: lane j's is the delta of row 32 j
          if (!BF16 && lane < 4 && 32 * lane < rows) first = first_delta(a, t.start + row + 32 * lane, walk.h * group + hh);
#pragma unroll
          for (int j = 0; j < 4; ++j) {      // negated; rows beyond the end: P = 2^-inf = 0
            const int k = lane + 32 * j;
            lse[j] = k < rows ? -a.lse[at + k] * kLog2e + (BF16 ? 0.f : 10.f) : -INFINITY;      // (kLiftP)
            delta[j] = k < rows ? -a.delta[at + k] * lift : 0.f;
          }
          if constexpr (!BF16) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float f = -__shfl_sync(0xffffffffu, first, j) * lift;
              if (lane == 0) delta[j] = f;
            }
          }
          if (!(ok = wait(row_empty + 8 * (u % SR), ((u / SR) & 1) ^ 1))) break;
          float* stats = row_stats + (u % SR) * 256;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            stats[lane + 32 * j] = lse[j];
            stats[128 + lane + 32 * j] = delta[j];
          }
          if (!BF16 && lane == 0) lift_of[u % SR] = lift;
          mbar_arrive(row_full + 8 * (u % SR));
        }
    }
  } else if (warp == 9) {
    // ================================================================= MMAs
    bool ok = true;
    BlockWalk as(a.tiles, heads, items, blocks), ad(a.tiles, heads, items, blocks), now(a.tiles, heads, items, blocks);
    auto score = [&]() {
      if (!as.valid()) return true;
      const uint32_t k = as.u;
      if (as.i == 0 && !wait(k_full, as.walk.round & 1)) return false;
      if (!wait(q_full + 8 * (k % SQ), (k / SQ) & 1)) return false;
      tc_fence_after();
      mma_columns<BF16, DP>(tmem + c_s, sk, sq + (k % SQ) * TILE);
      mma_commit(s_full);
      if (as.last()) mma_commit(k_empty);
      as.next();
      return true;
    };
    auto dprob = [&]() {
      if (!ad.valid()) return true;
      const uint32_t k = ad.u;
      if (ad.i == 0 && !wait(v_full, ad.walk.round & 1)) return false;
      if (!wait(do_full + 8 * (k % SQ), (k / SQ) & 1)) return false;
      tc_fence_after();
      mma_columns<BF16, DP>(tmem + c_dp, sv, sdo + (k % SQ) * TILE);
      mma_commit(dp_full);
      if (ad.last()) mma_commit(v_empty);
      ad.next();
      return true;
    };
    ok = score() && dprob();
    for (; ok && now.valid(); now.next()) {
      const uint32_t k = now.u, s = k % SQ;
      if (!(ok = wait(p_full, k & 1))) break;
      if (now.i == 0 && !(ok = wait(out_free, (now.walk.round & 1) ^ 1))) break;
      tc_fence_after();
      mma_rows<BF16, DP>(tmem + c_dv, tmem + c_s, 64, sdo + s * TILE, now.i > 0);
      mma_commit(do_empty + 8 * s);
      if (!(ok = score())) break;
      if (!(ok = wait(ds_full, k & 1))) break;
      tc_fence_after();
      mma_rows<BF16, DP>(tmem + c_dk, tmem + c_dp, 64, sq + s * TILE, now.i > 0);
      mma_commit(q_empty + 8 * s);
      if (now.last()) mma_commit(out_done);
      ok = dprob();
    }
    mma_commit(done);
    wait.drain(done, 0);
  } else {
    // ================================================================= P^T, dS^T, and the gradients' way out
    const int r = (warp & 3) * 32 + lane, h = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + c_s + 64 * h + lanes, td = tmem + c_dp + 64 * h + lanes;
    const float2 c2 = both(a.scale * kLog2e);
    uint32_t u = 0;
    bool ok = true;
    ItemWalk walk(a.tiles, heads, items);
    while (ok && walk.valid) {
      const AttnTile t = walk.t;
      const int kvh = walk.h, round = walk.round, per_head = per_head_of(t), n = group * per_head;
      float lift = 1.f;
      for (int i = 0, q = 0; i < n; ++i, ++u, q = q + 1 == per_head ? 0 : q + 1) {
        const uint32_t st = u % SR;
        const float4* lse4 = reinterpret_cast<const float4*>(row_stats + st * 256 + 64 * h);
        const float4* delta4 = lse4 + 32;
        if (!(ok = wait(row_full + 8 * st, (u / SR) & 1))) break;
        if constexpr (!BF16) lift = lift_of[st];
        if (!(ok = wait(s_full, u & 1))) break;
        tc_fence_after();
        uint32_t s[64];
        float2 p[32];
        load_row64(ts, s);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const float4 l = lse4[k];
          p[2 * k] = exp2_pair(fma2(two(s + 4 * k), c2, make_float2(l.x, l.y)), 2 * k);
          p[2 * k + 1] = exp2_pair(fma2(two(s + 4 * k + 2), c2, make_float2(l.z, l.w)), 2 * k + 1);
        }
        auto mask = [&]() {      // on the diagonal: queries before the key do not see it
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            if (64 * h + 2 * k < r) p[k].x = 0.f;
            if (64 * h + 2 * k + 1 < r) p[k].y = 0.f;
          }
        };
        if (q == 0) mask();
        store_pairs<BF16>(ts, p);
        mbar_arrive(p_full);
        if (!(ok = wait(dp_full, u & 1))) break;
        tc_fence_after();
        load_row64(td, s);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const float4 l = delta4[k];
          const float2 x = two(s + 4 * k), y = two(s + 4 * k + 2);
          p[2 * k] = mul2(p[2 * k], BF16 ? add2(x, make_float2(l.x, l.y)) : fma2(x, both(lift), make_float2(l.x, l.y)));
          p[2 * k + 1] = mul2(p[2 * k + 1], BF16 ? add2(y, make_float2(l.z, l.w)) : fma2(y, both(lift), make_float2(l.z, l.w)));
        }
        if (q == 0) mask();      // (0 times a non-finite value of a masked place is not 0)
        mbar_arrive(row_empty + 8 * st);
        store_pairs<BF16>(td, p);
        mbar_arrive(ds_full);
      }
      if (!ok) break;
      walk.next();
      if (!(ok = wait(out_done, round & 1))) break;
      tc_fence_after();
      const int row0 = t.row + (warp & 3) * 32;
      // half 0 writes dK, half 1 dV
      const AttnHeads& to = h ? a.dv : a.dk;
      const float back = BF16 ? 1.f : 1.f / kLiftP, factor = h ? back : BF16 ? a.scale : a.scale * back * power_inverse(lift);
      char* out = to.p + 2 * ((int64_t)(t.start + row0) * to.token + kvh * to.head);
      unsigned char* stage = base + (2 + 2 * SQ) * TILE + SR * 2 * 128 * sizeof(float) + warp * kStoreStage;
#pragma unroll 1
      for (int k = 0; k < DP; k += 32) {
        uint32_t o[32];
        tmem_ld_32(tmem + (h ? c_dv : c_dk) + k + lanes, o);
        tmem_ld_done<32>(o);
        store_rows<BF16>(stage, o, factor, out, 2 * to.token, t.len - row0, k, a.d, lane);
      }
      tc_fence_before();
      mbar_arrive(out_free);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

template <int DP, bool BF16>
int launch(const fgd_attn_plan* plan, AttnArgs a, cudaStream_t st) {
  const char* who = "fgd_attn_backward";
  CUtensorMap mq, mk, mv, mdo;
  auto map = [&](CUtensorMap* m, const AttnHeads& t, int heads) { return attn_tensor_map(plan->encode_tiled, m, BF16, t, a.tokens, heads, a.d); };
  const int64_t items_kv = (int64_t)plan->n_kv * a.hk, items_q = (int64_t)plan->n_q * a.hq;
  if (items_kv > 0x7fffffff - 1024 || items_q > 0x7fffffff - 1024) return op_fail(FGD_ERR_UNSUPPORTED, "%s: too many tiles", who);
  const int sms = sm_count();
  auto dq = attn_dq_tc_kernel<DP, BF16>;
  auto dkv = attn_dkv_tc_kernel<DP, BF16>;
  cudaError_t e = allow_smem<attn_dq_tc_kernel<DP, BF16>>(dq_smem<DP>());
  if (e == cudaSuccess) e = allow_smem<attn_dkv_tc_kernel<DP, BF16>>(dkv_smem<DP>());
  if (e != cudaSuccess) return op_fail(FGD_ERR_CUDA, "%s: %s", who, cudaGetErrorString(e));
  if (!map(&mq, a.q, a.hq) || !map(&mk, a.k, a.hk) || !map(&mv, a.v, a.hk) || !map(&mdo, a.dout, a.hq))
    return op_fail(FGD_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed", who);
  a.tiles = plan->kv_tiles;
  e = launch_early(dkv, dim3((unsigned)(items_kv < sms ? items_kv : sms)), kDkvThreads, dkv_smem<DP>(), st, a, FastDiv(a.hk), (int)items_kv, mq, mk, mv, mdo);
  if (e != cudaSuccess) return op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
  a.tiles = plan->q_tiles;
  e = launch_early(dq, dim3((unsigned)(items_q < sms ? items_q : sms)), kBwdThreads, dq_smem<DP>(), st, a, FastDiv(a.hq), (int)items_q, mq, mk, mv, mdo);
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

}  // namespace

namespace fgd {

int attn_backward_tc(const fgd_attn_plan* plan, int dtype, const AttnArgs& a, cudaStream_t st) {
  if (a.d <= 64) return dtype == FGD_BF16 ? launch<64, true>(plan, a, st) : launch<64, false>(plan, a, st);
  return dtype == FGD_BF16 ? launch<128, true>(plan, a, st) : launch<128, false>(plan, a, st);
}

}  // namespace fgd

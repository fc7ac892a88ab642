// Gradients of causal attention on the tensor cores (mathematics: fgd_attn_elem.cu), in two kernels: one owns
// query tiles and sums dQ over the keys, one owns key tiles and sums dK and dV over the queries of every head that shares the
// key.  Each recomputes S and dP, seven products instead of five, and in return every sum stays in one CTA's tensor
// memory: no atomics, no fp32 copy of dQ in memory, results that are bit-identical from run to run.
//
// Both kernels: ten warps, one CTA per SM, persistent.  The CTA's own tile is 128 rows (a tensor-memory lane each); the other side
// comes in blocks of 64 rows.  Two groups of four warps take the blocks by turns, one thread per row and 64 columns: each group has
// its own S and dP columns, so one group's waits (a product and its way to the waiting warp take about 450 clocks beyond the product
// itself) are the other's work, and the next block's products are issued before this block's sums.
// Warp 8 loads by TMA, warp 9 issues the MMAs.  A 16-bit factor goes back into tensor memory over the fp32 values it came from.
//
// Query kernel, tensor memory S0 | S1 | dP0 | dP1 | dQ | Q | dO:  S = Q K^T, dP = dO V^T, dS = P o (dP - delta) over dP, dQ += dS K.
//     Q and dO are operands from tensor memory, copied there once per item: with 64-row blocks a shared-memory A would be read
//     twice as often and shared memory, not the MMAs, would set the pace.
// Key kernel, tensor memory S0 | S1 | dP0 | dP1 | dV | dK:  S^T = K Q^T, P^T over S^T, dV += P^T dO, dP^T = V dO^T, dS^T over dP^T,
//     dK += dS^T Q.  K and V have two buffers, so that the next item's are there when its first product is due.
// `scale` multiplies dQ and dK once, at the end.
#include "fgd_attn_tc.cuh"

using namespace fgd;

namespace {

constexpr int kBwdThreads = 320;
constexpr int kBlock = 64;                            // rows of a block

template <int DP> constexpr uint32_t kTile = 128 * DP * 2;       // bytes of the CTA's own tile of one tensor
template <int DP> constexpr uint32_t kBlk = kBlock * DP * 2;     // bytes of a block of one tensor
// query kernel: stages of K (needed by two products) and of V
constexpr int kStagesK = 6, kStagesV = 3;
template <int DP> constexpr size_t dq_smem() { return 1024 + 2 * kTile<DP> + (kStagesK + kStagesV) * kBlk<DP>; }
// key kernel: two buffers of K and V, stages of (Q, dO) blocks, and their rows' lse and delta
template <int DP> constexpr int kStagesQ = DP == 128 ? 3 : 4;
template <int DP> constexpr size_t dkv_smem() { return 1024 + 4 * kTile<DP> + 2 * kStagesQ<DP> * kBlk<DP> + kStagesQ<DP> * 2 * kBlock * sizeof(float); }

template <bool BF16>
__device__ __forceinline__ void store_pairs(uint32_t addr, const float2 (&x)[32]) {
  uint32_t w[32];
#pragma unroll
  for (int k = 0; k < 32; ++k) w[k] = pack2<BF16>(x[k].x, x[k].y);
  tmem_st_32(addr, w);
  tmem_st_wait();
  tc_fence_before();
}
// 64 columns of this thread's row
__device__ __forceinline__ void load_row64(uint32_t addr, uint32_t (&s)[64]) {
  tmem_ld_32(addr, s);
  tmem_ld_32(addr + 32, s + 32);
  tmem_ld_done<64>(s);
}

// ------------------------------------------------------------------------------------------ dQ
// Blocks of an item: keys [64 j, 64 j + 64), from the last block that the tile's rows see down to block 0.
__device__ __forceinline__ int dq_blocks(const AttnTile& t) { return (min(t.row + kAttnRows, t.len) + kBlock - 1) / kBlock; }

// Two consecutive words of 16-bit values of a tile in shared memory (128-byte swizzle) go to tensor memory: row r of the tile to lane r.
template <int DP>
__device__ __forceinline__ void tile_row_to_tmem(const unsigned char* tile, int r, uint32_t addr) {
#pragma unroll
  for (int b = 0; b < DP / 64; ++b) {
    uint32_t w[32];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint4 v = *reinterpret_cast<const uint4*>(tile + b * kAttnBox + r * 128 + ((c ^ (r & 7)) << 4));
      w[4 * c] = v.x; w[4 * c + 1] = v.y; w[4 * c + 2] = v.z; w[4 * c + 3] = v.w;
    }
    tmem_st_32(addr + 32 * b, w);
  }
  tmem_st_wait();
  tc_fence_before();
}

template <int DP, bool BF16>
__global__ void __launch_bounds__(kBwdThreads, 1)
attn_dq_tc_kernel(const AttnArgs a, int items, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                  const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo) {
  constexpr uint32_t TILE = kTile<DP>, BLK = kBlk<DP>;
  constexpr int SK = kStagesK, SV = kStagesV;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) unsigned long long bars[14 + 2 * (SK + SV)];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sq = smem_u32(base), sdo = sq + TILE, sk = sdo + TILE, sv = sk + SK * BLK;
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  // qd_full: Q and dO are in shared memory; qd_read: and have been copied; qd_in: they are in tensor memory; qd_done: the item's
  // products with them are done
  const uint32_t b0 = smem_u32(bars), qd_full = b0, qd_read = b0 + 8, qd_in = b0 + 16, qd_done = b0 + 24, raw = b0 + 32, done = b0 + 40, dq_done = b0 + 48,
                 dq_free = b0 + 56, s_full = b0 + 64, dp_full = b0 + 80, ds_full = b0 + 96, k_full = b0 + 112, k_empty = k_full + 8 * SK,
                 v_full = k_empty + 8 * SK, v_empty = v_full + 8 * SV;
  if (tid == 0) {
    abort_flag = 0;
    for (uint32_t b : {qd_full, qd_done, raw, done, dq_done, s_full, s_full + 8, dp_full, dp_full + 8}) mbar_init(b, 1);
    for (uint32_t b : {qd_read, qd_in, dq_free}) mbar_init(b, 256);
    mbar_init(ds_full, 128);
    mbar_init(ds_full + 8, 128);
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
  const uint32_t tmem = (uint32_t)uniform((int)tmem_slot), c_dp = 128, c_dq = 256, c_q = 256 + DP, c_do = c_q + DP / 2;
  const AttnWait wait{&abort_flag, a.status};
  const int group = a.hq / a.hk;

  if (warp == 8) {
    // ================================================================= loads: K and V of every block, from the diagonal down
    uint32_t u = 0, n_raw = 0;
    bool ok = true;
    ItemWalk walk(a.tiles, a.hq, items);
    for (; ok && walk.valid; walk.next()) {
      const AttnTile t = walk.t;
      const int kvh = walk.h / group;
      if (!(ok = wait(qd_read, (walk.round & 1) ^ 1))) break;
      if (elect_one()) {
        mbar_expect_tx(qd_full, 2 * TILE);
        load_tile<DP>(sq, &mq, walk.h, t.start + t.row, qd_full);
        load_tile<DP>(sdo, &mdo, walk.h, t.start + t.row, qd_full);
      }
      for (int j = dq_blocks(t) - 1; ok && j >= 0; --j, ++u) {
        const int token = t.start + j * kBlock, rows = t.len - j * kBlock;
        const uint32_t ik = u % SK, iv = u % SV, kb = k_full + 8 * ik, vb = v_full + 8 * iv;
        if (!(ok = wait(k_empty + 8 * ik, ((u / SK) & 1) ^ 1))) break;
        if (rows >= kBlock) {
          if (elect_one()) {
            mbar_expect_tx(kb, BLK);
            load_tile<DP, kBlock>(sk + ik * BLK, &mk, kvh, token, kb);
          }
        } else {     // dQ = dS K must not meet the next sequence's keys
          if (elect_one()) {
            mbar_expect_tx(raw, BLK);
            load_tile<DP, kBlock>(sk + ik * BLK, &mk, kvh, token, raw);
          }
          ok = wait(raw, n_raw & 1);
          ++n_raw;
          if (!ok) { drain_wait(raw, (n_raw - 1) & 1); break; }
          zero_rows<DP, kBlock>(base + 2 * TILE + ik * BLK, rows, lane);
          if (elect_one()) mbar_arrive(kb);
        }
        if (!(ok = wait(v_empty + 8 * iv, ((u / SV) & 1) ^ 1))) break;
        if (elect_one()) {
          mbar_expect_tx(vb, BLK);
          load_tile<DP, kBlock>(sv + iv * BLK, &mv, kvh, token, vb);
        }
      }
    }
    if (wait.given_up()) {
      drain_wait(qd_full, walk.round & 1);
      if (walk.round > 0) drain_wait(qd_full, (walk.round - 1) & 1);
      for (uint32_t k = u > (uint32_t)SK ? u - SK : 0; k <= u; ++k) drain_wait(k_full + 8 * (k % SK), (k / SK) & 1);
      for (uint32_t k = u > (uint32_t)SV ? u - SV : 0; k <= u; ++k) drain_wait(v_full + 8 * (k % SV), (k / SV) & 1);
    }
  } else if (warp == 9) {
    // ================================================================= MMAs
    bool ok = true;
    // products of the block that `ahead` points at (block index ua over all items)
    ItemWalk ahead(a.tiles, a.hq, items);
    int ia = 0, na = ahead.valid ? dq_blocks(ahead.t) : 0;
    uint32_t ua = 0;
    auto products = [&]() {
      if (!ahead.valid) return true;
      if (ia == 0 && !wait(qd_in, ahead.round & 1)) return false;
      const uint32_t ik = ua % SK, iv = ua % SV, b = ua & 1;
      if (!wait(k_full + 8 * ik, (ua / SK) & 1)) return false;
      tc_fence_after();
      mma_columns_t<BF16, DP, kBlock>(tmem + 64 * b, tmem + c_q, sk + ik * BLK);
      mma_commit(s_full + 8 * b);
      if (!wait(v_full + 8 * iv, (ua / SV) & 1)) return false;
      tc_fence_after();
      mma_columns_t<BF16, DP, kBlock>(tmem + c_dp + 64 * b, tmem + c_do, sv + iv * BLK);
      mma_commit(dp_full + 8 * b);
      mma_commit(v_empty + 8 * iv);
      if (ia == na - 1) mma_commit(qd_done);
      ++ua;
      if (++ia == na) {
        ahead.next();
        ia = 0;
        na = ahead.valid ? dq_blocks(ahead.t) : 0;
      }
      return true;
    };
    ok = products() && products();
    uint32_t u = 0;
    for (ItemWalk walk(a.tiles, a.hq, items); ok && walk.valid; walk.next()) {
      const int n = dq_blocks(walk.t);
      for (int i = 0; i < n; ++i, ++u) {
        const uint32_t b = u & 1;
        if (!(ok = wait(ds_full + 8 * b, (u >> 1) & 1))) break;
        if (i == 0 && !(ok = wait(dq_free, (walk.round & 1) ^ 1))) break;
        tc_fence_after();
        mma_half_rows<BF16, DP, kBlock>(tmem + c_dq, tmem + c_dp + 64 * b, sk + (u % SK) * BLK, 0, i > 0);
        mma_commit(k_empty + 8 * (u % SK));
        if (i == n - 1) mma_commit(dq_done);
        if (!(ok = products())) break;
      }
    }
    mma_commit(done);
    drain_wait(done, 0);
  } else {
    // ================================================================= P, dS; Q and dO into tensor memory; dQ's way out
    const int r = (warp & 3) * 32 + lane, g = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + 64 * g + lanes, td = tmem + c_dp + 64 * g + lanes;
    const float2 c2 = both(a.scale * kLog2e);
    uint32_t u = 0;                // first block of the item
    uint32_t mine = 0;             // blocks this group has done
    bool ok = true;
    ItemWalk walk(a.tiles, a.hq, items);
    // group 0 copies Q, group 1 dO, once the previous item's products are done
    auto copy_in = [&](int round) {
      if (round > 0 && !wait(qd_done, (round - 1) & 1)) return false;
      if (!wait(qd_full, round & 1)) return false;
      tc_fence_after();
      tile_row_to_tmem<DP>(base + g * TILE, r, tmem + (g ? c_do : c_q) + lanes);
      mbar_arrive(qd_read);
      mbar_arrive(qd_in);
      return true;
    };
    if (walk.valid) ok = copy_in(0);
    while (ok && walk.valid) {
      const AttnTile t = walk.t;
      const int n = dq_blocks(t), head = walk.h, round = walk.round;
      const int64_t row = t.start + t.row + r, at = (int64_t)head * a.tokens + row;
      const bool real = t.row + r < t.len;
      const float2 lse2 = both(real ? -a.lse[at] * kLog2e : 0.f), delta2 = both(real ? -a.delta[at] : 0.f);
      for (int i = (g ^ u) & 1; i < n; i += 2, ++mine) {
        const int over = (n - 1 - i) * kBlock - t.row - r;      // column k is masked where k + over > 0
        if (!(ok = wait(s_full + 8 * g, mine & 1))) break;
        tc_fence_after();
        uint32_t s[64];
        float2 p[32];
        load_row64(ts, s);
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          p[k] = fma2(two(s + 2 * k), c2, lse2);
          p[k].x = exp2_fast(p[k].x);
          p[k].y = exp2_fast(p[k].y);
        }
        if (!(ok = wait(dp_full + 8 * g, mine & 1))) break;
        tc_fence_after();
        load_row64(td, s);
#pragma unroll
        for (int k = 0; k < 32; ++k) p[k] = mul2(p[k], add2(two(s + 2 * k), delta2));
        if (i < 2) {      // the blocks that the diagonal can cross (0 times a non-finite value of a masked place is not 0)
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            if (2 * k + over > 0) p[k].x = 0.f;
            if (2 * k + 1 + over > 0) p[k].y = 0.f;
          }
        }
        store_pairs<BF16>(td, p);
        mbar_arrive(ds_full + 8 * g);
      }
      if (!ok) break;
      u += n;
      walk.next();
      if (walk.valid && !(ok = copy_in(round + 1))) break;      // before the wait below: the MMA warp may be waiting for it
      if (!(ok = wait(dq_done, round & 1))) break;
      tc_fence_after();
      char* out = a.dq.p + 2 * (row * a.dq.token + head * a.dq.head);
#pragma unroll
      for (int k = 0; k < DP / 2; k += 32) {
        uint32_t o[32];
        tmem_ld_32(tmem + c_dq + g * (DP / 2) + k + lanes, o);
        tmem_ld_done<32>(o);
        if (real) store_columns<BF16, 32>(out, o, a.scale, g * (DP / 2) + k, a.d);
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
}

// ------------------------------------------------------------------------------------------ dK, dV
// Blocks of an item: for every query head of the group, queries [64 i, 64 i + 64) from the key tile's first row to the sequence's end.
__device__ __forceinline__ int dkv_blocks(const AttnTile& t) { return (t.len + kBlock - 1) / kBlock - t.row / kBlock; }

template <int DP, bool BF16>
__global__ void __launch_bounds__(kBwdThreads, 1)
attn_dkv_tc_kernel(const AttnArgs a, int items, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                   const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo) {
  constexpr uint32_t TILE = kTile<DP>, BLK = kBlk<DP>;
  constexpr int SQ = kStagesQ<DP>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) unsigned long long bars[16 + 6 * SQ];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  // K0 | V0 | K1 | V1 | Q stages | dO stages | [stage][lse | delta][64]
  const uint32_t skv = smem_u32(base), sq = skv + 4 * TILE, sdo = sq + SQ * BLK;
  float* row_stats = reinterpret_cast<float*>(base + 4 * TILE + 2 * SQ * BLK);
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  const uint32_t b0 = smem_u32(bars), raw = b0, done = b0 + 8, out_done = b0 + 16, out_free = b0 + 24, kv_full = b0 + 32, kv_empty = b0 + 48, s_full = b0 + 64,
                 p_full = b0 + 80, dp_full = b0 + 96, ds_full = b0 + 112, q_full = b0 + 128, q_empty = q_full + 8 * SQ, do_full = q_empty + 8 * SQ,
                 do_empty = do_full + 8 * SQ, row_full = do_empty + 8 * SQ, row_empty = row_full + 8 * SQ;
  if (tid == 0) {
    abort_flag = 0;
    for (uint32_t b : {raw, done, out_done, kv_full, kv_full + 8, kv_empty, kv_empty + 8, s_full, s_full + 8, dp_full, dp_full + 8}) mbar_init(b, 1);
    mbar_init(out_free, 256);
    for (uint32_t b : {p_full, p_full + 8, ds_full, ds_full + 8}) mbar_init(b, 128);
    for (int s = 0; s < 4 * SQ; ++s) mbar_init(q_full + 8 * s, 1);
    for (int s = 0; s < SQ; ++s) { mbar_init(row_full + 8 * s, 32); mbar_init(row_empty + 8 * s, 128); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)uniform((int)tmem_slot), c_dp = 128, c_dv = 256, c_dk = 256 + DP;
  const AttnWait wait{&abort_flag, a.status};
  const int group = a.hq / a.hk;

  if (warp == 8) {
    // ================================================================= loads
    uint32_t u = 0, n_raw = 0;
    bool ok = true;
    // one block of queries or output gradients; rows beyond the sequence become zero (P^T dO and dS^T Q run over them)
    auto block = [&](const CUtensorMap* map, uint32_t offset, uint32_t bar, int head, int token, int rows) {
      if (rows >= kBlock) {
        if (elect_one()) {
          mbar_expect_tx(bar, BLK);
          load_tile<DP, kBlock>(skv + offset, map, head, token, bar);
        }
        return true;
      }
      if (elect_one()) {
        mbar_expect_tx(raw, BLK);
        load_tile<DP, kBlock>(skv + offset, map, head, token, raw);
      }
      const bool here = wait(raw, n_raw & 1);
      ++n_raw;
      if (!here) { drain_wait(raw, (n_raw - 1) & 1); return false; }
      zero_rows<DP, kBlock>(base + offset, rows, lane);
      if (elect_one()) mbar_arrive(bar);
      return true;
    };
    ItemWalk walk(a.tiles, a.hk, items);
    for (; ok && walk.valid; walk.next()) {
      const AttnTile t = walk.t;
      const int kvh = walk.h, first = t.row / kBlock, per_head = dkv_blocks(t);
      const uint32_t kb = walk.round & 1;
      if (!(ok = wait(kv_empty + 8 * kb, ((walk.round >> 1) & 1) ^ 1))) break;
      if (elect_one()) {
        mbar_expect_tx(kv_full + 8 * kb, 2 * TILE);
        load_tile<DP>(skv + 2 * kb * TILE, &mk, kvh, t.start + t.row, kv_full + 8 * kb);
        load_tile<DP>(skv + (2 * kb + 1) * TILE, &mv, kvh, t.start + t.row, kv_full + 8 * kb);
      }
      for (int h = 0; ok && h < group; ++h)
        for (int i = 0; ok && i < per_head; ++i, ++u) {
          const int head = kvh * group + h, row = (first + i) * kBlock, rows = t.len - row;
          const uint32_t s = u % SQ, parity = ((u / SQ) & 1) ^ 1;
          if (!(ok = wait(q_empty + 8 * s, parity))) break;
          if (!(ok = block(&mq, 4 * TILE + s * BLK, q_full + 8 * s, head, t.start + row, rows))) break;
          if (!(ok = wait(do_empty + 8 * s, parity))) break;
          if (!(ok = block(&mdo, 4 * TILE + (SQ + s) * BLK, do_full + 8 * s, head, t.start + row, rows))) break;
          if (!(ok = wait(row_empty + 8 * s, parity))) break;
          float* stats = row_stats + s * 2 * kBlock;
          for (int k = lane; k < kBlock; k += 32) {      // negated; rows beyond the end: P = 2^-inf = 0
            const int64_t at = (int64_t)head * a.tokens + t.start + row + k;
            stats[k] = k < rows ? -a.lse[at] * kLog2e : -INFINITY;
            stats[kBlock + k] = k < rows ? -a.delta[at] : 0.f;
          }
          mbar_arrive(row_full + 8 * s);
        }
    }
    if (wait.given_up()) {
      for (int k = walk.round > 1 ? walk.round - 2 : 0; k <= walk.round; ++k) drain_wait(kv_full + 8 * (k & 1), (k >> 1) & 1);
      for (uint32_t k = u > (uint32_t)SQ ? u - SQ : 0; k <= u; ++k) {
        drain_wait(q_full + 8 * (k % SQ), (k / SQ) & 1);
        drain_wait(do_full + 8 * (k % SQ), (k / SQ) & 1);
      }
    }
  } else if (warp == 9) {
    // ================================================================= MMAs
    bool ok = true;
    ItemWalk ahead(a.tiles, a.hk, items);      // the item of block ua, whose S and dP are issued next
    int ia = 0, na = ahead.valid ? group * dkv_blocks(ahead.t) : 0;
    uint32_t ua = 0;
    auto score = [&]() {
      if (!ahead.valid) return true;
      const uint32_t s = ua % SQ, b = ua & 1, kb = ahead.round & 1;
      if (ia == 0 && !wait(kv_full + 8 * kb, (ahead.round >> 1) & 1)) return false;
      if (!wait(q_full + 8 * s, (ua / SQ) & 1)) return false;
      tc_fence_after();
      mma_columns<BF16, DP, kBlock>(tmem + 64 * b, skv + 2 * kb * TILE, sq + s * BLK);
      mma_commit(s_full + 8 * b);
      return true;
    };
    auto dprob = [&]() {
      if (!ahead.valid) return true;
      const uint32_t s = ua % SQ, b = ua & 1, kb = ahead.round & 1;
      if (!wait(do_full + 8 * s, (ua / SQ) & 1)) return false;
      tc_fence_after();
      mma_columns<BF16, DP, kBlock>(tmem + c_dp + 64 * b, skv + (2 * kb + 1) * TILE, sdo + s * BLK);
      mma_commit(dp_full + 8 * b);
      if (ia == na - 1) mma_commit(kv_empty + 8 * kb);
      ++ua;
      if (++ia == na) {
        ahead.next();
        ia = 0;
        na = ahead.valid ? group * dkv_blocks(ahead.t) : 0;
      }
      return true;
    };
    ok = score() && dprob() && score() && dprob();
    uint32_t u = 0;
    for (ItemWalk walk(a.tiles, a.hk, items); ok && walk.valid; walk.next()) {
      const int n = group * dkv_blocks(walk.t);
      for (int i = 0; i < n; ++i, ++u) {
        const uint32_t s = u % SQ, b = u & 1, parity = (u >> 1) & 1;
        if (!(ok = wait(p_full + 8 * b, parity))) break;
        if (i == 0 && !(ok = wait(out_free, (walk.round & 1) ^ 1))) break;
        tc_fence_after();
        mma_half_rows<BF16, DP, kBlock>(tmem + c_dv, tmem + 64 * b, sdo + s * BLK, 0, i > 0);
        mma_commit(do_empty + 8 * s);
        if (!(ok = wait(ds_full + 8 * b, parity))) break;
        tc_fence_after();
        mma_half_rows<BF16, DP, kBlock>(tmem + c_dk, tmem + c_dp + 64 * b, sq + s * BLK, 0, i > 0);
        mma_commit(q_empty + 8 * s);
        if (i == n - 1) mma_commit(out_done);
        if (!(ok = score() && dprob())) break;
      }
    }
    mma_commit(done);
    drain_wait(done, 0);
  } else {
    // ================================================================= P^T, dS^T, and the gradients' way out
    const int r = (warp & 3) * 32 + lane, g = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + 64 * g + lanes, td = tmem + c_dp + 64 * g + lanes;
    const float2 c2 = both(a.scale * kLog2e);
    uint32_t u = 0;                // first block of the item
    uint32_t mine = 0;
    bool ok = true;
    ItemWalk walk(a.tiles, a.hk, items);
    while (ok && walk.valid) {
      const AttnTile t = walk.t;
      const int kvh = walk.h, round = walk.round, per_head = dkv_blocks(t), n = group * per_head;
      int i = (int)((g ^ u) & 1), q = i;      // q: the block's number within its head
      for (; i < n; i += 2, q += 2, ++mine) {
        while (q >= per_head) q -= per_head;
        const uint32_t st = (u + i) % SQ, st_parity = ((u + i) / SQ) & 1;
        const float4* lse4 = reinterpret_cast<const float4*>(row_stats + st * 2 * kBlock);
        const float4* delta4 = lse4 + kBlock / 4;
        const int under = q * kBlock - r;                       // column k is masked where k + under < 0
        if (!(ok = wait(row_full + 8 * st, st_parity))) break;
        if (!(ok = wait(s_full + 8 * g, mine & 1))) break;
        tc_fence_after();
        uint32_t s[64];
        float2 p[32];
        load_row64(ts, s);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const float4 l = lse4[k];
          p[2 * k] = fma2(two(s + 4 * k), c2, make_float2(l.x, l.y));
          p[2 * k + 1] = fma2(two(s + 4 * k + 2), c2, make_float2(l.z, l.w));
          p[2 * k].x = exp2_fast(p[2 * k].x);
          p[2 * k].y = exp2_fast(p[2 * k].y);
          p[2 * k + 1].x = exp2_fast(p[2 * k + 1].x);
          p[2 * k + 1].y = exp2_fast(p[2 * k + 1].y);
        }
        auto mask = [&]() {
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            if (2 * k + under < 0) p[k].x = 0.f;
            if (2 * k + 1 + under < 0) p[k].y = 0.f;
          }
        };
        if (q < 2) mask();      // queries before the key do not see it
        store_pairs<BF16>(ts, p);
        mbar_arrive(p_full + 8 * g);
        if (!(ok = wait(dp_full + 8 * g, mine & 1))) break;
        tc_fence_after();
        load_row64(td, s);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const float4 l = delta4[k];
          p[2 * k] = mul2(p[2 * k], add2(two(s + 4 * k), make_float2(l.x, l.y)));
          p[2 * k + 1] = mul2(p[2 * k + 1], add2(two(s + 4 * k + 2), make_float2(l.z, l.w)));
        }
        if (q < 2) mask();      // (0 times a non-finite value of a masked place is not 0)
        mbar_arrive(row_empty + 8 * st);
        store_pairs<BF16>(td, p);
        mbar_arrive(ds_full + 8 * g);
      }
      if (!ok) break;
      u += n;
      walk.next();
      if (!(ok = wait(out_done, round & 1))) break;
      tc_fence_after();
      const bool real = t.row + r < t.len;
      const int64_t token = t.start + t.row + r;
      // group 0 writes dK, group 1 dV
      const AttnHeads& to = g ? a.dv : a.dk;
      char* out = to.p + 2 * (token * to.token + kvh * to.head);
#pragma unroll
      for (int k = 0; k < DP; k += 32) {
        uint32_t o[32];
        tmem_ld_32(tmem + (g ? c_dv : c_dk) + k + lanes, o);
        tmem_ld_done<32>(o);
        if (real) store_columns<BF16, 32>(out, o, g ? 1.f : a.scale, k, a.d);
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
  auto map = [&](CUtensorMap* m, const AttnHeads& t, int heads, int rows) { return attn_tensor_map(plan->encode_tiled, m, BF16, t, a.tokens, heads, a.d, rows); };
  const int64_t items_kv = (int64_t)plan->n_kv * a.hk, items_q = (int64_t)plan->n_q * a.hq;
  if (items_kv > 0x7fffffff - 1024 || items_q > 0x7fffffff - 1024) return op_fail(FGD_ERR_UNSUPPORTED, "%s: too many tiles", who);
  const int sms = sm_count();
  auto dq = attn_dq_tc_kernel<DP, BF16>;
  auto dkv = attn_dkv_tc_kernel<DP, BF16>;
  cudaError_t e = cudaFuncSetAttribute(dq, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)dq_smem<DP>());
  if (e == cudaSuccess) e = cudaFuncSetAttribute(dkv, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)dkv_smem<DP>());
  if (e != cudaSuccess) return op_fail(FGD_ERR_CUDA, "%s: %s", who, cudaGetErrorString(e));
  if (!map(&mq, a.q, a.hq, kBlock) || !map(&mk, a.k, a.hk, kAttnRows) || !map(&mv, a.v, a.hk, kAttnRows) || !map(&mdo, a.dout, a.hq, kBlock))
    return op_fail(FGD_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed", who);
  a.tiles = plan->kv_tiles;
  dkv<<<(unsigned)(items_kv < sms ? items_kv : sms), kBwdThreads, dkv_smem<DP>(), st>>>(a, (int)items_kv, mq, mk, mv, mdo);
  if (!map(&mq, a.q, a.hq, kAttnRows) || !map(&mk, a.k, a.hk, kBlock) || !map(&mv, a.v, a.hk, kBlock) || !map(&mdo, a.dout, a.hq, kAttnRows))
    return op_fail(FGD_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed", who);
  a.tiles = plan->q_tiles;
  dq<<<(unsigned)(items_q < sms ? items_q : sms), kBwdThreads, dq_smem<DP>(), st>>>(a, (int)items_q, mq, mk, mv, mdo);
  e = cudaGetLastError();
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

}  // namespace

namespace fgd {

int attn_backward_tc(const fgd_attn_plan* plan, int dtype, const AttnArgs& a, cudaStream_t st) {
  if (a.d <= 64) return dtype == FGD_BF16 ? launch<64, true>(plan, a, st) : launch<64, false>(plan, a, st);
  return dtype == FGD_BF16 ? launch<128, true>(plan, a, st) : launch<128, false>(plan, a, st);
}

}  // namespace fgd

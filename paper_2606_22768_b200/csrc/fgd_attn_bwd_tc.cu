// Gradients of causal attention on the tensor cores (mathematics: fgd_attn_elem.cu), in two kernels: one owns
// query tiles and sums dQ over the keys, one owns key tiles and sums dK and dV over the queries of every head that shares the
// key.  Each recomputes S and dP, seven products instead of five, and in return every sum stays in one CTA's tensor
// memory: no atomics, no fp32 copy of dQ in memory, results that are bit-identical from run to run.
//
// Both kernels: ten warps, one CTA per SM, persistent.  Warps 0-7 do the element-wise part, two threads per row: thread
// (half h, lane r) owns row r and columns [64 h, 64 h + 64) of a 128 x 128 tile; warp 8 loads by TMA, warp 9 issues MMAs.
// A 16-bit factor goes back into tensor memory over the fp32 scores it came from, inside the columns that the same thread
// has read: its two halves of 32 packed columns start 64 columns apart.
//
// Query kernel, tensor memory S0 | S1 | dP | dQ:   S = Q K^T (two buffers, one block ahead), dP = dO V^T,
//     dS = P o (dP - delta) over dP, dQ += dS K.
// Key kernel, tensor memory S^T | dP^T | dV | dK:  S^T = K Q^T, P^T over S^T, dV += P^T dO, and while dS^T is formed the next S^T runs;
//     dP^T = V dO^T, dS^T over dP^T, dK += dS^T Q, and while P^T of the next block is formed the next dP^T runs.
// `scale` multiplies dQ and dK once, at the end.
#include "fgd_attn_tc.cuh"

using namespace fgd;

namespace {

constexpr int kBwdThreads = 320;
constexpr int kQStagesK = 3, kQStagesV = 2;      // query kernel: K tiles stay for two products, V tiles for one

template <int DP> constexpr size_t dq_smem() { return 1024 + (size_t)(2 + kQStagesK + kQStagesV) * attn_tile_bytes<DP>(); }
// key kernel: K, V, two stages of Q and dO, and the rows' lse and delta beside each stage
template <int DP> constexpr size_t dkv_smem() { return 1024 + (size_t)6 * attn_tile_bytes<DP>() + 2 * 2 * 128 * sizeof(float); }

// p and dS of one thread's 64 columns; packs 16-bit values two to a register
template <bool BF16>
__device__ __forceinline__ void pack64(const float (&x)[64], uint32_t (&w)[32]) {
#pragma unroll
  for (int k = 0; k < 32; ++k) w[k] = pack2<BF16>(x[2 * k], x[2 * k + 1]);
}

// ------------------------------------------------------------------------------------------ dQ
template <int DP, bool BF16>
__global__ void __launch_bounds__(kBwdThreads, 1)
attn_dq_tc_kernel(const AttnArgs a, int64_t items, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                  const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo) {
  constexpr uint32_t TILE = attn_tile_bytes<DP>();
  constexpr int SK = kQStagesK, SV = kQStagesV;
  extern __shared__ unsigned char smem_raw[];
  // q_full, q_empty, raw, done, dp_full, ds_full, dq_done, dq_free | s_full[2] | k_full[SK], k_empty[SK], v_full[SV], v_empty[SV]
  __shared__ __align__(8) unsigned long long bars[10 + 2 * (SK + SV)];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sq = smem_u32(base), sdo = sq + TILE, sk = sdo + TILE, sv = sk + SK * TILE;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t b0 = smem_u32(bars);
  const uint32_t q_full = b0, q_empty = b0 + 8, raw = b0 + 16, done = b0 + 24, dp_full = b0 + 32, ds_full = b0 + 40, dq_done = b0 + 48, dq_free = b0 + 56,
                 s_full = b0 + 64, k_full = b0 + 80, k_empty = k_full + 8 * SK, v_full = k_empty + 8 * SK, v_empty = v_full + 8 * SV;
  if (tid == 0) {
    abort_flag = 0;
    for (uint32_t b : {q_full, q_empty, raw, done, dp_full, dq_done, s_full, s_full + 8}) mbar_init(b, 1);
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
  const uint32_t tmem = tmem_slot, c_dp = 256, c_dq = 384;
  const AttnWait wait{&abort_flag, a.status};
  const int group = a.hq / a.hk;
  auto item = [&](int64_t w, AttnTile& t, int& head, int& n) {
    t = a.tiles[(int)(w / a.hq)];
    head = (int)(w % a.hq);
    n = t.row / kAttnRows + 1;
  };

  if (warp == 8) {
    // ================================================================= loads: K and V of every block, from the diagonal down
    uint32_t u = 0, n_raw = 0;
    int round = 0;
    bool ok = true;
    for (; ok; ++round) {
      const int64_t w = work_item(round);
      if ((int64_t)round * gridDim.x >= items) break;
      if (w >= items) continue;
      AttnTile t;
      int head, n;
      item(w, t, head, n);
      if (!(ok = wait(q_empty, (round & 1) ^ 1))) break;
      if (elect_one()) {
        mbar_expect_tx(q_full, 2 * TILE);
        load_tile<DP>(sq, &mq, head, t.start + t.row, q_full);
        load_tile<DP>(sdo, &mdo, head, t.start + t.row, q_full);
      }
      for (int jb = n - 1; ok && jb >= 0; --jb, ++u) {
        const int token = t.start + jb * 128, rows = t.len - jb * 128;
        const uint32_t ik = u % SK, iv = u % SV, kb = k_full + 8 * ik, vb = v_full + 8 * iv;
        if (!(ok = wait(k_empty + 8 * ik, ((u / SK) & 1) ^ 1))) break;
        if (rows >= 128) {
          if (elect_one()) {
            mbar_expect_tx(kb, TILE);
            load_tile<DP>(sk + ik * TILE, &mk, head / group, token, kb);
          }
        } else {     // dQ = dS K must not meet the next sequence's keys
          if (elect_one()) {
            mbar_expect_tx(raw, TILE);
            load_tile<DP>(sk + ik * TILE, &mk, head / group, token, raw);
          }
          ok = wait(raw, n_raw & 1);
          ++n_raw;
          if (!ok) { drain_wait(raw, (n_raw - 1) & 1); break; }
          zero_rows<DP>(base + 2 * TILE + ik * TILE, rows, lane);
          if (elect_one()) mbar_arrive(kb);
        }
        if (!(ok = wait(v_empty + 8 * iv, ((u / SV) & 1) ^ 1))) break;
        if (elect_one()) {
          mbar_expect_tx(vb, TILE);
          load_tile<DP>(sv + iv * TILE, &mv, head / group, token, vb);
        }
      }
    }
    if (wait.given_up()) {
      const int r = round > 0 && !ok ? round : round - 1;
      if (r >= 0) drain_wait(q_full, r & 1);
      for (uint32_t k = u > (uint32_t)SK ? u - SK : 0; k <= u; ++k) drain_wait(k_full + 8 * (k % SK), (k / SK) & 1);
      for (uint32_t k = u > (uint32_t)SV ? u - SV : 0; k <= u; ++k) drain_wait(v_full + 8 * (k % SV), (k / SV) & 1);
    }
  } else if (warp == 9) {
    // ================================================================= MMAs
    uint32_t u = 0;         // block index over all items
    int n_ds = 0;
    bool ok = true;
    auto score = [&](uint32_t k) {      // S of block k into buffer k & 1
      if (!wait(k_full + 8 * (k % SK), (k / SK) & 1)) return false;
      tc_fence_after();
      if (elect_one()) {
        mma_columns<BF16, DP>(tmem + 128 * (k & 1), sq, sk + (k % SK) * TILE);
        umma_commit(s_full + 8 * (k & 1));
      }
      return true;
    };
    auto dprob = [&](uint32_t k) {
      if (!wait(v_full + 8 * (k % SV), (k / SV) & 1)) return false;
      tc_fence_after();
      if (elect_one()) {
        mma_columns<BF16, DP>(tmem + c_dp, sdo, sv + (k % SV) * TILE);
        umma_commit(dp_full);
        umma_commit(v_empty + 8 * (k % SV));
      }
      return true;
    };
    int done_items = 0;
    for (int round = 0; ok; ++round) {
      const int64_t w = work_item(round);
      if ((int64_t)round * gridDim.x >= items) break;
      if (w >= items) continue;
      AttnTile t;
      int head, n;
      item(w, t, head, n);
      if (!(ok = wait(q_full, round & 1))) break;
      if (!(ok = score(u) && dprob(u) && (n == 1 || score(u + 1)))) break;
      if (n == 1 && elect_one()) umma_commit(q_empty);
      for (int i = 0; i < n; ++i, ++u) {
        if (!(ok = wait(ds_full, n_ds & 1))) break;
        ++n_ds;
        if (i == 0 && !(ok = wait(dq_free, (done_items & 1) ^ 1))) break;
        tc_fence_after();
        if (elect_one()) {
          mma_rows<BF16, DP>(tmem + c_dq, tmem + c_dp, 64, sk + (u % SK) * TILE, i > 0);
          if (i == n - 1) umma_commit(dq_done);
          umma_commit(k_empty + 8 * (u % SK));
        }
        if (i + 1 < n && !(ok = dprob(u + 1))) break;
        if (i + 2 < n && !(ok = score(u + 2))) break;
        if (i + 2 == n && elect_one()) umma_commit(q_empty);      // the item's last product with Q and dO is on its way
      }
      ++done_items;
    }
    if (elect_one()) umma_commit(done);
    drain_wait(done, 0);
  } else {
    // ================================================================= P, dS, and dQ's way out
    const int r = (warp & 3) * 32 + lane, h = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float c = a.scale * kLog2e;
    uint32_t u = 0;
    int n_items = 0;
    bool ok = true;
    for (int round = 0; ok; ++round) {
      const int64_t w = work_item(round);
      if ((int64_t)round * gridDim.x >= items) break;
      if (w >= items) continue;
      AttnTile t;
      int head, n;
      item(w, t, head, n);
      const bool real = t.row + r < t.len;
      const int64_t at = (int64_t)head * a.tokens + t.start + t.row + r;
      const float lse = real ? a.lse[at] * kLog2e : 0.f, delta = real ? a.delta[at] : 0.f;
      for (int i = 0; i < n; ++i, ++u) {
        if (!(ok = wait(s_full + 8 * (u & 1), (u >> 1) & 1))) break;
        tc_fence_after();
        uint32_t s[64];
        const uint32_t ts = tmem + 128 * (u & 1) + 64 * h + lanes, td = tmem + c_dp + 64 * h + lanes;
        tmem_ld_32(ts, s);
        tmem_ld_32(ts + 32, s + 32);
        tmem_ld_done<64>(s);
        float p[64];
#pragma unroll
        for (int k = 0; k < 64; ++k) p[k] = exp2_fast(fmaf(__uint_as_float(s[k]), c, -lse));
        if (i == 0) {
#pragma unroll
          for (int k = 0; k < 64; ++k)
            if (64 * h + k > r) p[k] = 0.f;
        }
        if (!(ok = wait(dp_full, u & 1))) break;
        tc_fence_after();
        tmem_ld_32(td, s);
        tmem_ld_32(td + 32, s + 32);
        tmem_ld_done<64>(s);
        const bool diagonal = i == 0;
#pragma unroll
        for (int k = 0; k < 64; ++k) p[k] *= __uint_as_float(s[k]) - delta;
        if (diagonal) {      // (0 times a non-finite dP of a masked place)
#pragma unroll
          for (int k = 0; k < 64; ++k)
            if (64 * h + k > r) p[k] = 0.f;
        }
        uint32_t ds[32];
        pack64<BF16>(p, ds);
        tmem_st_32(td, ds);
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(ds_full);
      }
      if (!ok || !(ok = wait(dq_done, n_items & 1))) break;
      ++n_items;
      tc_fence_after();
      char* out = a.dq.p + 2 * ((int64_t)(t.start + t.row + r) * a.dq.token + head * a.dq.head);
#pragma unroll
      for (int k = 0; k < DP / 2; k += 32) {
        uint32_t o[32];
        tmem_ld_32(tmem + c_dq + h * (DP / 2) + k + lanes, o);
        tmem_ld_done<32>(o);
        if (real) store_columns<BF16, 32>(out, o, a.scale, h * (DP / 2) + k, a.d);
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
template <int DP, bool BF16>
__global__ void __launch_bounds__(kBwdThreads, 1)
attn_dkv_tc_kernel(const AttnArgs a, int64_t items, const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                   const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo) {
  constexpr uint32_t TILE = attn_tile_bytes<DP>();
  extern __shared__ unsigned char smem_raw[];
  // kv_full, kv_empty, raw, done, s_full, p_full, dp_full, ds_full, out_done, out_free | q_full[2], q_empty[2], do_full[2], do_empty[2], row_full[2], row_empty[2]
  __shared__ __align__(8) unsigned long long bars[22];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sk = smem_u32(base), sv = sk + TILE, sq = sv + TILE, sdo = sq + 2 * TILE;
  float* row_stats = reinterpret_cast<float*>(base + 6 * TILE);      // [stage][lse | delta][128]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t b0 = smem_u32(bars);
  const uint32_t kv_full = b0, kv_empty = b0 + 8, raw = b0 + 16, done = b0 + 24, s_full = b0 + 32, p_full = b0 + 40, dp_full = b0 + 48, ds_full = b0 + 56,
                 out_done = b0 + 64, out_free = b0 + 72, q_full = b0 + 80, q_empty = b0 + 96, do_full = b0 + 112, do_empty = b0 + 128, row_full = b0 + 144,
                 row_empty = b0 + 160;
  if (tid == 0) {
    abort_flag = 0;
    for (uint32_t b : {kv_full, kv_empty, raw, done, s_full, dp_full, out_done}) mbar_init(b, 1);
    for (uint32_t b : {p_full, ds_full, out_free}) mbar_init(b, 256);
    for (uint32_t b : {q_full, q_empty, do_full, do_empty}) { mbar_init(b, 1); mbar_init(b + 8, 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(row_full + 8 * s, 32); mbar_init(row_empty + 8 * s, 256); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot, c_s = 0, c_dp = 128, c_dv = 256, c_dk = 384;
  const AttnWait wait{&abort_flag, a.status};
  const int group = a.hq / a.hk;
  // an item is a key tile and a key head; its blocks are the query tiles from the diagonal to the end, head by head
  auto item = [&](int64_t w, AttnTile& t, int& kvh, int& first, int& per_head) {
    t = a.tiles[(int)(w / a.hk)];
    kvh = (int)(w % a.hk);
    first = t.row / kAttnRows;
    per_head = (t.len + kAttnRows - 1) / kAttnRows - first;
  };

  if (warp == 8) {
    // ================================================================= loads
    uint32_t u = 0, n_raw = 0;
    int round = 0;
    bool ok = true;
    // one tile of queries or output gradients; rows beyond the sequence become zero (P^T dO and dS^T Q run over them)
    auto rows_tile = [&](const CUtensorMap* map, uint32_t tile, uint32_t bar, int head, int token, int rows) {
      if (rows >= 128) {
        if (elect_one()) {
          mbar_expect_tx(bar, TILE);
          load_tile<DP>(sk + tile * TILE, map, head, token, bar);
        }
        return true;
      }
      if (elect_one()) {
        mbar_expect_tx(raw, TILE);
        load_tile<DP>(sk + tile * TILE, map, head, token, raw);
      }
      const bool here = wait(raw, n_raw & 1);
      ++n_raw;
      if (!here) { drain_wait(raw, (n_raw - 1) & 1); return false; }
      zero_rows<DP>(base + tile * TILE, rows, lane);
      if (elect_one()) mbar_arrive(bar);
      return true;
    };
    for (; ok; ++round) {
      const int64_t w = work_item(round);
      if ((int64_t)round * gridDim.x >= items) break;
      if (w >= items) continue;
      AttnTile t;
      int kvh, first, per_head;
      item(w, t, kvh, first, per_head);
      if (!(ok = wait(kv_empty, (round & 1) ^ 1))) break;
      if (elect_one()) {
        mbar_expect_tx(kv_full, 2 * TILE);
        load_tile<DP>(sk, &mk, kvh, t.start + t.row, kv_full);
        load_tile<DP>(sv, &mv, kvh, t.start + t.row, kv_full);
      }
      for (int h = 0; ok && h < group; ++h)
        for (int i = 0; ok && i < per_head; ++i, ++u) {
          const int head = kvh * group + h, row = (first + i) * 128, rows = t.len - row;
          const uint32_t s = u & 1, parity = ((u >> 1) & 1) ^ 1;
          if (!(ok = wait(q_empty + 8 * s, parity))) break;
          if (!(ok = rows_tile(&mq, 2 + s, q_full + 8 * s, head, t.start + row, rows))) break;
          if (!(ok = wait(row_empty + 8 * s, parity))) break;
          float* stats = row_stats + s * 256;
          for (int k = lane; k < 128; k += 32) {      // rows beyond the end: P = 2^-inf = 0
            const int64_t at = (int64_t)head * a.tokens + t.start + row + k;
            stats[k] = k < rows ? a.lse[at] * kLog2e : INFINITY;
            stats[128 + k] = k < rows ? a.delta[at] : 0.f;
          }
          mbar_arrive(row_full + 8 * s);
          if (!(ok = wait(do_empty + 8 * s, parity))) break;
          ok = rows_tile(&mdo, 4 + s, do_full + 8 * s, head, t.start + row, rows);
        }
    }
    if (wait.given_up()) {
      const int r = round > 0 && !ok ? round : round - 1;
      if (r >= 0) drain_wait(kv_full, r & 1);
      for (uint32_t k = u > 2 ? u - 2 : 0; k <= u; ++k) {
        drain_wait(q_full + 8 * (k & 1), (k >> 1) & 1);
        drain_wait(do_full + 8 * (k & 1), (k >> 1) & 1);
      }
    }
  } else if (warp == 9) {
    // ================================================================= MMAs
    uint32_t u = 0;
    int n_items = 0;
    bool ok = true;
    auto score = [&](uint32_t k) {
      if (!wait(q_full + 8 * (k & 1), (k >> 1) & 1)) return false;
      tc_fence_after();
      if (elect_one()) {
        mma_columns<BF16, DP>(tmem + c_s, sk, sq + (k & 1) * TILE);
        umma_commit(s_full);
      }
      return true;
    };
    auto dprob = [&](uint32_t k) {
      if (!wait(do_full + 8 * (k & 1), (k >> 1) & 1)) return false;
      tc_fence_after();
      if (elect_one()) {
        mma_columns<BF16, DP>(tmem + c_dp, sv, sdo + (k & 1) * TILE);
        umma_commit(dp_full);
      }
      return true;
    };
    for (int round = 0; ok; ++round) {
      const int64_t w = work_item(round);
      if ((int64_t)round * gridDim.x >= items) break;
      if (w >= items) continue;
      AttnTile t;
      int kvh, first, per_head;
      item(w, t, kvh, first, per_head);
      const int n = group * per_head;
      if (!(ok = wait(kv_full, round & 1))) break;
      if (!(ok = score(u) && dprob(u))) break;
      for (int i = 0; i < n; ++i, ++u) {
        if (!(ok = wait(p_full, u & 1))) break;
        if (i == 0 && !(ok = wait(out_free, (n_items & 1) ^ 1))) break;
        tc_fence_after();
        if (elect_one()) {
          mma_rows<BF16, DP>(tmem + c_dv, tmem + c_s, 64, sdo + (u & 1) * TILE, i > 0);
          umma_commit(do_empty + 8 * (u & 1));
        }
        if (i + 1 < n && !(ok = score(u + 1))) break;
        if (!(ok = wait(ds_full, u & 1))) break;
        tc_fence_after();
        if (elect_one()) {
          mma_rows<BF16, DP>(tmem + c_dk, tmem + c_dp, 64, sq + (u & 1) * TILE, i > 0);
          umma_commit(q_empty + 8 * (u & 1));
          if (i == n - 1) { umma_commit(out_done); umma_commit(kv_empty); }
        }
        if (i + 1 < n && !(ok = dprob(u + 1))) break;
      }
      ++n_items;
    }
    if (elect_one()) umma_commit(done);
    drain_wait(done, 0);
  } else {
    // ================================================================= P^T, dS^T, and the gradients' way out
    const int r = (warp & 3) * 32 + lane, h = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + c_s + 64 * h + lanes, td = tmem + c_dp + 64 * h + lanes;
    const float c = a.scale * kLog2e;
    uint32_t u = 0;
    int n_items = 0;
    bool ok = true;
    for (int round = 0; ok; ++round) {
      const int64_t w = work_item(round);
      if ((int64_t)round * gridDim.x >= items) break;
      if (w >= items) continue;
      AttnTile t;
      int kvh, first, per_head;
      item(w, t, kvh, first, per_head);
      for (int i = 0, q = 0; i < group * per_head; ++i, ++u, q = q + 1 == per_head ? 0 : q + 1) {
        const uint32_t st = u & 1;
        const float4* lse4 = reinterpret_cast<const float4*>(row_stats + st * 256 + 64 * h);
        const float4* delta4 = reinterpret_cast<const float4*>(row_stats + st * 256 + 128 + 64 * h);
        if (!(ok = wait(row_full + 8 * st, (u >> 1) & 1))) break;
        if (!(ok = wait(s_full, u & 1))) break;
        tc_fence_after();
        uint32_t s[64], w16[32];
        float p[64];
        tmem_ld_32(ts, s);
        tmem_ld_32(ts + 32, s + 32);
        tmem_ld_done<64>(s);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const float4 l = lse4[k];
          p[4 * k] = exp2_fast(fmaf(__uint_as_float(s[4 * k]), c, -l.x));
          p[4 * k + 1] = exp2_fast(fmaf(__uint_as_float(s[4 * k + 1]), c, -l.y));
          p[4 * k + 2] = exp2_fast(fmaf(__uint_as_float(s[4 * k + 2]), c, -l.z));
          p[4 * k + 3] = exp2_fast(fmaf(__uint_as_float(s[4 * k + 3]), c, -l.w));
        }
        if (q == 0) {      // on the diagonal: queries before the key do not see it
#pragma unroll
          for (int k = 0; k < 64; ++k)
            if (64 * h + k < r) p[k] = 0.f;
        }
        pack64<BF16>(p, w16);
        tmem_st_32(ts, w16);
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(p_full);
        if (!(ok = wait(dp_full, u & 1))) break;
        tc_fence_after();
        tmem_ld_32(td, s);
        tmem_ld_32(td + 32, s + 32);
        tmem_ld_done<64>(s);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const float4 l = delta4[k];
          p[4 * k] *= __uint_as_float(s[4 * k]) - l.x;
          p[4 * k + 1] *= __uint_as_float(s[4 * k + 1]) - l.y;
          p[4 * k + 2] *= __uint_as_float(s[4 * k + 2]) - l.z;
          p[4 * k + 3] *= __uint_as_float(s[4 * k + 3]) - l.w;
        }
        if (q == 0) {
#pragma unroll
          for (int k = 0; k < 64; ++k)
            if (64 * h + k < r) p[k] = 0.f;
        }
        mbar_arrive(row_empty + 8 * st);
        pack64<BF16>(p, w16);
        tmem_st_32(td, w16);
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(ds_full);
      }
      if (!ok || !(ok = wait(out_done, n_items & 1))) break;
      ++n_items;
      tc_fence_after();
      const bool real = t.row + r < t.len;
      const int64_t token = t.start + t.row + r;
      char *ok_ = a.dk.p + 2 * (token * a.dk.token + kvh * a.dk.head), *ov = a.dv.p + 2 * (token * a.dv.token + kvh * a.dv.head);
#pragma unroll
      for (int k = 0; k < DP / 2; k += 32) {
        uint32_t o[32];
        const int c0 = h * (DP / 2) + k;
        tmem_ld_32(tmem + c_dk + c0 + lanes, o);
        tmem_ld_done<32>(o);
        if (real) store_columns<BF16, 32>(ok_, o, a.scale, c0, a.d);
        tmem_ld_32(tmem + c_dv + c0 + lanes, o);
        tmem_ld_done<32>(o);
        if (real) store_columns<BF16, 32>(ov, o, 1.f, c0, a.d);
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
  if (!attn_tensor_map(plan->encode_tiled, &mq, BF16, a.q, a.tokens, a.hq, a.d) || !attn_tensor_map(plan->encode_tiled, &mk, BF16, a.k, a.tokens, a.hk, a.d) ||
      !attn_tensor_map(plan->encode_tiled, &mv, BF16, a.v, a.tokens, a.hk, a.d) || !attn_tensor_map(plan->encode_tiled, &mdo, BF16, a.dout, a.tokens, a.hq, a.d))
    return op_fail(FGD_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed", who);
  const int sms = sm_count();
  auto dq = attn_dq_tc_kernel<DP, BF16>;
  auto dkv = attn_dkv_tc_kernel<DP, BF16>;
  cudaError_t e = cudaFuncSetAttribute(dq, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)dq_smem<DP>());
  if (e == cudaSuccess) e = cudaFuncSetAttribute(dkv, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)dkv_smem<DP>());
  if (e == cudaSuccess) {
    int64_t items = (int64_t)plan->n_kv * a.hk;
    a.tiles = plan->kv_tiles;
    dkv<<<(unsigned)(items < sms ? items : sms), kBwdThreads, dkv_smem<DP>(), st>>>(a, items, mq, mk, mv, mdo);
    items = (int64_t)plan->n_q * a.hq;
    a.tiles = plan->q_tiles;
    dq<<<(unsigned)(items < sms ? items : sms), kBwdThreads, dq_smem<DP>(), st>>>(a, items, mq, mk, mv, mdo);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

}  // namespace

namespace fgd {

int attn_backward_tc(const fgd_attn_plan* plan, int dtype, const AttnArgs& a, cudaStream_t st) {
  if (a.d <= 64) return dtype == FGD_BF16 ? launch<64, true>(plan, a, st) : launch<64, false>(plan, a, st);
  return dtype == FGD_BF16 ? launch<128, true>(plan, a, st) : launch<128, false>(plan, a, st);
}

}  // namespace fgd

// Causal attention forward on the tensor cores (mathematics: fgd_attn_elem.cu).
//
// A CTA (one per SM) takes two tiles of 128 query rows that read the same key head -- two query heads that share it, or
// two neighbouring row tiles of one head -- so that every key / value tile that comes from L2 feeds 256 query rows.
// Ten warps:
//     0-3, 4-7  softmax of tile 0 and of tile 1: one thread per row.  It reads its 128 scores from tensor memory, keeps
//               the running maximum and sum, and writes P (16 bit) back over the scores;
//     8         loads: Q, then K and V tiles by TMA into a ring, from the diagonal block down to block 0;
//     9         MMAs: S = Q K^T, O += P V.
// Tensor memory (512 columns): S0 | S1 | O0 | O1, P over its own S.  While one tile's softmax runs, the other tile's
// O += P V and its next S run on the tensor cores.
//
// The running maximum only moves O when it has grown by more than 2^8 since O was last scaled: P and the row sum use the
// same stale maximum, so the quotient is exact, and the 16-bit P keeps its relative precision below 2^8 too.  In fp16 P is held times 2^7, at most
// 2^15, so that weights keep it down to 2^-21 of the largest; the sum has the factor too, and lse takes it back.
// Only the block on the diagonal is masked; rows of V beyond the sequence's end are zeroed in shared memory, so nothing of the
// next sequence (0 x inf) reaches a result.
//
// Rounding: P is rounded to the 16-bit type before P V (its sum is taken before, in fp32), one rounding per term next to the output's
// own: the error against 64 bits is .0020 of the result's norm in bf16, .0016 for the output's rounding alone.
//
// What bounds it: a tile's own chain, S (512 clocks at width 128) -> softmax (about 1850: 128 columns from tensor memory, maximum,
// exponentials, P back) -> P V (512) with a hop of 300 to 450 clocks between units, since P lies over S and the next S has to wait
// for P V.  Two tiles side by side hide half of it: 58 % of the tensor pipe's and 56 % of the exponential units' cycles are busy
// (8192 tokens, 16 heads of 128 over 4: 243 us, 1.13 PFLOP/s).  16384 tokens: 971 us, 70 % of the measured matrix peak (83 % of what it
// sustains).  Sequences of different lengths, 9 of 1 to 2011 tokens, 67 us, 41 %: beside the chain, the fixed back-and-forth walk over the
// items gives the fullest CTA 17 % more than the mean (longest first to whoever is free: 5 %), and a tile's end (last P V, output, next
// item's first P) costs about 3800 clocks, 7 us for 3.7 items.
// 168 registers a thread at 320 threads; 78 bytes spilt, in every instance.
// Slower: two threads per row (maxima traded through shared memory; 1025 us at 16384 tokens), the next item's first S before the other
// tile's last P V, outputs held back until after the
// next item's first P; for widths to 64, four query tiles and blocks of 64 keys (16 x 1024, 16 heads of 64: 96 against 80 us).
#include "fgd_attn_tc.cuh"

using namespace fgd;

namespace {

constexpr int kFwdThreads = 320;
template <int DP> constexpr int kFwdStages = DP == 128 ? 4 : 8;
constexpr float kRescale = 8.f;   // log2
template <bool BF16> constexpr float kLift = BF16 ? 0.f : 7.f;   // log2 of P's factor

template <int DP>
constexpr size_t fwd_smem() { return 1024 + (size_t)(2 + kFwdStages<DP>) * attn_tile_bytes<DP>() + 8 * kStoreStage; }

struct FwdItem {
  int start, len, kvh, nmax;
  int head[2], row[2], n[2];   // n: key blocks of the tile (0: no tile)
};
// pair_heads: heads 2 h and 2 h + 1 of one 128-row tile; otherwise rows [r, r + 256) of head h.
__device__ __forceinline__ FwdItem fwd_item(const AttnArgs& a, int pair_heads, const AttnTile& t, int h) {
  FwdItem it;
  it.start = t.start; it.len = t.len;
  it.head[0] = pair_heads ? 2 * h : h;
  it.head[1] = pair_heads ? 2 * h + 1 : h;
  it.row[0] = t.row;
  it.row[1] = pair_heads ? t.row : t.row + kAttnRows;
  it.n[0] = t.row / kAttnRows + 1;
  it.n[1] = it.row[1] < t.len ? it.row[1] / kAttnRows + 1 : 0;
  it.nmax = max(it.n[0], it.n[1]);
  it.kvh = (int)(((float)it.head[0] + 0.5f) * a.inv_group);      // (exact: heads are below 2^15)
  return it;
}

template <int DP, bool BF16>
__global__ void __launch_bounds__(kFwdThreads, 1)
attn_forward_tc_kernel(const AttnArgs a, int pair_heads, FastDiv per_tile, int items, const __grid_constant__ CUtensorMap mq,
                       const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv) {
  constexpr int ST = kFwdStages<DP>;
  constexpr uint32_t TILE = attn_tile_bytes<DP>();
  extern __shared__ unsigned char smem_raw[];
  // q_full, q_empty, raw, done | full[ST], empty[ST] | s_full[2], pv_done[2], o_free[2], p_full[2][2]
  __shared__ __align__(8) unsigned long long bars[4 + 2 * ST + 10];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  unsigned char* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sq = smem_u32(base), skv = sq + 2 * TILE;
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  const uint32_t b0 = smem_u32(bars);
  const uint32_t q_full = b0, q_empty = b0 + 8, raw = b0 + 16, done = b0 + 24, full = b0 + 32, empty = full + 8 * ST, s_full = empty + 8 * ST,
                 pv_done = s_full + 16, o_free = s_full + 32, p_full = s_full + 48;   // p_full + 16 t + 8 half: 64 columns of P each
  if (tid == 0) {
    abort_flag = 0;
    mbar_init(q_full, 1); mbar_init(q_empty, 1); mbar_init(raw, 1); mbar_init(done, 1);
    for (int s = 0; s < ST; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
    for (int t = 0; t < 2; ++t) {
      mbar_init(s_full + 8 * t, 1); mbar_init(pv_done + 8 * t, 1); mbar_init(o_free + 8 * t, 128);
      mbar_init(p_full + 16 * t, 128); mbar_init(p_full + 16 * t + 8, 128);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)uniform((int)tmem_slot);
  const AttnWait wait{&abort_flag, a.status, a.spin_limit};
  // tensor memory columns
  auto s_col = [](int t) { return (uint32_t)(128 * t); };
  auto o_col = [](int t) { return (uint32_t)(256 + 128 * t); };

  if (warp == 8) {
    // ================================================================= loads
    uint32_t u = 0, n_raw = 0;     // ring uses, repaired tiles
    bool ok = true;
    ItemWalk walk(a.tiles, per_tile, items);
    for (; ok && walk.valid; walk.next()) {
      const int round = walk.round;
      const FwdItem it = fwd_item(a, pair_heads, walk.t, walk.h);
      ok = wait(q_empty, (round & 1) ^ 1);
      if (!ok) break;
      if (elect_one()) {
        mbar_expect_tx(q_full, it.n[1] ? 2 * TILE : TILE);
        load_tile<DP>(sq, &mq, it.head[0], it.start + it.row[0], q_full);
        if (it.n[1]) load_tile<DP>(sq + TILE, &mq, it.head[1], it.start + it.row[1], q_full);
      }
      for (int jb = it.nmax - 1; ok && jb >= 0; --jb) {
        const int token = it.start + jb * 128, rows = it.len - jb * 128;
        for (int v = 0; v < 2; ++v, ++u) {
          const uint32_t s = u % ST, bar = full + 8 * s, dst = skv + s * TILE;
          ok = wait(empty + 8 * s, ((u / ST) & 1) ^ 1);
          if (!ok) break;
          if (v == 0 || rows >= 128) {
            if (elect_one()) {
              mbar_expect_tx(bar, TILE);
              if ((int)u != a.skip) load_tile<DP>(dst, v ? &mv : &mk, it.kvh, token, bar);
            }
          } else {     // the sequence ends inside this tile
            if (elect_one()) {
              mbar_expect_tx(raw, TILE);
              if ((int)u != a.skip) load_tile<DP>(dst, &mv, it.kvh, token, raw);
            }
            ok = wait(raw, n_raw & 1);
            ++n_raw;
            if (!ok) { wait.drain(raw, (n_raw - 1) & 1); break; }
            zero_rows<DP>(base + 2 * TILE + s * TILE, rows, lane);
            if (elect_one()) mbar_arrive(bar);
          }
        }
      }
    }
    // a CTA that gave up still waits for its own copies
    if (wait.given_up()) {
      wait.drain(q_full, walk.round & 1);
      if (walk.round > 0) wait.drain(q_full, (walk.round - 1) & 1);
      for (uint32_t k = u > (uint32_t)ST ? u - ST : 0; k < u; ++k) wait.drain(full + 8 * (k % ST), (k / ST) & 1);
    }
  } else if (warp == 9) {
    // ================================================================= MMAs
    uint32_t u = 0;
    uint32_t n_p[2] = {0, 0}, n_o[2] = {0, 0};
    bool ok = true;
    auto score = [&](int t, uint32_t stage) {
      mma_columns<BF16, DP>(tmem + s_col(t), sq + t * TILE, skv + stage * TILE);
      mma_commit(s_full + 8 * t);
    };
    auto release = [&](uint32_t use) { mma_commit(empty + 8 * (use % ST)); };
    auto arrived = [&](uint32_t use) { return wait(full + 8 * (use % ST), (use / ST) & 1); };
    for (ItemWalk walk(a.tiles, per_tile, items); ok && walk.valid; walk.next()) {
      const FwdItem it = fwd_item(a, pair_heads, walk.t, walk.h);
      if (!(ok = wait(q_full, walk.round & 1))) break;
      uint32_t uk = u++;
      if (!(ok = arrived(uk))) break;
      tc_fence_after();
      for (int t = 0; t < 2; ++t)
        if (it.nmax - 1 < it.n[t]) score(t, uk % ST);
      release(uk);
      if (it.nmax == 1) mma_commit(q_empty);
      for (int jb = it.nmax - 1; ok && jb >= 0; --jb) {
        const uint32_t uv = u++;
        uk = u;
        bool k_here = false;
        if (!(ok = arrived(uv))) break;
        for (int t = 0; ok && t < 2; ++t) {
          if (jb < it.n[t]) {
            const bool first = jb == it.n[t] - 1;
            for (int half = 0; ok && half < 2; ++half) {
              ok = wait(p_full + 16 * t + 8 * half, n_p[t] & 1);
              if (ok && first && half == 0) {      // the tile's previous output has been read
                ok = wait(o_free + 8 * t, (n_o[t] & 1) ^ 1);
                ++n_o[t];
              }
              if (!ok) break;
              tc_fence_after();
              mma_half_rows<BF16, DP>(tmem + o_col(t), tmem + s_col(t) + 32 * half, skv + (uv % ST) * TILE, half, !first || half == 1);
            }
            ++n_p[t];
            if (!ok) break;
            mma_commit(pv_done + 8 * t);
          }
          if (t == 1) release(uv);
          if (jb > 0 && jb - 1 < it.n[t]) {
            if (!k_here && !(ok = arrived(uk))) break;
            k_here = true;
            tc_fence_after();
            score(t, uk % ST);
          }
        }
        if (ok && jb > 0) { release(uk); ++u; }
        if (ok && jb == 1) mma_commit(q_empty);     // the last scores of this item are on their way
      }
      __syncwarp();
    }
    // tensor memory is not released under a running MMA
    mma_commit(done);
    wait.drain(done, 0);
  } else {
    // ================================================================= softmax
    const int t = warp >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + s_col(t) + lanes, to = tmem + o_col(t) + lanes;
    const float c = a.scale * kLog2e;
    uint32_t n_s = 0, n_pv = 0;
    bool ok = true;
    for (ItemWalk walk(a.tiles, per_tile, items); ok && walk.valid; walk.next()) {
      const FwdItem it = fwd_item(a, pair_heads, walk.t, walk.h);
      const int n = it.n[t];
      if (n == 0) continue;
      const bool real = it.row[t] + r < it.len;
      float m = 0.f;
      float2 l = make_float2(0.f, 0.f);
      for (int jb = n - 1; jb >= 0; --jb) {
        if (!(ok = wait(s_full + 8 * t, n_s & 1))) break;
        ++n_s;
        tc_fence_after();
        uint32_t s[128];
        tmem_ld_32(ts, s);
        tmem_ld_32(ts + 32, s + 32);
        tmem_ld_done<64>(s);
        tmem_ld_32(ts + 64, s + 64);          // on their way while the first half's maximum is found
        tmem_ld_32(ts + 96, s + 96);
        const bool diagonal = jb == n - 1;
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        auto half_max = [&](int from) {
          if (diagonal) {
#pragma unroll
            for (int k = 0; k < 64; ++k)
              if (from + k > r) s[from + k] = 0xFF800000u;
          }
#pragma unroll
          for (int k = 0; k < 64; k += 2) mx[(k >> 1) & 3] = max3(mx[(k >> 1) & 3], __uint_as_float(s[from + k]), __uint_as_float(s[from + k + 1]));
        };
        half_max(0);
        tmem_ld_done<64>(s + 64);
        half_max(64);
        const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * c;
        if (diagonal) {
          // No finite score here (an infinite key): a maximum that every later finite one exceeds, and from which -inf is still -inf away.
          m = top == -INFINITY ? -1.7e38f : top;
        } else if (__any_sync(0xffffffffu, real && top > m + kRescale)) {      // (rows of another sequence have no say in it)
          const float mn = fmaxf(m, top), f = exp2_fast(m - mn);
          if (!(ok = wait(pv_done + 8 * t, (n_pv - 1) & 1))) break;
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < DP; k += 16) {
            uint32_t o[16];
            tmem_ld_8(to + k, reinterpret_cast<float*>(o));
            tmem_ld_8(to + k + 8, reinterpret_cast<float*>(o + 8));
            tmem_ld_done<16>(o);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            tmem_st_16(to + k, o);
          }
          l.x *= f;
          l.y *= f;
          m = mn;
        }
        // p = 2^(c s - m), 32 columns at a time
        const float2 c2 = both(c), m2 = both(kLift<BF16> - m);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t p[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const float2 x = exp2_pair(fma2(two(s + 32 * q + 2 * k), c2, m2), k);
            l = add2(l, x);
            p[k] = pack2<BF16>(x.x, x.y);
          }
          tmem_st_16(ts + 16 * q, p);
          if (q & 1) {                        // half of P: its product can start
            tmem_st_wait();
            tc_fence_before();
            mbar_arrive(p_full + 16 * t + 8 * (q >> 1));
          }
        }
        ++n_pv;
      }
      if (!ok || !(ok = wait(pv_done + 8 * t, (n_pv - 1) & 1))) break;
      tc_fence_after();
      const float sum = l.x + l.y, f = 1.f / sum;
      const int row0 = it.row[t] + (warp & 3) * 32;      // the warp's first row
      char* out = a.o.p + 2 * ((int64_t)(it.start + row0) * a.o.token + it.head[t] * a.o.head);
#pragma unroll
      for (int k = 0; k < DP; k += 32) {
        uint32_t o[32];
        tmem_ld_32(to + k, o);
        tmem_ld_done<32>(o);
        store_rows<BF16>(base + (2 + ST) * TILE + warp * kStoreStage, o, f, out, 2 * a.o.token, it.len - row0, k, a.d, lane);
      }
      tc_fence_before();
      mbar_arrive(o_free + 8 * t);
      if (row0 + lane < it.len) a.lse[it.head[t] * a.tokens + it.start + row0 + lane] = (m + (log2f(sum) - kLift<BF16>)) * kLn2;
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
  const char* who = "fgd_attn_forward";
  const bool pair_heads = (a.hq / a.hk) % 2 == 0;
  a.tiles = pair_heads ? plan->q_tiles : plan->q2_tiles;
  a.n_tiles = pair_heads ? plan->n_q : plan->n_q2;
  const int per_tile = pair_heads ? a.hq / 2 : a.hq;
  const int64_t items = (int64_t)a.n_tiles * per_tile;
  if (items > 0x7fffffff - 1024) return op_fail(FGD_ERR_UNSUPPORTED, "%s: %lld tiles", who, (long long)items);
  CUtensorMap mq, mk, mv;
  if (!attn_tensor_map(plan->encode_tiled, &mq, BF16, a.q, a.tokens, a.hq, a.d) || !attn_tensor_map(plan->encode_tiled, &mk, BF16, a.k, a.tokens, a.hk, a.d) ||
      !attn_tensor_map(plan->encode_tiled, &mv, BF16, a.v, a.tokens, a.hk, a.d))
    return op_fail(FGD_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed", who);
  auto kern = attn_forward_tc_kernel<DP, BF16>;
  cudaError_t e = allow_smem<attn_forward_tc_kernel<DP, BF16>>(fwd_smem<DP>());
  if (e == cudaSuccess) {
    const int sms = sm_count();
    kern<<<(unsigned)(items < sms ? items : sms), kFwdThreads, fwd_smem<DP>(), st>>>(a, pair_heads, FastDiv(per_tile), (int)items, mq, mk, mv);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

}  // namespace

namespace fgd {

int attn_forward_tc(const fgd_attn_plan* plan, int dtype, const AttnArgs& a, cudaStream_t st) {
  if (a.d <= 64) return dtype == FGD_BF16 ? launch<64, true>(plan, a, st) : launch<64, false>(plan, a, st);
  return dtype == FGD_BF16 ? launch<128, true>(plan, a, st) : launch<128, false>(plan, a, st);
}

}  // namespace fgd

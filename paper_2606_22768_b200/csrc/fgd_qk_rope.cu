// Norms of queries and keys per head with the rotation by position in the same pass, for K workers at once.
//
//   z = x r w,  r = 1 / sqrt(mean(x^2) + eps)   (without weights: z = x)
//   (a, b) a pair of the first `rotary` channels of z:  a' = a cos - b sin,  b' = b cos + a sin,   cos, sin = tables[position][pair]
//   the other channels: z
// Gradients from x and dy (dz: the transposed rotation of dy):
//   dw = sum over tokens and heads of dz x r,   dx = r (dz w - x r^2 mean(dz w x))
// Without weights the backward pass is the transposed rotation alone: the forward kernel with -sin.
//
// Bound by HBM, and close to it by instructions: 8 x 4096 tokens of 16 + 4 heads of 128, bf16, forward 61 us (83 % of the copy peak; the same walk without norm and
// rotation 60), backward 95 us (81 %; 83 to 85); rotation alone of 16384 tokens 31 us (83 %).
//
// A lane holds 2 V channels of a head: a chunk of V consecutive ones and the chunk of their partners, so the rotation needs no other lane and the
// norm log2(lanes) shuffles.  LG lanes make a head, 32 / LG heads a warp.  Of those, gt (the most that divide their number and both head counts)
// belong to one token: a warp goes through its tokens' heads gt at a time, and a lane's cos and sin serve all that it has of a token.  It takes all
// its q first and then its k: so the weights and, in the backward pass, the sums of their gradients (CTAs belong to one worker) stay in
// registers, of one side at a time.  What the next steps need is on its way meanwhile: activations through a ring in shared memory that each lane
// fills for itself (cp.async), the next token's cos and sin in registers.
#include <cmath>

#include "fgd_dtype.cuh"
#include "fgd_heads.h"
#include "fgd_nvtx.h"

using namespace fgd;

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
// CTAs on an SM: what the kernels' registers allow, by the channels of a lane.  (Eight pairs: four and three; the backward pass with four, 128 registers a
// thread and some of them spilled, takes 109 us for 8 x 4096 tokens of 20 heads of 128 instead of 96.  Fewer pairs: one CTA more: 16384 tokens of 20
// heads, bf16, 72 wide (with 16 lanes) 40 and 69 us with four and three, 38 and 61 with five and four; 100 wide 65 and 120, 61 and 97; 66 wide 96 and 223, 89 and 170; 80 wide fp32
// 44 and 73, 41 and 62.  The one that loses: backward of 128 wide fp32, 85 and 92.)
constexpr int ctas_of(int v, int nc, bool grad) { return (grad ? 4 : 5) - (v == 8 || nc == 4); }
constexpr int kMostBackwardCtas = 4;
constexpr int kMaxDim = 256;

struct RopeHeads { char* p; int64_t ts, hs, step; };      // strides, and from one of a warp's batches to the next, in bytes
struct RopeSide {
  RopeHeads x, y, g;           // forward: input, output; backward: input, gradient out, gradient in
  const float* w; int64_t w_ld;
  int batches;                 // of gt heads of a token
};
struct RopeArgs {
  RopeSide side[2];
  const float *cos, *sin; int64_t cos_ld, sin_ld;
  const void* positions; int position_bytes;
  int64_t rows, table_rows;
  int d, rot, lg, pairs;       // lanes of a head; chunk pairs of a head
  int gt, split;               // lane groups that share a token; warps that share its batches
  float eps, inv_d, turn;      // turn: 1, or -1 for the transposed rotation
  float* partial;              // backward: [worker][cta][q or k][d]
};

// V consecutive values as they lie in memory.
template <typename T, int V>
struct Chunk {
  static constexpr int kBytes = V * sizeof(T), kWords = kBytes < 4 ? 1 : kBytes / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes == 16) { const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p)); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
    else if constexpr (kBytes == 8) { const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p)); w[0] = v.x; w[1] = v.y; }
    else if constexpr (kBytes == 4) w[0] = __ldcs(reinterpret_cast<const uint32_t*>(p));
    else w[0] = __ldcs(reinterpret_cast<const unsigned short*>(p));
  }
  __device__ __forceinline__ void from_shared(uint32_t p) {
    if constexpr (kBytes == 16) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(p) : "memory");
    else if constexpr (kBytes == 8) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(p) : "memory");
    else asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(p) : "memory");
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (kBytes == 16) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *reinterpret_cast<unsigned short*>(p) = (unsigned short)w[0];
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ void get(float* f) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        const float2 h = halves<T>(w[i]);
        f[2 * i] = h.x;
        if (V > 1) f[2 * i + 1] = h.y;
      }
    }
  }
  __device__ __forceinline__ void set(const float* f) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = __float_as_uint(f[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = from_pair<T>(f[2 * i], V > 1 ? f[2 * i + 1] : 0.f);
    }
  }
};

// Where a lane's chunk pairs lie in a head: chunk j's first channels c0 and c1, its first table column, and what of it exists.
template <int V, int NC, bool INTER>
struct Geometry {
  // Neighbouring pairs lie inside the chunks, half of them in each (a lane's two chunks are apart all the same: side by side, memory would be read in
  // half sectors, 43 us instead of 31 for 16384 tokens of 20 heads of 128); of single values the pair is the two chunks.
  static constexpr bool kInside = INTER && V > 1, kBeside = INTER && V == 1;
  int c0[NC], c1[NC], at[NC];
  bool has0[NC], has1[NC], turns[NC];
  __device__ __forceinline__ Geometry(int sub, const RopeArgs& a) {
    const int turning = a.rot / (2 * V), rest = a.pairs - turning;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int p = sub + j * a.lg;
      turns[j] = p < turning;
      at[j] = kInside ? p * V / 2 : p * V;
      if (turns[j]) { c0[j] = kBeside ? 2 * p : p * V; c1[j] = kBeside ? c0[j] + 1 : c0[j] + a.rot / 2; }
      else { c0[j] = a.rot + (p - turning) * V; c1[j] = c0[j] + rest * V; }
      has0[j] = p < a.pairs && c0[j] < a.d;
      has1[j] = p < a.pairs && c1[j] < a.d;
    }
  }
};

__device__ __forceinline__ int64_t position_of(const RopeArgs& a, int64_t token) {
  if (!a.positions) return token;
  return a.position_bytes == 8 ? __ldg(static_cast<const long long*>(a.positions) + token) : (int64_t)__ldg(static_cast<const int*>(a.positions) + token);
}
template <int V>
__device__ __forceinline__ void load_table(const float* p, float* f) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
      const float4 v = __ldg(reinterpret_cast<const float4*>(p) + i);
      f[4 * i] = v.x; f[4 * i + 1] = v.y; f[4 * i + 2] = v.z; f[4 * i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = __ldg(p + i);
  }
}
// cos and sin of a token for a lane's channels.  A position outside the tables turns the whole head into NaN: `good` is false.
template <int V, int NC>
struct Angles {
  float cs[NC][V], sn[NC][V];
  bool good;
  template <bool INTER>
  __device__ __forceinline__ void load(const RopeArgs& a, const Geometry<V, NC, INTER>& geo, int64_t pos) {
    good = pos >= 0 && pos < a.table_rows;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
#pragma unroll
      for (int i = 0; i < V; ++i) { cs[j][i] = 1.f; sn[j][i] = 0.f; }
      if (good && geo.turns[j] && geo.has0[j]) {
        const float *c = a.cos + pos * a.cos_ld + geo.at[j], *s = a.sin + pos * a.sin_ld + geo.at[j];
        if constexpr (Geometry<V, NC, INTER>::kInside) {
          load_table<V / 2>(c, cs[j]);
          load_table<V / 2>(s, sn[j]);
          load_table<V / 2>(c + a.rot / 4, cs[j] + V / 2);
          load_table<V / 2>(s + a.rot / 4, sn[j] + V / 2);
        } else {
          load_table<V>(c, cs[j]);
          load_table<V>(s, sn[j]);
        }
      }
    }
  }
};

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ float2 two(const float* f) { return make_float2(f[0], f[1]); }
__device__ __forceinline__ void put(float* f, float2 v) { f[0] = v.x; f[1] = v.y; }
// A lane's 2 V channels in registers: the pairs' first members, then their second ones, whichever way they lie in memory (neighbours where INTER).
template <int V, bool INTER>
__device__ __forceinline__ void to_pairs(float (&z)[2 * V]) {
  if constexpr (INTER) {
    float m[2 * V];
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) m[i] = z[i];
#pragma unroll
    for (int i = 0; i < V; ++i) { z[i] = m[2 * i]; z[V + i] = m[2 * i + 1]; }
  }
}
template <int V, bool INTER>
__device__ __forceinline__ void from_pairs(float (&z)[2 * V]) {
  if constexpr (INTER) {
    float m[2 * V];
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) m[i] = z[i];
#pragma unroll
    for (int i = 0; i < V; ++i) { z[2 * i] = m[i]; z[2 * i + 1] = m[V + i]; }
  }
}

// N tensors' chunk pairs of a step, kDepth - 1 steps ahead: in shared memory where a lane has one pair of at least 4 bytes each.  A lane reads back what
// it copied itself: no barrier.  A lane without a chunk reads the zeros that it put there first; of a token beyond the last it reads anything,
// and nothing is made of it.  Else one step ahead, in registers.
template <typename T, int V, int NC, int N>
struct Feed {
  static constexpr int kBytes = V * sizeof(T);
  static constexpr bool kRing = kBytes >= 4 && NC == 1;
  static constexpr int kDepth = kRing ? 4 : 2, kPart = 32 * kBytes, kSlot = N * 2 * kPart, kWarpBytes = kRing ? kDepth * kSlot : 0;
  uint32_t base, at;      // of the lane's part of a warp's ring; the slot of the current step
  Chunk<T, V> held[kRing ? 1 : N][kRing ? 1 : NC][2];
  __device__ __forceinline__ void start(unsigned char* ring, bool has) {
    if constexpr (kRing) {
      base = (uint32_t)__cvta_generic_to_shared(ring) + (threadIdx.x / 32) * kWarpBytes + (threadIdx.x & 31) * kBytes;
      at = 0;
      if (!has) {
#pragma unroll
        for (int i = 0; i < kDepth * N * 2; ++i)
#pragma unroll
          for (int b = 0; b < kBytes; b += 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(base + i * kPart + b), "r"(0) : "memory");
      }
    }
  }
  // The step `ahead` behind the current one; kDepth - 1: into the slot of the one before it.
  template <bool INTER>
  __device__ __forceinline__ void fetch(const char* const (&p)[N], bool real, bool all, int ahead, const Geometry<V, NC, INTER>& geo) {
    if constexpr (kRing) {
      const int partner = (geo.c1[0] - geo.c0[0]) * (int)sizeof(T);
      const uint32_t to = base + (at + ahead * kSlot) % kWarpBytes;
      if (real && geo.has0[0]) {
#pragma unroll
        for (int n = 0; n < N; ++n)
          if (n == 0 || all) {
            copy_async<kBytes>(to + 2 * n * kPart, p[n]);
            copy_async<kBytes>(to + (2 * n + 1) * kPart, p[n] + partner);
          }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            held[n][j][half].clear();
            if (real && (n == 0 || all) && (half ? geo.has1[j] : geo.has0[j])) held[n][j][half].load(reinterpret_cast<const T*>(p[n]) + (half ? geo.c1[j] : geo.c0[j]) - geo.c0[0]);
          }
    }
  }
  __device__ __forceinline__ void wait() {
    if constexpr (kRing) asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 2) : "memory");
  }
  template <bool INTER>
  __device__ __forceinline__ void get(float (&z)[NC][2 * V], int n, std::bool_constant<INTER>) {
#pragma unroll
    for (int j = 0; j < NC; ++j) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if constexpr (kRing) {
          Chunk<T, V> c;
          c.from_shared(base + at + (2 * n + half) * kPart);
          c.get(z[j] + half * V);
        } else {
          held[n][j][half].get(z[j] + half * V);
        }
      }
      to_pairs<V, INTER>(z[j]);
    }
  }
  __device__ __forceinline__ void next() {
    if constexpr (kRing) at = (at + kSlot) % kWarpBytes;
  }
};

// The pairs of a chunk and its partner, turned: turn is 1, or -1 for the transposed rotation.  Products and sums are rounded one by one, and every form
// of the rotation that computes in fp32 without contraction agrees with this one to the bit.  (A sum is written as a product with +-1, which is
// exact, because the compiler contracts a packed product and a packed sum into one operation; the factor is one that it does not know.)
template <int V>
__device__ __forceinline__ void rotate(float (&z)[2 * V], const float (&cs)[V], const float (&sn)[V], float turn) {
  if constexpr (V == 1) {
    const float a = z[0], b = z[1];
    z[0] = fmaf(__fmul_rn(b, sn[0]), -turn, __fmul_rn(a, cs[0]));
    z[1] = fmaf(__fmul_rn(a, sn[0]), turn, __fmul_rn(b, cs[0]));
  } else {
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const float2 a = two(z + i), b = two(z + V + i), c = two(cs + i), s = two(sn + i);
      put(z + i, fma2(mul2(b, s), both(-turn), mul2(a, c)));
      put(z + V + i, fma2(mul2(a, s), both(turn), mul2(b, c)));
    }
  }
}
// Sums over the lanes of a head, for each of them; `place` is a lane's in its head.  All lanes of the warp take part.  EXACT: any number of lanes, else
// a power of two.
template <bool EXACT, int N>
__device__ __forceinline__ void head_sums(float (&v)[N], int lg, int place) {
  if constexpr (EXACT) {      // folded in halves onto the first lane
#pragma unroll
    for (int o = 8; o > 0; o /= 2) {
      if (o >= lg) continue;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const float t = __shfl_down_sync(0xffffffffu, v[n], o);
        if (place + o < lg) v[n] += t;
      }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = __shfl_sync(0xffffffffu, v[n], (threadIdx.x & 31) - place);
  } else {
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      if (o >= lg) break;
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
    }
  }
}
template <typename T, int V, int NC, bool INTER>
__device__ __forceinline__ void store_head(float (&z)[NC][2 * V], T* p, bool real, const Geometry<V, NC, INTER>& geo) {
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    from_pairs<V, INTER>(z[j]);
    Chunk<T, V> c;
    c.set(z[j]);
    if (real && geo.has0[j]) c.store(p + geo.c0[j] - geo.c0[0]);
    c.set(z[j] + V);
    if (real && geo.has1[j]) c.store(p + geo.c1[j] - geo.c0[0]);
  }
}
template <int V, int NC, bool INTER>
__device__ __forceinline__ void load_weights(const float* w, const Geometry<V, NC, INTER>& geo, float (&f)[NC][2 * V]) {
#pragma unroll
  for (int j = 0; j < NC; ++j) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      f[j][i] = geo.has0[j] ? __ldg(w + geo.c0[j] + i) : 0.f;
      f[j][V + i] = geo.has1[j] ? __ldg(w + geo.c1[j] + i) : 0.f;
    }
    to_pairs<V, INTER>(f[j]);
  }
}
template <int V, int NC>
__device__ __forceinline__ void poison(float (&z)[NC][2 * V]) {
#pragma unroll
  for (int j = 0; j < NC; ++j)
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) z[j][i] = __int_as_float(0x7fffffff);
}

// GRAD: the backward pass with weights.  Otherwise the forward pass, or the transposed rotation alone.  EXACT: a.lg is any number of lanes up to 16.
template <typename T, int V, int NC, bool INTER, bool GRAD, bool EXACT>
__global__ void __launch_bounds__(kThreads, ctas_of(V, NC, GRAD)) rope_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int N = GRAD ? 2 : 1;      // tensors that are read: the gradient, x; or x alone
  using Ring = Feed<T, V, NC, N>;
  extern __shared__ __align__(16) unsigned char ring[];
  __shared__ float sums[GRAD ? 2 : 1][GRAD ? kWarps : 1][kMaxDim];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  // (lanes behind the last head that fits have no channels)
  const bool extra = EXACT && lane >= 32 / a.lg * a.lg;
  const int group = extra ? 0 : lane / a.lg, in_head = extra ? a.pairs : lane % a.lg, sub = group % a.gt;
  const uint32_t tokens = 32 / a.lg / a.gt, mine = group / a.gt;      // tokens of a warp at once, this lane's among them
  const uint32_t rows = (uint32_t)a.rows, place = blockIdx.x * kWarps + warp, stride = gridDim.x * kWarps / a.split * tokens, first = place / a.split * tokens;
  const int part = place % a.split;
  const Geometry<V, NC, INTER> geo(in_head, a);
  const int worker = wait_for_previous((int)blockIdx.y);
  const int64_t base = worker * a.rows + mine;
  if constexpr (GRAD) let_next_start();      // the sums' CTAs wait for this kernel's end on the SMs
  // The step that is fetched next, kDepth - 1 ahead: side, first token of the warp's group, batch, addresses.  (An address moves on by a constant
  // within a token; worked out anew in every step they were a third of the kernel's instructions.)
  int ahead_side = first >= rows ? 2 : part < a.side[0].batches ? 0 : 1, ahead_b = part;
  uint32_t ahead_t0 = first;
  const char* in[N];
  auto at = [&](const RopeHeads& h, uint32_t t0) { return h.p + (base + t0) * h.ts + (sub + part * a.gt) * h.hs + geo.c0[0] * (int)sizeof(T); };      // of a lane's first channel
  auto seek = [&](const RopeSide& s) {
    in[0] = at(GRAD ? s.g : s.x, ahead_t0);
    if constexpr (GRAD) in[N - 1] = at(s.x, ahead_t0);
  };
  auto advance = [&] {
    if (ahead_side == 2) return;
    const RopeSide& s = a.side[ahead_side];
    if ((ahead_b += a.split) < s.batches) {
      in[0] += GRAD ? s.g.step : s.x.step;
      if constexpr (GRAD) in[N - 1] += s.x.step;
      return;
    }
    ahead_b = part;
    ahead_t0 += stride;
    if (ahead_t0 >= rows) {
      ahead_t0 = first;
      if (++ahead_side == 1 && part >= a.side[1].batches) ahead_side = 2;
    }
    if (ahead_side < 2) seek(a.side[ahead_side]);
  };
  Ring feed;
  auto fetch = [&](int steps) {
    const bool real = ahead_side < 2 && ahead_t0 + mine < rows;
    feed.fetch(in, real, real && a.side[ahead_side & 1].w != nullptr, steps, geo);      // (without weights x may be absent)
  };
  if (ahead_side == 1 && part >= a.side[1].batches) ahead_side = 2;
  seek(a.side[ahead_side & 1]);
  feed.start(ring, geo.has0[0]);
#pragma unroll
  for (int i = 0; i < Ring::kDepth - 1; ++i) {
    fetch(i);
    advance();
  }
#pragma unroll 1
  for (int side = 0; side < 2; ++side) {
    const RopeSide& s = a.side[side];
    const bool norm = s.w != nullptr;      // (of the gradient's kernel: one of the sides may be the rotation alone)
    float w[NC][2 * V], dw[NC][2 * V];
    if (norm) load_weights(s.w + worker * s.w_ld, geo, w);
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) dw[j][i] = 0.f;
    // Forward: positions two tokens ahead, cos and sin one.  The backward pass has no registers for that: 99 us with them for 8 x 4096 tokens of 20
    // heads of 128, 95 without.
    auto position = [&](uint32_t t0) { return t0 + mine < rows ? position_of(a, base + t0) : (int64_t)-1; };
    Angles<V, NC> turn, next;
    if constexpr (!GRAD) next.load(a, geo, position(first));
    int64_t pos = position(GRAD ? first : first + stride);
    for (uint32_t t0 = part < s.batches ? first : rows; t0 < rows; t0 += stride) {
      const bool real = t0 + mine < rows;
      if constexpr (GRAD) {
        turn.load(a, geo, pos);
        pos = position(t0 + stride);
      } else {
        turn = next;
        next.load(a, geo, pos);
        pos = position(t0 + 2 * stride);
      }
      char* out = at(s.y, t0);
#pragma unroll (GRAD ? 1 : 2)
      for (int b = part; b < s.batches; b += a.split, out += s.y.step) {
        feed.wait();
        float z[NC][2 * V], v[NC][2 * V];
        feed.get(z, 0, std::bool_constant<INTER>{});
        if constexpr (GRAD) feed.get(v, 1, std::bool_constant<INTER>{});
        fetch(Ring::kDepth - 1);
        advance();
        feed.next();
        if constexpr (!GRAD) {
          if (norm) {
            float2 ss = both(0.f);
#pragma unroll
            for (int j = 0; j < NC; ++j)
#pragma unroll
              for (int i = 0; i < 2 * V; i += 2) ss = fma2(two(z[j] + i), two(z[j] + i), ss);
            float sum[1] = {ss.x + ss.y};
            head_sums<EXACT>(sum, a.lg, in_head);
            const float2 r = both(rsqrtf(fmaf(sum[0], a.inv_d, a.eps)));
#pragma unroll
            for (int j = 0; j < NC; ++j)
#pragma unroll
              for (int i = 0; i < 2 * V; i += 2) put(z[j] + i, mul2(two(z[j] + i), mul2(r, two(w[j] + i))));
          }
        }
#pragma unroll
        for (int j = 0; j < NC; ++j)
          if (geo.turns[j]) rotate<V>(z[j], turn.cs[j], turn.sn[j], a.turn);
        if (!turn.good) poison<V, NC>(z);
        if constexpr (GRAD) {
          if (norm) {
            // u = dz x: dw += u r, dx = r dz w - k x, k = r^3 mean(u w)
            float2 ss = both(0.f), sg = both(0.f);
#pragma unroll
            for (int j = 0; j < NC; ++j)
#pragma unroll
              for (int i = 0; i < 2 * V; i += 2) {
                const float2 x = two(v[j] + i);
                ss = fma2(x, x, ss);
                sg = fma2(mul2(two(z[j] + i), x), two(w[j] + i), sg);
              }
            float sum[2] = {ss.x + ss.y, sg.x + sg.y};
            head_sums<EXACT>(sum, a.lg, in_head);
            const float r = rsqrtf(fmaf(sum[0], a.inv_d, a.eps)), k = r * r * (r * sum[1] * a.inv_d);
            if (real) {
#pragma unroll
              for (int j = 0; j < NC; ++j)
#pragma unroll
                for (int i = 0; i < 2 * V; i += 2) {
                  const float2 x = two(v[j] + i), dz = two(z[j] + i);
                  put(dw[j] + i, fma2(mul2(dz, x), both(r), two(dw[j] + i)));
                  put(z[j] + i, fma2(both(r), mul2(dz, two(w[j] + i)), mul2(both(-k), x)));
                }
            }
          }
        }
        store_head<T, V, NC, INTER>(z, reinterpret_cast<T*>(out), real, geo);
      }
    }
    if constexpr (GRAD) {
      if (norm) {
#pragma unroll
        for (int j = 0; j < NC; ++j) from_pairs<V, INTER>(dw[j]);
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) {
            float t = dw[j][i];
            if constexpr (EXACT) {
              for (int o = a.lg; o + a.lg <= 32; o += a.lg) t += __shfl_sync(0xffffffffu, dw[j][i], (lane + o) & 31);
            } else {
              for (int o = a.lg; o < 32; o *= 2) t += __shfl_xor_sync(0xffffffffu, t, o);
            }
            const bool has = i < V ? geo.has0[j] : geo.has1[j];
            if (group == 0 && has) sums[side][warp][i < V ? geo.c0[j] + i : geo.c1[j] + i - V] = t;
          }
      }
    }
  }
  if constexpr (GRAD) {
    __syncthreads();
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      if (!a.side[side].w) continue;
      float* out = a.partial + (((int64_t)worker * gridDim.x + blockIdx.x) * 2 + side) * a.d;
      for (int c = threadIdx.x; c < a.d; c += kThreads) {
        float t = sums[side][0][c];
#pragma unroll
        for (int i = 1; i < kWarps; ++i) t += sums[side][i][c];
        out[c] = t;
      }
    }
  }
}

// dw of a worker and side: its CTAs' sums, 32 at a time added in order, 32 channels a CTA.
constexpr int kParts = 32;
struct RopeSums { const float* partial; float* dw[2]; int64_t ld[2]; int ctas, d; };
__global__ void __launch_bounds__(32 * kParts) rope_sums_kernel(const __grid_constant__ RopeSums a) {
  wait_for_previous();
  __shared__ float buf[kParts][32];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, worker = blockIdx.y, side = blockIdx.z;
  if (!a.dw[side]) return;
  const float* p = a.partial + ((int64_t)worker * a.ctas * 2 + side) * a.d + c;
  float t = 0.f;
  if (c < a.d) {
#pragma unroll 8
    for (int i = part; i < a.ctas; i += kParts) t += p[(int64_t)i * 2 * a.d];
  }
  buf[part][lane] = t;
  __syncthreads();
  if (part != 0 || c >= a.d) return;
#pragma unroll
  for (int i = 1; i < kParts; ++i) t += buf[i][lane];
  a.dw[side][worker * a.ld[side] + c] = t;
}

// ---- host
// The most of a warp's lane groups that can share a token's heads evenly: it divides their number and both head counts.
int group_of(int q_heads, int k_heads, int groups) {
  int g = groups;
  while (groups % g != 0 || q_heads % g != 0 || k_heads % g != 0) --g;
  return g;
}
// CTAs of one worker: its share of the SMs' places, and no more than there is work for.
int ctas_for(int per_sm, int64_t workers, int64_t rows, int64_t warp_tokens) {
  int64_t c = (int64_t)sm_count() * per_sm / workers;
  const int64_t most = (rows + kWarps * warp_tokens - 1) / (kWarps * warp_tokens);
  if (c > most) c = most;
  return (int)(c < 1 ? 1 : c);
}

bool vector_of(const void* p, int64_t s0, int64_t s1, int bytes, int vec) {
  return reinterpret_cast<uintptr_t>(p) % (uintptr_t)(vec * bytes) == 0 && s0 % vec == 0 && s1 % vec == 0;
}

struct Launch { int vec, lg, pairs; };

int64_t workspace_bytes(int workers, int d) { return ((int64_t)sm_count() * kMostBackwardCtas + workers) * 2 * d * (int64_t)sizeof(float); }

template <typename T, int V, int NC, bool INTER, bool GRAD, bool EXACT>
cudaError_t start(const RopeArgs& a, int workers, int ctas, cudaStream_t st) {
  constexpr size_t smem = kWarps * Feed<T, V, NC, GRAD ? 2 : 1>::kWarpBytes;
  cudaError_t e = smem > 32 * 1024 ? allow_smem<rope_kernel<T, V, NC, INTER, GRAD, EXACT>>(smem) : cudaSuccess;
  if (e == cudaSuccess) {
    // (starting while the kernel before it ends saves 0.2 to 0.6 us, among other work 2)
    e = launch_early(rope_kernel<T, V, NC, INTER, GRAD, EXACT>, dim3(ctas, workers), kThreads, smem, st, a);
  }
  return e;
}
template <typename T, int V, int NC>
cudaError_t launch(const RopeArgs& a, int workers, int ctas, bool grad, bool inter, cudaStream_t st) {
  if constexpr (V >= 4) {
    if ((a.lg & (a.lg - 1)) != 0) {
      if (inter) return grad ? start<T, V, NC, true, true, true>(a, workers, ctas, st) : start<T, V, NC, true, false, true>(a, workers, ctas, st);
      return grad ? start<T, V, NC, false, true, true>(a, workers, ctas, st) : start<T, V, NC, false, false, true>(a, workers, ctas, st);
    }
  }
  if (inter) return grad ? start<T, V, NC, true, true, false>(a, workers, ctas, st) : start<T, V, NC, true, false, false>(a, workers, ctas, st);
  return grad ? start<T, V, NC, false, true, false>(a, workers, ctas, st) : start<T, V, NC, false, false, false>(a, workers, ctas, st);
}

struct Mat { const char* name; const void* p; int64_t rows, width, ld; bool output; };

int run_rope(const fgd_qk_rope_args* b, bool backward, int device, void* stream) {
  const char* who = backward ? "fgd_qk_rope_backward" : "fgd_qk_rope_forward";
  if (!b) return op_fail(FGD_ERR_INVALID_ARG, "%s: NULL arguments", who);
  const int bytes = dtype_bytes(b->dtype), d = b->head_dim, rot = b->rotary_dim;
  if (bytes == 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: unknown dtype %d", who, b->dtype);
  if (b->workers < 1 || b->workers > FGD_MAX_K || b->rows < 0 || b->rows > 0x7fffffff) return op_fail(FGD_ERR_INVALID_ARG, "%s: workers=%d, rows=%lld out of range", who, b->workers, (long long)b->rows);
  if (b->n_q_heads < 1 || b->n_q_heads > 32768 || b->n_k_heads < 0 || b->n_k_heads > 32768) return op_fail(FGD_ERR_INVALID_ARG, "%s: %d query and %d key heads", who, b->n_q_heads, b->n_k_heads);
  if (d < 1) return op_fail(FGD_ERR_INVALID_ARG, "%s: head_dim %d", who, d);
  if (d > kMaxDim) return op_fail(FGD_ERR_UNSUPPORTED, "%s: head_dim %d above %d", who, d, kMaxDim);
  if (rot < 2 || rot % 2 != 0 || rot > d) return op_fail(FGD_ERR_INVALID_ARG, "%s: rotary_dim %d is not an even number up to head_dim", who, rot);
  if (b->position_bytes != 0 && b->position_bytes != 4 && b->position_bytes != 8) return op_fail(FGD_ERR_INVALID_ARG, "%s: position_bytes %d", who, b->position_bytes);
  if (!std::isfinite((float)b->eps) || b->eps < 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: eps is negative or not finite in fp32", who);
  const int64_t T = b->workers * b->rows;
  const bool use[2] = {true, b->n_k_heads > 0};
  const bool norm[2] = {b->w_q.p != nullptr, use[1] && b->w_k.p != nullptr}, any_norm = norm[0] || norm[1];
  if (!use[1] && b->w_k.p) return op_fail(FGD_ERR_INVALID_ARG, "%s: w_k without keys", who);
  if (b->table_rows < 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: table_rows %lld", who, (long long)b->table_rows);
  const bool has_positions = b->position_bytes != 0;
  if (has_positions && !b->positions && T > 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: positions is NULL", who);
  if (!has_positions && b->table_rows < T) return op_fail(FGD_ERR_INVALID_ARG, "%s: without positions the tables need a row for each of the %lld tokens", who, (long long)T);
  const fgd_heads* in[2] = {backward ? &b->dq_out : &b->q, backward ? &b->dk_out : &b->k};
  const fgd_heads* out[2] = {backward ? &b->dq : &b->q_out, backward ? &b->dk : &b->k_out};
  const fgd_heads* x[2] = {&b->q, &b->k};
  const fgd_mat* w[2] = {&b->w_q, &b->w_k};
  const fgd_mat* dw[2] = {&b->dw_q, &b->dw_k};
  const int heads[2] = {b->n_q_heads, b->n_k_heads};
  static const char* const in_name[2][2] = {{"q", "k"}, {"dq_out", "dk_out"}};
  static const char* const out_name[2][2] = {{"q_out", "k_out"}, {"dq", "dk"}};
  static const char* const x_name[2] = {"q", "k"};
  static const char* const w_name[2] = {"w_q", "w_k"};
  static const char* const dw_name[2] = {"dw_q", "dw_k"};

  // matrices: tables, weights and their gradients, positions, workspace
  Mat mats[8];      // cos, sin, two weights, two gradients, positions, workspace
  int n_mats = 0;
  auto mat = [&](const char* name, const fgd_mat& m, int64_t rows, int64_t width, bool output) -> int {
    if (!m.p && rows > 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: %s is NULL", who, name);
    if (m.ld < width) return op_fail(FGD_ERR_INVALID_ARG, "%s: row stride of %s is below its width", who, name);
    if (reinterpret_cast<uintptr_t>(m.p) % 4 != 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: %s is not on a boundary of its elements", who, name);
    mats[n_mats++] = Mat{name, m.p, rows, width, m.ld, output};
    return FGD_OK;
  };
  if (int rc = mat("cos", b->cos, b->table_rows, rot / 2, false)) return rc;
  if (int rc = mat("sin", b->sin, b->table_rows, rot / 2, false)) return rc;
  for (int i = 0; i < 2; ++i) {
    if (!norm[i]) continue;
    if (int rc = mat(w_name[i], *w[i], b->workers, d, false)) return rc;
    if (backward)
      if (int rc = mat(dw_name[i], *dw[i], b->workers, d, true)) return rc;
  }
  if (has_positions) {
    if (reinterpret_cast<uintptr_t>(b->positions) % b->position_bytes != 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: positions is not on a boundary of its elements", who);
    mats[n_mats++] = Mat{"positions", b->positions, 1, T * b->position_bytes / 4, T * b->position_bytes / 4, false};
  }

  // heads: (tensor, span, output)
  struct Tensor { const char* name; const fgd_heads* t; Span span; bool output; };
  Tensor tensors[6];
  int n_tensors = 0;
  Launch l = {0, 0, 0};
  int vec = 16 / bytes;
  auto chunked = [&](int v) { return (rot / 2) % v == 0 && (d - rot) % (2 * v) == 0; };
  if (T > 0) {
    for (int i = 0; i < 2; ++i) {
      if (!use[i]) continue;
      const HeadsArg args[] = {{in_name[backward][i], in[i], heads[i], false}, {out_name[backward][i], out[i], heads[i], true}, {x_name[i], x[i], heads[i], false}};
      for (int j = 0; j < (backward && norm[i] ? 3 : 2); ++j) {
        if (int rc = check_heads(who, args[j], T, d, bytes)) return rc;
        tensors[n_tensors++] = Tensor{args[j].name, args[j].t, heads_span(*args[j].t, T, heads[i], d, bytes), args[j].output};
      }
    }
    for (int i = 0; i < n_tensors; ++i) {
      if (!tensors[i].output) continue;
      for (int j = 0; j < n_tensors; ++j) {
        if (j == i || !tensors[i].span.overlaps(tensors[j].span)) continue;
        // q_out may be q itself, dq may be dq_out: a lane reads a head's channels before it writes the same ones
        const bool own = j == i - 1 && tensors[j].t->p == tensors[i].t->p && tensors[j].t->token_stride == tensors[i].t->token_stride &&
                         tensors[j].t->head_stride == tensors[i].t->head_stride;
        if (!own) return op_fail(FGD_ERR_ALIAS, "%s: %s overlaps %s", who, tensors[i].name, tensors[j].name);
      }
      for (int j = 0; j < n_mats; ++j)
        if (tensors[i].span.overlaps(span_of(mats[j].p, mats[j].rows, mats[j].width, mats[j].ld, 4))) return op_fail(FGD_ERR_ALIAS, "%s: %s overlaps %s", who, tensors[i].name, mats[j].name);
    }
    // Chunks of 16 bytes; of 8 or 4 where a half of the rotated channels, or of the others, is no multiple of that (16-bit heads of 72, of 100); else
    // one by one.
    for (; vec > 1; vec = bytes == 2 ? vec / 2 : 1) {
      bool fits = chunked(vec) && (vec == 2 ? d <= 128 : vector_of(b->cos.p, b->cos.ld, 0, 4, 4) && vector_of(b->sin.p, b->sin.ld, 0, 4, 4));
      for (int i = 0; i < n_tensors && fits; ++i) fits = vector_of(tensors[i].t->p, tensors[i].t->token_stride, tensors[i].t->head_stride, bytes, vec);
      if (fits) break;
    }
    l.pairs = vec == 1 ? rot / 2 + (d - rot + 1) / 2 : d / (2 * vec);
    l.lg = 1;
    while (l.lg < 32 && l.lg < l.pairs) l.lg *= 2;
    l.vec = vec;
  }
  const bool sums = backward && any_norm;
  if (sums) {
    if (!b->workspace || reinterpret_cast<uintptr_t>(b->workspace) % 4 != 0)
      return op_fail(FGD_ERR_INVALID_ARG, "%s: the workspace is NULL or not on a 4-byte boundary", who);
    const int64_t words = b->workspace_bytes / 4;
    mats[n_mats++] = Mat{"workspace", b->workspace, 1, words, words, true};
  }
  for (int i = 0; i < n_mats; ++i) {
    if (!mats[i].output) continue;
    const Span so = span_of(mats[i].p, mats[i].rows, mats[i].width, mats[i].ld, 4);
    for (int j = 0; j < n_mats; ++j)
      if (j != i && so.overlaps(span_of(mats[j].p, mats[j].rows, mats[j].width, mats[j].ld, 4))) return op_fail(FGD_ERR_ALIAS, "%s: %s overlaps %s", who, mats[i].name, mats[j].name);
    for (int j = 0; j < n_tensors; ++j)
      if (so.overlaps(tensors[j].span)) return op_fail(FGD_ERR_ALIAS, "%s: %s overlaps %s", who, mats[i].name, tensors[j].name);
  }
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  RopeArgs a = {};
  if (sums) {
    const int64_t need = workspace_bytes(b->workers, d);
    if (b->workspace_bytes < need)
      return op_fail(FGD_ERR_INVALID_ARG, "%s: needs a workspace of %lld bytes (fgd_qk_rope_workspace)", who, (long long)need);
    a.partial = static_cast<float*>(b->workspace);
  } else if (T == 0) {
    return FGD_OK;
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  RopeSums c = {};
  c.partial = a.partial; c.d = d;
  for (int i = 0; i < 2; ++i) {
    RopeSide& s = a.side[i];
    auto at = [&](const fgd_heads& t) { return RopeHeads{static_cast<char*>(t.p), t.token_stride * bytes, t.head_stride * bytes, 0}; };
    s.x = at(sums ? *x[i] : *in[i]); s.y = at(*out[i]); s.g = at(*in[i]);
    s.w = norm[i] ? static_cast<const float*>(w[i]->p) : nullptr;
    s.w_ld = w[i]->ld;
    c.dw[i] = norm[i] ? static_cast<float*>(dw[i]->p) : nullptr;
    c.ld[i] = dw[i]->ld;
  }
  cudaError_t e = cudaSuccess;
  if (T > 0) {
    a.cos = static_cast<const float*>(b->cos.p); a.sin = static_cast<const float*>(b->sin.p); a.cos_ld = b->cos.ld; a.sin_ld = b->sin.ld;
    a.positions = has_positions ? b->positions : nullptr; a.position_bytes = b->position_bytes;
    a.rows = b->rows; a.table_rows = b->table_rows;
    a.d = d; a.rot = rot; a.pairs = l.pairs;
    // Warps share a token's heads where that evens out the rounds of the SMs' warps over the tokens (a step for a batch, and two more for each token).
    const int per_sm = ctas_of(l.vec, l.vec > 1 ? 1 : l.pairs <= 64 ? 2 : 4, sums);
    struct Plan { int lg, gt, split; int64_t tokens; double steps; };
    auto plan = [&](int lg) {
      Plan p = {lg, group_of(heads[0], heads[1], 32 / lg), 1, 0, 0};
      p.tokens = 32 / lg / p.gt;
      const int64_t warps = b->workers * ((b->rows + p.tokens - 1) / p.tokens), places = (int64_t)sm_count() * per_sm * kWarps;
      int64_t least = 0;
      for (int split = 1; split <= kWarps; split *= 2) {
        const int64_t rounds = (warps * split + places - 1) / places;
        const int64_t batches = (heads[0] / p.gt + split - 1) / split + (heads[1] / p.gt + split - 1) / split + 2;
        const double steps = batches * (warps * split > places ? (double)(warps * split) / (double)places : 1.);
        if (split == 1 || rounds * batches < least) { least = rounds * batches; p.split = split; }
        if (split == 1 || steps < p.steps) p.steps = steps;
      }
      return p;
    };
    Plan p = plan(l.lg);
    // Heads of as many lanes as they have chunk pairs, instead of a power of two, where more of them fit a warp and that saves steps.  Chunks of 8 bytes are bound
    // by instructions: 16384 tokens of 16 + 4 heads of 72, bf16, 38 and 61 us with 16 lanes, 29 and 49 with nine; rotation alone 28 and 23.  Of 16 bytes the rotation
    // alone loses (32 + 32 heads of 80: 64 us with eight lanes, 69 with five: shorter pieces of memory), and with norms a third of the steps has to go:
    // 16 + 4 heads of 80 30 and 51 us, 26 and 48; of 48 (four lanes or three) 33 us backward would become 40.  (What the estimate gets wrong: backward of
    // 3000 tokens of 16 + 4 heads of 80, 18 us and 21.)
    if (l.vec >= 4 && l.pairs <= 16 && 32 / l.pairs > 32 / l.lg) {
      const Plan exact = plan(l.pairs);
      if (exact.steps < (l.vec * bytes < 16 ? 1. : any_norm ? 0.68 : 0.) * p.steps) p = exact;
    }
    a.lg = p.lg; a.gt = p.gt; a.split = p.split;
    for (int i = 0; i < 2; ++i) {
      RopeSide& side = a.side[i];
      side.batches = heads[i] / a.gt;
      for (RopeHeads* h : {&side.x, &side.y, &side.g}) h->step = h->hs * a.gt * a.split;
    }
    c.ctas = ctas_for(per_sm, b->workers, b->rows * a.split, p.tokens);
    a.eps = (float)b->eps; a.inv_d = 1.f / (float)d; a.turn = backward ? -1.f : 1.f;
    const bool inter = b->interleaved != 0;
    auto by_vec = [&](auto zero) {
      using E = decltype(zero);
      if constexpr (sizeof(E) == 2) {
        if (l.vec == 8) return launch<E, 8, 1>(a, b->workers, c.ctas, sums, inter, st);
        if (l.vec == 2) return launch<E, 2, 1>(a, b->workers, c.ctas, sums, inter, st);
      }
      if (l.vec == 4) return launch<E, 4, 1>(a, b->workers, c.ctas, sums, inter, st);
      return l.pairs <= 64 ? launch<E, 1, 2>(a, b->workers, c.ctas, sums, inter, st) : launch<E, 1, 4>(a, b->workers, c.ctas, sums, inter, st);
    };
    switch (b->dtype) {
      case FGD_F32: e = by_vec(float{}); break;
      case FGD_BF16: e = by_vec(__nv_bfloat16{}); break;
      default: e = by_vec(__half{}); break;
    }
  }
  if (e == cudaSuccess && sums) e = launch_early(rope_sums_kernel, dim3((unsigned)((d + 31) / 32), (unsigned)b->workers, 2), 32 * kParts, 0, st, c);
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

}  // namespace

extern "C" int64_t fgd_qk_rope_workspace(int device, int workers, int head_dim) {
  if (workers < 1 || workers > FGD_MAX_K || head_dim < 1 || head_dim > kMaxDim) return FGD_ERR_INVALID_ARG;
  DeviceScope dev(device);
  return workspace_bytes(workers, head_dim);
}
extern "C" int fgd_qk_rope_forward(int device, const fgd_qk_rope_args* args, void* stream) {
  FGD_NVTX_RANGE("fgd_qk_rope_forward");
  return run_rope(args, false, device, stream);
}
extern "C" int fgd_qk_rope_backward(int device, const fgd_qk_rope_args* args, void* stream) {
  FGD_NVTX_RANGE("fgd_qk_rope_backward");
  return run_rope(args, true, device, stream);
}

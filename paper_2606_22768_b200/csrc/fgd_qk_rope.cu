// Norms of queries and keys per head with the rotation by position in the same pass, for K workers at once.
//
//   z = x r w,  r = 1 / sqrt(mean(x^2) + eps)   (without weights: z = x)
//   (a, b) a pair of the first `rotary` channels of z:  a' = a cos - b sin,  b' = b cos + a sin,   cos, sin = tables[position][pair]
//   the other channels: z
// Gradients from x and dy (dz: the transposed rotation of dy):
//   dw = sum over tokens and heads of dz x r,   dx = r (dz w - x r^2 mean(dz w x))
// Without weights the backward pass is the transposed rotation alone: the forward kernel with -sin.
//
// A lane holds 2 V channels of a head: a chunk of V consecutive ones and the chunk of their partners, so the rotation needs no other lane and the
// norm log2(lanes) shuffles.  LG lanes make a head, 32 / LG heads a warp.  Of those, gt (the largest power of two that divides the head count)
// belong to one token, so a lane's cos and sin serve all its heads; CTAs belong to one worker and to q or k, so its weights, and in the
// backward pass the sums of their gradients, stay in registers.
#include <cmath>

#include "fgd_dtype.cuh"
#include "fgd_heads.h"
#include "fgd_nvtx.h"

using namespace fgd;

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxDim = 256;

struct RopeHeads { char* p; int64_t ts, hs; };
struct RopeSide {
  RopeHeads x, y, g;           // forward: input, output; backward: input, gradient out, gradient in
  const float* w; int64_t w_ld;
  int heads, gt, ctas;         // gt: lane groups that share a token; CTAs of one worker
};
struct RopeArgs {
  RopeSide side[2];
  const float *cos, *sin; int64_t cos_ld, sin_ld;
  const void* positions; int position_bytes;
  int64_t rows, table_rows;
  int d, rot, lg, pairs;       // lanes of a head; chunk pairs of a head
  float eps, inv_d, turn;      // turn: 1, or -1 for the transposed rotation
  float* partial;              // backward: [side][worker][cta][d]
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
  int c0[NC], c1[NC], at[NC];
  bool has0[NC], has1[NC], turns[NC];
  __device__ __forceinline__ Geometry(int sub, const RopeArgs& a) {
    const int turning = a.rot / (2 * V), rest = a.pairs - turning;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int p = sub + j * a.lg;
      turns[j] = p < turning;
      at[j] = p * V;
      if (turns[j]) { c0[j] = INTER ? 2 * p * V : p * V; c1[j] = INTER ? c0[j] + V : c0[j] + a.rot / 2; }
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
template <int V, int NC, bool INTER>
__device__ __forceinline__ bool load_angles(const RopeArgs& a, const Geometry<V, NC, INTER>& geo, int64_t token, bool real, float (&cs)[NC][V], float (&sn)[NC][V]) {
  const int64_t pos = real ? position_of(a, token) : 0;
  const bool good = pos >= 0 && pos < a.table_rows;
#pragma unroll
  for (int j = 0; j < NC; ++j) {
#pragma unroll
    for (int i = 0; i < V; ++i) { cs[j][i] = 1.f; sn[j][i] = 0.f; }
    if (real && good && geo.turns[j] && geo.has0[j]) {
      load_table<V>(a.cos + pos * a.cos_ld + geo.at[j], cs[j]);
      load_table<V>(a.sin + pos * a.sin_ld + geo.at[j], sn[j]);
    }
  }
  return good;
}
// The pairs of a chunk and its partner, turned by +-angle.  Products and sums are rounded one by one: so every form of the rotation that
// computes in fp32 without contraction agrees with this one to the bit.
template <int V, bool INTER>
__device__ __forceinline__ void rotate(float (&z)[2 * V], const float (&cs)[V], const float (&sn)[V], float turn) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float& a = z[INTER ? 2 * i : i];
    float& b = z[INTER ? 2 * i + 1 : V + i];
    const float s = turn * sn[i], p = __fsub_rn(__fmul_rn(a, cs[i]), __fmul_rn(b, s)), q = __fadd_rn(__fmul_rn(b, cs[i]), __fmul_rn(a, s));
    a = p; b = q;
  }
}
// Sum over the lanes of a head; all lanes of the warp take part.
__device__ __forceinline__ float head_sum(float v, int lg) {
  for (int o = 1; o < lg; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <typename T, int V, int NC, bool INTER>
__device__ __forceinline__ void load_head(Chunk<T, V> (&r)[NC][2], const T* p, bool real, const Geometry<V, NC, INTER>& geo) {
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    r[j][0].clear(); r[j][1].clear();
    if (real && geo.has0[j]) r[j][0].load(p + geo.c0[j]);
    if (real && geo.has1[j]) r[j][1].load(p + geo.c1[j]);
  }
}
template <typename T, int V, int NC, bool INTER>
__device__ __forceinline__ void store_head(const float (&z)[NC][2 * V], T* p, bool real, const Geometry<V, NC, INTER>& geo) {
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    Chunk<T, V> c;
    c.set(z[j]);
    if (real && geo.has0[j]) c.store(p + geo.c0[j]);
    c.set(z[j] + V);
    if (real && geo.has1[j]) c.store(p + geo.c1[j]);
  }
}
template <int V, int NC, bool INTER>
__device__ __forceinline__ void load_weights(const RopeSide& s, int worker, const Geometry<V, NC, INTER>& geo, float (&w)[NC][2 * V]) {
#pragma unroll
  for (int j = 0; j < NC; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      w[j][i] = geo.has0[j] ? __ldg(s.w + worker * s.w_ld + geo.c0[j] + i) : 0.f;
      w[j][V + i] = geo.has1[j] ? __ldg(s.w + worker * s.w_ld + geo.c1[j] + i) : 0.f;
    }
}

// UH: heads of a lane in flight at once.
template <typename T, int V, int NC, int UH, bool INTER>
__global__ void __launch_bounds__(kThreads) rope_forward_kernel(const RopeArgs a) {
  const bool is_k = (int)blockIdx.x >= a.side[0].ctas;
  const RopeSide& s = a.side[is_k];
  const int cta = blockIdx.x - (is_k ? a.side[0].ctas : 0), worker = blockIdx.y, lane = threadIdx.x & 31, group = lane / a.lg;
  const int tokens = 32 / a.lg / s.gt;      // of a warp at once
  const Geometry<V, NC, INTER> geo(lane % a.lg, a);
  const bool norm = s.w != nullptr;
  float w[NC][2 * V];
  if (norm) load_weights(s, worker, geo, w);
  const T* x = reinterpret_cast<const T*>(s.x.p);
  T* y = reinterpret_cast<T*>(s.y.p);
  for (int64_t t0 = (int64_t)(cta * kWarps + threadIdx.x / 32) * tokens; t0 < a.rows; t0 += (int64_t)s.ctas * kWarps * tokens) {
    const int64_t local = t0 + group / s.gt, token = worker * a.rows + local;
    const bool real = local < a.rows;
    float cs[NC][V], sn[NC][V];
    const bool good = load_angles(a, geo, token, real, cs, sn);
    for (int h0 = group % s.gt; h0 < s.heads; h0 += s.gt * UH) {      // gt divides the heads: the groups leave the loop together
      Chunk<T, V> raw[UH][NC][2];
#pragma unroll
      for (int u = 0; u < UH; ++u) load_head<T, V, NC, INTER>(raw[u], x + token * s.x.ts + (h0 + u * s.gt) * s.x.hs, real && h0 + u * s.gt < s.heads, geo);
#pragma unroll
      for (int u = 0; u < UH; ++u) {
        if (h0 + u * s.gt >= s.heads) break;
        float z[NC][2 * V];
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          raw[u][j][0].get(z[j]);
          raw[u][j][1].get(z[j] + V);
        }
        if (norm) {
#pragma unroll
          for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) ss = fmaf(z[j][i], z[j][i], ss);
          const float r = rsqrtf(fmaf(head_sum(ss, a.lg), a.inv_d, a.eps));
#pragma unroll
          for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) z[j][i] *= r * w[j][i];
        }
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          if (geo.turns[j]) rotate<V, INTER>(z[j], cs[j], sn[j], a.turn);
          if (!good) {
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) z[j][i] = __int_as_float(0x7fffffff);
          }
        }
        store_head<T, V, NC, INTER>(z, y + token * s.y.ts + (h0 + u * s.gt) * s.y.hs, real, geo);
      }
    }
  }
}

// With weights; UH as above.
template <typename T, int V, int NC, int UH, bool INTER>
__global__ void __launch_bounds__(kThreads) rope_backward_kernel(const RopeArgs a) {
  __shared__ float sums[kWarps][kMaxDim];
  const bool is_k = (int)blockIdx.x >= a.side[0].ctas;
  const RopeSide& s = a.side[is_k];
  const int cta = blockIdx.x - (is_k ? a.side[0].ctas : 0), worker = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x / 32, group = lane / a.lg;
  const int tokens = 32 / a.lg / s.gt;
  const Geometry<V, NC, INTER> geo(lane % a.lg, a);
  float w[NC][2 * V], dw[NC][2 * V];
  const bool norm = s.w != nullptr;      // (of one side only: the other is the rotation alone)
#pragma unroll
  for (int j = 0; j < NC; ++j)
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) w[j][i] = dw[j][i] = 0.f;
  if (norm) load_weights(s, worker, geo, w);
  let_next_start();
  const T* x = reinterpret_cast<const T*>(s.x.p);
  const T* g = reinterpret_cast<const T*>(s.g.p);
  T* y = reinterpret_cast<T*>(s.y.p);
  for (int64_t t0 = (int64_t)(cta * kWarps + warp) * tokens; t0 < a.rows; t0 += (int64_t)s.ctas * kWarps * tokens) {
    const int64_t local = t0 + group / s.gt, token = worker * a.rows + local;
    const bool real = local < a.rows;
    float cs[NC][V], sn[NC][V];
    const bool good = load_angles(a, geo, token, real, cs, sn);
    for (int h0 = group % s.gt; h0 < s.heads; h0 += s.gt * UH) {
      Chunk<T, V> rx[UH][NC][2], rg[UH][NC][2];
#pragma unroll
      for (int u = 0; u < UH; ++u) {
        const int h = h0 + u * s.gt;
        load_head<T, V, NC, INTER>(rg[u], g + token * s.g.ts + h * s.g.hs, real && h < s.heads, geo);
        load_head<T, V, NC, INTER>(rx[u], x + token * s.x.ts + h * s.x.hs, real && norm && h < s.heads, geo);
      }
#pragma unroll
      for (int u = 0; u < UH; ++u) {
        const int h = h0 + u * s.gt;
        if (h >= s.heads) break;
        float z[NC][2 * V], v[NC][2 * V];
        float ss = 0.f, sg = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          rg[u][j][0].get(z[j]); rg[u][j][1].get(z[j] + V);
          rx[u][j][0].get(v[j]); rx[u][j][1].get(v[j] + V);
          if (geo.turns[j]) rotate<V, INTER>(z[j], cs[j], sn[j], a.turn);
          if (!good) {
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) z[j][i] = __int_as_float(0x7fffffff);
          }
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) {
            ss = fmaf(v[j][i], v[j][i], ss);
            sg = fmaf(z[j][i] * w[j][i], v[j][i], sg);
          }
        }
        if (norm) {
          ss = head_sum(ss, a.lg);
          sg = head_sum(sg, a.lg);
          const float r = rsqrtf(fmaf(ss, a.inv_d, a.eps)), k = r * r * (r * sg * a.inv_d);
#pragma unroll
          for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) {
              const float t = z[j][i] * r;
              dw[j][i] = fmaf(t, v[j][i], dw[j][i]);
              z[j][i] = fmaf(t, w[j][i], -k * v[j][i]);
            }
        }
        store_head<T, V, NC, INTER>(z, y + token * s.y.ts + h * s.y.hs, real, geo);
      }
    }
  }
  if (!norm) return;      // (the whole CTA)
#pragma unroll
  for (int j = 0; j < NC; ++j)
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) {
      float t = dw[j][i];
      for (int o = a.lg; o < 32; o *= 2) t += __shfl_xor_sync(0xffffffffu, t, o);
      const bool has = i < V ? geo.has0[j] : geo.has1[j];
      if (group == 0 && has) sums[warp][i < V ? geo.c0[j] + i : geo.c1[j] + i - V] = t;
    }
  __syncthreads();
  float* out = a.partial + ((is_k ? (int64_t)gridDim.y * a.side[0].ctas : 0) + (int64_t)worker * s.ctas + cta) * a.d;
  for (int c = threadIdx.x; c < a.d; c += kThreads) {
    float t = sums[0][c];
#pragma unroll
    for (int i = 1; i < kWarps; ++i) t += sums[i][c];
    out[c] = t;
  }
}

// dw of a worker and side: its CTAs' sums, eight at a time added in order, 32 channels a CTA.
struct RopeSums { const float* partial; float* dw[2]; int64_t ld[2]; int ctas[2], d; };
__global__ void __launch_bounds__(256) rope_sums_kernel(const RopeSums a) {
  wait_for_previous();
  __shared__ float buf[8][32];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, worker = blockIdx.y, side = blockIdx.z;
  if (!a.dw[side]) return;
  const float* p = a.partial + ((side ? (int64_t)gridDim.y * a.ctas[0] : 0) + (int64_t)worker * a.ctas[side]) * a.d;
  float t = 0.f;
  if (c < a.d)
    for (int i = part; i < a.ctas[side]; i += 8) t += p[(int64_t)i * a.d + c];
  buf[part][lane] = t;
  __syncthreads();
  if (part != 0 || c >= a.d) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) t += buf[i][lane];
  a.dw[side][worker * a.ld[side] + c] = t;
}

// ---- host
constexpr int kCtasPerSm = 2;      // of the persistent grid

int64_t tokens_per_warp(int lg, int gt) { return 32 / lg / gt; }
int group_of(int heads, int groups) {      // the largest power of two that divides the heads, at most `groups`
  int g = 1;
  while (g < groups && heads % (2 * g) == 0) g *= 2;
  return g;
}
// CTAs of one worker for a side with `heads` of all `total` heads: its share of the SMs' places, and no more than there is work for.
int ctas_for(int64_t workers, int64_t rows, int heads, int total, int64_t warp_tokens) {
  if (heads == 0) return 0;
  int64_t c = (int64_t)sm_count() * kCtasPerSm * heads / ((int64_t)total * workers);
  const int64_t most = (rows + kWarps * warp_tokens - 1) / (kWarps * warp_tokens);
  if (c > most) c = most;
  return (int)(c < 1 ? 1 : c);
}

bool vector_of(const void* p, int64_t s0, int64_t s1, int bytes, int vec) {
  return reinterpret_cast<uintptr_t>(p) % (uintptr_t)(vec * bytes) == 0 && s0 % vec == 0 && s1 % vec == 0;
}

struct Launch { int vec, lg, pairs; };

int64_t workspace_bytes(int workers, int d) { return ((int64_t)sm_count() * kCtasPerSm + 2 * (int64_t)workers) * d * (int64_t)sizeof(float); }

template <typename T, int V, int NC>
cudaError_t launch(const RopeArgs& a, int workers, bool sums, bool inter, cudaStream_t st) {
  const dim3 grid(a.side[0].ctas + a.side[1].ctas, workers);
  constexpr int UF = NC > 1 ? 1 : 4, UB = NC > 1 ? 1 : 2;
  if (sums) {
    if (inter) rope_backward_kernel<T, V, NC, UB, true><<<grid, kThreads, 0, st>>>(a);
    else rope_backward_kernel<T, V, NC, UB, false><<<grid, kThreads, 0, st>>>(a);
  } else {
    if (inter) rope_forward_kernel<T, V, NC, UF, true><<<grid, kThreads, 0, st>>>(a);
    else rope_forward_kernel<T, V, NC, UF, false><<<grid, kThreads, 0, st>>>(a);
  }
  return cudaGetLastError();
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
  if (!std::isfinite(b->eps) || b->eps < 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: eps is negative or not finite", who);
  const int64_t T = b->workers * b->rows;
  const bool use[2] = {true, b->n_k_heads > 0};
  const bool norm[2] = {b->w_q.p != nullptr, use[1] && b->w_k.p != nullptr}, any_norm = norm[0] || norm[1];
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
    // Chunks of 16 bytes; of 8 where a half of the rotated channels is no multiple of that (16-bit heads of 72); else one by one.
    for (; vec > 1; vec = vec == 8 ? 4 : 1) {
      bool fits = chunked(vec) && vector_of(b->cos.p, b->cos.ld, 0, 4, 4) && vector_of(b->sin.p, b->sin.ld, 0, 4, 4);
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
    auto at = [](const fgd_heads& t) { return RopeHeads{static_cast<char*>(t.p), t.token_stride, t.head_stride}; };
    s.x = at(sums ? *x[i] : *in[i]); s.y = at(*out[i]); s.g = at(*in[i]);
    s.w = norm[i] ? static_cast<const float*>(w[i]->p) : nullptr;
    s.w_ld = w[i]->ld;
    s.heads = heads[i];
    if (T > 0) {
      s.gt = heads[i] ? group_of(heads[i], 32 / l.lg) : 1;
      s.ctas = ctas_for(b->workers, b->rows, heads[i], heads[0] + heads[1], tokens_per_warp(l.lg, s.gt));
    }
    c.dw[i] = norm[i] ? static_cast<float*>(dw[i]->p) : nullptr;
    c.ld[i] = dw[i]->ld;
    c.ctas[i] = s.ctas;
  }
  cudaError_t e = cudaSuccess;
  if (T > 0) {
    a.cos = static_cast<const float*>(b->cos.p); a.sin = static_cast<const float*>(b->sin.p); a.cos_ld = b->cos.ld; a.sin_ld = b->sin.ld;
    a.positions = has_positions ? b->positions : nullptr; a.position_bytes = b->position_bytes;
    a.rows = b->rows; a.table_rows = b->table_rows;
    a.d = d; a.rot = rot; a.lg = l.lg; a.pairs = l.pairs;
    a.eps = (float)b->eps; a.inv_d = 1.f / (float)d; a.turn = backward ? -1.f : 1.f;
    const bool inter = b->interleaved != 0;
    auto by_vec = [&](auto zero) {
      using E = decltype(zero);
      if constexpr (sizeof(E) == 2)
        if (l.vec == 8) return launch<E, 8, 1>(a, b->workers, sums, inter, st);
      if (l.vec == 4) return launch<E, 4, 1>(a, b->workers, sums, inter, st);
      return launch<E, 1, 4>(a, b->workers, sums, inter, st);
    };
    switch (b->dtype) {
      case FGD_F32: e = by_vec(float{}); break;
      case FGD_BF16: e = by_vec(__nv_bfloat16{}); break;
      default: e = by_vec(__half{}); break;
    }
  }
  if (e == cudaSuccess && sums) e = launch_early(rope_sums_kernel, dim3((unsigned)((d + 31) / 32), (unsigned)b->workers, 2), 256, 0, st, c);
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

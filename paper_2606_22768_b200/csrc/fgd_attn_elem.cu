// Causal attention over packed sequences on the CUDA cores: the kernels for what the tensor-core kernels do not
// take (fp32, widths that are not a multiple of 8 or exceed 128, bases and strides off the 16-byte grid).
//
//     S_ij = scale q_i . k_j  (j <= i, same sequence),  P = softmax(S),  O = P V,  lse_i = log sum_j exp(S_ij)
//     delta_i = dO_i . O_i,  dP = dO V^T,  dS = scale P o (dP - delta)
//     dQ = dS K,  dK = sum over the heads that share k of dS^T Q,  dV = the same of P^T dO
//
// A warp owns four rows (queries; keys in the key / value gradient); the other side comes in tiles of 32
// rows through shared memory, one row per lane for the scores, one column per lane and 32-column step for the
// products.  The softmax runs over the key tiles with a running maximum and sum; the gradient recomputes P from lse.
// Only unmasked pairs enter a product, so what stands in masked places never reaches a result.
// Bound by the shared-memory loads that feed the fp32 FMAs: a score's dot product takes two for one, the products with P and dS one for one,
// so the FMA units run at about a tenth of their rate: 16384 tokens, 16 heads of 128 over 4, forward 155 ms, where the tensor cores take
// 0.97; 4 x 1024 tokens of the same in fp32 forward 2.9 ms, forward + backward 12.9.  delta has kernels of its own for 16-byte rows
// (8 elements a lane, several rows to a warp; 14.6 us for 8192 tokens of 16 x 128, 4.6 TB/s).
#include "fgd_attn.h"
#include "fgd_dtype.cuh"

using namespace fgd;

namespace {

constexpr int kWarps = 4, kRows = 4;                    // warps per CTA, rows per warp
constexpr int kCtaRows = kWarps * kRows;
constexpr int kSub = kAttnRows / kCtaRows;              // CTAs per tile
constexpr int kCols = kAttnElemMaxDim / 32;             // columns per lane

template <typename T>
__device__ __forceinline__ const T* row_of(const AttnHeads& t, int64_t token, int head) {
  return reinterpret_cast<const T*>(t.p) + token * t.token + head * t.head;
}
template <typename T>
__device__ __forceinline__ T* row_out(const AttnHeads& t, int64_t token, int head) {
  return reinterpret_cast<T*>(t.p) + token * t.token + head * t.head;
}
// 32 rows [first, first + 32) of a head into shared memory as fp32, rows d + 1 apart; rows at or beyond `len` are zero.
template <typename T>
__device__ __forceinline__ void stage(float* dst, const AttnHeads& t, int64_t start, int head, int first, int len, int d) {
  for (int r = threadIdx.x >> 5; r < 32; r += kWarps) {
    const bool real = first + r < len;
    const T* src = row_of<T>(t, start + (real ? first + r : 0), head);
    for (int c = threadIdx.x & 31; c < d; c += 32) dst[r * (d + 1) + c] = real ? to_f32<T>(src[c]) : 0.f;
  }
}
__device__ __forceinline__ float dot(const float* a, const float* b, int d) {
  float s = 0.f;
  for (int c = 0; c < d; ++c) s = fmaf(a[c], b[c], s);
  return s;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}
// acc[k] += sum over n rows of w (lane r's value) * m[r][lane + 32 k], rows from `first`
__device__ __forceinline__ void accumulate(float (&acc)[kCols], float w, const float* m, int d, int first, int n, int lane) {
  for (int r = first; r < n; ++r) {
    const float p = __shfl_sync(0xffffffffu, w, r);
#pragma unroll
    for (int k = 0; k < kCols; ++k)
      if (lane + 32 * k < d) acc[k] = fmaf(p, m[r * (d + 1) + lane + 32 * k], acc[k]);
  }
}

template <typename T>
__global__ void __launch_bounds__(kWarps * 32) attn_forward_elem_kernel(const AttnArgs a) {
  extern __shared__ float smem[];
  const int d = a.d, ld = d + 1, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float *kt = smem, *vt = kt + 32 * ld, *qs = vt + 32 * ld;
  const AttnTile t = a.tiles[blockIdx.x / kSub];
  const int row0 = t.row + (blockIdx.x % kSub) * kCtaRows, head = blockIdx.y, kvh = head / (a.hq / a.hk);
  if (row0 >= t.len) return;                              // (uniform for the CTA)
  const int rows = min(kCtaRows, t.len - row0);
  for (int r = warp; r < kCtaRows; r += kWarps)
    for (int c = lane; c < d; c += 32) qs[r * ld + c] = r < rows ? to_f32<T>(row_of<T>(a.q, t.start + row0 + r, head)[c]) : 0.f;
  float m[kRows], l[kRows], o[kRows][kCols];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int k = 0; k < kCols; ++k) o[r][k] = 0.f;
  }
  for (int j0 = 0; j0 < row0 + rows; j0 += 32) {
    __syncthreads();
    stage<T>(kt, a.k, t.start, kvh, j0, t.len, d);
    stage<T>(vt, a.v, t.start, kvh, j0, t.len, d);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int i = row0 + warp * kRows + r;
      const int n = min(32, i + 1 - j0);                  // keys of this tile that the row sees
      if (i >= t.len || n <= 0) continue;
      float s = -INFINITY;
      if (lane < n) s = a.scale * dot(qs + (warp * kRows + r) * ld, kt + lane * ld, d);
      const float mn = fmaxf(m[r], warp_max(s));
      const float shift = mn == -INFINITY ? 0.f : mn;
      const float p = lane < n ? expf(s - shift) : 0.f, f = expf(m[r] - shift);
      m[r] = mn;
      l[r] = fmaf(l[r], f, warp_sum(p));
#pragma unroll
      for (int k = 0; k < kCols; ++k) o[r][k] *= f;
      accumulate(o[r], p, vt, d, 0, n, lane);
    }
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int i = row0 + warp * kRows + r;
    if (i >= t.len) continue;
    T* out = row_out<T>(a.o, t.start + i, head);
#pragma unroll
    for (int k = 0; k < kCols; ++k)
      if (lane + 32 * k < d) out[lane + 32 * k] = from_f32<T>(o[r][k] / l[r]);
    if (lane == 0) a.lse[(int64_t)head * a.tokens + t.start + i] = m[r] + logf(l[r]);
  }
}

template <typename T>
__global__ void __launch_bounds__(256) attn_delta_kernel(const AttnArgs a) {
  const int64_t pair = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (pair >= a.tokens * a.hq) return;
  const int64_t token = pair / a.hq;
  const int head = (int)(pair - token * a.hq), lane = threadIdx.x & 31;
  const T *o = row_of<T>(a.o, token, head), *g = row_of<T>(a.dout, token, head);
  float s = 0.f;
  for (int c = lane; c < a.d; c += 32) s = fmaf(to_f32<T>(o[c]), to_f32<T>(g[c]), s);
  s = warp_sum(s);
  if (lane == 0) a.delta[(int64_t)head * a.tokens + token] = s;
}

// The same for 16-bit values in 16-byte vectors: L lanes take a row, a warp 32 tokens of one head (so that its 32 results are one
// store), eight rows' loads per lane on their way at a time.  -> delta of token0 + lane, and, where TOP asks for it, the largest finite
// magnitudes of dout that this lane has met, of a word's low and high halves; tokens at or beyond `end` count as zero.
__device__ __forceinline__ __half2 top_of(__half2 top, uint32_t w) {
  const __half2 x = __habs2(*reinterpret_cast<const __half2*>(&w));
  return __hmax2(top, __hfma2(x, __float2half2_rn(0.f), x));      // x 0 + x: NaN where x is not finite, and the maximum passes a NaN over
}
__device__ __forceinline__ __half2 top_of(__half2 top, uint4 w) { return top_of(top_of(top_of(top_of(top, w.x), w.y), w.z), w.w); }
// of a warp, as bits
__device__ __forceinline__ uint16_t warp_top(__half2 top) {
  return (uint16_t)__reduce_max_sync(0xffffffffu, (uint32_t)__half_as_ushort(__hmax(__low2half(top), __high2half(top))));
}
template <typename T, int L, bool TOP>
__device__ __forceinline__ float delta_of_32(const AttnArgs& a, int head, int64_t token0, int64_t end, __half2& top) {
  constexpr int RPS = 32 / L, AT_ONCE = 8;                 // rows per step of the warp, steps at a time
  const int lane = threadIdx.x & 31, sub = lane / L, c = (lane % L) * 8;
  float mine = 0.f;
#pragma unroll
  for (int s0 = 0; s0 < L; s0 += AT_ONCE) {
    ActPack<T, 8> o[AT_ONCE], g[AT_ONCE];
#pragma unroll
    for (int s = 0; s < AT_ONCE; ++s) {
      const int64_t token = token0 + (s0 + s) * RPS + sub;
      if (token < end && c < a.d) {
        o[s] = load_stream<T, 8>(row_of<T>(a.o, token, head) + c);
        g[s] = load_stream<T, 8>(row_of<T>(a.dout, token, head) + c);
      } else {
        zero(o[s]);
        zero(g[s]);
      }
    }
#pragma unroll
    for (int s = 0; s < AT_ONCE; ++s) {
      const Vals<8> x = unpack<T, 8>(o[s]), y = unpack<T, 8>(g[s]);
      float2 v = both(0.f);
#pragma unroll
      for (int k = 0; k < 4; ++k) v = fma2(x.pair(k), y.pair(k), v);
      float sum = v.x + v.y;
#pragma unroll
      for (int off = L / 2; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      sum = __shfl_sync(0xffffffffu, sum, (lane % RPS) * L);
      if (lane / RPS == s0 + s) mine = sum;
      if constexpr (TOP) top = top_of(top, g[s].w);
    }
  }
  return mine;
}
template <int L>
__global__ void __launch_bounds__(256) attn_delta_bf16_kernel(const AttnArgs a) {
  let_next_start();
  const int lane = threadIdx.x & 31;
  const int64_t warp = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), head = warp % a.hq, token0 = warp / a.hq * 32;
  if (token0 >= a.tokens) return;
  __half2 unused{};
  const float delta = delta_of_32<__nv_bfloat16, L, false>(a, (int)head, token0, a.tokens, unused);
  if (token0 + lane < a.tokens) a.delta[head * a.tokens + token0 + lane] = delta;
}

// fp16: dS = P (dP - delta) goes back to the tensor cores in a type whose smallest normal value is 2^-14 and whose largest is 65504, while
// the gradients it comes from may have any size.  So it is held times a power of two, which the output's factor takes back.  The terms of a
// row are bounded by |dP|, |delta| <= width x (the largest |dout| of the row) x (the largest |v| of the keys that it sees): this kernel leaves
// both of every 32 rows (the largest finite ones: what is not finite makes its own terms so, and has no say in the others), and the gradient kernels choose from them (attn_lift), out of one sequence alone, so that no other
// sequence's values change a rounding.  Where: the two are fp16 values and fit one word, which takes the place of the first row's delta; that
// delta stands in the first word of the same row of dq, where its reader alone writes, later (a scratch of the call's own would have to be
// asked for; a kernel of its own for the largest |v| took 4 us longer on 288 tokens).  A warp: 32 rows of one tile and one head, of dout or of v.
template <int L>
__global__ void __launch_bounds__(256) attn_delta_f16_kernel(const AttnArgs a) {
  let_next_start();
  const int64_t warp = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int heads = a.hq + a.hk;
  const int64_t quarter = warp / heads;
  if (quarter >= 4 * (int64_t)a.n_tiles) return;
  const AttnTile t = a.tiles[quarter >> 2];
  const int lane = threadIdx.x & 31, head = (int)(warp - quarter * heads), row = t.row + 32 * (int)(quarter & 3);
  if (row >= t.len) return;
  const int64_t token0 = (int64_t)t.start + row, end = (int64_t)t.start + t.len;
  __half2 top = __float2half2_rn(0.f);
  if (head < a.hq) {
    const float delta = delta_of_32<__half, L, true>(a, head, token0, end, top);
    float* at = a.delta + head * a.tokens + token0;
    const uint16_t most = warp_top(top);
    if (lane == 0) {
      reinterpret_cast<uint16_t*>(at)[1] = most;
      *reinterpret_cast<float*>(row_out<__half>(a.dq, token0, head)) = delta;
    } else if (token0 + lane < end) {
      at[lane] = delta;
    }
  } else {
    constexpr int RPS = 32 / L, AT_ONCE = 8;
    const int kvh = head - a.hq, c = (lane % L) * 8;
#pragma unroll
    for (int s0 = 0; s0 < L; s0 += AT_ONCE) {
      ActPack<__half, 8> v[AT_ONCE];
#pragma unroll
      for (int s = 0; s < AT_ONCE; ++s) {
        const int64_t token = token0 + (s0 + s) * RPS + lane / L;
        if (token < end && c < a.d) v[s] = load_stream<__half, 8>(row_of<__half>(a.v, token, kvh) + c);
        else zero(v[s]);
      }
#pragma unroll
      for (int s = 0; s < AT_ONCE; ++s) top = top_of(top, v[s].w);
    }
    const uint16_t most = warp_top(top);
    if (lane == 0) reinterpret_cast<uint16_t*>(a.delta + (int64_t)kvh * (a.hq / a.hk) * a.tokens + token0)[0] = most;
  }
}

template <typename T>
__global__ void __launch_bounds__(kWarps * 32) attn_dq_elem_kernel(const AttnArgs a) {
  extern __shared__ float smem[];
  const int d = a.d, ld = d + 1, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float *kt = smem, *vt = kt + 32 * ld, *qs = vt + 32 * ld, *gs = qs + kCtaRows * ld;
  const AttnTile t = a.tiles[blockIdx.x / kSub];
  const int row0 = t.row + (blockIdx.x % kSub) * kCtaRows, head = blockIdx.y, kvh = head / (a.hq / a.hk);
  if (row0 >= t.len) return;
  const int rows = min(kCtaRows, t.len - row0);
  for (int r = warp; r < kCtaRows; r += kWarps)
    for (int c = lane; c < d; c += 32) {
      qs[r * ld + c] = r < rows ? to_f32<T>(row_of<T>(a.q, t.start + row0 + r, head)[c]) : 0.f;
      gs[r * ld + c] = r < rows ? to_f32<T>(row_of<T>(a.dout, t.start + row0 + r, head)[c]) : 0.f;
    }
  float acc[kRows][kCols];
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int k = 0; k < kCols; ++k) acc[r][k] = 0.f;
  for (int j0 = 0; j0 < row0 + rows; j0 += 32) {
    __syncthreads();
    stage<T>(kt, a.k, t.start, kvh, j0, t.len, d);
    stage<T>(vt, a.v, t.start, kvh, j0, t.len, d);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int lr = warp * kRows + r, i = row0 + lr, n = min(32, i + 1 - j0);
      if (i >= t.len || n <= 0) continue;
      const int64_t at = (int64_t)head * a.tokens + t.start + i;
      float ds = 0.f;
      if (lane < n) {
        const float p = expf(a.scale * dot(qs + lr * ld, kt + lane * ld, d) - a.lse[at]);
        ds = a.scale * p * (dot(gs + lr * ld, vt + lane * ld, d) - a.delta[at]);
      }
      accumulate(acc[r], ds, kt, d, 0, n, lane);
    }
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int i = row0 + warp * kRows + r;
    if (i >= t.len) continue;
    T* out = row_out<T>(a.dq, t.start + i, head);
#pragma unroll
    for (int k = 0; k < kCols; ++k)
      if (lane + 32 * k < d) out[lane + 32 * k] = from_f32<T>(acc[r][k]);
  }
}

template <typename T>
__global__ void __launch_bounds__(kWarps * 32) attn_dkv_elem_kernel(const AttnArgs a) {
  extern __shared__ float smem[];
  const int d = a.d, ld = d + 1, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = a.hq / a.hk;
  float *qt = smem, *gt = qt + 32 * ld, *ks = gt + 32 * ld, *vs = ks + kCtaRows * ld;
  const AttnTile t = a.tiles[blockIdx.x / kSub];
  const int row0 = t.row + (blockIdx.x % kSub) * kCtaRows, kvh = blockIdx.y;
  if (row0 >= t.len) return;
  const int rows = min(kCtaRows, t.len - row0);
  for (int r = warp; r < kCtaRows; r += kWarps)
    for (int c = lane; c < d; c += 32) {
      ks[r * ld + c] = r < rows ? to_f32<T>(row_of<T>(a.k, t.start + row0 + r, kvh)[c]) : 0.f;
      vs[r * ld + c] = r < rows ? to_f32<T>(row_of<T>(a.v, t.start + row0 + r, kvh)[c]) : 0.f;
    }
  float dk[kRows][kCols], dv[kRows][kCols];
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int k = 0; k < kCols; ++k) dk[r][k] = dv[r][k] = 0.f;
  for (int head = kvh * group; head < (kvh + 1) * group; ++head)
    for (int i0 = row0 / 32 * 32; i0 < t.len; i0 += 32) {
      __syncthreads();
      stage<T>(qt, a.q, t.start, head, i0, t.len, d);
      stage<T>(gt, a.dout, t.start, head, i0, t.len, d);
      __syncthreads();
      const int n = min(32, t.len - i0);
      const int64_t at = (int64_t)head * a.tokens + t.start + i0 + min(lane, n - 1);
      const float lse = a.lse[at], delta = a.delta[at];
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const int lr = warp * kRows + r, j = row0 + lr, first = max(0, j - i0);   // queries before the key do not see it
        if (j >= t.len || first >= n) continue;
        float p = 0.f, ds = 0.f;
        if (lane >= first && lane < n) {
          p = expf(a.scale * dot(ks + lr * ld, qt + lane * ld, d) - lse);
          ds = a.scale * p * (dot(vs + lr * ld, gt + lane * ld, d) - delta);
        }
        accumulate(dv[r], p, gt, d, first, n, lane);
        accumulate(dk[r], ds, qt, d, first, n, lane);
      }
    }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int j = row0 + warp * kRows + r;
    if (j >= t.len) continue;
    T *ok = row_out<T>(a.dk, t.start + j, kvh), *ov = row_out<T>(a.dv, t.start + j, kvh);
#pragma unroll
    for (int k = 0; k < kCols; ++k)
      if (lane + 32 * k < d) {
        ok[lane + 32 * k] = from_f32<T>(dk[r][k]);
        ov[lane + 32 * k] = from_f32<T>(dv[r][k]);
      }
  }
}

template <typename K>
int launch(K kern, const char* who, AttnArgs a, const AttnTile* tiles, int n_tiles, int heads, int own, cudaStream_t st) {
  const size_t smem = sizeof(float) * (size_t)(a.d + 1) * (64 + own * kCtaRows);
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess) {
    a.tiles = tiles;
    a.n_tiles = n_tiles;
    kern<<<dim3((unsigned)n_tiles * kSub, (unsigned)heads), kWarps * 32, smem, st>>>(a);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

}  // namespace

namespace fgd {

int attn_forward_elem(const fgd_attn_plan* plan, int dtype, const AttnArgs& a, cudaStream_t st) {
  const char* who = "fgd_attn_forward";
  switch (dtype) {
    case FGD_F32: return launch(attn_forward_elem_kernel<float>, who, a, plan->q_tiles, plan->n_q, a.hq, 1, st);
    case FGD_BF16: return launch(attn_forward_elem_kernel<__nv_bfloat16>, who, a, plan->q_tiles, plan->n_q, a.hq, 1, st);
    default: return launch(attn_forward_elem_kernel<__half>, who, a, plan->q_tiles, plan->n_q, a.hq, 1, st);
  }
}

int attn_delta(const fgd_attn_plan* plan, int dtype, bool vectors, AttnArgs a, cudaStream_t st) {
  const bool quarters = vectors && dtype == FGD_F16;
  a.tiles = plan->q_tiles;
  a.n_tiles = plan->n_q;
  const int64_t warps = quarters ? 4 * (int64_t)a.n_tiles * (a.hq + a.hk) : (vectors ? (a.tokens + 31) / 32 : a.tokens) * a.hq, blocks = (warps + 7) / 8;
  if (blocks > 0x7fffffff) return op_fail(FGD_ERR_INVALID_ARG, "fgd_attn_backward: too many rows");
  if (quarters && a.d <= 64) attn_delta_f16_kernel<8><<<(unsigned)blocks, 256, 0, st>>>(a);
  else if (quarters) attn_delta_f16_kernel<16><<<(unsigned)blocks, 256, 0, st>>>(a);
  else if (vectors && a.d <= 64) attn_delta_bf16_kernel<8><<<(unsigned)blocks, 256, 0, st>>>(a);
  else if (vectors) attn_delta_bf16_kernel<16><<<(unsigned)blocks, 256, 0, st>>>(a);
  else if (dtype == FGD_F32) attn_delta_kernel<float><<<(unsigned)blocks, 256, 0, st>>>(a);
  else if (dtype == FGD_BF16) attn_delta_kernel<__nv_bfloat16><<<(unsigned)blocks, 256, 0, st>>>(a);
  else attn_delta_kernel<__half><<<(unsigned)blocks, 256, 0, st>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "fgd_attn_backward: launch failed: %s", cudaGetErrorString(e));
}

int attn_backward_elem(const fgd_attn_plan* plan, int dtype, const AttnArgs& a, cudaStream_t st) {
  const char* who = "fgd_attn_backward";
  int rc;
  switch (dtype) {
    case FGD_F32:
      rc = launch(attn_dq_elem_kernel<float>, who, a, plan->q_tiles, plan->n_q, a.hq, 2, st);
      return rc ? rc : launch(attn_dkv_elem_kernel<float>, who, a, plan->kv_tiles, plan->n_kv, a.hk, 2, st);
    case FGD_BF16:
      rc = launch(attn_dq_elem_kernel<__nv_bfloat16>, who, a, plan->q_tiles, plan->n_q, a.hq, 2, st);
      return rc ? rc : launch(attn_dkv_elem_kernel<__nv_bfloat16>, who, a, plan->kv_tiles, plan->n_kv, a.hk, 2, st);
    default:
      rc = launch(attn_dq_elem_kernel<__half>, who, a, plan->q_tiles, plan->n_q, a.hq, 2, st);
      return rc ? rc : launch(attn_dkv_elem_kernel<__half>, who, a, plan->kv_tiles, plan->n_kv, a.hk, 2, st);
  }
}

}  // namespace fgd

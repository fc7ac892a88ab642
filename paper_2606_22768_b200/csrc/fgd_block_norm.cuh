// Norms before and after a block, fused with the block's gate and residual scale; forward and backward.
//
// Per row (token), with s the residual scale and g the gate (none, one per channel, or one per element):
//     u = y r_y w_post,  r_y = 1 / sqrt(mean y^2 + eps)       the norm after the block   (optional: u = y)
//     x' = x + s g o u                                        gate, scale, residual add  (optional: x' = x)
//     n = x' r_x w_pre,  r_x = 1 / sqrt(mean x'^2 + eps)      the norm before the next block (optional)
// Backward, from dn, dres (the gradient that reaches x' from elsewhere) and x', y as they were stored:
//     a = dn o w_pre,  xh = x' r_x,  dX = dres + r_x (a - xh mean(a o xh)),  dx = dX,  dw_pre = sum dn o xh
//     t = s dX o g,  yh = y r_y,  b = t o w_post,  dy = r_y (b - yh mean(b o yh))
//     dw_post = sum t o yh,  dgate = s dX o yh o w_post (summed over the rows where the gate is per channel)
// The statistics are computed again from x' and y, which are read anyway: nothing is kept for the backward
// pass but the activations themselves.
//
// HBM-bound: forward 4 activations' bytes per element, backward 6 (8 with an element-wise gate).  One CTA takes whole
// rows, every element stays in registers between its load and its store, and the next row is loaded
// before this row's sums are reduced.  The backward pass needs ONE reduction per row for all its means: with
// t0 = s g o w_post o y,
//     sum b o yh = r_y sum t0 o dX = r_y (sum t0 o dres + r_x sum t0 o a - r_x^2 mean(a o xh) sum t0 o x'),
// so the six sums of x'^2, y^2, a x', t0 dres, t0 a, t0 x' settle everything at once.  Gradients of weights and of a
// per-channel gate are column sums: every CTA keeps its own in registers over its rows and writes them
// once, and a second kernel adds the CTAs up in a fixed order (no atomics: bit-identical from run to run).
// The workers' rows never share a CTA's sums: each of the K workers has CTAs of its own.
#ifndef FGD_BLOCK_NORM_CUH_
#define FGD_BLOCK_NORM_CUH_

#include "fgd_dtype.cuh"

namespace fgd {

enum : int { GATE_NONE = 0, GATE_ROW = 1, GATE_FULL = 2 };

struct NormMat {
  char* p;       // nullptr: absent
  int64_t ld;    // elements between rows
};
struct NormArgs {
  NormMat x, y, gate, w_post, w_pre, x_new, n;       // forward: x in; backward: x_new in
  NormMat dn, dres, dx, dy, dgate, dw_post, dw_pre;
  float* partial;    // [gridDim.x][2][width] column sums of each CTA
  int64_t rows;      // per worker
  int width, gate_kind, ctas;   // ctas: CTAs per worker
  float eps, scale, inv_width;
};

template <typename T, int VEC>
struct RowVec {
  ActPack<T, VEC> r;
  __device__ __forceinline__ void load(const NormMat& m, int64_t row, int c, bool real) {
    if (real) r = load_stream<T, VEC>(reinterpret_cast<const T*>(m.p) + row * m.ld + c);
    else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) r.v[i] = from_f32<T>(0.f);
    }
  }
  __device__ __forceinline__ float operator[](int i) const { return to_f32<T>(r.v[i]); }
};

// VEC per-channel fp32 values (weights are read by every row: through the read-only cache).
template <int VEC>
__device__ __forceinline__ void load_channel(const NormMat& m, int64_t worker, int c, bool real, float fill, float (&w)[VEC]) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) w[i] = fill;
  if (m.p == nullptr || !real) return;
  const float* p = reinterpret_cast<const float*>(m.p) + worker * m.ld + c;
  if constexpr (VEC % 4 == 0) {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      const float4 t = __ldg(reinterpret_cast<const float4*>(p + i));
      w[i] = t.x; w[i + 1] = t.y; w[i + 2] = t.z; w[i + 3] = t.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) w[i] = __ldg(p + i);
  }
}

// Sums of N values over the CTA, in a fixed order, given to every thread.  `slot` alternates between calls, so
// one barrier per reduction is enough.
template <int N, int NT>
__device__ __forceinline__ void cta_sum(float (&v)[N], float (*buf)[N][NT / 32], int slot) {
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], off);
  if constexpr (NT > 32) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) buf[slot][k][warp] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < NT / 32; ++w) s += buf[slot][k][w];
      v[k] = s;
    }
  }
}

// Threads per row and vectors per thread for rows of `vecs` vectors; the kernels are compiled for
// exactly these.
struct NormShape { int nt, vpt; };

}  // namespace fgd
#endif

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
// rows.  A thread copies its vectors of the next rows into shared memory asynchronously (cp.async: a ring of
// rows that only this thread reads, so it needs no barrier and costs no registers) while it works on the current row.  The
// backward pass needs ONE reduction per row for all its means: with t0 = s g o w_post o y,
//     sum b o yh = r_y sum t0 o dX = r_y (sum t0 o dres + r_x sum t0 o a - r_x^2 mean(a o xh) sum t0 o x'),
// so the six sums of x'^2, y^2, a x', t0 dres, t0 a, t0 x' settle everything at once.  Gradients of weights and of a
// per-channel gate are column sums: every CTA keeps its own in registers over its rows and writes them
// once, and a second kernel adds the CTAs up in a fixed order (no atomics: bit-identical from run to run).
// Rows off their 16-byte boundaries go the same way in shifted chunks (fgd_shift.cuh).
// Measured, % of the copy peak at the activations' and weights' own bytes (8 workers, gate per channel, 2^26 elements a tensor in bf16, 2^25
// in fp32): forward bf16 80 at 2048 columns, 90 at 4096, 69 at 8192, 59 at 16384, backward 86, 86, 79, 40; fp32 82, 90, 72, 63 and 93, 93, 82, 37.
// Some instances spill, bytes a thread: fp32 above 8192 columns 36 to 832, 16-bit backward above 8192 204 to 432, and off the boundaries above
// 2048 columns 176 to 492.
// The workers' rows never share a CTA's sums: each of the K workers has CTAs of its own.
#ifndef FGD_BLOCK_NORM_CUH_
#define FGD_BLOCK_NORM_CUH_

#include "fgd_dtype.cuh"
#include "fgd_shift.cuh"

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
  int64_t rows, last_row;      // per worker; of all workers
  int width, gate_kind, ctas;   // ctas: CTAs per worker
  float eps, scale, inv_width;
};

// Columns c .. c + VEC - 1 of a row; all lanes call it together, whether c lies in the row or beyond it.  ANY: rows start anywhere.
template <typename T, int VEC, bool ANY>
__device__ __forceinline__ void store_vec(const NormMat& m, int64_t row, int c, int width, const Vals<VEC>& v) {
  T* p = reinterpret_cast<T*>(m.p) + row * m.ld + c;
  const ActPack<T, VEC> r = round_to<T, VEC>(v);
  if constexpr (ANY) {
    const uint32_t w[4] = {r.w.x, r.w.y, r.w.z, r.w.w};
    const int lane = threadIdx.x & 31;
    store_unit<sizeof(T), 4>(reinterpret_cast<char*>(p), (width - c) * (int)sizeof(T), lane > 0, lane < 31, w);
  } else {
    if (c < width) store_stream<T, VEC>(p, r);
  }
}

// VPT vectors of per-channel fp32 values (1 where the tensor is absent), c[j] the first column of vector j; what a column beyond the
// width gets is never used.  ANY: the row may start anywhere and end inside a vector.
template <int VEC, int VPT, bool ANY>
__device__ __forceinline__ void load_channel(const NormMat& m, int64_t worker, const int (&c)[VPT], int width, Vals<VEC> (&w)[VPT]) {
  if (m.p == nullptr) {
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) w[j].v[i] = 1.f;
    return;
  }
  const float* p = reinterpret_cast<const float*>(m.p) + worker * m.ld;
  const bool vectors = !ANY || (reinterpret_cast<uintptr_t>(p) & 15u) == 0;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const bool whole = ANY ? c[j] + VEC <= width : c[j] < width;
    if (!ANY || (vectors && whole)) {
      const float* q = p + (whole ? c[j] : 0);
#pragma unroll
      for (int i = 0; i < VEC; i += 4) {
        const float4 t = __ldg(reinterpret_cast<const float4*>(q + i));
        w[j].v[i] = t.x; w[j].v[i + 1] = t.y; w[j].v[i + 2] = t.z; w[j].v[i + 3] = t.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) w[j].v[i] = c[j] + i < width ? __ldg(p + c[j] + i) : 0.f;
    }
  }
}
// What multiplies y r_y per channel: res_scale, w_post, and the gate where it is per channel.
template <int VEC, int VPT, bool ANY>
__device__ __forceinline__ void post_factors(const NormArgs& a, int64_t worker, const int (&c)[VPT], Vals<VEC> (&w)[VPT]) {
  load_channel<VEC, VPT, ANY>(a.w_post, worker, c, a.width, w);
  if (a.gate_kind == GATE_ROW) {
    Vals<VEC> g[VPT];
    load_channel<VEC, VPT, ANY>(a.gate, worker, c, a.width, g);
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) w[j].v[i] *= g[j].v[i];
  }
#pragma unroll
  for (int j = 0; j < VPT; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) w[j].v[i] *= a.scale;
}

// The rows of up to N tensors that a thread is going to work on: a ring of STAGES rows in shared memory filled with cp.async
// (16-byte vectors), or, with STAGES = 0, the current row in registers.  Absent tensors and columns beyond the width read as zero.
// ANY: a row starts s bytes behind a 16-byte boundary.  The ring then holds the chunks from that boundary on; a vector lies in its
// own chunk and the next one, the next lane's.  So that no warp reads another's chunks, lane 31 fetches that one too.
template <typename T, int VEC, int NT, int VPT, int N, int STAGES, bool ANY>
struct RowFeed {
  static constexpr int SLOTS = ANY ? 33 : 32;      // of a warp
  static constexpr size_t kStageBytes = (size_t)VPT * (NT / 32) * SLOTS * 16;      // of one tensor
  unsigned char* ring;
  uint32_t use;               // bit k: tensor k is present
  int width, stage;
  int64_t last;               // the tensors' last row
  uint32_t shift[ANY ? N : 1];
  // The current row in registers: shifted once, read twice (ANY), or read once from the ring (backward, two sets of inputs in turn: 8 x 4096 x
  // 2048 bf16 150 us from the ring twice, 144 so; with a gate per element, N = 5, 178 against 183, and forward 103 against 105: from the ring).
  static constexpr bool HELD = STAGES == 0 || (ANY && VPT <= 2) || (N == 4 && VPT == 1);
  ActPack<T, VEC> cur[HELD ? N : 1][HELD ? VPT : 1];

  __device__ __forceinline__ int column(int j) const { return (int)(threadIdx.x + j * NT) * VEC; }
  __device__ __forceinline__ size_t slot(int s, int k, int j) const {
    const size_t row = (size_t)(s * N + k) * VPT + j;
    if constexpr (ANY) return ((row * (NT / 32) + threadIdx.x / 32) * SLOTS + threadIdx.x % 32) * 16;
    else return (row * NT + threadIdx.x) * 16;
  }
  static __device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  }
  // A chunk of a tensor that ends at hi and begins at lo: bytes outside are not read.
  static __device__ __forceinline__ void copy_chunk(uint32_t dst, const char* src, const char* lo, const char* hi) {
    if (src >= lo && src + 16 <= hi) {
      copy16(dst, src);
    } else {
      for (int b = 0; b < 16; b += (int)sizeof(T))
        if (src + b >= lo && src + b < hi) {
          const uint32_t v = load_elem<sizeof(T)>(src + b);
          if constexpr (sizeof(T) == 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst + b), "r"(v) : "memory");
          else asm volatile("st.shared.b16 [%0], %1;" ::"r"(dst + b), "h"((unsigned short)v) : "memory");
        }
    }
  }
  __device__ __forceinline__ void ask(int s, int64_t row, const NormMat (&t)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (use >> k & 1) {
        const char* p = t[k].p + row * t[k].ld * (int64_t)sizeof(T);
        const int sh = ANY ? (int)(reinterpret_cast<uintptr_t>(p) & 15u) : 0, bytes = sh + width * (int)sizeof(T);
        const char* lo = t[k].p;
        const char* hi = p + ((last - row) * t[k].ld + width) * (int64_t)sizeof(T);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
          const int b = (int)(threadIdx.x + j * NT) * 16;
          const uint32_t dst = (uint32_t)__cvta_generic_to_shared(ring + slot(s, k, j));
          if constexpr (ANY) {
            if (b < bytes) copy_chunk(dst, p - sh + b, lo, hi);
            if (threadIdx.x % 32 == 31 && b + 16 < bytes) copy_chunk(dst + 16, p - sh + b + 16, lo, hi);
          } else {
            if (b < bytes) copy16(dst, p + b);
          }
        }
      }
  }
  // Rows first, first + step, ... below end of tensors whose last row is `last`.
  __device__ __forceinline__ void start(const NormMat (&t)[N], int width_, unsigned char* ring_, int64_t first, int64_t step, int64_t end, int64_t last_) {
    ring = ring_; width = width_; stage = 0; use = 0; last = last_;
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (t[k].p != nullptr) use |= 1u << k;
    if constexpr (STAGES > 0) {
#pragma unroll
      for (int s = 0; s < STAGES; ++s)
        for (int k = 0; k < N; ++k)
          for (int j = 0; j < VPT; ++j)
            if (!(use >> k & 1) || (!ANY && column(j) >= width)) *reinterpret_cast<uint4*>(ring + slot(s, k, j)) = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int s = 0; s < STAGES - 1; ++s) {
        if (first + s * step < end) ask(s, first + s * step, t);
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
    }
  }
  // Makes row `row` the current one and asks for the row STAGES - 1 further on.
  __device__ __forceinline__ void next(const NormMat (&t)[N], int64_t row, int64_t step, int64_t end, bool first) {
    if constexpr (ANY) {
#pragma unroll
      for (int k = 0; k < N; ++k)      // (0 for an absent tensor: its zeros are in the lanes' own chunks alone)
        shift[k] = use >> k & 1 ? (uint32_t)((reinterpret_cast<uintptr_t>(t[k].p) + (uintptr_t)(row * t[k].ld) * sizeof(T)) & 15u) : 0u;
    }
    if constexpr (STAGES == 1) {
      if constexpr (ANY) __syncwarp();      // the lane before has read this lane's chunks
      ask(0, row, t);
      asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
      if constexpr (ANY) __syncwarp();
    } else if constexpr (STAGES > 1) {
      if (!first) stage = stage + 1 == STAGES ? 0 : stage + 1;
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
      if constexpr (ANY) __syncwarp();      // the lanes' chunks are there, and those of the row before have been read
      const int64_t far = row + (STAGES - 1) * step;
      const int into = stage == 0 ? STAGES - 1 : stage - 1;
      if (far < end) ask(into, far, t);
      asm volatile("cp.async.commit_group;" ::: "memory");
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
          const int c = column(j);
          const T* p = reinterpret_cast<const T*>(t[k].p) + row * t[k].ld;
          if constexpr (ANY) {
            zero(cur[k][j]);
            if (use >> k & 1) {
              const char* at = reinterpret_cast<const char*>(p + c);
              uint32_t w[4];
              load_unit<sizeof(T), 4>(at, c < width, threadIdx.x % 32 < 31 && c + VEC < width, t[k].p,
                                      reinterpret_cast<const char*>(p + (last - row) * t[k].ld + width), w);
              cur[k][j].w = make_uint4(w[0], w[1], w[2], w[3]);
            }
          } else {
            if ((use >> k & 1) && c < width) cur[k][j] = load_stream<T, VEC>(p + c);
            else zero(cur[k][j]);
          }
        }
    }
    if constexpr (HELD && STAGES > 0) {
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int j = 0; j < VPT; ++j) cur[k][j] = from_ring(k, j);
    }
  }
  __device__ __forceinline__ ActPack<T, VEC> from_ring(int k, int j) const {
    ActPack<T, VEC> p;
    const uint4* at = reinterpret_cast<const uint4*>(ring + slot(stage, k, j));
    p.w = at[0];
    if constexpr (ANY) {
      const uint4 next = at[1];
      const uint32_t x[8] = {p.w.x, p.w.y, p.w.z, p.w.w, next.x, next.y, next.z, next.w};
      uint32_t r[4];
      shift_words<4>(x, shift[k], r);
      p.w = make_uint4(r[0], r[1], r[2], r[3]);
    }
    return p;
  }
  __device__ __forceinline__ Vals<VEC> get(int k, int j) const {
    Vals<VEC> v;
    if constexpr (HELD) v = unpack<T, VEC>(cur[k][j]);
    else v = unpack<T, VEC>(from_ring(k, j));
    if constexpr (ANY) {
      const int left = width - column(j);
      if (left < VEC) {                     // beyond the row: the next row's values, or none
#pragma unroll
        for (int i = 0; i < VEC; ++i) v.v[i] = i < left ? v.v[i] : 0.f;
      }
    }
    return v;
  }
};

// Per-channel factors of a thread's columns: in registers (`held`), or in shared memory, where only this thread reads them.
template <int VEC, int VPT, int NT, bool KEEP>
struct Factors {
  float4* at;
  __device__ __forceinline__ void start(unsigned char* smem, int which, const Vals<VEC> (&held)[VPT]) {
    if constexpr (KEEP) {
      at = reinterpret_cast<float4*>(smem) + (size_t)which * VPT * (VEC / 4) * NT + threadIdx.x;
#pragma unroll
      for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int i = 0; i < VEC / 4; ++i)
          at[(j * (VEC / 4) + i) * NT] = make_float4(held[j].v[4 * i], held[j].v[4 * i + 1], held[j].v[4 * i + 2], held[j].v[4 * i + 3]);
    }
  }
  __device__ __forceinline__ Vals<VEC> get(const Vals<VEC> (&held)[VPT], int j) const {
    if constexpr (KEEP) {
      Vals<VEC> r;
#pragma unroll
      for (int i = 0; i < VEC / 4; ++i) {
        const float4 f = at[(j * (VEC / 4) + i) * NT];
        r.v[4 * i] = f.x; r.v[4 * i + 1] = f.y; r.v[4 * i + 2] = f.z; r.v[4 * i + 3] = f.w;
      }
      return r;
    } else {
      return held[j];
    }
  }
};

// Sums of N values over the CTA, in a fixed order, given to every thread.  `slot` alternates between calls, so
// one barrier per reduction is enough.  Inside a warp the lanes trade values as they add: after the first step a lane carries half of
// the N sums, after the third one of eight, so that six sums cost 9 shuffles instead of 30.
template <int N, int NT>
__device__ __forceinline__ void cta_sum(float (&v)[N], float (*buf)[N][NT / 32], int slot) {
  static_assert(N == 1 || N == 6, "one sum or six");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if constexpr (N == 1) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], off);
    if constexpr (NT > 32) {
      if (lane == 0) buf[slot][0][warp] = v[0];
    }
  } else {
    // bit 4, 3, 2 of the lane choose the upper half of what is left
    const bool up16 = lane & 16, up8 = lane & 8, up4 = lane & 4;
    float a[4], b[2], c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float hi = i < 2 ? v[i + 4] : 0.f;
      a[i] = (up16 ? hi : v[i]) + __shfl_xor_sync(0xffffffffu, up16 ? v[i] : hi, 16);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) b[i] = (up8 ? a[i + 2] : a[i]) + __shfl_xor_sync(0xffffffffu, up8 ? a[i] : a[i + 2], 8);
    c = (up4 ? b[1] : b[0]) + __shfl_xor_sync(0xffffffffu, up4 ? b[0] : b[1], 4);
    c += __shfl_xor_sync(0xffffffffu, c, 2);
    c += __shfl_xor_sync(0xffffffffu, c, 1);
    const int k = (lane >> 4) * 4 + ((lane >> 3) & 1) * 2 + ((lane >> 2) & 1);     // which sum this lane has
    if constexpr (NT > 32) {
      if ((lane & 3) == 0 && k < N) buf[slot][k][warp] = c;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, c, (i >> 2) * 16 + ((i >> 1) & 1) * 8 + (i & 1) * 4);
    }
  }
  if constexpr (NT > 32) {
    constexpr int W = NT / 32;
    __syncthreads();
    if constexpr (N == 1) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += buf[slot][0][w];
      v[0] = s;
    } else {
      // four lanes per sum add the warps' parts, then every lane takes all six
      const int k = lane >> 2, part = lane & 3;
      float s = 0.f;
      if (k < N) {
#pragma unroll
        for (int w = 0; w < (W + 3) / 4; ++w)
          if (W % 4 == 0 || part * ((W + 3) / 4) + w < W) s += buf[slot][k][part * ((W + 3) / 4) + w];
      }
      s += __shfl_xor_sync(0xffffffffu, s, 1);
      s += __shfl_xor_sync(0xffffffffu, s, 2);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, s, 4 * i);
    }
  }
}

}  // namespace fgd
#endif

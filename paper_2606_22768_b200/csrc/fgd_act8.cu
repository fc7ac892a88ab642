// Activation checkpoints in 8 bits, and the SwiGLU that keeps its inputs in them.
//
// A row is cut into groups of 32 consecutive values.  A group stores 32 signed bytes q and one byte e:
//     value = q 2^(e-127),   e = max(biased exponent of the group's largest magnitude - 6, 1),
//     q = round-to-nearest-even(x 2^(127-e)), held to [-127, 127].
// The largest magnitude of a group lands in [64, 128), so the step is at most 1/64 of it.  A power of
// two rather than amax/127 as the step costs up to one bit of resolution and makes every operation but
// the rounding exact: save and load need no division, a bf16 value read back is exactly the stored one
// (7 bits into 8), and any two implementations agree bit for bit.  A group that holds an infinity or a
// NaN stores e = 255 and reads back as NaN, so an overflow in the forward pass stays visible.
//
// SwiGLU: h = silu(g) u with g, u the two halves of a row.  The backward pass reads only the
// checkpoint (g^, u^), never g and u:
//     sg = 1 / (1 + exp(-g^)),  du = dh g^ sg,  dg = dh u^ sg (1 + g^ (1 - sg)),  h = g^ sg u^ (again).
//
// All four are bound by HBM: one pass, every byte read or written once.
//
// Vector kernels (rows and bases on 16-byte boundaries, width a multiple of 8): a thread takes 8
// consecutive values, four neighbouring lanes make a group, so the group's largest magnitude is two
// shuffles away.  Element kernels (any width and stride): a warp takes a group, a lane a value.
#include "fgd_dtype.cuh"
#include "fgd_nvtx.h"

using namespace fgd;

namespace {

constexpr int kGroup = 32;
constexpr int kBlock8 = 256;

// Step exponent of a group from the bits of its largest magnitude (sign bit clear; NaN and infinity
// have exponent 255 and are the largest as integers too, so an integer maximum finds them).
__device__ __forceinline__ uint32_t step_exponent(uint32_t amax_bits) {
  const uint32_t eb = amax_bits >> 23;
  if (eb >= 255u) return 255u;
  return eb > 7u ? eb - 6u : 1u;
}
__device__ __forceinline__ float step_of(uint32_t e) { return e >= 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(e << 23); }
__device__ __forceinline__ float inverse_step(uint32_t e) { return e >= 255u ? 0.f : __uint_as_float((254u - e) << 23); }
__device__ __forceinline__ int to_q8(float x, float inv) {
  return __float2int_rn(fminf(fmaxf(x * inv, -127.f), 127.f));
}
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

__device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.f, 1.f + __expf(-g)); }

// Largest magnitude bits over the four lanes of a group.
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  return max(m, __shfl_xor_sync(0xffffffffu, m, 2));
}
__device__ __forceinline__ uint32_t warp_max(uint32_t m) { return __reduce_max_sync(0xffffffffu, m); }

// 8 consecutive values starting at p, as fp32.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&f)[8]) {
  constexpr int N = 16 / sizeof(T);
#pragma unroll
  for (int j = 0; j < 8; j += N) {
    const Vals<N> r = unpack<T, N>(load_stream<T, N>(p + j));
#pragma unroll
    for (int i = 0; i < N; ++i) f[j + i] = r.v[i];
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
  constexpr int N = 16 / sizeof(T);
#pragma unroll
  for (int j = 0; j < 8; j += N) {
    Vals<N> r;
#pragma unroll
    for (int i = 0; i < N; ++i) r.v[i] = f[j + i];
    store_stream<T, N>(p + j, round_to<T, N>(r));
  }
}
__device__ __forceinline__ uint2 quantise8(const float (&f)[8], float inv) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i >> 2] |= (uint32_t)(to_q8(f[i], inv) & 255) << (8 * (i & 3));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void dequantise8(uint2 q, float step, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (float)(int8_t)(((i < 4 ? q.x : q.y) >> (8 * (i & 3))) & 255u) * step;
}
__device__ __forceinline__ uint32_t amax8(const float (&f)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, abs_bits(f[i]));
  return m;
}

struct Act8Args {
  const void* x; int64_t ld_x;       // save: source; load: destination (non-const there)
  void* out; int64_t ld_out;
  int8_t* q; int64_t ld_q;
  uint8_t* e; int64_t ld_e;
  int64_t rows, width;
};

// A walk over (row, unit) with `units` units per row, gridDim x blockDim units at a time, without a
// division in the loop.
struct Walk {
  int64_t row, step_row;
  int unit, step_unit, units;
  __device__ __forceinline__ Walk(int64_t first, int64_t stride, int units_) : units(units_) {
    row = first / units; unit = (int)(first - row * units);
    step_row = stride / units; step_unit = (int)(stride - step_row * units);
  }
  __device__ __forceinline__ void next() {
    row += step_row; unit += step_unit;
    if (unit >= units) { unit -= units; ++row; }
  }
};

// ---- vector kernels: a unit is 8 values; every row is padded to whole groups, i.e. to a multiple of four
// units, so that the four lanes of a group always work together
template <typename T>
__global__ void __launch_bounds__(kBlock8) act8_save_kernel(const Act8Args a) {
  const int units = (int)((a.width + kGroup - 1) / kGroup) * 4;
  const int64_t total = a.rows * units, padded = (total + 31) / 32 * 32;   // whole warps stay in the loop for the shuffles
  Walk w((int64_t)blockIdx.x * kBlock8 + threadIdx.x, (int64_t)gridDim.x * kBlock8, units);
  for (int64_t i = (int64_t)blockIdx.x * kBlock8 + threadIdx.x; i < padded; i += (int64_t)gridDim.x * kBlock8, w.next()) {
    const int c = w.unit * 8;
    const bool real = i < total && c < a.width;
    float f[8] = {};
    if (real) load8<T>(static_cast<const T*>(a.x) + w.row * a.ld_x + c, f);
    const uint32_t e = step_exponent(quad_max(amax8(f)));
    if (real) *reinterpret_cast<uint2*>(a.q + w.row * a.ld_q + c) = quantise8(f, inverse_step(e));
    if (i < total && (w.unit & 3) == 0) a.e[w.row * a.ld_e + (w.unit >> 2)] = (uint8_t)e;
  }
}
template <typename T>
__global__ void __launch_bounds__(kBlock8) act8_load_kernel(const Act8Args a) {
  const int units = (int)(a.width / 8);
  const int64_t total = a.rows * units;
  Walk w((int64_t)blockIdx.x * kBlock8 + threadIdx.x, (int64_t)gridDim.x * kBlock8, units);
  for (int64_t i = (int64_t)blockIdx.x * kBlock8 + threadIdx.x; i < total; i += (int64_t)gridDim.x * kBlock8, w.next()) {
    const int c = w.unit * 8;
    float f[8];
    dequantise8(__ldcs(reinterpret_cast<const uint2*>(a.q + w.row * a.ld_q + c)), step_of(a.e[w.row * a.ld_e + (w.unit >> 2)]), f);
    store8<T>(static_cast<T*>(a.out) + w.row * a.ld_out + c, f);
  }
}
template <typename T>
__global__ void __launch_bounds__(kBlock8) swiglu8_forward_kernel(const Act8Args a) {
  const int groups = (int)((a.width + kGroup - 1) / kGroup), units = groups * 4;
  const int64_t total = a.rows * units, padded = (total + 31) / 32 * 32;
  Walk w((int64_t)blockIdx.x * kBlock8 + threadIdx.x, (int64_t)gridDim.x * kBlock8, units);
  for (int64_t i = (int64_t)blockIdx.x * kBlock8 + threadIdx.x; i < padded; i += (int64_t)gridDim.x * kBlock8, w.next()) {
    const int c = w.unit * 8;
    const bool real = i < total && c < a.width;
    float g[8] = {}, u[8] = {};
    if (real) {
      const T* row = static_cast<const T*>(a.x) + w.row * a.ld_x + c;
      load8<T>(row, g);
      load8<T>(row + a.width, u);
    }
    const uint32_t eg = step_exponent(quad_max(amax8(g))), eu = step_exponent(quad_max(amax8(u)));
    if (real) {
      int8_t* q = a.q + w.row * a.ld_q + c;
      *reinterpret_cast<uint2*>(q) = quantise8(g, inverse_step(eg));
      *reinterpret_cast<uint2*>(q + a.width) = quantise8(u, inverse_step(eu));
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = g[j] * sigmoid(g[j]) * u[j];
      store8<T>(static_cast<T*>(a.out) + w.row * a.ld_out + c, g);
    }
    if (i < total && (w.unit & 3) == 0) {
      uint8_t* e = a.e + w.row * a.ld_e + (w.unit >> 2);
      e[0] = (uint8_t)eg;
      e[groups] = (uint8_t)eu;
    }
  }
}
struct Swiglu8BackArgs {
  const void* dh; int64_t ld_dh;
  const int8_t* q; int64_t ld_q;
  const uint8_t* e; int64_t ld_e;
  void* dgu; int64_t ld_dgu;
  void* h; int64_t ld_h;             // NULL: not wanted
  int64_t rows, width;
};
__device__ __forceinline__ void swiglu_back(float dh, float g, float u, float& dg, float& du, float& h) {
  const float s = sigmoid(g), gs = g * s;
  h = gs * u;
  du = dh * gs;
  dg = dh * u * s * fmaf(g, 1.f - s, 1.f);
}
template <typename T>
__global__ void __launch_bounds__(kBlock8) swiglu8_backward_kernel(const Swiglu8BackArgs a) {
  const int groups = (int)((a.width + kGroup - 1) / kGroup), units = (int)(a.width / 8);
  const int64_t total = a.rows * units;
  Walk w((int64_t)blockIdx.x * kBlock8 + threadIdx.x, (int64_t)gridDim.x * kBlock8, units);
  for (int64_t i = (int64_t)blockIdx.x * kBlock8 + threadIdx.x; i < total; i += (int64_t)gridDim.x * kBlock8, w.next()) {
    const int c = w.unit * 8;
    const int8_t* q = a.q + w.row * a.ld_q + c;
    const uint8_t* e = a.e + w.row * a.ld_e + (w.unit >> 2);
    const uint2 qg = __ldcs(reinterpret_cast<const uint2*>(q)), qu = __ldcs(reinterpret_cast<const uint2*>(q + a.width));
    float dh[8], g[8], u[8], h[8];
    load8<T>(static_cast<const T*>(a.dh) + w.row * a.ld_dh + c, dh);
    dequantise8(qg, step_of(e[0]), g);
    dequantise8(qu, step_of(e[groups]), u);
#pragma unroll
    for (int j = 0; j < 8; ++j) swiglu_back(dh[j], g[j], u[j], g[j], u[j], h[j]);
    T* out = static_cast<T*>(a.dgu) + w.row * a.ld_dgu + c;
    store8<T>(out, g);
    store8<T>(out + a.width, u);
    if (a.h) store8<T>(static_cast<T*>(a.h) + w.row * a.ld_h + c, h);
  }
}

// ---- element kernels: a warp is a group, a lane a value
template <typename T>
__global__ void __launch_bounds__(kBlock8) act8_save_elem_kernel(const Act8Args a) {
  const int groups = (int)((a.width + kGroup - 1) / kGroup), lane = threadIdx.x & 31;
  const int64_t stride = (int64_t)gridDim.x * (kBlock8 / 32), total = a.rows * groups;
  int64_t i = (int64_t)blockIdx.x * (kBlock8 / 32) + (threadIdx.x >> 5);
  Walk w(i, stride, groups);
  for (; i < total; i += stride, w.next()) {
    const int64_t c = (int64_t)w.unit * kGroup + lane;
    const bool real = c < a.width;
    const float f = real ? to_f32<T>(static_cast<const T*>(a.x)[w.row * a.ld_x + c]) : 0.f;
    const uint32_t e = step_exponent(warp_max(abs_bits(f)));
    if (real) a.q[w.row * a.ld_q + c] = (int8_t)to_q8(f, inverse_step(e));
    if (lane == 0) a.e[w.row * a.ld_e + w.unit] = (uint8_t)e;
  }
}
template <typename T>
__global__ void __launch_bounds__(kBlock8) act8_load_elem_kernel(const Act8Args a) {
  const int groups = (int)((a.width + kGroup - 1) / kGroup), lane = threadIdx.x & 31;
  const int64_t stride = (int64_t)gridDim.x * (kBlock8 / 32), total = a.rows * groups;
  int64_t i = (int64_t)blockIdx.x * (kBlock8 / 32) + (threadIdx.x >> 5);
  Walk w(i, stride, groups);
  for (; i < total; i += stride, w.next()) {
    const int64_t c = (int64_t)w.unit * kGroup + lane;
    if (c < a.width) static_cast<T*>(a.out)[w.row * a.ld_out + c] = from_f32<T>((float)a.q[w.row * a.ld_q + c] * step_of(a.e[w.row * a.ld_e + w.unit]));
  }
}
template <typename T>
__global__ void __launch_bounds__(kBlock8) swiglu8_forward_elem_kernel(const Act8Args a) {
  const int groups = (int)((a.width + kGroup - 1) / kGroup), lane = threadIdx.x & 31;
  const int64_t stride = (int64_t)gridDim.x * (kBlock8 / 32), total = a.rows * groups;
  int64_t i = (int64_t)blockIdx.x * (kBlock8 / 32) + (threadIdx.x >> 5);
  Walk w(i, stride, groups);
  for (; i < total; i += stride, w.next()) {
    const int64_t c = (int64_t)w.unit * kGroup + lane;
    const bool real = c < a.width;
    const T* row = static_cast<const T*>(a.x) + w.row * a.ld_x;
    const float g = real ? to_f32<T>(row[c]) : 0.f, u = real ? to_f32<T>(row[a.width + c]) : 0.f;
    const uint32_t eg = step_exponent(warp_max(abs_bits(g))), eu = step_exponent(warp_max(abs_bits(u)));
    if (real) {
      int8_t* q = a.q + w.row * a.ld_q + c;
      q[0] = (int8_t)to_q8(g, inverse_step(eg));
      q[a.width] = (int8_t)to_q8(u, inverse_step(eu));
      static_cast<T*>(a.out)[w.row * a.ld_out + c] = from_f32<T>(g * sigmoid(g) * u);
    }
    if (lane == 0) {
      uint8_t* e = a.e + w.row * a.ld_e + w.unit;
      e[0] = (uint8_t)eg;
      e[groups] = (uint8_t)eu;
    }
  }
}
template <typename T>
__global__ void __launch_bounds__(kBlock8) swiglu8_backward_elem_kernel(const Swiglu8BackArgs a) {
  const int groups = (int)((a.width + kGroup - 1) / kGroup), lane = threadIdx.x & 31;
  const int64_t stride = (int64_t)gridDim.x * (kBlock8 / 32), total = a.rows * groups;
  int64_t i = (int64_t)blockIdx.x * (kBlock8 / 32) + (threadIdx.x >> 5);
  Walk w(i, stride, groups);
  for (; i < total; i += stride, w.next()) {
    const int64_t c = (int64_t)w.unit * kGroup + lane;
    if (c >= a.width) continue;
    const int8_t* q = a.q + w.row * a.ld_q + c;
    const uint8_t* e = a.e + w.row * a.ld_e + w.unit;
    float dg, du, h;
    swiglu_back(to_f32<T>(static_cast<const T*>(a.dh)[w.row * a.ld_dh + c]), (float)q[0] * step_of(e[0]), (float)q[a.width] * step_of(e[groups]), dg, du, h);
    T* out = static_cast<T*>(a.dgu) + w.row * a.ld_dgu + c;
    out[0] = from_f32<T>(dg);
    out[a.width] = from_f32<T>(du);
    if (a.h) static_cast<T*>(a.h)[w.row * a.ld_h + c] = from_f32<T>(h);
  }
}

bool on16(const void* p, int64_t ld, int bytes) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * bytes) % 16 == 0; }
bool on8(const void* p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0 && ld % 8 == 0; }

int check_dims(const char* who, int dtype, int64_t rows, int64_t width) {
  if (dtype_bytes(dtype) == 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (rows < 0 || width < 0 || width > ((int64_t)1 << 29)) return op_fail(FGD_ERR_INVALID_ARG, "%s: rows=%lld, width=%lld out of range", who, (long long)rows, (long long)width);
  return FGD_OK;
}

// Threads enough to cover the work, at most eight CTAs per SM of a grid that strides over the rest.
unsigned grid_for(int64_t threads) {
  const int64_t want = (threads + kBlock8 - 1) / kBlock8, most = (int64_t)sm_count() * 8;
  return (unsigned)(want < most ? want : most);
}

int launched(const char* who) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

#define FGD_BY_DTYPE(dtype, KERNEL, ...)                                             \
  switch (dtype) {                                                                   \
    case FGD_F32: KERNEL<float><<<__VA_ARGS__>>>(a); break;                          \
    case FGD_BF16: KERNEL<__nv_bfloat16><<<__VA_ARGS__>>>(a); break;                 \
    default: KERNEL<__half><<<__VA_ARGS__>>>(a); break;                              \
  }

}  // namespace

extern "C" int fgd_act_save8(int device, int dtype, int64_t rows, int64_t width, const void* x, int64_t ld_x, int8_t* q8, int64_t ld_q, uint8_t* e8,
                             int64_t ld_e, void* stream) {
  FGD_NVTX_RANGE("fgd_act_save8");
  if (int rc = check_dims("fgd_act_save8", dtype, rows, width)) return rc;
  if (rows == 0 || width == 0) return FGD_OK;
  const int64_t groups = (width + kGroup - 1) / kGroup;
  if (!x || !q8 || !e8) return op_fail(FGD_ERR_INVALID_ARG, "fgd_act_save8: NULL pointer");
  if (ld_x < width || ld_q < width || ld_e < groups) return op_fail(FGD_ERR_INVALID_ARG, "fgd_act_save8: a row stride is below the row's width");
  const int b = dtype_bytes(dtype);
  const Span sx = span_of(x, rows, width, ld_x, b), sq = span_of(q8, rows, width, ld_q, 1), se = span_of(e8, rows, groups, ld_e, 1);
  if (sx.overlaps(sq) || sx.overlaps(se) || sq.overlaps(se)) return op_fail(FGD_ERR_ALIAS, "fgd_act_save8: tensors overlap");
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  const Act8Args a{x, ld_x, nullptr, 0, q8, ld_q, e8, ld_e, rows, width};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (width % 8 == 0 && on16(x, ld_x, b) && on8(q8, ld_q)) {
    FGD_BY_DTYPE(dtype, act8_save_kernel, grid_for(rows * groups * 4), kBlock8, 0, st)
  } else {
    FGD_BY_DTYPE(dtype, act8_save_elem_kernel, grid_for(rows * groups * 32), kBlock8, 0, st)
  }
  return launched("fgd_act_save8");
}

extern "C" int fgd_act_load8(int device, int dtype, int64_t rows, int64_t width, const int8_t* q8, int64_t ld_q, const uint8_t* e8, int64_t ld_e, void* out,
                             int64_t ld_out, void* stream) {
  FGD_NVTX_RANGE("fgd_act_load8");
  if (int rc = check_dims("fgd_act_load8", dtype, rows, width)) return rc;
  if (rows == 0 || width == 0) return FGD_OK;
  const int64_t groups = (width + kGroup - 1) / kGroup;
  if (!out || !q8 || !e8) return op_fail(FGD_ERR_INVALID_ARG, "fgd_act_load8: NULL pointer");
  if (ld_out < width || ld_q < width || ld_e < groups) return op_fail(FGD_ERR_INVALID_ARG, "fgd_act_load8: a row stride is below the row's width");
  const int b = dtype_bytes(dtype);
  const Span so = span_of(out, rows, width, ld_out, b);
  if (so.overlaps(span_of(q8, rows, width, ld_q, 1)) || so.overlaps(span_of(e8, rows, groups, ld_e, 1))) return op_fail(FGD_ERR_ALIAS, "fgd_act_load8: tensors overlap");
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  const Act8Args a{nullptr, 0, out, ld_out, const_cast<int8_t*>(q8), ld_q, const_cast<uint8_t*>(e8), ld_e, rows, width};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (width % 8 == 0 && on16(out, ld_out, b) && on8(q8, ld_q)) {
    FGD_BY_DTYPE(dtype, act8_load_kernel, grid_for(rows * (width / 8)), kBlock8, 0, st)
  } else {
    FGD_BY_DTYPE(dtype, act8_load_elem_kernel, grid_for(rows * groups * 32), kBlock8, 0, st)
  }
  return launched("fgd_act_load8");
}

extern "C" int fgd_swiglu8_forward(int device, int dtype, int64_t rows, int64_t width, const void* gu, int64_t ld_gu, void* h, int64_t ld_h, int8_t* q8,
                                   int64_t ld_q, uint8_t* e8, int64_t ld_e, void* stream) {
  FGD_NVTX_RANGE("fgd_swiglu8_forward");
  if (int rc = check_dims("fgd_swiglu8_forward", dtype, rows, width)) return rc;
  if (rows == 0 || width == 0) return FGD_OK;
  const int64_t groups = (width + kGroup - 1) / kGroup;
  if (!gu || !h || !q8 || !e8) return op_fail(FGD_ERR_INVALID_ARG, "fgd_swiglu8_forward: NULL pointer");
  if (ld_gu < 2 * width || ld_h < width || ld_q < 2 * width || ld_e < 2 * groups)
    return op_fail(FGD_ERR_INVALID_ARG, "fgd_swiglu8_forward: a row stride is below the row's width");
  const int b = dtype_bytes(dtype);
  const Span sx = span_of(gu, rows, 2 * width, ld_gu, b), sh = span_of(h, rows, width, ld_h, b), sq = span_of(q8, rows, 2 * width, ld_q, 1),
             se = span_of(e8, rows, 2 * groups, ld_e, 1);
  if (sx.overlaps(sh) || sx.overlaps(sq) || sx.overlaps(se) || sh.overlaps(sq) || sh.overlaps(se) || sq.overlaps(se))
    return op_fail(FGD_ERR_ALIAS, "fgd_swiglu8_forward: tensors overlap");
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  const Act8Args a{gu, ld_gu, h, ld_h, q8, ld_q, e8, ld_e, rows, width};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (width % 8 == 0 && on16(gu, ld_gu, b) && on16(h, ld_h, b) && on8(q8, ld_q)) {
    FGD_BY_DTYPE(dtype, swiglu8_forward_kernel, grid_for(rows * groups * 4), kBlock8, 0, st)
  } else {
    FGD_BY_DTYPE(dtype, swiglu8_forward_elem_kernel, grid_for(rows * groups * 32), kBlock8, 0, st)
  }
  return launched("fgd_swiglu8_forward");
}

extern "C" int fgd_swiglu8_backward(int device, int dtype, int64_t rows, int64_t width, const void* dh, int64_t ld_dh, const int8_t* q8, int64_t ld_q,
                                    const uint8_t* e8, int64_t ld_e, void* dgu, int64_t ld_dgu, void* h, int64_t ld_h, void* stream) {
  FGD_NVTX_RANGE("fgd_swiglu8_backward");
  if (int rc = check_dims("fgd_swiglu8_backward", dtype, rows, width)) return rc;
  if (rows == 0 || width == 0) return FGD_OK;
  const int64_t groups = (width + kGroup - 1) / kGroup;
  if (!dh || !dgu || !q8 || !e8) return op_fail(FGD_ERR_INVALID_ARG, "fgd_swiglu8_backward: NULL pointer");
  if (ld_dh < width || ld_dgu < 2 * width || (h && ld_h < width) || ld_q < 2 * width || ld_e < 2 * groups)
    return op_fail(FGD_ERR_INVALID_ARG, "fgd_swiglu8_backward: a row stride is below the row's width");
  const int b = dtype_bytes(dtype);
  const Span sd = span_of(dh, rows, width, ld_dh, b), so = span_of(dgu, rows, 2 * width, ld_dgu, b), sh = span_of(h, rows, width, ld_h, b),
             sq = span_of(q8, rows, 2 * width, ld_q, 1), se = span_of(e8, rows, 2 * groups, ld_e, 1);
  if (so.overlaps(sd) || so.overlaps(sh) || so.overlaps(sq) || so.overlaps(se) || sh.overlaps(sd) || sh.overlaps(sq) || sh.overlaps(se))
    return op_fail(FGD_ERR_ALIAS, "fgd_swiglu8_backward: tensors overlap");
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  const Swiglu8BackArgs a{dh, ld_dh, q8, ld_q, e8, ld_e, dgu, ld_dgu, h, ld_h, rows, width};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (width % 8 == 0 && on16(dh, ld_dh, b) && on16(dgu, ld_dgu, b) && (!h || on16(h, ld_h, b)) && on8(q8, ld_q)) {
    FGD_BY_DTYPE(dtype, swiglu8_backward_kernel, grid_for(rows * (width / 8)), kBlock8, 0, st)
  } else {
    FGD_BY_DTYPE(dtype, swiglu8_backward_elem_kernel, grid_for(rows * groups * 32), kBlock8, 0, st)
  }
  return launched("fgd_swiglu8_backward");
}

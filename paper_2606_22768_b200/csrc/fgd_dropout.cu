// Dropout whose mask is a function of (seed, offset, row, column) and is never stored:
//     out[r][c] = keep ? x[r][c] / (1 - p) : 0,   keep = word(r, c) >= p 2^32,
//     word(r, c) = word c % 4 of Philox4x32 with seven rounds, counter (c / 4, r, offset low, offset high), key (seed low, seed high)
// (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011; seven rounds are the fewest that pass their tests).
// The backward pass is the same call on the gradient.  A function of the row and column, not of the address: any width, stride, launch shape
// and device gives the same mask.
//
// A thread takes 16 bytes: two groups of four words for 16-bit activations, one for fp32.
#include <cmath>

#include "fgd_dtype.cuh"
#include "fgd_nvtx.h"
#include "fgd_units.cuh"

using namespace fgd;

namespace {

constexpr int kThreads = 256;

struct DropoutArgs {
  const char* x; int64_t ld_x;
  char* out; int64_t ld_out;
  int64_t rows, width;
  uint32_t k0, k1;
  uint64_t offset;
  const int64_t* counter;      // added to the offset, or nullptr
  uint32_t threshold;          // dropped below it
  float scale;
};

__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 7; ++i) {
    const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)q;
    c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// The values of a unit of V columns from column c of row r on.
template <int V>
__device__ __forceinline__ Vals<V> drop(const Vals<V>& x, uint32_t c, uint32_t r, uint64_t offset, const DropoutArgs& a) {
  Vals<V> y;
#pragma unroll
  for (int g = 0; g < V / 4; ++g) {
    const uint4 w = philox(c / 4 + g, r, (uint32_t)offset, (uint32_t)(offset >> 32), a.k0, a.k1);
    y.v[4 * g] = w.x >= a.threshold ? x.v[4 * g] * a.scale : 0.f;
    y.v[4 * g + 1] = w.y >= a.threshold ? x.v[4 * g + 1] * a.scale : 0.f;
    y.v[4 * g + 2] = w.z >= a.threshold ? x.v[4 * g + 2] * a.scale : 0.f;
    y.v[4 * g + 3] = w.w >= a.threshold ? x.v[4 * g + 3] * a.scale : 0.f;
  }
  return y;
}

// SHIFTED: rows that start off the 16-byte boundaries, or do not end on one.
template <typename T, bool SHIFTED>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropoutArgs a) {
  constexpr int V = 16 / sizeof(T);
  const int units = (int)((a.width + V - 1) / V);
  const int64_t total = a.rows * units, stride = (int64_t)gridDim.x * kThreads;
  const uint64_t offset = a.offset + (a.counter ? (uint64_t)*a.counter : 0u);
  const T* x = reinterpret_cast<const T*>(a.x);
  T* out = reinterpret_cast<T*>(a.out);
  int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  Walk w(i, stride, units);
  if constexpr (SHIFTED) {
    const T* end = x + (a.rows - 1) * a.ld_x + a.width;
    const int64_t padded = (total + 31) / 32 * 32;      // whole warps stay for the shuffles
    for (; i < padded; i += stride, w.next()) {
      const ShiftedUnit<V> u(w, i < total, a.width);
      const Vals<V> v = load_shifted<T, V>(x + w.row * a.ld_x + u.c, u, x, end);
      store_shifted<T, V>(out + w.row * a.ld_out + u.c, u, drop<V>(v, (uint32_t)u.c, (uint32_t)w.row, offset, a));
    }
  } else {
    for (; i < total; i += stride, w.next()) {
      const int64_t c = (int64_t)w.unit * V;
      const Vals<V> v = unpack<T, V>(load_stream<T, V>(x + w.row * a.ld_x + c));
      store_stream<T, V>(out + w.row * a.ld_out + c, round_to<T, V>(drop<V>(v, (uint32_t)c, (uint32_t)w.row, offset, a)));
    }
  }
}

template <auto KERNEL>
cudaError_t go(const DropoutArgs& a, int64_t units, int waves, cudaStream_t st) {
  static int cached[64] = {};
  int dev = 0, fit = 0;
  const bool known = cudaGetDevice(&dev) == cudaSuccess && dev < 64;
  if (known) fit = cached[dev];
  if (fit == 0) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, KERNEL, kThreads, 0) != cudaSuccess || fit < 1) fit = 1;
    if (known) cached[dev] = fit;
  }
  const int64_t want = (units + kThreads - 1) / kThreads, most = (int64_t)sm_count() * fit * waves;
  KERNEL<<<(unsigned)(want < most ? want : most), kThreads, 0, st>>>(a);
  return cudaGetLastError();
}

bool on16(const void* p, int64_t ld, int bytes) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * bytes) % 16 == 0; }

}  // namespace

extern "C" int fgd_dropout(int device, int dtype, int64_t rows, int64_t width, const void* x, int64_t ld_x, void* out, int64_t ld_out, double p, uint64_t seed,
                           uint64_t offset, const int64_t* counter, void* stream) {
  FGD_NVTX_RANGE("fgd_dropout");
  const int b = dtype_bytes(dtype);
  if (b == 0) return op_fail(FGD_ERR_INVALID_ARG, "fgd_dropout: unknown dtype %d", dtype);
  if (rows < 0 || rows > 0xffffffffll || width < 0 || width > 0x7fffffffll - 64)
    return op_fail(FGD_ERR_INVALID_ARG, "fgd_dropout: rows=%lld, width=%lld out of range", (long long)rows, (long long)width);
  if (!(p >= 0.0 && p < 1.0)) return op_fail(FGD_ERR_INVALID_ARG, "fgd_dropout: p=%g is not in [0, 1)", p);
  if (rows == 0 || width == 0) return FGD_OK;
  if (!x || !out) return op_fail(FGD_ERR_INVALID_ARG, "fgd_dropout: NULL pointer");
  if (ld_x < width || ld_out < width) return op_fail(FGD_ERR_INVALID_ARG, "fgd_dropout: a row stride is below the width");
  if (reinterpret_cast<uintptr_t>(x) % b != 0 || reinterpret_cast<uintptr_t>(out) % b != 0 || reinterpret_cast<uintptr_t>(counter) % 8 != 0)
    return op_fail(FGD_ERR_INVALID_ARG, "fgd_dropout: a pointer is not on a boundary of its elements");
  const Span so = span_of(out, rows, width, ld_out, b);
  if (so.overlaps(span_of(x, rows, width, ld_x, b)) && !(x == out && ld_x == ld_out)) return op_fail(FGD_ERR_ALIAS, "fgd_dropout: out overlaps x and is not x itself");
  if (so.overlaps(span_of(counter, 1, 1, 1, 8))) return op_fail(FGD_ERR_ALIAS, "fgd_dropout: out overlaps the counter");
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  DropoutArgs a = {};
  a.x = static_cast<const char*>(x); a.ld_x = ld_x; a.out = static_cast<char*>(out); a.ld_out = ld_out;
  a.rows = rows; a.width = width;
  a.k0 = (uint32_t)seed; a.k1 = (uint32_t)(seed >> 32);
  a.offset = offset; a.counter = counter;
  const double t = std::nearbyint(p * 4294967296.0);
  a.threshold = t > 4294967295.0 ? 4294967295u : (uint32_t)t;      // (2^32: p within 2^-33 of 1)
  a.scale = (float)(1.0 / (1.0 - p));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int64_t units = rows * ((width * b + 15) / 16);
  const bool aligned = (width * b) % 16 == 0 && on16(x, ld_x, b) && on16(out, ld_out, b);
  cudaError_t e;
  switch (dtype) {
    case FGD_F32: e = aligned ? go<dropout_kernel<float, false>>(a, units, 4, st) : go<dropout_kernel<float, true>>(a, units, 4, st); break;
    case FGD_BF16: e = aligned ? go<dropout_kernel<__nv_bfloat16, false>>(a, units, 4, st) : go<dropout_kernel<__nv_bfloat16, true>>(a, units, 4, st); break;
    default: e = aligned ? go<dropout_kernel<__half, false>>(a, units, 4, st) : go<dropout_kernel<__half, true>>(a, units, 4, st); break;
  }
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "fgd_dropout: launch failed: %s", cudaGetErrorString(e));
}

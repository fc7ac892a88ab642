// Activation types of the training operators and the few helpers that all of them use: 16-byte
// vectors of activations, their conversion to and from fp32, argument checks on the host.
#ifndef FGD_DTYPE_CUH_
#define FGD_DTYPE_CUH_

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "fgd_internal.h"

namespace fgd {

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// N consecutive activations as they lie in memory; 16 bytes (or one element on the element-wise paths).
template <typename T, int N>
struct alignas(sizeof(T) * N) ActPack {
  T v[N];
};
// Streaming access: activations are read once and written once per call, so they leave L1 alone.
template <typename T, int N>
__device__ __forceinline__ ActPack<T, N> load_stream(const T* p) {
  ActPack<T, N> r;
  if constexpr (sizeof(T) * N == 16) {
    *reinterpret_cast<uint4*>(&r) = __ldcs(reinterpret_cast<const uint4*>(p));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) r.v[i] = p[i];
  }
  return r;
}
template <typename T, int N>
__device__ __forceinline__ void store_stream(T* p, const ActPack<T, N>& r) {
  if constexpr (sizeof(T) * N == 16) {
    __stcs(reinterpret_cast<uint4*>(p), *reinterpret_cast<const uint4*>(&r));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = r.v[i];
  }
}

inline int op_fail(int status, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_thread_error, sizeof(g_thread_error), fmt, ap);
  va_end(ap);
  return status;
}

inline int dtype_bytes(int dtype) { return dtype == FGD_F32 ? 4 : (dtype == FGD_BF16 || dtype == FGD_F16) ? 2 : 0; }

// Selects the CUDA device for the duration of a call.
class DeviceScope {
 public:
  explicit DeviceScope(int device) {
    if (cudaGetDevice(&prev_) != cudaSuccess) { prev_ = -1; return; }
    ok_ = prev_ == device || cudaSetDevice(device) == cudaSuccess;
    moved_ = ok_ && prev_ != device;
  }
  ~DeviceScope() { if (moved_) cudaSetDevice(prev_); }
  DeviceScope(const DeviceScope&) = delete;
  DeviceScope& operator=(const DeviceScope&) = delete;
  bool ok() const { return ok_; }

 private:
  int prev_ = -1;
  bool ok_ = false, moved_ = false;
};

// SM count of the current device, asked for once per device.
inline int sm_count() {
  static int cached[64] = {};
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 1;
  if (dev < 64 && cached[dev]) return cached[dev];
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) n = 1;
  if (dev < 64) cached[dev] = n;
  return n;
}

// The bytes that a matrix of `rows` rows of `width` elements, `ld` apart, touches.
struct Span {
  uintptr_t lo = 0, hi = 0, ld = 0, width = 0;   // all in bytes; lo == hi: nothing
  bool overlaps(const Span& o) const {
    if (!(lo < hi && o.lo < o.hi && lo < o.hi && o.lo < hi)) return false;
    if (ld == o.ld && width <= ld && o.width <= ld) {   // column ranges of one larger matrix?
      const uintptr_t d = o.lo >= lo ? (o.lo - lo) % ld : (ld - (lo - o.lo) % ld) % ld;
      if (d >= width && d + o.width <= ld) return false;
    }
    return true;
  }
};
inline Span span_of(const void* p, int64_t rows, int64_t width, int64_t ld, int bytes) {
  Span s;
  if (p == nullptr || rows < 1 || width < 1) return s;
  s.lo = reinterpret_cast<uintptr_t>(p);
  s.hi = s.lo + (uintptr_t)(((rows - 1) * ld + width) * bytes);
  s.ld = (uintptr_t)(ld * bytes);
  s.width = (uintptr_t)(width * bytes);
  return s;
}

}  // namespace fgd
#endif

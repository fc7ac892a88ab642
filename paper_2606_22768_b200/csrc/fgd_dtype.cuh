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
#include <type_traits>
#include <utility>

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

// N consecutive activations as they lie in memory: 16 bytes.  Kept as whole words (as an array of 16-bit values the compiler gives
// each a register of its own and spends more instructions on taking the words apart and together than on the arithmetic).
template <typename T, int N>
struct ActPack {
  static_assert(sizeof(T) * N == 16, "a 16-byte vector");
  uint4 w;
};
// Streaming access: activations are read once and written once per call, so they leave L1 alone.
template <typename T, int N>
__device__ __forceinline__ ActPack<T, N> load_stream(const T* p) {
  return ActPack<T, N>{__ldcs(reinterpret_cast<const uint4*>(p))};
}
template <typename T, int N>
__device__ __forceinline__ void store_stream(T* p, const ActPack<T, N>& r) {
  __stcs(reinterpret_cast<uint4*>(p), r.w);
}
template <typename T, int N>
__device__ __forceinline__ void zero(ActPack<T, N>& r) {
  r.w = make_uint4(0u, 0u, 0u, 0u);
}

// Two fp32 operations per instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// N consecutive values as fp32, handled in pairs.
template <int N>
struct Vals {
  static_assert(N % 2 == 0, "pairs");
  float v[N];
  __device__ __forceinline__ float2 pair(int i) const { return make_float2(v[2 * i], v[2 * i + 1]); }
  __device__ __forceinline__ void set(int i, float2 p) { v[2 * i] = p.x; v[2 * i + 1] = p.y; }
};
// Two 16-bit values of a word.
template <typename T>
__device__ __forceinline__ float2 halves(uint32_t w) {
  if constexpr (std::is_same_v<T, __nv_bfloat16>) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  } else {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  }
}
template <typename T>
__device__ __forceinline__ uint32_t from_pair(float lo, float hi) {
  uint32_t w;
  if constexpr (std::is_same_v<T, __nv_bfloat16>) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}
template <typename T, int N>
__device__ __forceinline__ Vals<N> unpack(const ActPack<T, N>& p) {
  Vals<N> r;
  if constexpr (sizeof(T) == 4) {
    r.v[0] = __uint_as_float(p.w.x); r.v[1] = __uint_as_float(p.w.y); r.v[2] = __uint_as_float(p.w.z); r.v[3] = __uint_as_float(p.w.w);
  } else {
    r.set(0, halves<T>(p.w.x)); r.set(1, halves<T>(p.w.y)); r.set(2, halves<T>(p.w.z)); r.set(3, halves<T>(p.w.w));
  }
  return r;
}
template <typename T, int N>
__device__ __forceinline__ ActPack<T, N> round_to(const Vals<N>& a) {
  ActPack<T, N> r;
  if constexpr (sizeof(T) == 4) {
    r.w = make_uint4(__float_as_uint(a.v[0]), __float_as_uint(a.v[1]), __float_as_uint(a.v[2]), __float_as_uint(a.v[3]));
  } else {
    r.w = make_uint4(from_pair<T>(a.v[0], a.v[1]), from_pair<T>(a.v[2], a.v[3]), from_pair<T>(a.v[4], a.v[5]), from_pair<T>(a.v[6], a.v[7]));
  }
  return r;
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

// Programmatic dependent launch.  A kernel started with launch_early may begin while the kernel before it in the stream still runs,
// once every CTA of that one has called let_next_start (or has ended); wait_for_previous then waits for its end and its writes.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename... P, typename... A>
cudaError_t launch_early(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, A&&... args) {
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = grid;
  c.blockDim = dim3(threads);
  c.dynamicSmemBytes = smem;
  c.stream = st;
  c.attrs = &attr;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, kernel, P(std::forward<A>(args))...);
}

// Opts a kernel in to `smem` bytes of dynamic shared memory, once per kernel (KERNEL names the instance) and device.
template <auto KERNEL>
cudaError_t allow_smem(size_t smem) {
  static bool done[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && done[dev])) return e;
  e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess && dev < 64) done[dev] = true;
  return e;
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

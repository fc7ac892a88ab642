// Dropout whose mask is a function of (seed, offset, row, column) and is never stored:
//     out[r][c] = keep ? x[r][c] / (1 - p) : 0,   keep = word(r, c) >= p 2^32,
//     word(r, c) = word c % 4 of Philox4x32 with seven rounds, counter (c / 4, r, offset low, offset high), key (seed low, seed high)
// (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011; seven rounds are the fewest that pass their tests).
// The backward pass is the same call on the gradient.  A function of the row and column, not of the address: any width, stride, launch shape
// and device gives the same mask.
//
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

// The generator for one row.  Of the first two rounds' four products one depends on the offset alone and one on the row alone: they are made once.
struct RowWords {
  uint32_t low1, high2, low2, c3, k0, k1;
  __device__ __forceinline__ RowWords(uint32_t row, uint64_t offset, const DropoutArgs& a) : c3((uint32_t)(offset >> 32)), k0(a.k0), k1(a.k1) {
    const uint64_t q = (uint64_t)(uint32_t)offset * kM1;
    low1 = (uint32_t)q;
    const uint64_t p = (uint64_t)((uint32_t)(q >> 32) ^ row ^ k0) * kM0;
    high2 = (uint32_t)(p >> 32);
    low2 = (uint32_t)p;
  }
  // the four words of columns 4 c0 .. 4 c0 + 3
  __device__ __forceinline__ uint4 words(uint32_t group) const {
    const uint64_t p = (uint64_t)group * kM0;
    const uint64_t q = (uint64_t)((uint32_t)(p >> 32) ^ c3 ^ k1) * kM1;
    uint32_t a = (uint32_t)(q >> 32) ^ low1 ^ (k0 + kW0), b = (uint32_t)q, c = high2 ^ (uint32_t)p ^ (k1 + kW1), d = low2;
#pragma unroll
    for (uint32_t i = 2; i < 7; ++i) {
      const uint64_t s = (uint64_t)a * kM0, t = (uint64_t)c * kM1;
      a = (uint32_t)(t >> 32) ^ b ^ (k0 + i * kW0);
      b = (uint32_t)t;
      c = (uint32_t)(s >> 32) ^ d ^ (k1 + i * kW1);
      d = (uint32_t)s;
    }
    return make_uint4(a, b, c, d);
  }

 private:
  static constexpr uint32_t kM0 = 0xD2511F53u, kM1 = 0xCD9E8D57u, kW0 = 0x9E3779B9u, kW1 = 0xBB67AE85u;
};

// V values from column 4 group on.
template <int V>
__device__ __forceinline__ Vals<V> drop(const Vals<V>& x, uint32_t group, const RowWords& row, const DropoutArgs& a) {
  Vals<V> y;
#pragma unroll
  for (int g = 0; g < V / 4; ++g) {
    const uint4 w = row.words(group + g);
    const float2 lo = mul2(x.pair(2 * g), both(a.scale)), hi = mul2(x.pair(2 * g + 1), both(a.scale));
    y.v[4 * g] = w.x >= a.threshold ? lo.x : 0.f;
    y.v[4 * g + 1] = w.y >= a.threshold ? lo.y : 0.f;
    y.v[4 * g + 2] = w.z >= a.threshold ? hi.x : 0.f;
    y.v[4 * g + 3] = w.w >= a.threshold ? hi.y : 0.f;
  }
  return y;
}
// The generator's verdicts on V columns from column 4 group on, a bit each.
template <int V>
__device__ __forceinline__ uint32_t verdicts(uint32_t group, const RowWords& row, const DropoutArgs& a) {
  uint32_t keep = 0;
#pragma unroll
  for (int g = 0; g < V / 4; ++g) {
    const uint4 w = row.words(group + g);
    keep |= (w.x >= a.threshold ? 1u << 4 * g : 0u) | (w.y >= a.threshold ? 2u << 4 * g : 0u) | (w.z >= a.threshold ? 4u << 4 * g : 0u) | (w.w >= a.threshold ? 8u << 4 * g : 0u);
  }
  return keep;
}

// (volatile: not before the wait for the kernel that may have written it)
__device__ __forceinline__ uint64_t offset_of(const DropoutArgs& a) { return a.offset + (a.counter ? (uint64_t)*(const volatile int64_t*)a.counter : 0u); }

// A warp takes strips of kStrip x 32 chunks of 16 bytes of a row.  32768 x 4096 bf16: 86 us, 95 % of the copy peak (with one chunk a thread and nothing
// shared between them 106 us: bound by the generator's instructions).
// INSIDE: rows that start inside a chunk, x and out at the same place of one.  A row's chunks are then those of memory; its first and last are
// taken value by value.  Where columns of a chunk begin m behind a group of the generator, a lane makes V verdicts from that group on and gets
// the m that it lacks from the next lane.
constexpr int kStrip = 4;
// The values of a chunk at p that are columns of the row: c is the first one's.
template <typename T, int V>
__device__ __forceinline__ ActPack<T, V> load_some(const T* p, int c, int width) {
  Vals<V> v;
#pragma unroll
  for (int j = 0; j < V; ++j) v.v[j] = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (c + j >= 0 && c + j < width) v.v[j] = to_f32(p[j]);
  return round_to<T, V>(v);
}
template <typename T, int V>
__device__ __forceinline__ void store_some(T* p, const ActPack<T, V>& y, int c, int width) {
  const Vals<V> v = unpack<T, V>(y);
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (c + j >= 0 && c + j < width) p[j] = from_f32<T>(v.v[j]);
}
template <typename T, bool INSIDE>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropoutArgs a) {
  constexpr int V = 16 / sizeof(T), kColumns = 32 * kStrip * V;
  const int cta = wait_for_previous((int)blockIdx.x);
  const uint64_t offset = offset_of(a);
  const int lane = threadIdx.x & 31, strips = (int)((a.width + (INSIDE ? V - 1 : 0) + kColumns - 1) / kColumns);
  const int64_t total = a.rows * strips, stride = (int64_t)gridDim.x * (kThreads / 32);
  int64_t i = ((int64_t)cta * kThreads + threadIdx.x) / 32;
  Walk w(i, stride, strips);
  for (; i < total; i += stride, w.next()) {
    const T* x = reinterpret_cast<const T*>(a.x) + w.row * a.ld_x;
    T* out = reinterpret_cast<T*>(a.out) + w.row * a.ld_out;
    const int before = INSIDE ? (int)((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(T)) : 0;      // columns that the row's first chunk has before it
    const int c0 = (w.unit * (32 * kStrip) + lane) * V - before, width = (int)a.width;      // (they end below 2^31: see the launch)
    const RowWords row((uint32_t)w.row, offset, a);
    ActPack<T, V> raw[kStrip];
#pragma unroll
    for (int k = 0; k < kStrip; ++k) {
      const int c = c0 + k * 32 * V;
      if (!INSIDE ? c < width : c >= 0 && c + V <= width) raw[k] = load_stream<T, V>(x + c);
      else if (INSIDE && c > -V && c < width) raw[k] = load_some<T, V>(x + c, c, width);
    }
    if constexpr (INSIDE) {
      const int m = -before & 3;      // c0 - m is a multiple of 4 (-4 in a row's first chunk, where what is made of that group is not used)
      const int group = (c0 - m) >> 2, chunks = (width - c0 + lane * V + V - 1) / V;      // (of the row from this strip's first on: the same in all lanes)
      uint32_t keep[kStrip + 1];      // (also behind the row's last chunk where that is lane 31's: its last m columns belong to the group after its own)
#pragma unroll
      for (int k = 0; k <= kStrip; ++k)
        if (k * 32 <= chunks) keep[k] = k < kStrip ? verdicts<V>((uint32_t)(group + k * 8 * V), row, a) : verdicts<4>((uint32_t)(group + k * 8 * V), row, a);
#pragma unroll
      for (int k = 0; k < kStrip; ++k) {
        if (k * 32 >= chunks) break;
        const uint32_t above = __shfl_down_sync(0xffffffffu, keep[k], 1), first = (k + 1) * 32 <= chunks ? __shfl_sync(0xffffffffu, keep[k + 1], 0) : 0u;
        const uint32_t bits = (keep[k] | (lane == 31 ? first : above) << V) >> m;
        const int c = c0 + k * 32 * V;
        Vals<V> y = unpack<T, V>(raw[k]);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
          const float2 t = mul2(y.pair(j / 2), both(a.scale));
          y.v[j] = bits >> j & 1u ? t.x : 0.f;
          y.v[j + 1] = bits >> j & 2u ? t.y : 0.f;
        }
        if (c >= 0 && c + V <= width) store_stream<T, V>(out + c, round_to<T, V>(y));
        else if (c < width) store_some<T, V>(out + c, round_to<T, V>(y), c, width);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kStrip; ++k) {
        const int c = c0 + k * 32 * V;
        if (c < width) store_stream<T, V>(out + c, round_to<T, V>(drop<V>(unpack<T, V>(raw[k]), (uint32_t)c / 4, row, a)));
      }
    }
  }
}

// Every other row: units of 16 values, moved with shifts (fgd_units.cuh).  fp32 70 % of the copy peak, bf16 33 to 54 %: what the shifts and the generator cost
// in instructions.
template <typename T>
__global__ void __launch_bounds__(kThreads) dropout_shifted_kernel(const DropoutArgs a) {
  constexpr int V = 16;
  const int cta = wait_for_previous((int)blockIdx.x);
  const uint64_t offset = offset_of(a);
  const int units = (int)((a.width + V - 1) / V);
  const int64_t total = a.rows * units, padded = (total + 31) / 32 * 32, stride = (int64_t)gridDim.x * kThreads;      // whole warps stay for the shuffles
  const T* x = reinterpret_cast<const T*>(a.x);
  const T* end = x + (a.rows - 1) * a.ld_x + a.width;
  T* out = reinterpret_cast<T*>(a.out);
  int64_t i = (int64_t)cta * kThreads + threadIdx.x;
  Walk w(i, stride, units);
  for (; i < padded; i += stride, w.next()) {
    const ShiftedUnit<V> u(w, i < total, a.width);
    const Vals<V> v = load_shifted<T, V>(x + w.row * a.ld_x + u.c, u, x, end);
    const RowWords row((uint32_t)w.row, offset, a);
    store_shifted<T, V>(out + w.row * a.ld_out + u.c, u, drop<V>(v, (uint32_t)u.c / 4, row, a));
  }
}

template <auto KERNEL>
cudaError_t go(const DropoutArgs& a, int64_t threads, int waves, cudaStream_t st) {
  static int cached[64] = {};
  int dev = 0, fit = 0;
  const bool known = cudaGetDevice(&dev) == cudaSuccess && dev < 64;
  if (known) fit = cached[dev];
  if (fit == 0) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, KERNEL, kThreads, 0) != cudaSuccess || fit < 1) fit = 1;
    if (known) cached[dev] = fit;
  }
  const int64_t want = (threads + kThreads - 1) / kThreads, most = (int64_t)sm_count() * fit * waves;
  // (starting while the kernel before it ends saves 0.4 to 0.7 us, among other work 2)
  return launch_early(KERNEL, dim3((unsigned)(want < most ? want : most)), kThreads, 0, st, a);
}

bool on16(const void* p, int64_t ld, int bytes) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * bytes) % 16 == 0; }

}  // namespace

extern "C" int fgd_dropout(int device, int dtype, int64_t rows, int64_t width, const void* x, int64_t ld_x, void* out, int64_t ld_out, double p, uint64_t seed,
                           uint64_t offset, const int64_t* counter, void* stream) {
  FGD_NVTX_RANGE("fgd_dropout");
  const int b = dtype_bytes(dtype);
  if (b == 0) return op_fail(FGD_ERR_INVALID_ARG, "fgd_dropout: unknown dtype %d", dtype);
  if (rows < 0 || rows > 0xffffffffll || width < 0 || width > 0x7fffffffll - 4096)
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
  // 100 MB of bf16: strips where rows are on 16-byte boundaries and give a warp a full pass (256 columns 46 us against 57 by shifts, 128 columns 84
  // against 57); inside chunks where both sides lie alike and rows are long (3033 columns 58 against 68, 1025 92 against 72; fp32 37 against 42 and
  // 43 against 44); else by shifts.  CTAs for each place on the SMs: of 1, 4, 16, 64 for strips 92, 86, 90, 94 us (32768 x 4096), by shifts 35, 36, 39, 38
  // (5003 x 4097 fp32); chunks to a lane of a strip: of 2, 4, 8 92, 86, 93.
  const bool strips = (width * b) % 16 == 0 && width * b >= 32 * 16 && on16(x, ld_x, b) && on16(out, ld_out, b);
  const bool together = width * b >= 4096 && ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(out)) & 15u) == 0 && ((ld_x - ld_out) * b) % 16 == 0;
  auto launch = [&](auto zero) {
    using T = decltype(zero);
    constexpr int64_t V = 16 / sizeof(T), strip = 32 * kStrip * V;
    if (strips) return go<dropout_kernel<T, false>>(a, rows * ((width + strip - 1) / strip) * 32, 4, st);
    if (together) return go<dropout_kernel<T, true>>(a, rows * ((width + V - 1 + strip - 1) / strip) * 32, 4, st);
    return go<dropout_shifted_kernel<T>>(a, rows * ((width + 15) / 16), 1, st);
  };
  const cudaError_t e = dtype == FGD_F32 ? launch(float{}) : dtype == FGD_BF16 ? launch(__nv_bfloat16{}) : launch(__half{});
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "fgd_dropout: launch failed: %s", cudaGetErrorString(e));
}

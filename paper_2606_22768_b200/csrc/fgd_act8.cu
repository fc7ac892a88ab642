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
// All four are bound by HBM: one pass, every byte read or written once.  Measured, of the copy peak, bf16: save 96 %, load 90 % (32768 x
// 4096: 65 and 69 us), SwiGLU forward 88 %, backward 98 % (16384 x 5632: 130 and 144 us); fp32 save 95, load 85, SwiGLU 99 and 92 to 95.
//
// Vector kernels (rows and bases on 16-byte boundaries, width a multiple of 16 or 8): a thread takes 16 or 8
// consecutive values, two or four neighbouring lanes make a group, so the group's largest magnitude is one or two
// shuffles away.  Any other width, base or stride: 16 values to a lane as well, moved with shifts (fgd_units.cuh).
#include "fgd_dtype.cuh"
#include "fgd_nvtx.h"
#include "fgd_units.cuh"

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

// 1 / (1 + exp(-g)).
// fp32 activations: e = exp(-|g|) from the hardware's 2^x with what rounding -|g| log2 e lost put back, 1 / (1 + e) with one Newton step, and for
// g below 0 times e: the exponential's own 2^-22 and a few roundings, whatever the size of g, and nothing overflows (with -g log2 e as it
// is rounded the error grows with |g|, to 2^-18 at 60).  5957 x 5632 forward + backward 172 to 177 us, 4001 x 5003 179; the short form 171 to 173
// and 173, expf and a correctly rounded quotient 177 to 183 and 199.
// 16-bit ones: 1 / (1 + 2^(-g log2 e)) in short: 2^-20 (1 + |g|), far below their rounding; a denominator beyond fp32 gives 0.
template <typename T>
__device__ __forceinline__ float2 sigmoid2(float2 g) {
  constexpr float kHi = 1.4426950408889634f, kLo = (float)(1.4426950408889634074 - (double)kHi);
  if constexpr (sizeof(T) == 4) {
    float2 t = make_float2(-fabsf(g.x), -fabsf(g.y));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(t.x) : "f"(-128.f));      // (e is 0 there; an infinite y would lose infinitely much)
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(t.y) : "f"(-128.f));
    const float2 y = mul2(t, both(kHi));
    const float2 lost = fma2(t, both(kLo), fma2(t, both(kHi), mul2(y, both(-1.f))));
    float2 e = y;
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.x));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.y));
    e = fma2(e, mul2(lost, both(0.6931471805599453f)), e);
    const float2 d = add2(e, both(1.f));
    float2 r = d;
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r.x));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r.y));
    r = fma2(r, fma2(d, mul2(r, both(-1.f)), both(1.f)), r);
    const float2 n = mul2(e, r);
    return make_float2(g.x < 0.f ? n.x : r.x, g.y < 0.f ? n.y : r.y);
  }
  float2 x = mul2(g, both(-kHi));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(x.x));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(x.y));
  x = add2(x, both(1.f));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(x.x));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(x.y));
  return x;
}

// Largest magnitude bits over the 32 / V neighbouring lanes of a group.
template <int V>
__device__ __forceinline__ uint32_t group_max(uint32_t m) {
#pragma unroll
  for (int k = 1; k < kGroup / V; k <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, k));
  return m;
}

// V consecutive values starting at p, as fp32.
template <typename T, int V>
__device__ __forceinline__ Vals<V> load_vals(const T* p) {
  constexpr int N = 16 / sizeof(T);
  Vals<V> f;
#pragma unroll
  for (int j = 0; j < V; j += N) {
    const Vals<N> r = unpack<T, N>(load_stream<T, N>(p + j));
#pragma unroll
    for (int i = 0; i < N; ++i) f.v[j + i] = r.v[i];
  }
  return f;
}
template <typename T, int V>
__device__ __forceinline__ void store_vals(T* p, const Vals<V>& f) {
  constexpr int N = 16 / sizeof(T);
#pragma unroll
  for (int j = 0; j < V; j += N) {
    Vals<N> r;
#pragma unroll
    for (int i = 0; i < N; ++i) r.v[i] = f.v[j + i];
    store_stream<T, N>(p + j, round_to<T, N>(r));
  }
}
template <int V>
__device__ __forceinline__ Vals<V> no_vals() {
  Vals<V> f;
#pragma unroll
  for (int i = 0; i < V; ++i) f.v[i] = 0.f;
  return f;
}
// Largest magnitude of the values as bits; a NaN among them gives NaN bits.
template <int V>
__device__ __forceinline__ uint32_t amax_of(const Vals<V>& f) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < V; i += 2) asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(fabsf(f.v[i])), "f"(fabsf(f.v[i + 1])));
  return __float_as_uint(m);
}
// V stored bytes as they lie in memory: 4, 8 or 16.
template <int V>
using Bytes = std::conditional_t<V == 16, uint4, std::conditional_t<V == 8, uint2, uint32_t>>;
// Quantisation in the mantissa: x / step + 1.5 2^23 rounds to nearest-even at the units place, and the low byte of the sum's bits is
// q in two's complement.  No clamp is needed unless the largest magnitude reaches 127.5 steps, which the caller tells.
template <int V>
__device__ __forceinline__ Bytes<V> quantise(const Vals<V>& f, float inv, bool clamp) {
  const float2 inv2 = both(inv), magic = both(12582912.f);
  uint32_t w[V / 4];
#pragma unroll
  for (int j = 0; j < V / 4; ++j) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float2 y = fma2(f.pair(2 * j + i), inv2, magic);
      if (clamp) {
        y.x = fminf(fmaxf(y.x, 12582912.f - 127.f), 12582912.f + 127.f);
        y.y = fminf(fmaxf(y.y, 12582912.f - 127.f), 12582912.f + 127.f);
      }
      b[2 * i] = __float_as_uint(y.x);
      b[2 * i + 1] = __float_as_uint(y.y);
    }
    w[j] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  }
  if constexpr (V == 16) return make_uint4(w[0], w[1], w[2], w[3]);
  else return make_uint2(w[0], w[1]);
}
// Does a group with this largest magnitude reach 127.5 steps?  (mantissa at or above 127.5 / 128)
__device__ __forceinline__ bool tops_out(uint32_t amax_bits) { return (amax_bits & 0x7FFFFFu) >= 0x7F0000u; }
// And back: q + 128 in the low byte of 2^23 is 2^23 + 128 + q; the offset comes off before the step is applied, both exactly.  (One fused
// operation with offset x step would do, but that product is beyond fp32 for steps from 2^105 on: groups above 2^111.)
template <int V>
__device__ __forceinline__ Vals<V> dequantise(const Bytes<V>& q, float step) {
  uint32_t w[V / 4];
  if constexpr (V == 16) { w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w; }
  else if constexpr (V == 8) { w[0] = q.x; w[1] = q.y; }
  else w[0] = q;
  const float2 step2 = both(step), off = both(-8388736.f);
  Vals<V> f;
#pragma unroll
  for (int j = 0; j < V / 4; ++j) {
    const uint32_t u = w[j] ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 y = make_float2(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440 + 2 * i)), __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440 + 2 * i + 1)));
      f.set(2 * j + i, mul2(add2(y, off), step2));
    }
  }
  return f;
}

struct Act8Args {
  const void* x; int64_t ld_x;       // save: source; load: destination (non-const there)
  void* out; int64_t ld_out;
  int8_t* q; int64_t ld_q;
  uint8_t* e; int64_t ld_e;
  int64_t rows, width;
};

// ---- vector kernels: a unit is V values; every row is padded to whole groups, so that the lanes of a group always work together.
// V = 16 for 16-bit activations (16-byte stores of the checkpoint: save of 32768 x 4096 bf16 71.5 us against 78.6 with 8), 8 for fp32
// (57 against 60) and for widths that are not a multiple of 16.
template <typename T, int V>
__global__ void __launch_bounds__(kBlock8) act8_save_kernel(const Act8Args a) {
  constexpr int L = kGroup / V;      // lanes of a group
  const int units = (int)((a.width + kGroup - 1) / kGroup) * L;
  const int64_t total = a.rows * units, padded = (total + 31) / 32 * 32, stride = (int64_t)gridDim.x * kBlock8;   // whole warps stay in the loop for the shuffles
  int64_t i = (int64_t)blockIdx.x * kBlock8 + threadIdx.x;
  Walk w(i, stride, units);
  for (; i < padded; i += stride, w.next()) {
    const int c = w.unit * V;
    const bool real = i < total && c < a.width;
    const Vals<V> f = real ? load_vals<T, V>(static_cast<const T*>(a.x) + w.row * a.ld_x + c) : no_vals<V>();
    const uint32_t m = group_max<V>(amax_of<V>(f)), e = step_exponent(m);
    const Bytes<V> q = __any_sync(0xffffffffu, tops_out(m)) ? quantise<V>(f, inverse_step(e), true) : quantise<V>(f, inverse_step(e), false);
    if (real) __stcs(reinterpret_cast<Bytes<V>*>(a.q + w.row * a.ld_q + c), q);
    if (i < total && w.unit % L == 0) a.e[w.row * a.ld_e + w.unit / L] = (uint8_t)e;
  }
}
// Reading back, a thread takes what makes one 16-byte store, so that a warp's stores are whole lines (two stores 32 bytes apart cost
// 13 points of bandwidth), and has four such pieces on their way.
template <typename T>
__global__ void __launch_bounds__(kBlock8) act8_load_kernel(const Act8Args a) {
  constexpr int V = 16 / sizeof(T), L = kGroup / V, U = 4;
  const int units = (int)(a.width / V);
  const int64_t total = a.rows * units, stride = (int64_t)gridDim.x * kBlock8;
  int64_t i = (int64_t)blockIdx.x * kBlock8 + threadIdx.x;
  Walk w(i, stride, units);
  while (i < total) {
    Bytes<V> q[U];
    float step[U];
    T* out[U];
#pragma unroll
    for (int k = 0; k < U; ++k, i += stride, w.next()) {
      out[k] = nullptr;
      if (i >= total) continue;
      const int c = w.unit * V;
      q[k] = __ldcs(reinterpret_cast<const Bytes<V>*>(a.q + w.row * a.ld_q + c));
      step[k] = step_of(a.e[w.row * a.ld_e + w.unit / L]);
      out[k] = static_cast<T*>(a.out) + w.row * a.ld_out + c;
    }
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (out[k]) store_vals<T, V>(out[k], dequantise<V>(q[k], step[k]));
  }
}
template <typename T, int V>
__global__ void __launch_bounds__(kBlock8) swiglu8_forward_kernel(const Act8Args a) {
  constexpr int L = kGroup / V;
  const int groups = (int)((a.width + kGroup - 1) / kGroup), units = groups * L;
  const int64_t total = a.rows * units, padded = (total + 31) / 32 * 32, stride = (int64_t)gridDim.x * kBlock8;
  int64_t i = (int64_t)blockIdx.x * kBlock8 + threadIdx.x;
  Walk w(i, stride, units);
  for (; i < padded; i += stride, w.next()) {
    const int c = w.unit * V;
    const bool real = i < total && c < a.width;
    const T* row = static_cast<const T*>(a.x) + w.row * a.ld_x + c;
    const Vals<V> g = real ? load_vals<T, V>(row) : no_vals<V>(), u = real ? load_vals<T, V>(row + a.width) : no_vals<V>();
    const uint32_t mg = group_max<V>(amax_of<V>(g)), mu = group_max<V>(amax_of<V>(u)), eg = step_exponent(mg), eu = step_exponent(mu);
    Bytes<V> qg, qu;
    if (__any_sync(0xffffffffu, tops_out(mg) || tops_out(mu))) {
      qg = quantise<V>(g, inverse_step(eg), true);
      qu = quantise<V>(u, inverse_step(eu), true);
    } else {
      qg = quantise<V>(g, inverse_step(eg), false);
      qu = quantise<V>(u, inverse_step(eu), false);
    }
    if (real) {
      int8_t* q = a.q + w.row * a.ld_q + c;
      __stcs(reinterpret_cast<Bytes<V>*>(q), qg);
      __stcs(reinterpret_cast<Bytes<V>*>(q + a.width), qu);
      Vals<V> h;
#pragma unroll
      for (int j = 0; j < V / 2; ++j) h.set(j, mul2(mul2(g.pair(j), sigmoid2<T>(g.pair(j))), u.pair(j)));
      store_vals<T, V>(static_cast<T*>(a.out) + w.row * a.ld_out + c, h);
    }
    if (i < total && w.unit % L == 0) {
      uint8_t* e = a.e + w.row * a.ld_e + w.unit / L;
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
// h = g s u, du = dh g s, dg = dh u s (1 + g - g s)
template <typename T>
__device__ __forceinline__ void swiglu_back(float2 dh, float2 g, float2 u, float2& dg, float2& du, float2& h) {
  const float2 s = sigmoid2<T>(g), gs = mul2(g, s);
  h = mul2(gs, u);
  du = mul2(dh, gs);
  dg = mul2(mul2(mul2(dh, u), s), add2(fma2(gs, both(-1.f), g), both(1.f)));
}
template <typename T, int V>
__global__ void __launch_bounds__(kBlock8, 4) swiglu8_backward_kernel(const Swiglu8BackArgs a) {
  constexpr int L = kGroup / V;
  const int groups = (int)((a.width + kGroup - 1) / kGroup), units = (int)(a.width / V);
  const int64_t total = a.rows * units, stride = (int64_t)gridDim.x * kBlock8;
  int64_t i = (int64_t)blockIdx.x * kBlock8 + threadIdx.x;
  Walk w(i, stride, units);
  for (; i < total; i += stride, w.next()) {
    const int c = w.unit * V;
    const int8_t* q = a.q + w.row * a.ld_q + c;
    const uint8_t* e = a.e + w.row * a.ld_e + w.unit / L;
    const Bytes<V> qg = __ldcs(reinterpret_cast<const Bytes<V>*>(q)), qu = __ldcs(reinterpret_cast<const Bytes<V>*>(q + a.width));
    const Vals<V> dh = load_vals<T, V>(static_cast<const T*>(a.dh) + w.row * a.ld_dh + c);
    const Vals<V> g = dequantise<V>(qg, step_of(e[0])), u = dequantise<V>(qu, step_of(e[groups]));
    Vals<V> dg, du, h;
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      float2 x, y, z;
      swiglu_back<T>(dh.pair(j), g.pair(j), u.pair(j), x, y, z);
      dg.set(j, x); du.set(j, y); h.set(j, z);
    }
    T* out = static_cast<T*>(a.dgu) + w.row * a.ld_dgu + c;
    store_vals<T, V>(out, dg);
    store_vals<T, V>(out + a.width, du);
    if (a.h) store_vals<T, V>(static_cast<T*>(a.h) + w.row * a.ld_h + c, h);
  }
}

// ---- kernels for every other width, base and stride: a unit is 16 values, moved by fgd_units.cuh
constexpr int kAny = 16;
constexpr int kAnyWaves = 4;      // (1 to 8 are within 3 %, 16 is 6 % slower)
using AnyUnit = ShiftedUnit<kAny>;
__device__ __forceinline__ uint4 any_load8(const int8_t* p, const AnyUnit& u, const int8_t* lo, const int8_t* hi) {
  uint32_t w[4];
  load_unit<1, 4>(reinterpret_cast<const char*>(p), u.mine, u.has_next, reinterpret_cast<const char*>(lo), reinterpret_cast<const char*>(hi), w);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void any_store8(int8_t* p, const AnyUnit& u, uint4 q) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  store_unit<1, 4>(reinterpret_cast<char*>(p), u.valid, u.has_prev, u.has_next, w);
}

template <typename T>
__global__ void __launch_bounds__(kBlock8) act8_save_any_kernel(const Act8Args a) {
  const int units = (int)((a.width + kGroup - 1) / kGroup) * 2;
  const int64_t total = a.rows * units, padded = (total + 31) / 32 * 32, stride = (int64_t)gridDim.x * kBlock8;
  int64_t i = (int64_t)blockIdx.x * kBlock8 + threadIdx.x;
  Walk w(i, stride, units);
  const T* x = static_cast<const T*>(a.x);
  const T* end = x + (a.rows - 1) * a.ld_x + a.width;
  for (; i < padded; i += stride, w.next()) {
    const AnyUnit u(w, i < total, a.width);
    const Vals<kAny> f = load_shifted<T, kAny>(x + w.row * a.ld_x + u.c, u, x, end);
    const uint32_t m = group_max<kAny>(u.mine ? amax_of<kAny>(f) : 0u), e = step_exponent(m);
    const uint4 q = __any_sync(0xffffffffu, tops_out(m)) ? quantise<kAny>(f, inverse_step(e), true) : quantise<kAny>(f, inverse_step(e), false);
    any_store8(a.q + w.row * a.ld_q + u.c, u, q);
    if (i < total && w.unit % 2 == 0) a.e[w.row * a.ld_e + w.unit / 2] = (uint8_t)e;
  }
}
template <typename T>
__global__ void __launch_bounds__(kBlock8) act8_load_any_kernel(const Act8Args a) {
  const int units = (int)((a.width + kAny - 1) / kAny);
  const int64_t total = a.rows * units, padded = (total + 31) / 32 * 32, stride = (int64_t)gridDim.x * kBlock8;
  int64_t i = (int64_t)blockIdx.x * kBlock8 + threadIdx.x;
  Walk w(i, stride, units);
  const int8_t* end = a.q + (a.rows - 1) * a.ld_q + a.width;
  for (; i < padded; i += stride, w.next()) {
    const AnyUnit u(w, i < total, a.width);
    const float step = u.mine ? step_of(a.e[w.row * a.ld_e + w.unit / 2]) : 0.f;
    const uint4 q = any_load8(a.q + w.row * a.ld_q + u.c, u, a.q, end);
    store_shifted<T, kAny>(static_cast<T*>(a.out) + w.row * a.ld_out + u.c, u, dequantise<kAny>(q, step));
  }
}
template <typename T>
__global__ void __launch_bounds__(kBlock8) swiglu8_forward_any_kernel(const Act8Args a) {
  const int groups = (int)((a.width + kGroup - 1) / kGroup), units = groups * 2;
  const int64_t total = a.rows * units, padded = (total + 31) / 32 * 32, stride = (int64_t)gridDim.x * kBlock8;
  int64_t i = (int64_t)blockIdx.x * kBlock8 + threadIdx.x;
  Walk w(i, stride, units);
  const T* x = static_cast<const T*>(a.x);
  const T* end = x + (a.rows - 1) * a.ld_x + 2 * a.width;
  for (; i < padded; i += stride, w.next()) {
    const AnyUnit n(w, i < total, a.width);
    const T* row = x + w.row * a.ld_x + n.c;
    const Vals<kAny> g = load_shifted<T, kAny>(row, n, x, end), u = load_shifted<T, kAny>(row + a.width, n, x, end);
    const uint32_t mg = group_max<kAny>(n.mine ? amax_of<kAny>(g) : 0u), mu = group_max<kAny>(n.mine ? amax_of<kAny>(u) : 0u), eg = step_exponent(mg),
                   eu = step_exponent(mu);
    const bool clamp = __any_sync(0xffffffffu, tops_out(mg) || tops_out(mu));
    int8_t* q = a.q + w.row * a.ld_q + n.c;
    any_store8(q, n, clamp ? quantise<kAny>(g, inverse_step(eg), true) : quantise<kAny>(g, inverse_step(eg), false));
    any_store8(q + a.width, n, clamp ? quantise<kAny>(u, inverse_step(eu), true) : quantise<kAny>(u, inverse_step(eu), false));
    Vals<kAny> h;
#pragma unroll
    for (int j = 0; j < kAny / 2; ++j) h.set(j, mul2(mul2(g.pair(j), sigmoid2<T>(g.pair(j))), u.pair(j)));
    store_shifted<T, kAny>(static_cast<T*>(a.out) + w.row * a.ld_out + n.c, n, h);
    if (i < total && w.unit % 2 == 0) {
      uint8_t* e = a.e + w.row * a.ld_e + w.unit / 2;
      e[0] = (uint8_t)eg;
      e[groups] = (uint8_t)eu;
    }
  }
}
template <typename T>
__global__ void __launch_bounds__(kBlock8) swiglu8_backward_any_kernel(const Swiglu8BackArgs a) {
  const int groups = (int)((a.width + kGroup - 1) / kGroup), units = (int)((a.width + kAny - 1) / kAny);
  const int64_t total = a.rows * units, padded = (total + 31) / 32 * 32, stride = (int64_t)gridDim.x * kBlock8;
  int64_t i = (int64_t)blockIdx.x * kBlock8 + threadIdx.x;
  Walk w(i, stride, units);
  const T* dh = static_cast<const T*>(a.dh);
  const T* end = dh + (a.rows - 1) * a.ld_dh + a.width;
  const int8_t* end8 = a.q + (a.rows - 1) * a.ld_q + 2 * a.width;
  for (; i < padded; i += stride, w.next()) {
    const AnyUnit n(w, i < total, a.width);
    const int8_t* q = a.q + w.row * a.ld_q + n.c;
    const uint8_t* e = a.e + w.row * a.ld_e + w.unit / 2;
    const float sg = n.mine ? step_of(e[0]) : 0.f, su = n.mine ? step_of(e[groups]) : 0.f;
    const uint4 qg = any_load8(q, n, a.q, end8), qu = any_load8(q + a.width, n, a.q, end8);
    const Vals<kAny> d = load_shifted<T, kAny>(dh + w.row * a.ld_dh + n.c, n, dh, end), g = dequantise<kAny>(qg, sg), u = dequantise<kAny>(qu, su);
    Vals<kAny> dg, du, h;
#pragma unroll
    for (int j = 0; j < kAny / 2; ++j) {
      float2 x, y, z;
      swiglu_back<T>(d.pair(j), g.pair(j), u.pair(j), x, y, z);
      dg.set(j, x); du.set(j, y); h.set(j, z);
    }
    T* out = static_cast<T*>(a.dgu) + w.row * a.ld_dgu + n.c;
    store_shifted<T, kAny>(out, n, dg);
    store_shifted<T, kAny>(out + a.width, n, du);
    if (a.h) store_shifted<T, kAny>(static_cast<T*>(a.h) + w.row * a.ld_h + n.c, n, h);
  }
}

// Is the pointer on a boundary of its elements?  (Rows then are too.)
bool on_elements(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }
bool on16(const void* p, int64_t ld, int bytes) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * bytes) % 16 == 0; }
// Values per thread that width, base and stride of the stored bytes allow: 16 (16-bit activations), 8, or none (0).
int unit_for(int dtype, const void* q, int64_t ld, int64_t width) {
  for (int v : {16, 8})
    if ((v == 8 || dtype != FGD_F32) && width % v == 0 && ld % v == 0 && (reinterpret_cast<uintptr_t>(q) & (uintptr_t)(v - 1)) == 0) return v;
  return 0;
}

int check_dims(const char* who, int dtype, int64_t rows, int64_t width) {
  if (dtype_bytes(dtype) == 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (rows < 0 || width < 0 || width > ((int64_t)1 << 29)) return op_fail(FGD_ERR_INVALID_ARG, "%s: rows=%lld, width=%lld out of range", who, (long long)rows, (long long)width);
  return FGD_OK;
}

// Launches KERNEL with threads enough to cover the work, at most `waves` times as many CTAs as run at once: they stride over the rest.
// What is best was measured, per kernel, over 1 to 64 waves: the kernels that write least or most against what they read want many short
// CTAs, which the hardware hands out as others end (bf16, 32768 x 4096 save: 71 us with 1 wave, 65 with 8 and 16, 67 with 32; 16384 x 5632
// SwiGLU backward 190, 154 with 8, 149 with 16, 153 with 32); the other two want one wave (load 69, 73 with 8, 82 with 32; SwiGLU
// forward 131 and 135; but with fp32 16 waves, forward + backward of 5957 x 5632 182 with one, 170 so).
template <auto KERNEL, typename A>
void go(int waves, int64_t threads, cudaStream_t st, const A& a) {
  static int cached[64] = {};
  int dev = 0, fit = 0;
  const bool known = cudaGetDevice(&dev) == cudaSuccess && dev < 64;
  if (known) fit = cached[dev];
  if (fit == 0) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, KERNEL, kBlock8, 0) != cudaSuccess || fit < 1) fit = 1;
    if (known) cached[dev] = fit;
  }
  const int64_t want = (threads + kBlock8 - 1) / kBlock8, most = (int64_t)sm_count() * fit * waves;
  KERNEL<<<(unsigned)(want < most ? want : most), kBlock8, 0, st>>>(a);
}

int launched(const char* who) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

// f(a value of the activation type)
template <typename F>
void by_dtype(int dtype, F f) {
  if (dtype == FGD_F32) f(float{});
  else if (dtype == FGD_BF16) f(__nv_bfloat16{});
  else f(__half{});
}
// KERNEL<type, 16 or 8 values per thread>, or KERNEL_any<type> where `unit` is 0.
#define FGD_LAUNCH_DTYPE(KERNEL, WAVES, THREADS16, THREADS8)                                              \
  by_dtype(dtype, [&](auto zero) {                                                                         \
    using T = decltype(zero);                                                                              \
    if constexpr (sizeof(T) == 2)                                                                          \
      if (unit == 16) { go<KERNEL##_kernel<T, 16>>(WAVES, THREADS16, st, a); return; }                     \
    if (unit == 8) go<KERNEL##_kernel<T, 8>>(WAVES, THREADS8, st, a);                                      \
    else go<KERNEL##_any_kernel<T>>(kAnyWaves, rows * groups * 2, st, a);                                  \
  });

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
  if (!on_elements(x, b)) return op_fail(FGD_ERR_INVALID_ARG, "fgd_act_save8: a pointer is not on a boundary of its elements");
  const Span sx = span_of(x, rows, width, ld_x, b), sq = span_of(q8, rows, width, ld_q, 1), se = span_of(e8, rows, groups, ld_e, 1);
  if (sx.overlaps(sq) || sx.overlaps(se) || sq.overlaps(se)) return op_fail(FGD_ERR_ALIAS, "fgd_act_save8: tensors overlap");
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  const Act8Args a{x, ld_x, nullptr, 0, q8, ld_q, e8, ld_e, rows, width};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int unit = on16(x, ld_x, b) ? unit_for(dtype, q8, ld_q, width) : 0;
  FGD_LAUNCH_DTYPE(act8_save, 8, rows * groups * 2, rows * groups * 4)
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
  if (!on_elements(out, b)) return op_fail(FGD_ERR_INVALID_ARG, "fgd_act_load8: a pointer is not on a boundary of its elements");
  const Span so = span_of(out, rows, width, ld_out, b);
  if (so.overlaps(span_of(q8, rows, width, ld_q, 1)) || so.overlaps(span_of(e8, rows, groups, ld_e, 1))) return op_fail(FGD_ERR_ALIAS, "fgd_act_load8: tensors overlap");
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  const Act8Args a{nullptr, 0, out, ld_out, const_cast<int8_t*>(q8), ld_q, const_cast<uint8_t*>(e8), ld_e, rows, width};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int unit = on16(out, ld_out, b) ? unit_for(dtype, q8, ld_q, width) : 0;
  by_dtype(dtype, [&](auto zero) {
    using T = decltype(zero);
    if (unit) go<act8_load_kernel<T>>(1, rows * (width * (int64_t)sizeof(T) / 16), st, a);
    else go<act8_load_any_kernel<T>>(kAnyWaves, rows * groups * 2, st, a);
  });
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
  if (!on_elements(gu, b) || !on_elements(h, b)) return op_fail(FGD_ERR_INVALID_ARG, "fgd_swiglu8_forward: a pointer is not on a boundary of its elements");
  const Span sx = span_of(gu, rows, 2 * width, ld_gu, b), sh = span_of(h, rows, width, ld_h, b), sq = span_of(q8, rows, 2 * width, ld_q, 1),
             se = span_of(e8, rows, 2 * groups, ld_e, 1);
  if (sx.overlaps(sh) || sx.overlaps(sq) || sx.overlaps(se) || sh.overlaps(sq) || sh.overlaps(se) || sq.overlaps(se))
    return op_fail(FGD_ERR_ALIAS, "fgd_swiglu8_forward: tensors overlap");
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  const Act8Args a{gu, ld_gu, h, ld_h, q8, ld_q, e8, ld_e, rows, width};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int unit = on16(gu, ld_gu, b) && on16(h, ld_h, b) ? unit_for(dtype, q8, ld_q, width) : 0;
  FGD_LAUNCH_DTYPE(swiglu8_forward, sizeof(T) == 4 ? 16 : 1, rows * groups * 2, rows * groups * 4)
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
  if (!on_elements(dh, b) || !on_elements(dgu, b) || !on_elements(h, b)) return op_fail(FGD_ERR_INVALID_ARG, "fgd_swiglu8_backward: a pointer is not on a boundary of its elements");
  const Span sd = span_of(dh, rows, width, ld_dh, b), so = span_of(dgu, rows, 2 * width, ld_dgu, b), sh = span_of(h, rows, width, ld_h, b),
             sq = span_of(q8, rows, 2 * width, ld_q, 1), se = span_of(e8, rows, 2 * groups, ld_e, 1);
  if (so.overlaps(sd) || so.overlaps(sh) || so.overlaps(sq) || so.overlaps(se) || sh.overlaps(sd) || sh.overlaps(sq) || sh.overlaps(se))
    return op_fail(FGD_ERR_ALIAS, "fgd_swiglu8_backward: tensors overlap");
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  const Swiglu8BackArgs a{dh, ld_dh, q8, ld_q, e8, ld_e, dgu, ld_dgu, h, ld_h, rows, width};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int unit = on16(dh, ld_dh, b) && on16(dgu, ld_dgu, b) && (!h || on16(h, ld_h, b)) ? unit_for(dtype, q8, ld_q, width) : 0;
  FGD_LAUNCH_DTYPE(swiglu8_backward, 16, rows * (width / 16), rows * (width / 8))
  return launched("fgd_swiglu8_backward");
}

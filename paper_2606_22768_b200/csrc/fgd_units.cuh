// Units of N consecutive values of a row: how a kernel's threads walk over all rows' units, and units of rows that start anywhere in
// memory (fgd_shift.cuh).
#ifndef FGD_UNITS_CUH_
#define FGD_UNITS_CUH_

#include "fgd_dtype.cuh"
#include "fgd_shift.cuh"

namespace fgd {

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

template <typename T, int N>
constexpr int kUnitWords = N * (int)sizeof(T) / 4;

// Unit (row, unit) of a lane in the padded walk, and who its neighbours in the warp are.
template <int N>
struct ShiftedUnit {
  int c, left, valid;            // first column; columns from there to the row's end, clipped to [-N, N]
  bool mine, has_prev, has_next;
  __device__ __forceinline__ ShiftedUnit(const Walk& w, bool in_range, int64_t width) {
    const int lane = threadIdx.x & 31;
    c = w.unit * N;
    const int64_t l = width - c;
    left = (int)(l > N ? N : l < -N ? -N : l);
    mine = in_range && left > 0;
    valid = mine ? left : -4 * N;   // (of a lane without a unit nothing is stored)
    has_prev = lane > 0 && w.unit > 0;
    has_next = mine && lane < 31 && l > N;
  }
};
template <typename T, int N>
__device__ __forceinline__ Vals<N> unit_vals(const uint32_t (&w)[kUnitWords<T, N>], int left) {
  Vals<N> f;
#pragma unroll
  for (int i = 0; i < kUnitWords<T, N>; ++i) {
    if constexpr (sizeof(T) == 4) f.v[i] = __uint_as_float(w[i]);
    else f.set(i, halves<T>(w[i]));
  }
  if (left < N) {             // beyond the row: the next row's values, or none
#pragma unroll
    for (int i = 0; i < N; ++i) f.v[i] = i < left ? f.v[i] : 0.f;
  }
  return f;
}
template <typename T, int N>
__device__ __forceinline__ Vals<N> load_shifted(const T* p, const ShiftedUnit<N>& u, const T* lo, const T* hi) {
  uint32_t w[kUnitWords<T, N>];
  load_unit<sizeof(T), kUnitWords<T, N>>(reinterpret_cast<const char*>(p), u.mine, u.has_next, reinterpret_cast<const char*>(lo), reinterpret_cast<const char*>(hi), w);
  return unit_vals<T, N>(w, u.left);
}
template <typename T, int N>
__device__ __forceinline__ void store_shifted(T* p, const ShiftedUnit<N>& u, const Vals<N>& f) {
  uint32_t w[kUnitWords<T, N>];
#pragma unroll
  for (int i = 0; i < kUnitWords<T, N>; ++i) {
    if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(f.v[i]);
    else w[i] = from_pair<T>(f.v[2 * i], f.v[2 * i + 1]);
  }
  store_unit<sizeof(T), kUnitWords<T, N>>(reinterpret_cast<char*>(p), u.valid * (int)sizeof(T), u.has_prev, u.has_next, w);
}

}  // namespace fgd
#endif

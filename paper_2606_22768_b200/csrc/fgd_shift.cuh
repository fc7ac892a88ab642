// Rows that start anywhere in memory, moved in 16-byte chunks all the same.
//
// Lane i of a warp owns a unit: 4 NW consecutive bytes, those after lane i - 1's where both lie in one row.  A unit starts s bytes
// behind a 16-byte boundary.  Reading, a lane fetches the chunks from that boundary on, gets the one after its last from the next
// lane, and takes its unit out of the two with funnel shifts; writing, it takes the end of the unit before its own from the
// previous lane.  Only where a row, or the warp's part of it, begins or ends inside a chunk are fewer than 16 bytes written.
// What it gave against one element per lane and access, in % of the copy peak at odd widths, bf16: 8-bit save + load 16 to 50 (777 columns),
// SwiGLU 28 to 46, block norm forward 14 to 42 (1001 columns) and 33 (5003), backward 9 to 34 and 23.  What is left is the shifting itself
// and the cut chunks, not memory: 16-byte aligned rows reach 67 to 90.
// Bytes around a row are read with it, but none outside [lo, hi), the tensor; only the unit's own are ever written.
#ifndef FGD_SHIFT_CUH_
#define FGD_SHIFT_CUH_

#include <cstdint>
#include <type_traits>

namespace fgd {

// r = the 4 N bytes of x from byte k on, 0 <= k <= 16.  The lanes of a row agree on k, so the word offset is a branch that all of them
// take: N funnel shifts instead of 3 N selects before them.
template <int N>
__device__ __forceinline__ void shift_words(const uint32_t (&x)[N + 4], uint32_t k, uint32_t (&r)[N]) {
  const uint32_t bits = 8 * (k & 3);
  auto from = [&](auto offset) {
    constexpr int W = decltype(offset)::value;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = __funnelshift_r(x[i + W], x[i + W + 1 < N + 4 ? i + W + 1 : N + 3], bits);
  };
  switch (k >> 2) {
    case 0: from(std::integral_constant<int, 0>{}); break;
    case 1: from(std::integral_constant<int, 1>{}); break;
    case 2: from(std::integral_constant<int, 2>{}); break;
    case 3: from(std::integral_constant<int, 3>{}); break;
    default: from(std::integral_constant<int, 4>{}); break;      // k == 16
  }
}

template <int ES>
__device__ __forceinline__ uint32_t load_elem(const char* p) {
  if constexpr (ES == 4) return *reinterpret_cast<const uint32_t*>(p);
  else if constexpr (ES == 2) return *reinterpret_cast<const uint16_t*>(p);
  else return *reinterpret_cast<const uint8_t*>(p);
}
template <int ES>
__device__ __forceinline__ void store_elem(char* p, uint32_t v) {
  if constexpr (ES == 4) *reinterpret_cast<uint32_t*>(p) = v;
  else if constexpr (ES == 2) *reinterpret_cast<uint16_t*>(p) = (uint16_t)v;
  else *reinterpret_cast<uint8_t*>(p) = (uint8_t)v;
}

// The unit at p, elements of ES bytes; all lanes of the warp call it together.  `mine`: the lane has a unit; has_next: so has the next
// lane, right behind this one.  Elements of the unit beyond its row come back as whatever is there.
template <int ES, int NW>
__device__ __forceinline__ void load_unit(const char* p, bool mine, bool has_next, const char* lo, const char* hi, uint32_t (&r)[NW]) {
  constexpr int C = NW / 4;
  const uint32_t s = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u);
  const char* base = p - s;
  uint32_t x[NW + 4];
#pragma unroll
  for (int j = 0; j <= C; ++j) {
    uint4 c = make_uint4(0u, 0u, 0u, 0u);
    if (mine && (j < C || (s != 0 && !has_next)) && base + 16 * j >= lo && base + 16 * j + 16 <= hi) c = __ldcs(reinterpret_cast<const uint4*>(base) + j);
    x[4 * j] = c.x; x[4 * j + 1] = c.y; x[4 * j + 2] = c.z; x[4 * j + 3] = c.w;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t next = __shfl_down_sync(0xffffffffu, x[i], 1);
    if (has_next) x[NW + i] = next;
  }
  shift_words<NW>(x, s, r);
  if (mine && (base < lo || base + 4 * NW + 16 > hi)) {      // the tensor's first and last units, element by element
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      r[i] = 0u;
#pragma unroll
      for (int b = 0; b < 4; b += ES)
        if (p + 4 * i + b < hi) r[i] |= load_elem<ES>(p + 4 * i + b) << (8 * b);
    }
  }
}

// Bytes [from, 16) or [0, to) of the chunk w at p, in pieces of 8, 4, 2 and 1 bytes.
template <int ES>
__device__ __forceinline__ void store_end_of_chunk(char* p, const uint32_t (&w)[4], uint32_t from) {
  if constexpr (ES == 1)
    if (from & 1) {
      const uint32_t v = from & 8 ? (from & 4 ? w[3] : w[2]) : (from & 4 ? w[1] : w[0]);
      store_elem<1>(p + from, v >> (8 * (from & 3)));
      ++from;
    }
  if constexpr (ES <= 2)
    if (from & 2) {
      const uint32_t v = from & 8 ? (from & 4 ? w[3] : w[2]) : (from & 4 ? w[1] : w[0]);
      store_elem<2>(p + from, v >> 16);
      from += 2;
    }
  if (from & 4) {
    store_elem<4>(p + from, from & 8 ? w[3] : w[1]);
    from += 4;
  }
  if (from & 8) *reinterpret_cast<uint2*>(p + 8) = make_uint2(w[2], w[3]);
}
template <int ES>
__device__ __forceinline__ void store_start_of_chunk(char* p, const uint32_t (&w)[4], uint32_t to) {
  if (to & 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  if (to & 4) store_elem<4>(p + (to & 8), to & 8 ? w[2] : w[0]);
  const uint32_t v = to & 8 ? (to & 4 ? w[3] : w[2]) : (to & 4 ? w[1] : w[0]);
  if constexpr (ES <= 2)
    if (to & 2) store_elem<2>(p + (to & 12), v);
  if constexpr (ES == 1)
    if (to & 1) store_elem<1>(p + (to & 14), to & 2 ? v >> 16 : v);
}

// Writes the unit w at p; all lanes of the warp call it together.  `valid`: the bytes from p to the end of the row (a lane whose p
// lies beyond it passes a negative count); has_prev: the previous lane's unit lies right before this one; has_next: the next lane
// takes what this unit leaves over of its last chunk, though its own unit may lie beyond the row.
template <int ES, int NW>
__device__ __forceinline__ void store_unit(char* p, int valid, bool has_prev, bool has_next, const uint32_t (&w)[NW]) {
  constexpr int C = NW / 4;
  const int s = (int)(reinterpret_cast<uintptr_t>(p) & 15u), bytes = s + (valid < 4 * NW ? valid : 4 * NW);     // from the first chunk's start
  char* base = p - s;
  uint32_t x[NW + 8], r[NW + 4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = __shfl_up_sync(0xffffffffu, w[NW - 4 + i], 1);
    x[NW + 4 + i] = 0u;
  }
#pragma unroll
  for (int i = 0; i < NW; ++i) x[4 + i] = w[i];
  shift_words<NW + 4>(x, 16 - s, r);
  const bool cut = s != 0 && !has_prev;      // the first chunk begins with bytes that are not ours
#pragma unroll
  for (int j = 0; j < C; ++j)
    if (16 * j + 16 <= bytes && !(j == 0 && cut)) __stcs(reinterpret_cast<uint4*>(base) + j, make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]));
  if (cut && valid > 0) {
    uint32_t c[4] = {r[0], r[1], r[2], r[3]};
    if (bytes >= 16) {
      store_end_of_chunk<ES>(base, c, s);
    } else {                                 // a row inside one chunk
#pragma unroll
      for (int b = 0; b < 16; b += ES)
        if (b >= s && b < bytes) store_elem<ES>(base + b, c[b / 4] >> (8 * (b % 4)));
    }
  }
  const int last = bytes >> 4;
  if (bytes > 0 && (bytes & 15) && (last < C || !has_next) && !(last == 0 && cut)) {
    uint32_t c[4] = {r[0], r[1], r[2], r[3]};
#pragma unroll
    for (int j = 1; j <= C; ++j)
      if (last == j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = r[4 * j + i];
      }
    store_start_of_chunk<ES>(base + 16 * last, c, (uint32_t)(bytes & 15));
  }
}

}  // namespace fgd
#endif

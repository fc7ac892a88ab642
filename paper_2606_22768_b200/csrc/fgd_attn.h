// Causal attention over packed sequences: what the entry points, the tensor-core kernels and the
// element-wise kernels share.
#ifndef FGD_ATTN_H_
#define FGD_ATTN_H_

#include <cuda_runtime.h>

#include <cstdint>

#include "fgd.h"

namespace fgd {

// A tile of rows of one sequence.  Tiles do not depend on heads or widths: a CTA's (tile, head) pair
// comes from its index.
struct alignas(16) AttnTile {
  int32_t start;   // first token of the sequence
  int32_t len;     // tokens of the sequence
  int32_t row;     // first row of the tile, counted from the sequence's start
  int32_t unused;
};

constexpr int kAttnRows = 128;   // rows of a tile
constexpr uint32_t kAttnSpin = 1u << 22;   // polls before a wait gives up

struct AttnHeads {
  char* p;
  int64_t token, head;   // strides in elements
};

struct AttnArgs {
  AttnHeads q, k, v, o, dout, dq, dk, dv;
  float* lse;      // [n_q_heads, tokens]
  float* delta;    // [n_q_heads, tokens]: sum over the width of o * dout
  int64_t tokens;
  int hq, hk, d;
  float scale, inv_group;   // inv_group: n_kv_heads / n_q_heads
  const AttnTile* tiles;
  int n_tiles;
  int* status;
  uint32_t spin_limit;   // polls before a wait gives up
  int skip;              // test hook: the streamed tile of every CTA whose load is announced but not issued (-1: none)
};

}  // namespace fgd

// Tiles in the order in which CTAs take them: most work first.
struct fgd_attn_plan {
  int device = 0;
  int64_t tokens = 0;
  int n_q = 0, n_q2 = 0, n_kv = 0;
  fgd::AttnTile* q_tiles = nullptr;    // 128 rows each, by descending row (a row meets the keys before it)
  fgd::AttnTile* q2_tiles = nullptr;   // 256 rows each
  fgd::AttnTile* kv_tiles = nullptr;   // 128 rows each, by descending number of rows that follow
  int* status = nullptr;               // set by a device-side wait that gave up
  void* encode_tiled = nullptr;        // cuTensorMapEncodeTiled
  uint32_t dbg_spin_limit = 0;         // fgd_attn_debug_set: 0 = the default
  int dbg_skip = -1;
};

namespace fgd {
// Element-wise kernels: any type, stride and width up to kAttnElemMaxDim.
constexpr int kAttnElemMaxDim = 256;
int attn_forward_elem(const fgd_attn_plan* plan, int dtype, const AttnArgs& a, cudaStream_t st);
int attn_backward_elem(const fgd_attn_plan* plan, int dtype, const AttnArgs& a, cudaStream_t st);
// Tensor-core kernels: bf16 and fp16, width a multiple of 8 up to 128, 16-byte rows, scale > 0.
int attn_forward_tc(const fgd_attn_plan* plan, int dtype, const AttnArgs& a, cudaStream_t st);
int attn_backward_tc(const fgd_attn_plan* plan, int dtype, const AttnArgs& a, cudaStream_t st);
// delta of every (token, head); `vectors`: o and dout are 16-bit, in 16-byte vectors, at most 128 wide (then, in fp16, also what
// the tensor-core kernels choose their factors' scale from, in delta and dq)
int attn_delta(const fgd_attn_plan* plan, int dtype, bool vectors, AttnArgs a, cudaStream_t st);
}  // namespace fgd
#endif

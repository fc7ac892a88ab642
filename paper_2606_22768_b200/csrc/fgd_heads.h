// Host-side checks of [tokens, heads, head_dim] tensors.
#ifndef FGD_HEADS_H_
#define FGD_HEADS_H_

#include "fgd_dtype.cuh"

namespace fgd {

struct HeadsArg { const char* name; const fgd_heads* t; int heads; bool output; };

// The bytes of a [tokens, heads, d] tensor as a two-level layout: the axis with the larger stride outside.
inline Span heads_span(const fgd_heads& t, int64_t tokens, int heads, int d, int bytes) {
  const bool token_major = heads == 1 || t.token_stride >= t.head_stride;
  if (token_major) return span_of(t.p, tokens, (heads - 1) * t.head_stride + d, t.token_stride, bytes);
  return span_of(t.p, heads, (tokens - 1) * t.token_stride + d, t.head_stride, bytes);
}

inline int check_heads(const char* who, const HeadsArg& h, int64_t tokens, int d, int bytes) {
  if (!h.t->p) return op_fail(FGD_ERR_INVALID_ARG, "%s: %s is NULL", who, h.name);
  if (reinterpret_cast<uintptr_t>(h.t->p) % bytes != 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: %s is not on a boundary of its elements", who, h.name);
  const int64_t ts = h.t->token_stride, hs = h.t->head_stride;
  if (ts < 0 || hs < 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: %s has a negative stride", who, h.name);
  if (!h.output) return FGD_OK;
  // rows of an output may not overlap one another
  const bool token_major = h.heads == 1 || ts >= hs;
  const int64_t inner = token_major ? hs : ts, outer = token_major ? ts : hs, n_in = token_major ? h.heads : tokens, n_out = token_major ? tokens : h.heads;
  if ((n_in > 1 && inner < d) || (n_out > 1 && outer < (n_in - 1) * inner + d))
    return op_fail(FGD_ERR_INVALID_ARG, "%s: rows of %s overlap one another (strides %lld, %lld)", who, h.name, (long long)ts, (long long)hs);
  return FGD_OK;
}

}  // namespace fgd
#endif

// Entry points of causal attention over packed sequences with grouped heads: the plan (which tiles exist and
// in which order CTAs take them), the checks of arguments, and the choice of kernels.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "fgd_attn.h"
#include "fgd_attn_tc.cuh"
#include "fgd_dtype.cuh"
#include "fgd_heads.h"
#include "fgd_nvtx.h"

using namespace fgd;

namespace {

int check_common(const char* who, const fgd_attn_plan* plan, const fgd_attn_args* b) {
  if (!plan || !b) return op_fail(FGD_ERR_INVALID_ARG, "%s: NULL plan or arguments", who);
  if (dtype_bytes(b->dtype) == 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: unknown dtype %d", who, b->dtype);
  if (b->n_q_heads < 1 || b->n_kv_heads < 1 || b->n_q_heads % b->n_kv_heads != 0 || b->n_q_heads > 32768)
    return op_fail(FGD_ERR_INVALID_ARG, "%s: %d query heads do not share %d key heads", who, b->n_q_heads, b->n_kv_heads);
  if (b->head_dim < 1) return op_fail(FGD_ERR_INVALID_ARG, "%s: head_dim %d", who, b->head_dim);
  if (b->head_dim > kAttnElemMaxDim) return op_fail(FGD_ERR_UNSUPPORTED, "%s: head_dim %d above %d", who, b->head_dim, kAttnElemMaxDim);
  if (!std::isfinite(b->scale)) return op_fail(FGD_ERR_INVALID_ARG, "%s: scale is not finite", who);
  if (!b->lse && plan->tokens > 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: lse is NULL", who);
  if (reinterpret_cast<uintptr_t>(b->lse) % sizeof(float) != 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: lse is not on a boundary of its elements", who);
  return FGD_OK;
}

AttnHeads heads_of(const fgd_heads& t) { return AttnHeads{static_cast<char*>(t.p), t.token_stride, t.head_stride}; }

AttnArgs kernel_args(const fgd_attn_plan* plan, const fgd_attn_args* b) {
  AttnArgs a = {};
  a.q = heads_of(b->q); a.k = heads_of(b->k); a.v = heads_of(b->v); a.o = heads_of(b->o);
  a.dout = heads_of(b->dout); a.dq = heads_of(b->dq); a.dk = heads_of(b->dk); a.dv = heads_of(b->dv);
  a.lse = b->lse; a.delta = b->delta; a.tokens = plan->tokens;
  a.hq = b->n_q_heads; a.hk = b->n_kv_heads; a.d = b->head_dim; a.scale = (float)b->scale;
  a.inv_group = (float)b->n_kv_heads / (float)b->n_q_heads;
  a.status = plan->status;
  a.spin_limit = plan->dbg_spin_limit ? plan->dbg_spin_limit : kAttnSpin;
  a.skip = plan->dbg_skip;
  return a;
}

// The tensor-core kernels read their inputs by TMA (16-byte rows) and need a positive scale (the maximum of the scores is
// found before they are scaled; a masked score is -inf).
bool on_tensor_cores(const fgd_attn_plan* plan, const fgd_attn_args* b, const HeadsArg* all, int n) {
  if (!plan->encode_tiled || dtype_bytes(b->dtype) != 2 || b->head_dim % 8 != 0 || b->head_dim > 128 || !(b->scale >= 1e-20)) return false;
  for (int i = 0; i < n; ++i)
    if (!attn_tc_heads(heads_of(*all[i].t), plan->tokens, all[i].heads)) return false;
  return true;
}

}  // namespace

extern "C" int fgd_attn_plan_create(fgd_attn_plan** out, int device, int n_seqs, const int64_t* cu_seqlens) {
  if (!out) return op_fail(FGD_ERR_INVALID_ARG, "fgd_attn_plan_create: out is NULL");
  *out = nullptr;
  if (n_seqs < 0 || !cu_seqlens) return op_fail(FGD_ERR_INVALID_ARG, "fgd_attn_plan_create: n_seqs=%d, cu_seqlens=%p", n_seqs, (const void*)cu_seqlens);
  if (cu_seqlens[0] != 0) return op_fail(FGD_ERR_INVALID_ARG, "fgd_attn_plan_create: cu_seqlens[0] is %lld, not 0", (long long)cu_seqlens[0]);
  for (int i = 0; i < n_seqs; ++i)
    if (cu_seqlens[i + 1] < cu_seqlens[i]) return op_fail(FGD_ERR_INVALID_ARG, "fgd_attn_plan_create: cu_seqlens decreases at %d", i + 1);
  const int64_t tokens = cu_seqlens[n_seqs];
  if (tokens > 0x7fffffff - 4096) return op_fail(FGD_ERR_INVALID_ARG, "fgd_attn_plan_create: %lld tokens", (long long)tokens);
  try {
    std::vector<AttnTile> q, q2, kv;
    for (int i = 0; i < n_seqs; ++i) {
      const int32_t start = (int32_t)cu_seqlens[i], len = (int32_t)(cu_seqlens[i + 1] - cu_seqlens[i]);
      for (int32_t r = 0; r < len; r += kAttnRows) q.push_back({start, len, r, 0});
      for (int32_t r = 0; r < len; r += 2 * kAttnRows) q2.push_back({start, len, r, 0});
    }
    kv = q;
    auto by_row = [](const AttnTile& a, const AttnTile& b) { return a.row > b.row; };
    std::stable_sort(q.begin(), q.end(), by_row);
    std::stable_sort(q2.begin(), q2.end(), by_row);
    std::stable_sort(kv.begin(), kv.end(), [](const AttnTile& a, const AttnTile& b) { return a.len - a.row > b.len - b.row; });
    std::vector<AttnTile> all(q);
    all.insert(all.end(), q2.begin(), q2.end());
    all.insert(all.end(), kv.begin(), kv.end());
    all.push_back({0, 0, 0, 0});   // the status word
    fgd_attn_plan* p = new fgd_attn_plan;   // the last allocation that can throw
    p->device = device; p->tokens = tokens;
    p->n_q = (int)q.size(); p->n_q2 = (int)q2.size(); p->n_kv = (int)kv.size();
    DeviceScope dev(device);
    const size_t bytes = sizeof(AttnTile) * all.size();
    cudaError_t e = dev.ok() ? cudaMalloc(reinterpret_cast<void**>(&p->q_tiles), bytes) : cudaErrorInvalidDevice;
    if (e == cudaSuccess) {
      p->q2_tiles = p->q_tiles + q.size();
      p->kv_tiles = p->q2_tiles + q2.size();
      p->status = reinterpret_cast<int*>(p->kv_tiles + kv.size());
      e = cudaMemcpy(p->q_tiles, all.data(), bytes, cudaMemcpyHostToDevice);
      // From pageable memory that call may return before the bytes are on the device, and streams that do not wait for the default one may
      // use the plan next.
      if (e == cudaSuccess) e = cudaStreamSynchronize(cudaStreamLegacy);
    }
    if (e == cudaSuccess) {
      cudaDriverEntryPointQueryResult qr;
      if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p->encode_tiled, cudaEnableDefault, &qr) != cudaSuccess || qr != cudaDriverEntryPointSuccess)
        p->encode_tiled = nullptr;   // the element-wise kernels still work
    }
    if (e != cudaSuccess) {
      if (p->q_tiles) cudaFree(p->q_tiles);
      delete p;
      cudaGetLastError();
      return op_fail(FGD_ERR_CUDA, "fgd_attn_plan_create: device %d: %s", device, cudaGetErrorString(e));
    }
    *out = p;
  } catch (const std::bad_alloc&) {
    return op_fail(FGD_ERR_INVALID_ARG, "fgd_attn_plan_create: out of host memory");
  }
  return FGD_OK;
}

extern "C" int fgd_attn_plan_destroy(fgd_attn_plan* plan) {
  if (!plan) return FGD_OK;
  DeviceScope dev(plan->device);
  if (plan->q_tiles) cudaFree(plan->q_tiles);
  delete plan;
  return FGD_OK;
}

extern "C" int fgd_attn_debug_set(fgd_attn_plan* plan, int key, int64_t value) {
  if (!plan) return op_fail(FGD_ERR_INVALID_ARG, "fgd_attn_debug_set: NULL plan");
  switch (key) {
    case FGD_DEBUG_SPIN_LIMIT:
      if (value < 0 || value > (int64_t)0xffffffffu) return op_fail(FGD_ERR_INVALID_ARG, "fgd_attn_debug_set: spin limit %lld out of range", (long long)value);
      plan->dbg_spin_limit = (uint32_t)value;
      return FGD_OK;
    case FGD_DEBUG_SKIP_TILE:
      if (value < -1 || value > 0x7fffffff) return op_fail(FGD_ERR_INVALID_ARG, "fgd_attn_debug_set: tile index %lld out of range", (long long)value);
      plan->dbg_skip = (int)value;
      return FGD_OK;
    default:
      return op_fail(FGD_ERR_INVALID_ARG, "fgd_attn_debug_set: unknown key %d", key);
  }
}

extern "C" int fgd_attn_status(fgd_attn_plan* plan, void* stream) {
  if (!plan) return op_fail(FGD_ERR_INVALID_ARG, "fgd_attn_status: NULL plan");
  DeviceScope dev(plan->device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", plan->device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int word = 0;
  cudaError_t e = cudaMemcpyAsync(&word, plan->status, sizeof(int), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaMemsetAsync(plan->status, 0, sizeof(int), st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return op_fail(FGD_ERR_CUDA, "fgd_attn_status: %s", cudaGetErrorString(e));
  if (word != 0) return op_fail(FGD_ERR_TIMEOUT, "a device-side wait of an attention kernel gave up; the outputs of that call are invalid");
  return FGD_OK;
}

extern "C" int fgd_attn_forward(fgd_attn_plan* plan, const fgd_attn_args* b, void* stream) {
  FGD_NVTX_RANGE("fgd_attn_forward");
  const char* who = "fgd_attn_forward";
  if (int rc = check_common(who, plan, b)) return rc;
  if (plan->tokens == 0) return FGD_OK;
  const HeadsArg all[] = {{"q", &b->q, b->n_q_heads, false}, {"k", &b->k, b->n_kv_heads, false}, {"v", &b->v, b->n_kv_heads, false}, {"o", &b->o, b->n_q_heads, true}};
  const int bytes = dtype_bytes(b->dtype);
  for (const HeadsArg& h : all)
    if (int rc = check_heads(who, h, plan->tokens, b->head_dim, bytes)) return rc;
  const Span so = heads_span(b->o, plan->tokens, b->n_q_heads, b->head_dim, bytes), sl = span_of(b->lse, b->n_q_heads, plan->tokens, plan->tokens, 4);
  for (int i = 0; i < 3; ++i) {
    const Span s = heads_span(*all[i].t, plan->tokens, all[i].heads, b->head_dim, bytes);
    if (so.overlaps(s) || sl.overlaps(s)) return op_fail(FGD_ERR_ALIAS, "%s: an output overlaps %s", who, all[i].name);
  }
  if (so.overlaps(sl)) return op_fail(FGD_ERR_ALIAS, "%s: o and lse overlap", who);
  DeviceScope dev(plan->device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", plan->device);
  const AttnArgs a = kernel_args(plan, b);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return on_tensor_cores(plan, b, all, 4) ? attn_forward_tc(plan, b->dtype, a, st) : attn_forward_elem(plan, b->dtype, a, st);
}

extern "C" int fgd_attn_backward(fgd_attn_plan* plan, const fgd_attn_args* b, void* stream) {
  FGD_NVTX_RANGE("fgd_attn_backward");
  const char* who = "fgd_attn_backward";
  if (int rc = check_common(who, plan, b)) return rc;
  if (plan->tokens == 0) return FGD_OK;
  if (!b->delta) return op_fail(FGD_ERR_INVALID_ARG, "%s: delta is NULL", who);
  if (reinterpret_cast<uintptr_t>(b->delta) % sizeof(float) != 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: delta is not on a boundary of its elements", who);
  const HeadsArg all[] = {{"q", &b->q, b->n_q_heads, false}, {"k", &b->k, b->n_kv_heads, false}, {"v", &b->v, b->n_kv_heads, false},
                          {"o", &b->o, b->n_q_heads, false}, {"dout", &b->dout, b->n_q_heads, false},
                          {"dq", &b->dq, b->n_q_heads, true}, {"dk", &b->dk, b->n_kv_heads, true}, {"dv", &b->dv, b->n_kv_heads, true}};
  const int bytes = dtype_bytes(b->dtype);
  Span spans[10];
  for (int i = 0; i < 8; ++i) {
    if (int rc = check_heads(who, all[i], plan->tokens, b->head_dim, bytes)) return rc;
    spans[i] = heads_span(*all[i].t, plan->tokens, all[i].heads, b->head_dim, bytes);
  }
  spans[8] = span_of(b->lse, b->n_q_heads, plan->tokens, plan->tokens, 4);
  spans[9] = span_of(b->delta, b->n_q_heads, plan->tokens, plan->tokens, 4);
  for (int i : {5, 6, 7, 9})
    for (int j = 0; j < 10; ++j)
      if (i != j && spans[i].overlaps(spans[j])) return op_fail(FGD_ERR_ALIAS, "%s: %s overlaps another tensor", who, i == 9 ? "delta" : all[i].name);
  DeviceScope dev(plan->device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", plan->device);
  const AttnArgs a = kernel_args(plan, b);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool tc = on_tensor_cores(plan, b, all, 8);
  if (int rc = attn_delta(plan, b->dtype, tc, a, st)) return rc;
  return tc ? attn_backward_tc(plan, b->dtype, a, st) : attn_backward_elem(plan, b->dtype, a, st);
}

// Entry points and kernels of the fused block norm (mathematics and layout: fgd_block_norm.cuh).
#include "fgd_block_norm.cuh"
#include "fgd_nvtx.h"

using namespace fgd;

namespace {

template <typename T, int VEC, int NT, int VPT>
__global__ void __launch_bounds__(NT) norm_forward_kernel(const NormArgs a) {
  __shared__ float buf[2][1][NT / 32 > 0 ? NT / 32 : 1];
  const int64_t worker = blockIdx.x / a.ctas, row0 = worker * a.rows, end = row0 + a.rows;
  int64_t row = row0 + blockIdx.x % a.ctas;
  const bool has_y = a.y.p != nullptr, full = a.gate_kind == GATE_FULL, post = a.w_post.p != nullptr;
  int c[VPT];
  bool real[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) { c[j] = (threadIdx.x + j * NT) * VEC; real[j] = c[j] < a.width; }
  RowVec<T, VEC> x[VPT], y[VPT], g[VPT];
  auto fetch = [&](int64_t r) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      x[j].load(a.x, r, c[j], real[j]);
      if (has_y) y[j].load(a.y, r, c[j], real[j]);
      if (full) g[j].load(a.gate, r, c[j], real[j]);
    }
  };
  if (row < end) fetch(row);
  for (int slot = 0; row < end; row += a.ctas) {
    float v[VPT][VEC], ss[1] = {0.f};
    if (has_y) {
      float ry = 1.f;
      if (post) {
#pragma unroll
        for (int j = 0; j < VPT; ++j)
#pragma unroll
          for (int i = 0; i < VEC; ++i) ss[0] = fmaf(y[j][i], y[j][i], ss[0]);
        cta_sum<1, NT>(ss, buf, slot); slot ^= 1;
        ry = rsqrtf(fmaf(ss[0], a.inv_width, a.eps));
      }
      ry *= a.scale;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        float w[VEC], gr[VEC];
        load_channel<VEC>(a.w_post, worker, c[j], real[j], 1.f, w);
        if (a.gate_kind == GATE_ROW) load_channel<VEC>(a.gate, worker, c[j], real[j], 1.f, gr);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float u = y[j][i] * ry * w[i];
          if (full) u *= g[j][i];
          else if (a.gate_kind == GATE_ROW) u *= gr[i];
          v[j][i] = x[j][i] + u;
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[j][i] = x[j][i];
    }
    if (row + a.ctas < end) fetch(row + a.ctas);
    if (a.x_new.p) {
#pragma unroll
      for (int j = 0; j < VPT; ++j)
        if (real[j]) {
          ActPack<T, VEC> o;
#pragma unroll
          for (int i = 0; i < VEC; ++i) o.v[i] = from_f32<T>(v[j][i]);
          store_stream<T, VEC>(reinterpret_cast<T*>(a.x_new.p) + row * a.x_new.ld + c[j], o);
        }
    }
    if (a.n.p) {
      ss[0] = 0.f;
#pragma unroll
      for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) ss[0] = fmaf(v[j][i], v[j][i], ss[0]);
      cta_sum<1, NT>(ss, buf, slot); slot ^= 1;
      const float rx = rsqrtf(fmaf(ss[0], a.inv_width, a.eps));
#pragma unroll
      for (int j = 0; j < VPT; ++j)
        if (real[j]) {
          float w[VEC];
          load_channel<VEC>(a.w_pre, worker, c[j], true, 1.f, w);
          ActPack<T, VEC> o;
#pragma unroll
          for (int i = 0; i < VEC; ++i) o.v[i] = from_f32<T>(v[j][i] * rx * w[i]);
          store_stream<T, VEC>(reinterpret_cast<T*>(a.n.p) + row * a.n.ld + c[j], o);
        }
    }
  }
}

template <typename T, int VEC, int NT, int VPT>
__global__ void __launch_bounds__(NT) norm_backward_kernel(const NormArgs a) {
  __shared__ float buf[2][6][NT / 32 > 0 ? NT / 32 : 1];
  const int64_t worker = blockIdx.x / a.ctas, row0 = worker * a.rows, end = row0 + a.rows;
  int64_t row = row0 + blockIdx.x % a.ctas;
  const bool has_y = a.y.p != nullptr, full = a.gate_kind == GATE_FULL, post = a.w_post.p != nullptr, pre = a.dn.p != nullptr, dres = a.dres.p != nullptr;
  int c[VPT];
  bool real[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) { c[j] = (threadIdx.x + j * NT) * VEC; real[j] = c[j] < a.width; }
  RowVec<T, VEC> x[VPT], y[VPT], g[VPT], n[VPT], d[VPT];
  auto fetch = [&](int64_t r) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      x[j].load(a.x_new, r, c[j], real[j] && pre);
      y[j].load(a.y, r, c[j], real[j] && has_y);
      n[j].load(a.dn, r, c[j], real[j] && pre);
      d[j].load(a.dres, r, c[j], real[j] && dres);
      if (full) g[j].load(a.gate, r, c[j], real[j]);
    }
  };
  float acc_pre[VPT][VEC], acc_post[VPT][VEC];
#pragma unroll
  for (int j = 0; j < VPT; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc_pre[j][i] = acc_post[j][i] = 0.f;
  for (int slot = 0; row < end; row += a.ctas) {
    fetch(row);
    // t0 = s g w_post y; the six sums
    float s[6] = {};
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      float wn[VEC], wp[VEC], gr[VEC];
      load_channel<VEC>(a.w_pre, worker, c[j], real[j], 1.f, wn);
      load_channel<VEC>(a.w_post, worker, c[j], real[j], 1.f, wp);
      if (a.gate_kind == GATE_ROW) load_channel<VEC>(a.gate, worker, c[j], real[j], 1.f, gr);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float xv = x[j][i], yv = y[j][i], av = n[j][i] * wn[i], dv = d[j][i];
        float t0 = a.scale * wp[i] * yv;
        if (full) t0 *= g[j][i];
        else if (a.gate_kind == GATE_ROW) t0 *= gr[i];
        s[0] = fmaf(xv, xv, s[0]);
        s[1] = fmaf(yv, yv, s[1]);
        s[2] = fmaf(av, xv, s[2]);
        s[3] = fmaf(t0, dv, s[3]);
        s[4] = fmaf(t0, av, s[4]);
        s[5] = fmaf(t0, xv, s[5]);
      }
    }
    cta_sum<6, NT>(s, buf, slot); slot ^= 1;
    const float rx = pre ? rsqrtf(fmaf(s[0], a.inv_width, a.eps)) : 0.f;
    const float ry = post ? rsqrtf(fmaf(s[1], a.inv_width, a.eps)) : 1.f;
    const float k = rx * rx * (rx * s[2] * a.inv_width);                       // dX = dres + rx a - k x'
    const float m = post ? ry * ry * a.inv_width * (s[3] + rx * s[4] - k * s[5]) : 0.f;   // dy = ry (b - m y)
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      if (!real[j]) continue;
      float wn[VEC], wp[VEC], gr[VEC];
      load_channel<VEC>(a.w_pre, worker, c[j], true, 1.f, wn);
      load_channel<VEC>(a.w_post, worker, c[j], true, 1.f, wp);
      if (a.gate_kind == GATE_ROW) load_channel<VEC>(a.gate, worker, c[j], true, 1.f, gr);
      ActPack<T, VEC> ox, oy, og;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float xv = x[j][i], yv = y[j][i], nv = n[j][i];
        const float dX = fmaf(-k, xv, fmaf(rx, nv * wn[i], d[j][i]));
        const float gv = full ? g[j][i] : a.gate_kind == GATE_ROW ? gr[i] : 1.f;
        const float sd = a.scale * dX, yh = yv * ry;
        ox.v[i] = from_f32<T>(dX);
        oy.v[i] = from_f32<T>(ry * fmaf(-m, yv, sd * gv * wp[i]));
        acc_pre[j][i] = fmaf(nv, xv * rx, acc_pre[j][i]);
        acc_post[j][i] = fmaf(full ? sd * gv : sd, yh, acc_post[j][i]);
        if (full) og.v[i] = from_f32<T>(sd * yh * wp[i]);
      }
      store_stream<T, VEC>(reinterpret_cast<T*>(a.dx.p) + row * a.dx.ld + c[j], ox);
      if (has_y) store_stream<T, VEC>(reinterpret_cast<T*>(a.dy.p) + row * a.dy.ld + c[j], oy);
      if (full) store_stream<T, VEC>(reinterpret_cast<T*>(a.dgate.p) + row * a.dgate.ld + c[j], og);
    }
  }
  float* out = a.partial + (size_t)blockIdx.x * 2 * a.width;
#pragma unroll
  for (int j = 0; j < VPT; ++j)
    if (real[j])
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        out[c[j] + i] = acc_pre[j][i];
        out[a.width + c[j] + i] = acc_post[j][i];
      }
}

// Column sums over the CTAs of one worker, 32 columns per CTA, eight partial sums per column added in order.
__global__ void __launch_bounds__(256) norm_columns_kernel(const NormArgs a) {
  __shared__ float buf[2][8][32];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  const int64_t worker = blockIdx.y;
  float s[2] = {0.f, 0.f};
  if (c < a.width)
    for (int i = part; i < a.ctas; i += 8) {
      const float* p = a.partial + (size_t)(worker * a.ctas + i) * 2 * a.width + c;
      s[0] += p[0];
      s[1] += p[a.width];
    }
  buf[0][part][lane] = s[0];
  buf[1][part][lane] = s[1];
  __syncthreads();
  if (part != 0 || c >= a.width) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) { s[0] += buf[0][i][lane]; s[1] += buf[1][i][lane]; }
  auto at = [&](const NormMat& m) -> float& { return reinterpret_cast<float*>(m.p)[worker * m.ld + c]; };
  if (a.dw_pre.p) at(a.dw_pre) = s[0];
  if (a.dw_post.p) at(a.dw_post) = a.gate_kind == GATE_ROW ? s[1] * at(a.gate) : s[1];
  if (a.gate_kind == GATE_ROW) at(a.dgate) = a.w_post.p ? s[1] * at(a.w_post) : s[1];
}

// ---- host
constexpr int kMaxWidth = 16384;
struct Shape { int nt, vpt; };
// Threads per row x vectors per thread: one vector while a row fits 512 threads of them.
Shape shape_for(int width, int vec) {
  const int vecs = (width + vec - 1) / vec;
  if (vec > 1) {
    if (vecs <= 32) return {32, 1};
    if (vecs <= 128) return {128, 1};
    if (vecs <= 256) return {256, 1};
    if (vecs <= 512) return {512, 1};
    if (vecs <= 1024) return {512, 2};
    return {1024, 4};
  }
  if (vecs <= 128) return {128, 1};
  if (vecs <= 1024) return {256, 4};
  if (vecs <= 4096) return {512, 8};
  return {1024, 16};
}
int ctas_per_worker(int64_t workers, int64_t rows, int nt) {
  int64_t c = ((int64_t)sm_count() * (nt >= 1024 ? 1 : 1024 / nt > 16 ? 16 : 1024 / nt) + workers - 1) / workers;
  if (c > rows) c = rows;
  return (int)(c < 1 ? 1 : c);
}

template <typename T, int VEC, int NT, int VPT>
void launch_norm(const NormArgs& a, unsigned grid, bool backward, cudaStream_t st) {
  if (backward) norm_backward_kernel<T, VEC, NT, VPT><<<grid, NT, 0, st>>>(a);
  else norm_forward_kernel<T, VEC, NT, VPT><<<grid, NT, 0, st>>>(a);
}
template <typename T>
void launch_norm_shape(const NormArgs& a, Shape s, bool vec, unsigned grid, bool backward, cudaStream_t st) {
  constexpr int V = 16 / sizeof(T);
  if (vec) {
    if (s.nt == 32) launch_norm<T, V, 32, 1>(a, grid, backward, st);
    else if (s.nt == 128) launch_norm<T, V, 128, 1>(a, grid, backward, st);
    else if (s.nt == 256) launch_norm<T, V, 256, 1>(a, grid, backward, st);
    else if (s.nt == 512 && s.vpt == 1) launch_norm<T, V, 512, 1>(a, grid, backward, st);
    else if (s.nt == 512) launch_norm<T, V, 512, 2>(a, grid, backward, st);
    else launch_norm<T, V, 1024, 4>(a, grid, backward, st);
  } else {
    if (s.nt == 128) launch_norm<T, 1, 128, 1>(a, grid, backward, st);
    else if (s.nt == 256) launch_norm<T, 1, 256, 4>(a, grid, backward, st);
    else if (s.nt == 512) launch_norm<T, 1, 512, 8>(a, grid, backward, st);
    else launch_norm<T, 1, 1024, 16>(a, grid, backward, st);
  }
}

struct Named { const char* name; const fgd_mat* m; bool wanted, present_needed, channel; };

int run_norm(const fgd_block_norm_args* b, bool backward, int device, void* stream) {
  const char* who = backward ? "fgd_block_norm_backward" : "fgd_block_norm_forward";
  if (!b) return op_fail(FGD_ERR_INVALID_ARG, "%s: NULL arguments", who);
  const int bytes = dtype_bytes(b->dtype);
  if (bytes == 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: unknown dtype %d", who, b->dtype);
  if (b->workers < 1 || b->workers > FGD_MAX_K || b->rows < 0 || b->rows > 0x7fffffff || b->width < 1)
    return op_fail(FGD_ERR_INVALID_ARG, "%s: workers=%d, rows=%lld, width=%lld out of range", who, b->workers, (long long)b->rows, (long long)b->width);
  if (b->width > kMaxWidth) return op_fail(FGD_ERR_UNSUPPORTED, "%s: width %lld above %d", who, (long long)b->width, kMaxWidth);
  if (b->gate_kind < GATE_NONE || b->gate_kind > GATE_FULL) return op_fail(FGD_ERR_INVALID_ARG, "%s: gate_kind %d", who, b->gate_kind);
  const bool y = b->y.p != nullptr, post = b->w_post.p != nullptr, gate = b->gate_kind != GATE_NONE, full = b->gate_kind == GATE_FULL;
  const bool pre = backward ? b->dn.p != nullptr : b->n.p != nullptr;
  if (!y && (post || gate)) return op_fail(FGD_ERR_INVALID_ARG, "%s: w_post and gate need a block output y", who);
  // name, matrix, used by this call, required, per channel
  const Named all[] = {
      {"x", &b->x, !backward, true, false},
      {"x_new", &b->x_new, true, backward ? pre : y, false},
      {"y", &b->y, y, false, false},
      {"gate", &b->gate, gate, true, !full},
      {"w_post", &b->w_post, post, false, true},
      {"w_pre", &b->w_pre, pre, true, true},
      {"n", &b->n, !backward && pre, true, false},
      {"dn", &b->dn, backward && pre, true, false},
      {"dres", &b->dres, backward, !pre, false},
      {"dx", &b->dx, backward, true, false},
      {"dy", &b->dy, backward && y, true, false},
      {"dgate", &b->dgate, backward && gate, true, !full},
      {"dw_post", &b->dw_post, backward && post, true, true},
      {"dw_pre", &b->dw_pre, backward && pre, true, true},
  };
  const int vec = 16 / bytes;
  bool aligned = b->width % vec == 0;
  const int64_t T = b->workers * b->rows;
  for (const Named& e : all) {
    if (!e.wanted) continue;
    if (!e.m->p) {
      if (e.present_needed) return op_fail(FGD_ERR_INVALID_ARG, "%s: %s is NULL", who, e.name);
      continue;
    }
    if (e.m->ld < b->width) return op_fail(FGD_ERR_INVALID_ARG, "%s: row stride of %s is below the width", who, e.name);
    const int64_t size = e.channel ? 4 : bytes;
    if (reinterpret_cast<uintptr_t>(e.m->p) % 16 != 0 || (e.m->ld * size) % 16 != 0) aligned = false;
  }
  if (!backward && !pre && !y) return op_fail(FGD_ERR_INVALID_ARG, "%s: nothing to do (neither y nor n)", who);
  // outputs may not overlap anything, except that x_new may be x itself and dx may be dres itself (a row is
  // read whole before it is written)
  for (const Named& o : all) {
    const bool out = o.m == &b->dx || o.m == &b->dy || o.m == &b->dgate || o.m == &b->dw_post || o.m == &b->dw_pre || o.m == &b->n || (!backward && o.m == &b->x_new);
    if (!out || !o.wanted || !o.m->p) continue;
    for (const Named& e : all) {
      if (!e.wanted || !e.m->p || e.m == o.m) continue;
      const bool in_place = e.m->p == o.m->p && e.m->ld == o.m->ld && ((o.m == &b->x_new && e.m == &b->x) || (o.m == &b->dx && e.m == &b->dres));
      if (in_place || (o.m == &b->x && e.m == &b->x_new)) continue;
      const Span so = span_of(o.m->p, o.channel ? b->workers : T, b->width, o.m->ld, o.channel ? 4 : bytes);
      const Span se = span_of(e.m->p, e.channel ? b->workers : T, b->width, e.m->ld, e.channel ? 4 : bytes);
      if (so.overlaps(se)) return op_fail(FGD_ERR_ALIAS, "%s: %s overlaps %s", who, o.name, e.name);
    }
  }
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool columns = backward && (pre || post || b->gate_kind == GATE_ROW);
  if (T == 0 && !columns) return FGD_OK;
  const Shape s = shape_for((int)b->width, aligned ? vec : 1);
  NormArgs a = {};
  auto mat = [](const fgd_mat& m, bool use) { return NormMat{use ? static_cast<char*>(m.p) : nullptr, m.ld}; };
  a.x = mat(b->x, !backward); a.y = mat(b->y, y); a.gate = mat(b->gate, gate); a.w_post = mat(b->w_post, post); a.w_pre = mat(b->w_pre, pre);
  a.x_new = mat(b->x_new, backward ? pre : (y || b->x_new.p != b->x.p)); a.n = mat(b->n, !backward && pre);
  a.dn = mat(b->dn, backward && pre); a.dres = mat(b->dres, backward); a.dx = mat(b->dx, backward); a.dy = mat(b->dy, backward && y);
  a.dgate = mat(b->dgate, backward && gate); a.dw_post = mat(b->dw_post, backward && post); a.dw_pre = mat(b->dw_pre, backward && pre);
  a.rows = b->rows; a.width = (int)b->width; a.gate_kind = b->gate_kind;
  a.ctas = ctas_per_worker(b->workers, b->rows, s.nt);
  a.eps = (float)b->eps; a.scale = (float)b->res_scale; a.inv_width = 1.f / (float)b->width;
  const int64_t grid = (int64_t)b->workers * a.ctas;
  if (grid > 0x7fffffff) return op_fail(FGD_ERR_INVALID_ARG, "%s: too many workers", who);
  if (backward) {
    const int64_t need = grid * 2 * b->width * (int64_t)sizeof(float);
    if (!b->workspace || b->workspace_bytes < need || reinterpret_cast<uintptr_t>(b->workspace) % 4 != 0)
      return op_fail(FGD_ERR_INVALID_ARG, "%s: needs a workspace of %lld bytes (fgd_block_norm_workspace)", who, (long long)need);
    a.partial = static_cast<float*>(b->workspace);
  }
  switch (b->dtype) {
    case FGD_F32: launch_norm_shape<float>(a, s, aligned, (unsigned)grid, backward, st); break;
    case FGD_BF16: launch_norm_shape<__nv_bfloat16>(a, s, aligned, (unsigned)grid, backward, st); break;
    default: launch_norm_shape<__half>(a, s, aligned, (unsigned)grid, backward, st); break;
  }
  if (columns) norm_columns_kernel<<<dim3((unsigned)((b->width + 31) / 32), (unsigned)b->workers), 256, 0, st>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
  return FGD_OK;
}

}  // namespace

extern "C" int64_t fgd_block_norm_workspace(int device, int dtype, int workers, int64_t rows, int64_t width) {
  const int bytes = dtype_bytes(dtype);
  if (bytes == 0 || workers < 1 || workers > FGD_MAX_K || rows < 0 || rows > 0x7fffffff || width < 1 || width > kMaxWidth) return FGD_ERR_INVALID_ARG;
  DeviceScope dev(device);
  // the element-wise shapes have no fewer threads per row than the vector shapes, so no more CTAs
  return (int64_t)workers * ctas_per_worker(workers, rows, shape_for((int)width, 16 / bytes).nt) * 2 * width * (int64_t)sizeof(float);
}
extern "C" int fgd_block_norm_forward(int device, const fgd_block_norm_args* args, void* stream) {
  FGD_NVTX_RANGE("fgd_block_norm_forward");
  return run_norm(args, false, device, stream);
}
extern "C" int fgd_block_norm_backward(int device, const fgd_block_norm_args* args, void* stream) {
  FGD_NVTX_RANGE("fgd_block_norm_backward");
  return run_norm(args, true, device, stream);
}

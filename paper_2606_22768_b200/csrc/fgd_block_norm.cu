// Entry points and kernels of the fused block norm (mathematics and layout: fgd_block_norm.cuh).
#include "fgd_block_norm.cuh"
#include "fgd_nvtx.h"

using namespace fgd;

namespace {

// A thread with at most 8 elements of a row keeps the per-channel factors in registers for all its rows.  With more it keeps them in
// shared memory (KEEP, behind the ring), or, where that is full, reads them again in every row.  Arithmetic runs on pairs of fp32 values: with 16-bit activations a scalar version is bound by its
// instructions, not by HBM.
template <typename T, int VEC, int NT, int VPT, int STAGES, bool FULL, bool ANY, bool KEEP>
__global__ void __launch_bounds__(NT, NT * VPT <= 1024 ? 1024 / NT > 16 ? 16 : 1024 / NT : 1) norm_forward_kernel(const NormArgs a) {
  constexpr bool HOLD = VEC * VPT <= 8;
  constexpr int P = VEC / 2;
  enum { X, Y, G, N = FULL ? 3 : 2 };
  extern __shared__ __align__(16) unsigned char ring[];
  __shared__ __align__(16) float buf[2][1][NT / 32];
  const int64_t worker = blockIdx.x / a.ctas, row0 = worker * a.rows, end = row0 + a.rows, first = row0 + blockIdx.x % a.ctas;
  const bool post = a.w_post.p != nullptr;
  NormMat in[N] = {a.x, a.y};
  if constexpr (FULL) in[G] = a.gate;
  int c[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) c[j] = (threadIdx.x + j * NT) * VEC;
  Vals<VEC> wt[VPT], wn[VPT];
  if constexpr (HOLD || KEEP) {
    post_factors<VEC, VPT, ANY>(a, worker, c, wt);
    load_channel<VEC, VPT, ANY>(a.w_pre, worker, c, a.width, wn);
  }
  Factors<VEC, VPT, NT, KEEP> ft, fn;
  ft.start(ring + STAGES * N * RowFeed<T, VEC, NT, VPT, N, STAGES, ANY>::kStageBytes, 0, wt);
  fn.start(ring + STAGES * N * RowFeed<T, VEC, NT, VPT, N, STAGES, ANY>::kStageBytes, 1, wn);
  RowFeed<T, VEC, NT, VPT, N, STAGES, ANY> feed;
  feed.start(in, a.width, ring, first, a.ctas, end, a.last_row);
  int slot = 0;
  for (int64_t row = first; row < end; row += a.ctas) {
    feed.next(in, row, a.ctas, end, row == first);
    Vals<VEC> v[VPT];
    float ss[1], ry = 1.f;
    float2 sum = both(0.f);
    if (post) {
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const Vals<VEC> y = feed.get(Y, j);
#pragma unroll
        for (int i = 0; i < P; ++i) sum = fma2(y.pair(i), y.pair(i), sum);
      }
      ss[0] = sum.x + sum.y;
      cta_sum<1, NT>(ss, buf, slot); slot ^= 1;
      ry = rsqrtf(fmaf(ss[0], a.inv_width, a.eps));
    }
    if constexpr (!HOLD && !KEEP) post_factors<VEC, VPT, ANY>(a, worker, c, wt);
    sum = both(0.f);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      v[j] = feed.get(X, j);
      const Vals<VEC> y = feed.get(Y, j), ftj = ft.get(wt, j);
      Vals<VEC> g;
      if constexpr (FULL) g = feed.get(G, j);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        float2 u = mul2(y.pair(i), both(ry));
        if constexpr (FULL) u = mul2(u, g.pair(i));
        const float2 x = fma2(u, ftj.pair(i), v[j].pair(i));
        v[j].set(i, x);
        sum = fma2(x, x, sum);
      }
      if (a.x_new.p) store_vec<T, VEC, ANY>(a.x_new, row, c[j], a.width, v[j]);
    }
    if (a.n.p) {
      ss[0] = sum.x + sum.y;
      cta_sum<1, NT>(ss, buf, slot); slot ^= 1;
      const float2 rx = both(rsqrtf(fmaf(ss[0], a.inv_width, a.eps)));
      if constexpr (!HOLD && !KEEP) load_channel<VEC, VPT, ANY>(a.w_pre, worker, c, a.width, wn);
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const Vals<VEC> fnj = fn.get(wn, j);
#pragma unroll
        for (int i = 0; i < P; ++i) v[j].set(i, mul2(mul2(v[j].pair(i), rx), fnj.pair(i)));
        store_vec<T, VEC, ANY>(a.n, row, c[j], a.width, v[j]);
      }
    }
  }
}

template <typename T, int VEC, int NT, int VPT, int STAGES, bool FULL, bool ANY, bool KEEP>
__global__ void __launch_bounds__(NT, NT <= 512 ? 512 / NT : 1) norm_backward_kernel(const NormArgs a) {
  constexpr bool HOLD = VEC * VPT <= 8;
  constexpr int P = VEC / 2;
  enum { X, Y, DN, DR, G, N = FULL ? 5 : 4 };
  extern __shared__ __align__(16) unsigned char ring[];
  __shared__ __align__(16) float buf[2][6][NT / 32];
  const int64_t worker = blockIdx.x / a.ctas, row0 = worker * a.rows, end = row0 + a.rows, first = row0 + blockIdx.x % a.ctas;
  const bool has_y = a.y.p != nullptr, post = a.w_post.p != nullptr, pre = a.dn.p != nullptr;
  NormMat in[N] = {a.x_new, a.y, a.dn, a.dres};
  if constexpr (FULL) in[G] = a.gate;
  int c[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) c[j] = (threadIdx.x + j * NT) * VEC;
  Vals<VEC> acc_pre[VPT], acc_post[VPT], wt[VPT], wn[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc_pre[j].v[i] = acc_post[j].v[i] = 0.f;
  if constexpr (HOLD || KEEP) {
    post_factors<VEC, VPT, ANY>(a, worker, c, wt);
    load_channel<VEC, VPT, ANY>(a.w_pre, worker, c, a.width, wn);
  }
  Factors<VEC, VPT, NT, KEEP> ft, fn;
  ft.start(ring + STAGES * N * RowFeed<T, VEC, NT, VPT, N, STAGES, ANY>::kStageBytes, 0, wt);
  fn.start(ring + STAGES * N * RowFeed<T, VEC, NT, VPT, N, STAGES, ANY>::kStageBytes, 1, wn);
  RowFeed<T, VEC, NT, VPT, N, STAGES, ANY> feed;
  feed.start(in, a.width, ring, first, a.ctas, end, a.last_row);
  let_next_start();      // the column sums' CTAs wait for this kernel's end on the SMs
  int slot = 0;
  for (int64_t row = first; row < end; row += a.ctas) {
    feed.next(in, row, a.ctas, end, row == first);
    if constexpr (!HOLD && !KEEP) {
      post_factors<VEC, VPT, ANY>(a, worker, c, wt);
      load_channel<VEC, VPT, ANY>(a.w_pre, worker, c, a.width, wn);
    }
    // the six sums; t0 = s g w_post y
    float2 s2[6];
#pragma unroll
    for (int k = 0; k < 6; ++k) s2[k] = both(0.f);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const Vals<VEC> x = feed.get(X, j), y = feed.get(Y, j), n = feed.get(DN, j), d = feed.get(DR, j), ftj = ft.get(wt, j), fnj = fn.get(wn, j);
      Vals<VEC> g;
      if constexpr (FULL) g = feed.get(G, j);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float2 xv = x.pair(i), yv = y.pair(i), av = mul2(n.pair(i), fnj.pair(i));
        float2 t0 = mul2(ftj.pair(i), yv);
        if constexpr (FULL) t0 = mul2(t0, g.pair(i));
        s2[0] = fma2(xv, xv, s2[0]);
        s2[1] = fma2(yv, yv, s2[1]);
        s2[2] = fma2(av, xv, s2[2]);
        s2[3] = fma2(t0, d.pair(i), s2[3]);
        s2[4] = fma2(t0, av, s2[4]);
        s2[5] = fma2(t0, xv, s2[5]);
      }
    }
    float s[6];
#pragma unroll
    for (int k = 0; k < 6; ++k) s[k] = s2[k].x + s2[k].y;
    cta_sum<6, NT>(s, buf, slot); slot ^= 1;
    const float rx = pre ? rsqrtf(fmaf(s[0], a.inv_width, a.eps)) : 0.f;
    const float ry = post ? rsqrtf(fmaf(s[1], a.inv_width, a.eps)) : 1.f;
    const float k = rx * rx * (rx * s[2] * a.inv_width);                       // dX = dres + rx a - k x'
    const float m = post ? ry * ry * a.inv_width * (s[3] + rx * s[4] - k * s[5]) : 0.f;   // dy = ry (b - m y)
    const float2 rx2 = both(rx), mk2 = both(-k), ry2 = both(ry), mr2 = both(-m * ry), sry2 = both(a.scale * ry);
    if constexpr (!HOLD && !KEEP) {
      post_factors<VEC, VPT, ANY>(a, worker, c, wt);
      load_channel<VEC, VPT, ANY>(a.w_pre, worker, c, a.width, wn);
    }
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const Vals<VEC> x = feed.get(X, j), y = feed.get(Y, j), n = feed.get(DN, j), d = feed.get(DR, j), ftj = ft.get(wt, j), fnj = fn.get(wn, j);
      Vals<VEC> g, ox, oy, og;
      if constexpr (FULL) g = feed.get(G, j);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float2 xv = x.pair(i), yv = y.pair(i), nv = n.pair(i), xr = mul2(xv, rx2);
        acc_pre[j].set(i, fma2(nv, xr, acc_pre[j].pair(i)));
        const float2 dX = fma2(mk2, xv, fma2(rx2, mul2(nv, fnj.pair(i)), d.pair(i)));
        const float2 syh = mul2(yv, sry2), dg = FULL ? mul2(dX, g.pair(i)) : dX;          // syh = s yh
        ox.set(i, dX);
        oy.set(i, fma2(mr2, yv, mul2(mul2(dg, ftj.pair(i)), ry2)));
        acc_post[j].set(i, fma2(dg, syh, acc_post[j].pair(i)));
        if constexpr (FULL) og.set(i, mul2(mul2(dX, mul2(yv, ry2)), ftj.pair(i)));      // (ft is s w_post here)
      }
      store_vec<T, VEC, ANY>(a.dx, row, c[j], a.width, ox);
      if (has_y) store_vec<T, VEC, ANY>(a.dy, row, c[j], a.width, oy);
      if constexpr (FULL) store_vec<T, VEC, ANY>(a.dgate, row, c[j], a.width, og);
    }
  }
  float* out = a.partial + (size_t)blockIdx.x * 2 * a.width;
#pragma unroll
  for (int j = 0; j < VPT; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (c[j] + i < a.width) {
        out[c[j] + i] = acc_pre[j].v[i];
        out[a.width + c[j] + i] = acc_post[j].v[i];
      }
}

// Column sums over the CTAs of one worker, 32 columns per CTA, eight partial sums per column added in order.
__global__ void __launch_bounds__(256) norm_columns_kernel(const NormArgs a) {
  wait_for_previous();
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
constexpr size_t kMaxSmem = 226 * 1024;      // of a CTA, beside what the kernels hold statically
struct Shape { int nt, vpt; };
// Threads per row x vectors per thread: one vector while a row fits 512 threads of them.
Shape shape_for(int width, int vec, bool backward) {
  const int vecs = (width + vec - 1) / vec;
  if (vecs <= 32) return {32, 1};
  if (vecs <= 64) return {64, 1};
  if (vecs <= 128) return {128, 1};
  if (vecs <= 256) return {256, 1};
  if (vecs <= 512) return backward ? Shape{256, 2} : Shape{512, 1};
  if (vecs <= 1024) return {512, 2};
  if (vecs <= 2048) return {512, 4};
  return {1024, 4};      // fp32 above 8192 columns
}
// CTAs that share an SM: the kernels' launch bounds leave registers for them; `smem` is the dynamic part of what each of them takes.
int ctas_per_sm(int nt, bool backward, size_t smem) {
  const int regs = (backward ? 512 : 1024) / nt, room = (int)(228 * 1024 / (smem + 2 * 1024)), c = regs < room ? regs : room;
  return c < 1 ? 1 : c > 16 ? 16 : c;
}
int ctas_per_worker(int64_t workers, int64_t rows, int nt, bool backward, size_t smem) {
  int64_t c = (int64_t)sm_count() * ctas_per_sm(nt, backward, smem) / workers;      // (rounded down: a CTA too many takes as long as all of them, 267 against 151 us for 8 x 1024 x 8192 bf16 backward)
  if (c > rows) c = rows;
  return (int)(c < 1 ? 1 : c);
}

// Launches with as many CTAs as fit the SMs beside each other (their number: a.ctas per worker).
template <auto KERNEL>
cudaError_t start(NormArgs& a, int64_t workers, bool backward, int threads, size_t smem, cudaStream_t st) {
  a.ctas = ctas_per_worker(workers, a.rows, threads, backward, smem);
  cudaError_t e = smem > 32 * 1024 ? allow_smem<KERNEL>(smem) : cudaSuccess;
  if (e == cudaSuccess) {
    KERNEL<<<(unsigned)(workers * a.ctas), threads, smem, st>>>(a);
    e = cudaGetLastError();
  }
  return e;
}
template <typename T, int NT, int VPT, int SF, int SB, bool ANY>
cudaError_t launch_norm(NormArgs& a, int64_t workers, bool backward, cudaStream_t st) {
  constexpr int VEC = 16 / sizeof(T);
  constexpr size_t stage = (size_t)VPT * (NT / 32) * (ANY ? 33 : 32) * 16;      // of one tensor
  constexpr size_t factors = VEC * VPT > 8 ? (size_t)VPT * NT * VEC * 8 : 0;
  // The backward pass reads the factors twice a row: in shared memory wherever they fit (2048 rows x 8 of 4096 bf16: 209 us from L1 and
  // L2, 140 so).  Forward, once a row, they take a second CTA's place on the SM (8192 columns, 74 % of the copy peak without): only
  // where weights off their 16-byte boundaries would be read one by one (8 x 1676 x 5003 bf16: 444 us without, 246 so).
  constexpr bool kb4 = factors && SB * 4 * stage + factors <= kMaxSmem, kb5 = factors && SB * 5 * stage + factors <= kMaxSmem,
                 kf2 = ANY && factors && SF * 2 * stage + factors <= kMaxSmem, kf3 = ANY && factors && SF * 3 * stage + factors <= kMaxSmem;
  if (a.gate_kind == GATE_FULL)
    return backward ? start<norm_backward_kernel<T, VEC, NT, VPT, SB, true, ANY, kb5>>(a, workers, backward, NT, SB * 5 * stage + kb5 * factors, st)
                    : start<norm_forward_kernel<T, VEC, NT, VPT, SF, true, ANY, kf3>>(a, workers, backward, NT, SF * 3 * stage + kf3 * factors, st);
  return backward ? start<norm_backward_kernel<T, VEC, NT, VPT, SB, false, ANY, kb4>>(a, workers, backward, NT, SB * 4 * stage + kb4 * factors, st)
                  : start<norm_forward_kernel<T, VEC, NT, VPT, SF, false, ANY, kf2>>(a, workers, backward, NT, SF * 2 * stage + kf2 * factors, st);
}
template <typename T, bool ANY>
cudaError_t launch_norm_shape(NormArgs& a, Shape s, int64_t workers, bool backward, cudaStream_t st) {
  // rows in flight: forward 3 x 8 to 24 KB, backward 2 x 16 to 20 KB per 256 threads; two vectors per thread leave room for one.
  // (Forward, 512 x 2: fp32 is faster without a ring, 94 against 85 % of the copy peak at 4096 columns, 16-bit with one, 66 against 57 % at 8192.)
  if (s.nt == 32) return launch_norm<T, 32, 1, 4, 3, ANY>(a, workers, backward, st);
  if (s.nt == 64) return launch_norm<T, 64, 1, 4, 3, ANY>(a, workers, backward, st);
  if (s.nt == 128) return launch_norm<T, 128, 1, 4, 3, ANY>(a, workers, backward, st);
  if (s.nt == 256 && s.vpt == 1) return launch_norm<T, 256, 1, 4, 3, ANY>(a, workers, backward, st);
  if (s.nt == 256) return launch_norm<T, 256, 2, 2, 2, ANY>(a, workers, backward, st);
  if (s.vpt == 1) return launch_norm<T, 512, 1, 4, 3, ANY>(a, workers, backward, st);
  if (s.vpt == 2) return launch_norm<T, 512, 2, sizeof(T) == 4 ? (ANY ? 2 : 0) : (ANY ? 1 : 2), 2, ANY>(a, workers, backward, st);
  if (s.nt == 512) return launch_norm<T, 512, 4, 1, 1, ANY>(a, workers, backward, st);
  if constexpr (sizeof(T) == 4) return launch_norm<T, 1024, 4, 0, 0, ANY>(a, workers, backward, st);
  return cudaErrorInvalidValue;
}

// The column sums of the most CTAs that a backward pass of this shape can start.
int64_t workspace_bytes(int64_t workers, int64_t rows, int nt, int64_t width) {
  return workers * ctas_per_worker(workers, rows, nt, true, 0) * 2 * width * (int64_t)sizeof(float);
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
  const bool dpre = backward && (pre || b->dw_pre.p != nullptr);      // without dn it is zero
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
      {"dw_pre", &b->dw_pre, dpre, true, true},
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
    if (reinterpret_cast<uintptr_t>(e.m->p) % size != 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: %s is not on a boundary of its elements", who, e.name);
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
      if (in_place) continue;
      const Span so = span_of(o.m->p, o.channel ? b->workers : T, b->width, o.m->ld, o.channel ? 4 : bytes);
      const Span se = span_of(e.m->p, e.channel ? b->workers : T, b->width, e.m->ld, e.channel ? 4 : bytes);
      if (so.overlaps(se)) return op_fail(FGD_ERR_ALIAS, "%s: %s overlaps %s", who, o.name, e.name);
    }
  }
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool columns = dpre || (backward && (post || b->gate_kind == GATE_ROW));
  if (T == 0 && !columns) return FGD_OK;
  const Shape s = shape_for((int)b->width, vec, backward);
  NormArgs a = {};
  auto mat = [](const fgd_mat& m, bool use) { return NormMat{use ? static_cast<char*>(m.p) : nullptr, m.ld}; };
  a.x = mat(b->x, !backward); a.y = mat(b->y, y); a.gate = mat(b->gate, gate); a.w_post = mat(b->w_post, post); a.w_pre = mat(b->w_pre, pre);
  a.x_new = mat(b->x_new, backward ? pre : (y || b->x_new.p != b->x.p)); a.n = mat(b->n, !backward && pre);
  a.dn = mat(b->dn, backward && pre); a.dres = mat(b->dres, backward); a.dx = mat(b->dx, backward); a.dy = mat(b->dy, backward && y);
  a.dgate = mat(b->dgate, backward && gate); a.dw_post = mat(b->dw_post, backward && post); a.dw_pre = mat(b->dw_pre, dpre);
  a.rows = b->rows; a.last_row = T - 1; a.width = (int)b->width; a.gate_kind = b->gate_kind;
  a.eps = (float)b->eps; a.scale = (float)b->res_scale; a.inv_width = 1.f / (float)b->width;
  if (backward) {
    const int64_t need = workspace_bytes(b->workers, b->rows, s.nt, b->width);
    if (!b->workspace || b->workspace_bytes < need || reinterpret_cast<uintptr_t>(b->workspace) % 4 != 0)
      return op_fail(FGD_ERR_INVALID_ARG, "%s: needs a workspace of %lld bytes (fgd_block_norm_workspace)", who, (long long)need);
    a.partial = static_cast<float*>(b->workspace);
  }
  cudaError_t e;
  auto launch = [&](auto any) {
    constexpr bool ANY = decltype(any)::value;
    switch (b->dtype) {
      case FGD_F32: return launch_norm_shape<float, ANY>(a, s, b->workers, backward, st);
      case FGD_BF16: return launch_norm_shape<__nv_bfloat16, ANY>(a, s, b->workers, backward, st);
      default: return launch_norm_shape<__half, ANY>(a, s, b->workers, backward, st);
    }
  };
  e = aligned ? launch(std::false_type{}) : launch(std::true_type{});
  if (e == cudaSuccess && columns) {
    e = launch_early(norm_columns_kernel, dim3((unsigned)((b->width + 31) / 32), (unsigned)b->workers), 256, 0, st, a);
  }
  if (e != cudaSuccess) return op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
  return FGD_OK;
}

}  // namespace

extern "C" int64_t fgd_block_norm_workspace(int device, int dtype, int workers, int64_t rows, int64_t width) {
  const int bytes = dtype_bytes(dtype);
  if (bytes == 0 || workers < 1 || workers > FGD_MAX_K || rows < 0 || rows > 0x7fffffff || width < 1 || width > kMaxWidth) return FGD_ERR_INVALID_ARG;
  DeviceScope dev(device);
  return workspace_bytes(workers, rows, shape_for((int)width, 16 / bytes, true).nt, width);
}
extern "C" int fgd_block_norm_forward(int device, const fgd_block_norm_args* args, void* stream) {
  FGD_NVTX_RANGE("fgd_block_norm_forward");
  return run_norm(args, false, device, stream);
}
extern "C" int fgd_block_norm_backward(int device, const fgd_block_norm_args* args, void* stream) {
  FGD_NVTX_RANGE("fgd_block_norm_backward");
  return run_norm(args, true, device, stream);
}

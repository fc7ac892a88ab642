// Embeddings of K workers' tokens, and the gradient of their tables.
//
// Forward: a row of the table, scaled and rounded once, for every token.
// Backward: dtable[v] = scale * sum of dout[t] over the tokens t that are v, for every row v.  Text repeats few tokens very often (the
// commonest may be 7 % of a batch) and most of a vocabulary not at all, so the work is cut by tokens, not by rows, without atomics on floats:
//   sort   each worker's (token, position) pairs by token, stable, in one launch: a cluster of CTAs per worker, radix passes of up to ten bits;
//          histograms cross the cluster through distributed shared memory.  Marks the tokens that occur in a bitmap.
//   rows   the sorted list in chunks of 64: a warp adds up the runs of equal tokens within its chunk, for 32 lanes x 16 bytes of columns.  A run that
//          lies inside the chunk is a finished row; the pieces of one that crosses chunks go to scratch.  Other warps write the rows of
//          absent tokens with zeros.
//   joins  the pieces of a run, added in order by the chunk that it starts in.
// The order of every sum depends on the tokens alone.
#include <cooperative_groups.h>

#include <cmath>

#include "fgd_dtype.cuh"
#include "fgd_nvtx.h"

using namespace fgd;
namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kCluster = 8;           // CTAs that sort one worker's tokens
constexpr int kSortFew = 4096;        // up to so many a single one does
constexpr int kMaxItems = 4;          // keys of a thread in one tile
constexpr int kMaxBits = 10;          // of a radix pass
constexpr int kChunk = 64;            // sorted tokens that a warp adds up
constexpr int64_t kMaxWidth = 65536, kMaxVocab = 1 << 30;

struct Tokens {
  const void* p; int bytes; int64_t ld;
  __device__ __forceinline__ int64_t at(int64_t worker, int64_t i) const {
    return bytes == 8 ? __ldg(static_cast<const long long*>(p) + worker * ld + i) : (int64_t)__ldg(static_cast<const int*>(p) + worker * ld + i);
  }
};

// 16 bytes of activations, or as many values 32 columns apart where rows are off the 16-byte boundaries: value j of a lane is column
// col(j) of its warp's slab of 32 V.
template <typename T, bool ANY>
struct Slab {
  static constexpr int V = 16 / sizeof(T), kColumns = 32 * V;
  static __device__ __forceinline__ int col(int j) { return ANY ? (threadIdx.x & 31) + 32 * j : (threadIdx.x & 31) * V + j; }
};

struct EmbedArgs {
  Tokens tokens;
  const float* table; int64_t worker_stride, row_stride;
  char* out; int64_t ld_out;
  int64_t rows, tokens_total, vocab;
  int width, parts;            // slabs of a row that a warp takes together are kSlabs
  float scale;
};
constexpr int kSlabs = 4;

template <typename T, bool ANY>
__global__ void __launch_bounds__(kThreads) embed_forward_kernel(const EmbedArgs a) {
  using S = Slab<T, ANY>;
  constexpr int V = S::V;
  const int64_t items = a.tokens_total * a.parts;
  for (int64_t item = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; item < items; item += (int64_t)gridDim.x * kWarps) {
    const int64_t t = item / a.parts, worker = t / a.rows;
    const int c0 = (int)(item - t * a.parts) * (kSlabs * S::kColumns);
    const int64_t tok = a.tokens.at(worker, t - worker * a.rows);
    const bool real = tok >= 0 && tok < a.vocab;
    const float other = tok < 0 ? 0.f : __int_as_float(0x7fffffff);
    const float* row = a.table + worker * a.worker_stride + (real ? tok : 0) * a.row_stride;
    T* out = reinterpret_cast<T*>(a.out) + t * a.ld_out;
    Vals<V> v[kSlabs];
#pragma unroll
    for (int s = 0; s < kSlabs; ++s) {
      const int c = c0 + s * S::kColumns;
      if constexpr (ANY) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[s].v[j] = real && c + S::col(j) < a.width ? __ldg(row + c + S::col(j)) : other;
      } else {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
          float4 f = make_float4(other, other, other, other);
          if (real && c + S::col(0) < a.width) f = __ldg(reinterpret_cast<const float4*>(row + c + S::col(j)));
          v[s].v[j] = f.x; v[s].v[j + 1] = f.y; v[s].v[j + 2] = f.z; v[s].v[j + 3] = f.w;
        }
      }
    }
#pragma unroll
    for (int s = 0; s < kSlabs; ++s) {
      const int c = c0 + s * S::kColumns;
#pragma unroll
      for (int j = 0; j < V; ++j) v[s].v[j] *= a.scale;
      if constexpr (ANY) {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (c + S::col(j) < a.width) out[c + S::col(j)] = from_f32<T>(v[s].v[j]);
      } else {
        if (c + S::col(0) < a.width) store_stream<T, V>(out + c + S::col(0), round_to<T, V>(v[s]));
      }
    }
  }
}

// ---- sort
struct SortArgs {
  Tokens tokens;
  int64_t vocab;
  int rows, cluster, bits, passes;
  uint2 *pairs, *other;        // [worker][rows]: the result, and what the passes alternate with
  uint32_t* present; int words;      // [worker][words] bitmap of the vocabulary
};

// Pairs (token, position); a token outside the vocabulary counts as `vocab` and comes last.
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(const SortArgs a) {
  const cg::cluster_group cluster = cg::this_cluster();
  extern __shared__ __align__(16) unsigned char smem[];
  const int bins = 1 << a.bits, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x % a.cluster;
  const int64_t worker = blockIdx.x / a.cluster;
  uint32_t* hist = reinterpret_cast<uint32_t*>(smem);                       // [bins] of this CTA's part
  uint32_t* base = hist + bins;                                              // [bins] where the next key of a digit goes
  unsigned short* count = reinterpret_cast<unsigned short*>(base + bins);    // [warp][bins] of a tile
  __shared__ uint32_t warp_total[kSortWarps];
  uint32_t* present = a.present + worker * a.words;
  for (int i = rank * kSortThreads + tid; i < a.words; i += a.cluster * kSortThreads) present[i] = 0u;
  const int part = (a.rows + a.cluster - 1) / a.cluster, first = min(rank * part, a.rows), n = min(part, a.rows - first);
  const int items = part >= kMaxItems * kSortThreads ? kMaxItems : (part + kSortThreads - 1) / kSortThreads;
  uint2 *dst = a.passes & 1 ? a.pairs : a.other, *src = a.passes & 1 ? a.other : a.pairs;      // the last pass writes the result
  dst += worker * a.rows; src += worker * a.rows;
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = pass * a.bits;
    auto load = [&](int i) -> uint2 {
      if (pass > 0) return __ldcg(src + first + i);
      const int64_t tok = a.tokens.at(worker, first + i);
      return make_uint2(tok >= 0 && tok < a.vocab ? (uint32_t)tok : (uint32_t)a.vocab, (uint32_t)(first + i));
    };
    for (int b = tid; b < bins; b += kSortThreads) hist[b] = 0u;
    __syncthreads();
    for (int i0 = warp * 32; i0 < n; i0 += kSortThreads) {
      const int i = i0 + lane;
      const uint32_t digit = i < n ? load(i).x >> shift & (bins - 1) : 0xffffffffu;
      const uint32_t same = __match_any_sync(0xffffffffu, digit);
      if (i < n && (same & ((1u << lane) - 1)) == 0) atomicAdd(&hist[digit], (uint32_t)__popc(same));
    }
    cluster.sync();
    // where each digit starts: keys of smaller digits anywhere, and of this digit in the CTAs before; bins <= kSortThreads
    uint32_t before = 0, total = 0;
    if (tid < bins)
      for (int r = 0; r < a.cluster; ++r) {
        const uint32_t h = cluster.map_shared_rank(hist, r)[tid];
        total += h;
        if (r < rank) before += h;
      }
    uint32_t scan = total;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, scan, o);
      if (lane >= o) scan += v;
    }
    if (lane == 31) warp_total[warp] = scan;
    __syncthreads();
    if (warp == 0) {
      uint32_t v = warp_total[lane];
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
      }
      warp_total[lane] = v;
    }
    __syncthreads();
    if (tid < bins) base[tid] = scan - total + (warp ? warp_total[warp - 1] : 0u) + before;
    // tiles: a warp's keys are consecutive, so ranks follow the order of the keys
    for (int t0 = 0; t0 < n; t0 += items * kSortThreads) {
      for (int b = tid; b < kSortWarps * bins / 2; b += kSortThreads) reinterpret_cast<uint32_t*>(count)[b] = 0u;
      __syncthreads();
      uint2 key[kMaxItems];
      uint32_t before_me[kMaxItems];
      unsigned short* mine = count + warp * bins;
#pragma unroll
      for (int j = 0; j < kMaxItems; ++j) {
        const int i = t0 + (warp * items + j) * 32 + lane;
        const bool real = j < items && i < n;
        key[j] = real ? load(i) : make_uint2(0u, 0u);
        const uint32_t digit = real ? key[j].x >> shift & (bins - 1) : 0xffffffffu;
        const uint32_t same = __match_any_sync(0xffffffffu, digit), lower = same & ((1u << lane) - 1);
        const uint32_t old = real ? mine[digit] : 0u;
        __syncwarp();
        if (real && lower == 0) mine[digit] = (unsigned short)(old + __popc(same));
        __syncwarp();
        before_me[j] = old + __popc(lower);
      }
      __syncthreads();
      uint32_t sum = 0;
      if (tid < bins)
        for (int w = 0; w < kSortWarps; ++w) {
          const uint32_t c = count[w * bins + tid];
          count[w * bins + tid] = (unsigned short)sum;
          sum += c;
        }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kMaxItems; ++j) {
        const int i = t0 + (warp * items + j) * 32 + lane;
        if (j < items && i < n) {
          const uint32_t digit = key[j].x >> shift & (bins - 1);
          dst[base[digit] + mine[digit] + before_me[j]] = key[j];
        }
      }
      __syncthreads();
      if (tid < bins) base[tid] += sum;
    }
    cluster.sync();      // the pass has been written, and every histogram read
    uint2* t = src; src = dst; dst = t;
  }
  for (int i = tid; i < n; i += kSortThreads) {
    const uint32_t key = __ldcg(src + first + i).x;
    if (key < a.vocab && (first + i == 0 || __ldcg(src + first + i - 1).x != key)) atomicOr(present + key / 32, 1u << (key % 32));
  }
}

// ---- rows
struct RowsArgs {
  const uint2* pairs; const uint32_t* present; int words;
  const char* dout; int64_t ld;
  float* table; int64_t worker_stride, row_stride;
  float* pieces;               // [worker][chunk][2][width]: of a run that began before the chunk, and of one that goes on behind it
  int64_t vocab;
  int workers, rows, chunks, slabs, width, sum_ctas;
  float scale;
};

template <typename T, bool ANY>
__device__ __forceinline__ void write_floats(float* row, const float (&f)[Slab<T, ANY>::V], float scale, int c, int width) {
  using S = Slab<T, ANY>;
  if constexpr (ANY) {
#pragma unroll
    for (int j = 0; j < S::V; ++j)
      if (c + S::col(j) < width) row[c + S::col(j)] = f[j] * scale;
  } else {
    if (c + S::col(0) < width) {
#pragma unroll
      for (int j = 0; j < S::V; j += 4)
        __stcs(reinterpret_cast<float4*>(row + c + S::col(j)), make_float4(f[j] * scale, f[j + 1] * scale, f[j + 2] * scale, f[j + 3] * scale));
    }
  }
}

template <typename T, bool ANY>
__global__ void __launch_bounds__(kThreads) embed_rows_kernel(const RowsArgs a) {
  using S = Slab<T, ANY>;
  constexpr int V = S::V, kAhead = 8;
  wait_for_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  if ((int)blockIdx.x >= a.sum_ctas) {      // rows of absent tokens: 32 of them, a word of the bitmap, per CTA
    const int64_t word = blockIdx.x - a.sum_ctas, worker = word / a.words;
    const int v0 = (int)(word - worker * a.words) * 32;
    const uint32_t present = a.present[word];
    for (int i = warp; i < 32 && v0 + i < a.vocab; i += kWarps) {
      if (present >> i & 1u) continue;
      float* row = a.table + worker * a.worker_stride + (int64_t)(v0 + i) * a.row_stride;
      if constexpr (ANY) {
        for (int c = lane; c < a.width; c += 32) row[c] = 0.f;
      } else {
        for (int c = lane * 4; c < a.width; c += 128) __stcs(reinterpret_cast<float4*>(row + c), make_float4(0.f, 0.f, 0.f, 0.f));
      }
    }
    return;
  }
  const int64_t item = (int64_t)blockIdx.x * kWarps + warp;
  if (item >= (int64_t)a.workers * a.chunks * a.slabs) return;
  const int64_t wc = item / a.slabs, worker = wc / a.chunks;
  const int c = (int)(item - wc * a.slabs) * S::kColumns, first = (int)(wc - worker * a.chunks) * kChunk, n = min(kChunk, a.rows - first);
  const uint2* e = a.pairs + worker * a.rows + first;
  const T* dout = reinterpret_cast<const T*>(a.dout) + worker * a.rows * a.ld;
  // this chunk's pairs, two a lane, and the tokens beside it (all ones: none)
  const uint2 none = make_uint2(0xffffffffu, 0u);
  const uint2 p0 = lane < n ? e[lane] : none, p1 = lane + 32 < n ? e[lane + 32] : none;
  const uint32_t before = first > 0 ? e[-1].x : 0xffffffffu, after = first + n < a.rows ? e[n].x : 0xffffffffu;
  // real tokens come first; a pair ends a run where the next one's token differs
  uint32_t next0 = __shfl_down_sync(0xffffffffu, p0.x, 1), next1 = __shfl_down_sync(0xffffffffu, p1.x, 1);
  const uint32_t head1 = __shfl_sync(0xffffffffu, p1.x, 0);
  if (lane == 31) { next0 = head1; next1 = after; }
  if (lane == n - 1) next0 = after;
  if (lane + 32 == n - 1) next1 = after;
  const int real = __popc(__ballot_sync(0xffffffffu, p0.x < (uint32_t)a.vocab)) + __popc(__ballot_sync(0xffffffffu, p1.x < (uint32_t)a.vocab));
  const uint64_t ends = (uint64_t)__ballot_sync(0xffffffffu, p1.x != next1) << 32 | __ballot_sync(0xffffffffu, p0.x != next0);
  float* pieces = a.pieces + wc * 2 * a.width;
  bool cut = before == __shfl_sync(0xffffffffu, p0.x, 0);      // the current run began before this chunk
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
  for (int i0 = 0; i0 < real; i0 += kAhead) {
    Vals<V> x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = i0 + k;
      const uint32_t at = __shfl_sync(0xffffffffu, i0 < 32 ? p0.y : p1.y, i & 31);
      const T* row = dout + (int64_t)at * a.ld;
      if constexpr (ANY) {
#pragma unroll
        for (int j = 0; j < V; ++j) x[k].v[j] = i < real && c + S::col(j) < a.width ? to_f32(row[c + S::col(j)]) : 0.f;
      } else {
        ActPack<T, V> r;
        zero(r);
        if (i < real && c + S::col(0) < a.width) r = load_stream<T, V>(row + c + S::col(0));
        x[k] = unpack<T, V>(r);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = i0 + k;
      if (i >= real) break;
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] += x[k].v[j];
      if (ends >> i & 1u) {
        const uint32_t key = __shfl_sync(0xffffffffu, i < 32 ? p0.x : p1.x, i & 31);
        if (cut) write_floats<T, ANY>(pieces, acc, 1.f, c, a.width);
        else write_floats<T, ANY>(a.table + worker * a.worker_stride + (int64_t)key * a.row_stride, acc, a.scale, c, a.width);
        cut = false;
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
      }
    }
  }
  if (real > 0 && !(ends >> (real - 1) & 1u)) write_floats<T, ANY>(cut ? pieces : pieces + a.width, acc, 1.f, c, a.width);      // goes on in the next chunk
}

// A run that crosses chunks belongs to the chunk that it starts in.
template <typename T, bool ANY>
__global__ void __launch_bounds__(kThreads) embed_joins_kernel(const RowsArgs a) {
  using S = Slab<T, ANY>;
  constexpr int V = S::V;
  wait_for_previous();
  const int64_t item = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32;
  if (item >= (int64_t)a.workers * a.chunks * a.slabs) return;
  const int64_t wc = item / a.slabs, worker = wc / a.chunks;
  const int c = (int)(item - wc * a.slabs) * S::kColumns, chunk = (int)(wc - worker * a.chunks), first = chunk * kChunk, end = first + kChunk;
  const uint2* e = a.pairs + worker * a.rows;
  if (end >= a.rows) return;
  const uint32_t key = e[end - 1].x;
  if (key >= (uint32_t)a.vocab || e[end].x != key || (first > 0 && e[first - 1].x == key)) return;
  const float* piece = a.pieces + wc * 2 * a.width;
  auto read = [&](const float* p, float (&f)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] += c + S::col(j) < a.width ? p[c + S::col(j)] : 0.f;
  };
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
  read(piece + a.width, acc);
  for (int k = chunk + 1; k < a.chunks && e[k * kChunk].x == key; ++k) {
    piece += 2 * a.width;
    read(piece, acc);
  }
  write_floats<T, ANY>(a.table + worker * a.worker_stride + (int64_t)key * a.row_stride, acc, a.scale, c, a.width);
}

// ---- host
int check_common(const char* who, int dtype, int workers, int64_t rows, int64_t vocab, int64_t width, const void* tokens, int token_bytes, int64_t ld_tokens,
                 const float* table, int64_t worker_stride, int64_t row_stride, double scale, const void* x, int64_t ld_x) {
  const int b = dtype_bytes(dtype);
  if (b == 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (workers < 1 || workers > FGD_MAX_K || rows < 0 || rows > 0x7fffffff - 65536 || vocab < 1 || vocab > kMaxVocab || width < 1)
    return op_fail(FGD_ERR_INVALID_ARG, "%s: workers=%d, rows=%lld, vocab=%lld, width=%lld out of range", who, workers, (long long)rows, (long long)vocab, (long long)width);
  if (width > kMaxWidth) return op_fail(FGD_ERR_UNSUPPORTED, "%s: width %lld above %lld", who, (long long)width, (long long)kMaxWidth);
  if (token_bytes != 4 && token_bytes != 8) return op_fail(FGD_ERR_INVALID_ARG, "%s: token_bytes %d", who, token_bytes);
  if (!std::isfinite(scale)) return op_fail(FGD_ERR_INVALID_ARG, "%s: scale is not finite", who);
  if (!table || (rows > 0 && (!tokens || !x))) return op_fail(FGD_ERR_INVALID_ARG, "%s: NULL pointer", who);
  if (rows > 0 && (ld_tokens < rows || ld_x < width)) return op_fail(FGD_ERR_INVALID_ARG, "%s: a row stride is below the row's width", who);
  if (row_stride < width || (workers > 1 && worker_stride < (vocab - 1) * row_stride + width))
    return op_fail(FGD_ERR_INVALID_ARG, "%s: rows of the table overlap one another", who);
  if (reinterpret_cast<uintptr_t>(tokens) % token_bytes != 0 || reinterpret_cast<uintptr_t>(table) % 4 != 0 || reinterpret_cast<uintptr_t>(x) % b != 0)
    return op_fail(FGD_ERR_INVALID_ARG, "%s: a pointer is not on a boundary of its elements", who);
  return FGD_OK;
}
Span table_span(const float* table, int workers, int64_t vocab, int64_t width, int64_t worker_stride, int64_t row_stride) {
  return span_of(table, workers, (vocab - 1) * row_stride + width, worker_stride, 4);
}
// 16-byte accesses everywhere?
bool aligned(const float* table, int64_t worker_stride, int64_t row_stride, int workers, const void* x, int64_t ld, int b, int64_t width) {
  return ((reinterpret_cast<uintptr_t>(table) | reinterpret_cast<uintptr_t>(x)) & 15u) == 0 && (workers == 1 || worker_stride % 4 == 0) && row_stride % 4 == 0 &&
         (ld * b) % 16 == 0 && (width * b) % 16 == 0;
}

int64_t round16(int64_t n) { return (n + 15) / 16 * 16; }
struct Layout { int64_t pairs, other, present, pieces, total; int chunks, words; };
Layout layout_of(int64_t workers, int64_t rows, int64_t vocab, int64_t width) {
  Layout l;
  l.chunks = (int)((rows + kChunk - 1) / kChunk);
  l.words = (int)((vocab + 31) / 32);
  l.pairs = 0;
  l.other = l.pairs + round16(workers * rows * (int64_t)sizeof(uint2));
  l.present = l.other + round16(workers * rows * (int64_t)sizeof(uint2));
  l.pieces = l.present + round16(workers * l.words * 4);
  l.total = l.pieces + (l.chunks > 1 ? workers * l.chunks * 2 * round16(width * 4) : 0);
  return l;
}

template <typename T, bool ANY>
cudaError_t forward(const EmbedArgs& e, cudaStream_t st) {
  EmbedArgs a = e;
  a.parts = (a.width + kSlabs * Slab<T, ANY>::kColumns - 1) / (kSlabs * Slab<T, ANY>::kColumns);
  const int64_t ctas = (a.tokens_total * a.parts + kWarps - 1) / kWarps, most = (int64_t)sm_count() * 64;
  embed_forward_kernel<T, ANY><<<(unsigned)(ctas < most ? ctas : most), kThreads, 0, st>>>(a);
  return cudaGetLastError();
}
template <typename T, bool ANY>
cudaError_t backward(const RowsArgs& r, cudaStream_t st) {
  RowsArgs a = r;
  a.slabs = (a.width + Slab<T, ANY>::kColumns - 1) / Slab<T, ANY>::kColumns;
  const int64_t sums = ((int64_t)a.workers * a.chunks * a.slabs + kWarps - 1) / kWarps;
  a.sum_ctas = (int)sums;
  cudaError_t e = launch_early(embed_rows_kernel<T, ANY>, dim3((unsigned)(sums + (int64_t)a.workers * a.words)), kThreads, 0, st, a);
  if (e == cudaSuccess && a.chunks > 1) e = launch_early(embed_joins_kernel<T, ANY>, dim3((unsigned)sums), kThreads, 0, st, a);
  return e;
}
cudaError_t sort(const SortArgs& a, int workers, cudaStream_t st) {
  const size_t smem = ((size_t)8 << a.bits) + ((size_t)kSortWarps * 2 << a.bits);
  cudaError_t e = allow_smem<embed_sort_kernel>(((size_t)8 << kMaxBits) + ((size_t)kSortWarps * 2 << kMaxBits));
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = a.cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3((unsigned)(workers * a.cluster));
  c.blockDim = dim3(kSortThreads);
  c.dynamicSmemBytes = smem;
  c.stream = st;
  c.attrs = &attr;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, embed_sort_kernel, a);
}

// f(a value of the activation type, 16-byte accesses or not)
template <typename F>
cudaError_t by_type(int dtype, bool any, F f) {
  switch (dtype) {
    case FGD_F32: return any ? f(float{}, std::true_type{}) : f(float{}, std::false_type{});
    case FGD_BF16: return any ? f(__nv_bfloat16{}, std::true_type{}) : f(__nv_bfloat16{}, std::false_type{});
    default: return any ? f(__half{}, std::true_type{}) : f(__half{}, std::false_type{});
  }
}

}  // namespace

extern "C" int64_t fgd_embed_workspace(int workers, int64_t rows, int64_t vocab, int64_t width) {
  if (workers < 1 || workers > FGD_MAX_K || rows < 0 || rows > 0x7fffffff - 65536 || vocab < 1 || vocab > kMaxVocab || width < 1 || width > kMaxWidth) return FGD_ERR_INVALID_ARG;
  return layout_of(workers, rows, vocab, width).total;
}

extern "C" int fgd_embed_forward(int device, int dtype, int workers, int64_t rows, int64_t vocab, int64_t width, const void* tokens, int token_bytes,
                                 int64_t ld_tokens, const float* table, int64_t worker_stride, int64_t row_stride, double scale, void* out, int64_t ld_out,
                                 void* stream) {
  FGD_NVTX_RANGE("fgd_embed_forward");
  const char* who = "fgd_embed_forward";
  if (int rc = check_common(who, dtype, workers, rows, vocab, width, tokens, token_bytes, ld_tokens, table, worker_stride, row_stride, scale, out, ld_out)) return rc;
  if (rows == 0) return FGD_OK;
  const int b = dtype_bytes(dtype);
  const Span so = span_of(out, workers * rows, width, ld_out, b);
  if (so.overlaps(table_span(table, workers, vocab, width, worker_stride, row_stride)) || so.overlaps(span_of(tokens, workers, rows, ld_tokens, token_bytes)))
    return op_fail(FGD_ERR_ALIAS, "%s: out overlaps the tokens or the table", who);
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  EmbedArgs a = {};
  a.tokens = Tokens{tokens, token_bytes, ld_tokens};
  a.table = table; a.worker_stride = worker_stride; a.row_stride = row_stride;
  a.out = static_cast<char*>(out); a.ld_out = ld_out;
  a.rows = rows; a.tokens_total = workers * rows; a.vocab = vocab; a.width = (int)width; a.scale = (float)scale;
  const cudaError_t e = by_type(dtype, !aligned(table, worker_stride, row_stride, workers, out, ld_out, b, width),
                                [&](auto zero, auto any) { return forward<decltype(zero), decltype(any)::value>(a, static_cast<cudaStream_t>(stream)); });
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

extern "C" int fgd_embed_backward(int device, int dtype, int workers, int64_t rows, int64_t vocab, int64_t width, const void* tokens, int token_bytes,
                                  int64_t ld_tokens, const void* dout, int64_t ld_dout, double scale, float* dtable, int64_t worker_stride, int64_t row_stride,
                                  void* workspace, int64_t workspace_bytes, void* stream) {
  FGD_NVTX_RANGE("fgd_embed_backward");
  const char* who = "fgd_embed_backward";
  if (int rc = check_common(who, dtype, workers, rows, vocab, width, tokens, token_bytes, ld_tokens, dtable, worker_stride, row_stride, scale, dout, ld_dout)) return rc;
  const int b = dtype_bytes(dtype);
  const Layout l = layout_of(workers, rows, vocab, width);
  if (!workspace || workspace_bytes < l.total || reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
    return op_fail(FGD_ERR_INVALID_ARG, "%s: needs a workspace of %lld bytes on a 16-byte boundary (fgd_embed_workspace)", who, (long long)l.total);
  const Span st_ = table_span(dtable, workers, vocab, width, worker_stride, row_stride), sw = span_of(workspace, 1, l.total, l.total, 1);
  const Span sx = span_of(dout, workers * rows, width, ld_dout, b), sk = span_of(tokens, workers, rows, ld_tokens, token_bytes);
  if (st_.overlaps(sx) || st_.overlaps(sk) || st_.overlaps(sw) || sw.overlaps(sx) || sw.overlaps(sk)) return op_fail(FGD_ERR_ALIAS, "%s: dtable or the workspace overlaps another tensor", who);
  const int64_t ctas = (int64_t)workers * l.words + (int64_t)workers * l.chunks * ((width + 127) / 128);
  if (ctas > 0x7fffffff) return op_fail(FGD_ERR_UNSUPPORTED, "%s: more work than one launch holds", who);
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  char* ws = static_cast<char*>(workspace);
  SortArgs s = {};
  s.tokens = Tokens{tokens, token_bytes, ld_tokens};
  s.vocab = vocab; s.rows = (int)rows;
  s.cluster = rows <= kSortFew ? 1 : kCluster;
  int bits = 1;
  while ((int64_t)1 << bits <= vocab) ++bits;      // keys 0 .. vocab
  s.passes = (bits + kMaxBits - 1) / kMaxBits;
  s.bits = (bits + s.passes - 1) / s.passes;
  s.pairs = reinterpret_cast<uint2*>(ws + l.pairs); s.other = reinterpret_cast<uint2*>(ws + l.other);
  s.present = reinterpret_cast<uint32_t*>(ws + l.present); s.words = l.words;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = sort(s, workers, st);
  if (e == cudaSuccess) {
    RowsArgs r = {};
    r.pairs = s.pairs; r.present = s.present; r.words = l.words;
    r.dout = static_cast<const char*>(dout); r.ld = ld_dout;
    r.table = dtable; r.worker_stride = worker_stride; r.row_stride = row_stride;
    r.pieces = reinterpret_cast<float*>(ws + l.pieces);
    r.vocab = vocab; r.workers = workers; r.rows = (int)rows; r.chunks = l.chunks; r.width = (int)width; r.scale = (float)scale;
    e = by_type(dtype, !aligned(dtable, worker_stride, row_stride, workers, dout, ld_dout, b, width),
                [&](auto zero, auto any) { return backward<decltype(zero), decltype(any)::value>(r, st); });
  }
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

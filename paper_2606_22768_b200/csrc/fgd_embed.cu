// Embeddings of K workers' tokens, and the gradient of their tables.
//
// Forward: a row of the table, scaled and rounded once, for every token.
// Backward: dtable[v] = scale * sum of dout[t] over the tokens t that are v, for every row v.  Text repeats few tokens very often (the
// commonest may be 7 % of a batch) and most of a vocabulary not at all, so the work is cut by tokens, not by rows, without atomics on floats:
//   sort   each worker's (token, position) pairs by token, stable, in one launch: a cluster of CTAs per worker, radix passes of up to ten bits;
//          histograms cross the cluster through distributed shared memory.  Marks the tokens that occur in a bitmap.
//   rows   the sorted list in chunks: a warp adds up the runs of equal tokens within its chunk, for 32 lanes x 16 bytes of columns.  A run that
//          lies inside the chunk is a finished row; the pieces of one that crosses chunks go to scratch.  Other CTAs write the rows of
//          absent tokens with zeros.
//   joins  the pieces of the runs that cross chunks, which are few, eight warps to a run.
// A few tokens need no sort: a warp looks through all of them for the one that its row of the table stands for, in one launch.
// The order of every sum depends on the tokens and the sizes alone: workers, rows, vocabulary and width say which kernels run and how long the chunks are.
// 4 x 8192 tokens of 32000 rows, 2048 wide, bf16: 187 us, 95 % of the copy peak (sort 13, rows and zeros 168, joins 6); 65536 tokens of 50257, 1536 wide, f16:
// 121 us (25, 84, 12).
#include <cooperative_groups.h>

#include <cmath>

#include "fgd_dtype.cuh"
#include "fgd_nvtx.h"

using namespace fgd;
namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kCluster = 16;          // CTAs that sort one worker's tokens, at most
constexpr int kItems = 8;             // keys of a thread in one tile
constexpr int kMaxBits = 10;          // of a radix pass
constexpr int kChunk = 64, kShortChunk = 16;      // sorted tokens that a warp adds up
constexpr int kNoSort = 512;          // tokens of a worker up to which they may go unsorted
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
  int64_t rows, vocab;
  int width;
  float scale;
};
constexpr int kSlabs = 4;

// A warp has kSlabs slabs on their way at once: of one row, or where a row is no more than one (SHORT) of as many rows.  4 x 8192 tokens of 2048 bf16
// 39 us, 94 % of the copy peak (with rows and slabs mixed freely 61: every slab then has its own token, and its place to be worked out); 41160 tokens of
// 1002 columns 22 us, 57 %.  CTAs to an SM: as many as the registers of the loads in flight allow (six of five: 45 us).
template <typename T, bool ANY, bool SHORT>
__global__ void __launch_bounds__(kThreads, SHORT ? 3 : ANY ? 4 : 5) embed_forward_kernel(const EmbedArgs a) {
  using S = Slab<T, ANY>;
  constexpr int V = S::V, ROWS = SHORT ? kSlabs : 1;
  // the worker is the grid's second axis: 64-bit divisions would be a good part of the instructions
  const int64_t worker = wait_for_previous((int)blockIdx.y), t0 = ((int64_t)blockIdx.x * kWarps + threadIdx.x / 32) * ROWS;
  if (t0 >= a.rows) return;
  const float* row[ROWS];
  float other[ROWS];           // of a token outside the vocabulary
  bool real[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int64_t tok = a.tokens.at(worker, t0 + r < a.rows ? t0 + r : t0);
    real[r] = tok >= 0 && tok < a.vocab;
    other[r] = tok < 0 ? 0.f : __int_as_float(0x7fffffff);
    row[r] = a.table + worker * a.worker_stride + (real[r] ? tok : 0) * a.row_stride;
  }
  T* const out0 = reinterpret_cast<T*>(a.out) + (worker * a.rows + t0) * a.ld_out;
  for (int c0 = blockIdx.z * (kSlabs * S::kColumns); c0 < a.width; c0 += gridDim.z * (kSlabs * S::kColumns)) {
    Vals<V> v[kSlabs];
#pragma unroll
    for (int s = 0; s < kSlabs; ++s) {
      const int r = SHORT ? s : 0, c = SHORT ? 0 : c0 + s * S::kColumns;
      if constexpr (ANY) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[s].v[j] = real[r] && c + S::col(j) < a.width ? __ldg(row[r] + c + S::col(j)) : other[r];
      } else {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
          float4 f = make_float4(other[r], other[r], other[r], other[r]);
          if (real[r] && c + S::col(0) < a.width) f = __ldg(reinterpret_cast<const float4*>(row[r] + c + S::col(j)));
          v[s].v[j] = f.x; v[s].v[j + 1] = f.y; v[s].v[j + 2] = f.z; v[s].v[j + 3] = f.w;
        }
      }
    }
#pragma unroll
    for (int s = 0; s < kSlabs; ++s) {
      if (SHORT && t0 + s >= a.rows) break;
      T* out = out0 + (SHORT ? s : 0) * a.ld_out;
      const int c = SHORT ? 0 : c0 + s * S::kColumns;
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
  int workers, rows, cluster, bits, passes;
  uint2 *pairs, *other;        // [worker][rows]: the result, and what the passes alternate with
  uint32_t* present; int words;      // [worker][words] bitmap of the vocabulary
  int* joins;                  // length of the list of runs that cross chunks: cleared here
};

// Lanes whose digit is this lane's: a ballot for every bit.  (`real` lanes among themselves.)
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, bool real, int bits) {
  uint32_t same = __ballot_sync(0xffffffffu, real);
  for (int b = 0; b < bits; ++b) {
    const bool one = digit >> b & 1u;
    const uint32_t ones = __ballot_sync(0xffffffffu, one);
    same &= one ? ones : ~ones;
  }
  return same;
}

// Pairs (token, position); a token outside the vocabulary counts as `vocab` and comes last.
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(const SortArgs a) {
  const cg::cluster_group cluster = cg::this_cluster();
  asm volatile("barrier.cluster.arrive;" ::: "memory");      // its wait: before the first store to another CTA, which has to be there by then
  extern __shared__ __align__(16) unsigned char smem[];
  const int bins = 1 << a.bits, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x % a.cluster;
  const int64_t worker = wait_for_previous((int)(blockIdx.x / a.cluster));
  uint32_t* hist = reinterpret_cast<uint32_t*>(smem);                       // [cluster][bins] of all CTAs' parts
  uint32_t* base = hist + a.cluster * bins;                                  // [bins] where the next key of a digit goes
  unsigned short* count = reinterpret_cast<unsigned short*>(base + bins);    // [warp][bins] of a tile
  __shared__ uint32_t warp_total[kSortWarps];
  uint32_t* present = a.present + worker * a.words;
  for (int i = rank * kSortThreads + tid; i < a.words; i += a.cluster * kSortThreads) present[i] = 0u;
  if (blockIdx.x == 0 && tid == 0) *a.joins = 0;
  const int part = (a.rows + a.cluster - 1) / a.cluster, first = min(rank * part, a.rows), n = min(part, a.rows - first);
  const int items = part >= kItems * kSortThreads ? kItems : (part + kSortThreads - 1) / kSortThreads, tile = items * kSortThreads;
  uint2 *dst = a.passes & 1 ? a.pairs : a.other, *src = a.passes & 1 ? a.other : a.pairs;      // the last pass writes the result
  dst += worker * a.rows; src += worker * a.rows;
  unsigned short* mine = count + warp * bins;
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = pass * a.bits;
    uint2 key[kItems];
    uint32_t before_me[kItems];      // keys of the same digit earlier in the warp's part of the tile
    // a warp's keys are consecutive, so ranks follow the order of the keys
    auto load = [&](int t0) {
#pragma unroll
      for (int j = 0; j < kItems; ++j) {
        const int i = t0 + (warp * items + j) * 32 + lane;
        if (j >= items || i >= n) continue;
        if (pass > 0) {
          key[j] = __ldcg(src + first + i);
        } else {
          const int64_t tok = a.tokens.at(worker, first + i);
          key[j] = make_uint2(tok >= 0 && tok < a.vocab ? (uint32_t)tok : (uint32_t)a.vocab, (uint32_t)(first + i));
        }
      }
    };
    auto rank_tile = [&](int t0) {      // -> before_me and the warps' counts
      for (int b = tid; b < kSortWarps * bins / 2; b += kSortThreads) reinterpret_cast<uint32_t*>(count)[b] = 0u;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kItems; ++j) {
        if (j >= items) break;
        const bool real = t0 + (warp * items + j) * 32 + lane < n;
        const uint32_t digit = real ? key[j].x >> shift & (bins - 1) : 0u;
        const uint32_t same = same_digit(digit, real, a.bits), lower = same & ((1u << lane) - 1);
        const uint32_t old = real ? mine[digit] : 0u;
        __syncwarp();
        if (real && lower == 0) mine[digit] = (unsigned short)(old + __popc(same));
        __syncwarp();
        before_me[j] = old + __popc(lower);
      }
      __syncthreads();
    };
    auto sum_warps = [&]() -> uint32_t {      // counts become those of the warps before; -> the tile's of bin `tid`
      uint32_t sum = 0;
      if (tid < bins) {
        uint32_t c[kSortWarps];
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) c[w] = count[w * bins + tid];
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
          count[w * bins + tid] = (unsigned short)sum;
          sum += c[w];
        }
      }
      return sum;
    };
    // this CTA's histogram: of its only tile as it is ranked, of several beforehand
    const bool single = n <= tile;
    uint32_t tile_sum = 0;
    if (single) {
      load(0);
      rank_tile(0);
      tile_sum = sum_warps();
    } else {
      if (tid < bins) base[tid] = 0u;
      for (int t0 = 0; t0 < n; t0 += tile) {
        load(t0);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kItems; ++j) {
          const bool real = j < items && t0 + (warp * items + j) * 32 + lane < n;
          const uint32_t digit = real ? key[j].x >> shift & (bins - 1) : 0u;
          const uint32_t same = same_digit(digit, real, a.bits);
          if (real && (same & ((1u << lane) - 1)) == 0) atomicAdd(&base[digit], (uint32_t)__popc(same));
        }
      }
      __syncthreads();
    }
    // to every CTA of the cluster: stores, which nothing waits for as it would for loads (4 x 8192 tokens 1 us less)
    if (pass == 0) asm volatile("barrier.cluster.wait;" ::: "memory");
    if (tid < bins) {
      const uint32_t h = single ? tile_sum : base[tid];
      for (int r = 0; r < a.cluster; ++r) cluster.map_shared_rank(hist, r)[rank * bins + tid] = h;
    }
    cluster.sync();
    // where each digit starts: keys of smaller digits anywhere, and of this digit in the CTAs before; bins <= kSortThreads
    uint32_t before = 0, total = 0;
    if (tid < bins) {
#pragma unroll
      for (int r = 0; r < kCluster; ++r)
        if (r < a.cluster) {
          const uint32_t h = hist[r * bins + tid];
          total += h;
          if (r < rank) before += h;
        }
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
    for (int t0 = 0; t0 < n; t0 += tile) {
      if (!single) {
        load(t0);
        rank_tile(t0);
        tile_sum = sum_warps();
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kItems; ++j) {
        if (j < items && t0 + (warp * items + j) * 32 + lane < n) {
          const uint32_t digit = key[j].x >> shift & (bins - 1);
          dst[base[digit] + mine[digit] + before_me[j]] = key[j];
        }
      }
      __syncthreads();
      if (tid < bins) base[tid] += tile_sum;
    }
    cluster.sync();      // the pass has been written, and every histogram read
    uint2* t = src; src = dst; dst = t;
  }
  for (int i0 = 0; i0 < n; i0 += kItems * kSortThreads) {
    uint32_t key[kItems], prev[kItems];
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
      const int i = i0 + j * kSortThreads + tid;
      key[j] = i < n ? __ldcg(src + first + i).x : (uint32_t)a.vocab;
      prev[j] = i < n && first + i > 0 ? __ldcg(src + first + i - 1).x : 0xffffffffu;
    }
#pragma unroll
    for (int j = 0; j < kItems; ++j)
      if (key[j] < a.vocab && prev[j] != key[j]) atomicOr(present + key[j] / 32, 1u << (key[j] % 32));
  }
}

// ---- rows
struct RowsArgs {
  const uint2* pairs; const uint32_t* present; int words;
  const char* dout; int64_t ld;
  float* table; int64_t worker_stride, row_stride;
  float* pieces;               // [worker][chunk][2][width]: of a run that began before the chunk, and of one that goes on behind it
  int64_t vocab;
  int* joins; uint2* list;     // how many runs cross chunks; the chunks (of all workers) that they start in, their tokens
  int workers, rows, chunk, chunks, slabs, width, sum_ctas, cta_words, zero_lanes;
  float scale;
};

// A lane's values of a row, slab at column c.  ANY: loads without a condition, of the last column where there is none (what comes of it is never
// written): as branches around a load and its conversion they would wait for one another, 44 us instead of 11 for 8 x 107 tokens of 438 columns.
template <typename T, bool ANY>
__device__ __forceinline__ Vals<Slab<T, ANY>::V> load_values(const T* row, int c, int width, bool real) {
  using S = Slab<T, ANY>;
  Vals<S::V> x;
  if constexpr (ANY) {
#pragma unroll
    for (int j = 0; j < S::V; ++j) x.v[j] = to_f32(row[min(c + S::col(j), width - 1)]);
  } else {
    ActPack<T, S::V> r;
    zero(r);
    if (real && c + S::col(0) < width) r = load_stream<T, S::V>(row + c + S::col(0));
    x = unpack<T, S::V>(r);
  }
  return x;
}
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
  if ((int)blockIdx.x >= a.sum_ctas) {      // rows of absent tokens: some words of the bitmap, 32 rows each
    const int per_worker = (a.words + a.cta_words - 1) / a.cta_words, cta = blockIdx.x - a.sum_ctas;
    const int64_t worker = cta / per_worker;
    const int first = (int)(cta - worker * per_worker) * a.cta_words, last = min(first + a.cta_words, a.words);
    float* table = a.table + worker * a.worker_stride;
    // zero_lanes of a warp to a row
    const int group = lane / a.zero_lanes, groups = 32 / a.zero_lanes, l = lane % a.zero_lanes;
    for (int64_t v = (int64_t)first * 32 + warp * groups + group; v < (int64_t)last * 32 && v < a.vocab; v += kWarps * groups) {
      if (a.present[worker * a.words + v / 32] >> (v % 32) & 1u) continue;
      float* row = table + v * a.row_stride;
      if constexpr (ANY) {
        for (int c = l; c < a.width; c += a.zero_lanes) row[c] = 0.f;
      } else {
        for (int c = l * 4; c < a.width; c += a.zero_lanes * 4) __stcs(reinterpret_cast<float4*>(row + c), make_float4(0.f, 0.f, 0.f, 0.f));
      }
    }
    return;
  }
  const int64_t item = (int64_t)blockIdx.x * kWarps + warp;
  if (item >= (int64_t)a.workers * a.chunks * a.slabs) return;
  const int64_t wc = item / a.slabs, worker = wc / a.chunks;
  const int c = (int)(item - wc * a.slabs) * S::kColumns, first = (int)(wc - worker * a.chunks) * a.chunk, n = min(a.chunk, a.rows - first);
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
      const uint32_t at = __shfl_sync(0xffffffffu, i0 < 32 ? p0.y : p1.y, i & 31);      // (0 behind the last)
      x[k] = load_values<T, ANY>(dout + (int64_t)at * a.ld, c, a.width, i < real);
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
  if (real > 0 && !(ends >> (real - 1) & 1u)) {      // goes on in the next chunk
    write_floats<T, ANY>(cut ? pieces : pieces + a.width, acc, 1.f, c, a.width);
    const uint32_t key = __shfl_sync(0xffffffffu, real > 32 ? p1.x : p0.x, (real - 1) & 31);
    if (!cut && c == 0 && lane == 0) a.list[atomicAdd(a.joins, 1)] = make_uint2((uint32_t)wc, key);
  }
}

// Runs that cross chunks, listed in no particular order by the chunk that they start in.  128 columns to a CTA, a run to each of its warps, from all over
// the list: long runs stand together in it where common tokens have neighbouring numbers (65536 tokens 4 us less than with eight in a row).  Where the run
// has more than kPieces further pieces, all warps share it: of 8 kPieces consecutive ones each adds kPieces, and their sums are added in
// the warps' order.
constexpr int kPieces = 8;
__global__ void __launch_bounds__(kThreads) embed_joins_kernel(const RowsArgs a) {
  __shared__ __align__(16) float sums[kWarps][128];
  __shared__ uint2 shared_run[kWarps];
  wait_for_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, c0 = blockIdx.y * 128 + lane;
  const int runs = *a.joins;
  // adds the pieces of the run with this token in the chunks from k on, kPieces at most; -> how many there were.  FIRST: the one in chunk k is
  // known to exist, and is fetched with the tokens that tell of the others.
  auto add = [&](auto first, float (&acc)[4], const uint2* e, const float* pieces, uint32_t key, int64_t k) -> int {
    constexpr bool FIRST = decltype(first)::value;
    const bool has = lane < kPieces && k + lane < a.chunks && e[(k + lane) * a.chunk].x == key;
    float p[kPieces][4];
    if constexpr (FIRST) {
#pragma unroll
      for (int j = 0; j < 4; ++j) p[0][j] = c0 + 32 * j < a.width ? pieces[k * 2 * a.width + c0 + 32 * j] : 0.f;
    }
    const int n = __popc(__ballot_sync(0xffffffffu, has));      // (the first n)
#pragma unroll
    for (int i = FIRST; i < kPieces; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) p[i][j] = i < n && c0 + 32 * j < a.width ? pieces[(k + i) * 2 * a.width + c0 + 32 * j] : 0.f;
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] += p[i][j];
    return n;
  };
  for (int run0 = blockIdx.x; run0 < runs; run0 += gridDim.x * kWarps) {
    const int mine = run0 + warp * gridDim.x;
    uint2 run = make_uint2(0u, 0u);
    bool longer = false;
    if (mine < runs) {
      run = a.list[mine];
      const int64_t worker = run.x / (uint32_t)a.chunks, chunk = run.x % (uint32_t)a.chunks;
      const uint2* e = a.pairs + worker * a.rows;
      const float* pieces = a.pieces + worker * a.chunks * 2 * a.width;
      const int64_t next = chunk + 1 + kPieces;
      longer = next < a.chunks && e[next * a.chunk].x == run.y;
      float acc[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = c0 + 32 * j < a.width ? pieces[(chunk * 2 + 1) * a.width + c0 + 32 * j] : 0.f;
      if (!longer) {
        add(std::true_type{}, acc, e, pieces, run.y, chunk + 1);
        float* row = a.table + worker * a.worker_stride + (int64_t)run.y * a.row_stride;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c0 + 32 * j < a.width) row[c0 + 32 * j] = acc[j] * a.scale;
      }
    }
    if (!__syncthreads_or(longer)) continue;
    if (lane == 0) shared_run[warp] = longer ? run : make_uint2(0xffffffffu, 0u);
    __syncthreads();
    for (int i = 0; i < kWarps; ++i) {
      const uint2 r = shared_run[i];
      if (r.x == 0xffffffffu) continue;
      const int64_t worker = r.x / (uint32_t)a.chunks, chunk = r.x % (uint32_t)a.chunks;
      const uint2* e = a.pairs + worker * a.rows;
      const float* pieces = a.pieces + worker * a.chunks * 2 * a.width;
      float acc[4] = {0.f, 0.f, 0.f, 0.f};
      for (int64_t k = chunk + 1 + warp * kPieces; add(std::false_type{}, acc, e, pieces, r.y, k) == kPieces; k += kWarps * kPieces) {}
#pragma unroll
      for (int j = 0; j < 4; ++j) sums[warp][lane + 32 * j] = acc[j];
      __syncthreads();
      const int c = blockIdx.y * 128 + threadIdx.x;
      if (threadIdx.x < 128 && c < a.width) {
        float t = pieces[(chunk * 2 + 1) * a.width + c];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) t += sums[w][threadIdx.x];
        a.table[worker * a.worker_stride + (int64_t)r.y * a.row_stride + c] = t * a.scale;
      }
      __syncthreads();
    }
    __syncthreads();
  }
}

// ---- few tokens
struct FewArgs {
  Tokens tokens;
  const char* dout; int64_t ld;
  float* table; int64_t worker_stride, row_stride, vocab;
  int rows, width, slabs;
  float scale;
};
constexpr int kTogether = 32;      // tokens of one row above which all warps add them up together

// A warp has a row of the table: it lists the tokens that are that row's and adds up what belongs to them, eight at a time on their way.
template <typename T, bool ANY>
__global__ void __launch_bounds__(kThreads) embed_few_kernel(const FewArgs a) {
  using S = Slab<T, ANY>;
  constexpr int V = S::V, kAhead = 8;
  __shared__ int tokens[kNoSort];
  __shared__ unsigned short list[kWarps][kNoSort];
  __shared__ int lengths[kWarps];
  __shared__ __align__(16) float sums[kWarps][S::kColumns];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const int64_t worker = wait_for_previous((int)blockIdx.y), v0 = (int64_t)blockIdx.x * kWarps, v = v0 + warp;
  for (int i = threadIdx.x; i < a.rows; i += kThreads) {
    const int64_t tok = a.tokens.at(worker, i);
    tokens[i] = tok >= 0 && tok < a.vocab ? (int)tok : -1;
  }
  __syncthreads();
  int n = 0;
  for (int i0 = 0; i0 < a.rows; i0 += 32) {
    const bool hit = i0 + lane < a.rows && tokens[i0 + lane] == v;
    const uint32_t hits = __ballot_sync(0xffffffffu, hit);
    if (hit) list[warp][n + __popc(hits & ((1u << lane) - 1))] = (unsigned short)(i0 + lane);
    n += __popc(hits);
  }
  if (lane == 0) lengths[warp] = n;
  __syncthreads();
  const T* dout = reinterpret_cast<const T*>(a.dout) + worker * a.rows * a.ld;
  float* table = a.table + worker * a.worker_stride;
  // positions [from, to) of a list
  auto add = [&](const unsigned short* which, int from, int to, int c, float (&acc)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
    for (int i0 = from; i0 < to; i0 += kAhead) {
      Vals<V> x[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const bool real = i0 + k < to;
        x[k] = load_values<T, ANY>(dout + (real ? which[i0 + k] : 0) * a.ld, c, a.width, real);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (i0 + k < to) {
#pragma unroll
          for (int j = 0; j < V; ++j) acc[j] += x[k].v[j];
        }
    }
  };
  float acc[V];
  for (int slab = blockIdx.z; slab < a.slabs; slab += gridDim.z) {
    const int c = slab * S::kColumns;
    if (v < a.vocab && n <= kTogether) {
      add(list[warp], 0, n, c, acc);
      write_floats<T, ANY>(table + v * a.row_stride, acc, a.scale, c, a.width);
    }
    for (int w = 0; w < kWarps; ++w) {
      const int all = lengths[w];
      if (all <= kTogether) continue;      // (the whole CTA)
      const int each = (all + kWarps - 1) / kWarps, from = min(warp * each, all);
      add(list[w], from, min(from + each, all), c, acc);
#pragma unroll
      for (int j = 0; j < V; ++j) sums[warp][S::col(j)] = acc[j];
      __syncthreads();
      for (int i = threadIdx.x; i < S::kColumns; i += kThreads) {
        float t = sums[0][i];
#pragma unroll
        for (int k = 1; k < kWarps; ++k) t += sums[k][i];
        if (c + i < a.width) table[(v0 + w) * a.row_stride + c + i] = t * a.scale;
      }
      __syncthreads();
    }
  }
}

// ---- host
int check_common(const char* who, int dtype, int workers, int64_t rows, int64_t vocab, int64_t width, const void* tokens, int token_bytes, int64_t ld_tokens,
                 const float* table, int64_t worker_stride, int64_t row_stride, bool output, double scale, const void* x, int64_t ld_x) {
  const int b = dtype_bytes(dtype);
  if (b == 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  if (workers < 1 || workers > FGD_MAX_K || rows < 0 || rows > 0x7fffffff - 65536 || vocab < 1 || vocab > kMaxVocab || width < 1)
    return op_fail(FGD_ERR_INVALID_ARG, "%s: workers=%d, rows=%lld, vocab=%lld, width=%lld out of range", who, workers, (long long)rows, (long long)vocab, (long long)width);
  if (width > kMaxWidth) return op_fail(FGD_ERR_UNSUPPORTED, "%s: width %lld above %lld", who, (long long)width, (long long)kMaxWidth);
  if (token_bytes != 4 && token_bytes != 8) return op_fail(FGD_ERR_INVALID_ARG, "%s: token_bytes %d", who, token_bytes);
  if (!std::isfinite((float)scale)) return op_fail(FGD_ERR_INVALID_ARG, "%s: scale is not finite in fp32", who);
  if (!table || (rows > 0 && (!tokens || !x))) return op_fail(FGD_ERR_INVALID_ARG, "%s: NULL pointer", who);
  if (rows > 0 && (ld_tokens < rows || ld_x < width)) return op_fail(FGD_ERR_INVALID_ARG, "%s: a row stride is below the row's width", who);
  if (row_stride < width || worker_stride < 0) return op_fail(FGD_ERR_INVALID_ARG, "%s: a stride of the table is below its row's width, or negative", who);
  if (output && workers > 1 && worker_stride < (vocab - 1) * row_stride + width) return op_fail(FGD_ERR_INVALID_ARG, "%s: the workers' tables overlap one another", who);
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
// Few tokens and little of a table: every warp looks through all tokens for its row.  4 x 384 tokens of 256, 256 wide, bf16: 6.2 us, sorted 20; but
// 4 x 203 of 1195, 2240 wide, 42 us (one warp adds up all columns of a common token), sorted 26, and 2 x 419 of 94350, 264 wide, fp32, 154 us (the looking),
// sorted 47.
bool no_sort(int64_t workers, int64_t rows, int64_t vocab, int64_t width) { return rows <= kNoSort && workers * vocab * ((width + 255) / 256) <= 16384; }
struct Layout { int64_t pairs, other, present, joins, list, pieces, total; int chunk, chunks, words; };
Layout layout_of(int64_t workers, int64_t rows, int64_t vocab, int64_t width) {
  Layout l = {};
  if (no_sort(workers, rows, vocab, width)) return l;
  // Short chunks where long ones would be too few for the SMs' warps.
  l.chunk = workers * (rows / kChunk) * ((width + 255) / 256) < 16 * 148 ? kShortChunk : kChunk;
  l.chunks = (int)((rows + l.chunk - 1) / l.chunk);
  l.words = (int)((vocab + 31) / 32);
  l.other = l.pairs + round16(workers * rows * (int64_t)sizeof(uint2));
  l.present = l.other + round16(workers * rows * (int64_t)sizeof(uint2));
  l.joins = l.present + round16(workers * l.words * 4);
  l.list = l.joins + 16;
  l.pieces = l.list + round16(workers * l.chunks * (int64_t)sizeof(uint2));
  l.total = l.pieces + workers * l.chunks * 2 * round16(width * 4);
  return l;
}

template <typename T, bool ANY>
cudaError_t forward(const EmbedArgs& a, int workers, cudaStream_t st) {
  const int slabs = (a.width + Slab<T, ANY>::kColumns - 1) / Slab<T, ANY>::kColumns;
  const int64_t rows = slabs == 1 ? (a.rows + kSlabs - 1) / kSlabs : a.rows, ctas = (rows + kWarps - 1) / kWarps;
  // a warp goes through its whole row, unless there are few rows: then its parts go to several
  const int64_t parts = (slabs + kSlabs - 1) / kSlabs, cuts = (int64_t)sm_count() * 4 / (ctas * workers) + 1;
  const dim3 grid((unsigned)ctas, (unsigned)workers, (unsigned)(cuts < parts ? cuts : parts));
  // (starting while the kernel before it ends saves 0.2 to 0.5 us, among other work 2)
  return launch_early(slabs == 1 ? embed_forward_kernel<T, ANY, true> : embed_forward_kernel<T, ANY, false>, grid, kThreads, 0, st, a);
}
template <typename T, bool ANY>
cudaError_t backward(const RowsArgs& r, cudaStream_t st) {
  RowsArgs a = r;
  a.slabs = (a.width + Slab<T, ANY>::kColumns - 1) / Slab<T, ANY>::kColumns;
  a.sum_ctas = (int)(((int64_t)a.workers * a.chunks * a.slabs + kWarps - 1) / kWarps);
  // zeros: 256 KB to a CTA, or 32 rows; a float4 (or float) to a lane, as many lanes to a row as have one
  a.cta_words = (int)((256 * 1024) / ((int64_t)a.width * 4 * 32));
  const int64_t share = (int64_t)a.workers * a.words / ((int64_t)sm_count() * 8);      // (no fewer CTAs than the SMs hold)
  if (a.cta_words > share) a.cta_words = (int)share;
  if (a.cta_words < 1) a.cta_words = 1;
  for (a.zero_lanes = 1; a.zero_lanes < 32 && a.zero_lanes * (ANY ? 1 : 4) < a.width;) a.zero_lanes *= 2;
  const int64_t zeros = (int64_t)a.workers * ((a.words + a.cta_words - 1) / a.cta_words);
  cudaError_t e = launch_early(embed_rows_kernel<T, ANY>, dim3((unsigned)(a.sum_ctas + zeros)), kThreads, 0, st, a);
  if (e == cudaSuccess && a.chunks > 0) {
    // the CTAs that the SMs hold at once, three of 70 registers each: a few more are a second round (of 65536 tokens 3 us)
    const int64_t columns = (a.width + 127) / 128, most = ((int64_t)a.workers * a.chunks + kWarps - 1) / kWarps, want = (int64_t)sm_count() * 3 / columns;
    e = launch_early(embed_joins_kernel, dim3((unsigned)(want < 1 ? 1 : want < most ? want : most), (unsigned)columns), kThreads, 0, st, a);
  }
  return e;
}
template <typename T, bool ANY>
cudaError_t few(const FewArgs& f, int workers, cudaStream_t st) {
  FewArgs a = f;
  a.slabs = (a.width + Slab<T, ANY>::kColumns - 1) / Slab<T, ANY>::kColumns;
  // every CTA looks through the tokens, so columns are cut only as far as the SMs would stay empty
  const int64_t ctas = (a.vocab + kWarps - 1) / kWarps, want = (int64_t)sm_count() * 4 / (ctas * workers) + 1;
  return launch_early(embed_few_kernel<T, ANY>, dim3((unsigned)ctas, workers, (unsigned)(want < a.slabs ? want : a.slabs)), kThreads, 0, st, a);
}
// CTAs of a cluster that sorts many tokens: sixteen where the device can place so many (of 65536 tokens 25 us, eight 35), which CUDA does not promise.
cudaError_t cluster_size(int* size, size_t smem) {
  static int cached[64] = {};
  int dev = 0, active = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 64 && cached[dev]) { *size = cached[dev]; return cudaSuccess; }
  *size = kCluster / 2;
  if (cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess) {
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = kCluster;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(kCluster);
    c.blockDim = dim3(kSortThreads);
    c.dynamicSmemBytes = smem;
    c.attrs = &attr;
    c.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&active, embed_sort_kernel, &c) == cudaSuccess && active > 0) *size = kCluster;
  }
  (void)cudaGetLastError();      // (a refusal is an answer)
  if (dev < 64) cached[dev] = *size;
  return cudaSuccess;
}
cudaError_t sort(SortArgs& a, cudaStream_t st) {
  const auto smem = [&](int cluster, int bits) { return ((size_t)(4 * cluster + 4 + 2 * kSortWarps) << bits); };
  const size_t most = smem(kCluster, kMaxBits);
  cudaError_t e = allow_smem<embed_sort_kernel>(most);
  // 3000 tokens of 20000: one CTA 18.2 us, four 10.8, eight 11.6, sixteen 14.1; 8000: four 14.4, eight 12.6, sixteen 14.3; 30000: 31, 21, 18.
  a.cluster = a.rows <= 4096 ? 4 : 8;
  if (e == cudaSuccess && a.rows > 16384) e = cluster_size(&a.cluster, most);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = a.cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3((unsigned)(a.workers * a.cluster));
  c.blockDim = dim3(kSortThreads);
  c.dynamicSmemBytes = smem(a.cluster, a.bits);
  c.stream = st;
  c.attrs = attr;
  c.numAttrs = 2;
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
  if (int rc = check_common(who, dtype, workers, rows, vocab, width, tokens, token_bytes, ld_tokens, table, worker_stride, row_stride, false, scale, out, ld_out)) return rc;
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
  a.rows = rows; a.vocab = vocab; a.width = (int)width; a.scale = (float)scale;
  const cudaError_t e = by_type(dtype, !aligned(table, worker_stride, row_stride, workers, out, ld_out, b, width),
                                [&](auto zero, auto any) { return forward<decltype(zero), decltype(any)::value>(a, workers, static_cast<cudaStream_t>(stream)); });
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

extern "C" int fgd_embed_backward(int device, int dtype, int workers, int64_t rows, int64_t vocab, int64_t width, const void* tokens, int token_bytes,
                                  int64_t ld_tokens, const void* dout, int64_t ld_dout, double scale, float* dtable, int64_t worker_stride, int64_t row_stride,
                                  void* workspace, int64_t workspace_bytes, void* stream) {
  FGD_NVTX_RANGE("fgd_embed_backward");
  const char* who = "fgd_embed_backward";
  if (int rc = check_common(who, dtype, workers, rows, vocab, width, tokens, token_bytes, ld_tokens, dtable, worker_stride, row_stride, true, scale, dout, ld_dout)) return rc;
  const int b = dtype_bytes(dtype);
  const Layout l = layout_of(workers, rows, vocab, width);
  if (l.total > 0 && (!workspace || workspace_bytes < l.total || reinterpret_cast<uintptr_t>(workspace) % 16 != 0))
    return op_fail(FGD_ERR_INVALID_ARG, "%s: needs a workspace of %lld bytes on a 16-byte boundary (fgd_embed_workspace)", who, (long long)l.total);
  const Span st_ = table_span(dtable, workers, vocab, width, worker_stride, row_stride), sw = l.total > 0 ? span_of(workspace, 1, l.total, l.total, 1) : Span{};
  const Span sx = span_of(dout, workers * rows, width, ld_dout, b), sk = span_of(tokens, workers, rows, ld_tokens, token_bytes);
  if (st_.overlaps(sx) || st_.overlaps(sk) || st_.overlaps(sw) || sw.overlaps(sx) || sw.overlaps(sk)) return op_fail(FGD_ERR_ALIAS, "%s: dtable or the workspace overlaps another tensor", who);
  const int64_t ctas = no_sort(workers, rows, vocab, width) ? (vocab + kWarps - 1) / kWarps : (int64_t)workers * l.words + (int64_t)workers * l.chunks * ((width + 127) / 128);
  if (ctas > 0x7fffffff) return op_fail(FGD_ERR_UNSUPPORTED, "%s: more work than one launch holds", who);
  DeviceScope dev(device);
  if (!dev.ok()) return op_fail(FGD_ERR_CUDA, "cannot select device %d", device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool any = !aligned(dtable, worker_stride, row_stride, workers, dout, ld_dout, b, width);
  if (no_sort(workers, rows, vocab, width)) {
    FewArgs f = {};
    f.tokens = Tokens{tokens, token_bytes, ld_tokens};
    f.dout = static_cast<const char*>(dout); f.ld = ld_dout;
    f.table = dtable; f.worker_stride = worker_stride; f.row_stride = row_stride; f.vocab = vocab;
    f.rows = (int)rows; f.width = (int)width; f.scale = (float)scale;
    const cudaError_t e = by_type(dtype, any, [&](auto zero, auto any_) { return few<decltype(zero), decltype(any_)::value>(f, workers, st); });
    return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
  }
  char* ws = static_cast<char*>(workspace);
  SortArgs s = {};
  s.tokens = Tokens{tokens, token_bytes, ld_tokens};
  s.vocab = vocab; s.rows = (int)rows;
  int bits = 1;
  while ((int64_t)1 << bits <= vocab) ++bits;      // keys 0 .. vocab
  s.passes = (bits + kMaxBits - 1) / kMaxBits;
  s.bits = (bits + s.passes - 1) / s.passes;
  s.pairs = reinterpret_cast<uint2*>(ws + l.pairs); s.other = reinterpret_cast<uint2*>(ws + l.other);
  s.present = reinterpret_cast<uint32_t*>(ws + l.present); s.words = l.words;
  s.joins = reinterpret_cast<int*>(ws + l.joins);
  s.workers = workers;
  cudaError_t e = sort(s, st);
  if (e == cudaSuccess) {
    RowsArgs r = {};
    r.pairs = s.pairs; r.present = s.present; r.words = l.words;
    r.dout = static_cast<const char*>(dout); r.ld = ld_dout;
    r.table = dtable; r.worker_stride = worker_stride; r.row_stride = row_stride;
    r.pieces = reinterpret_cast<float*>(ws + l.pieces);
    r.vocab = vocab; r.workers = workers; r.rows = (int)rows; r.chunk = l.chunk; r.chunks = l.chunks;
    r.joins = s.joins; r.list = reinterpret_cast<uint2*>(ws + l.list); r.width = (int)width; r.scale = (float)scale;
    e = by_type(dtype, any, [&](auto zero, auto any_) { return backward<decltype(zero), decltype(any_)::value>(r, st); });
  }
  return e == cudaSuccess ? FGD_OK : op_fail(FGD_ERR_CUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
}

// Token eviction from a stored prefix: the choice of the tokens to keep, their copy into a shorter prefix,
// and the CUDA-core form of the accumulated attention weights (fp32, head dims other than 128).
#pragma once
#include <cuda_bf16.h>
#include "common.cuh"
#include "simt_kernels.cuh"

namespace bicache {

// ---------------------------------------------------------------------------------------------
// Lists in the kernel parameters.  Page lists and batch descriptions of these calls travel as launch
// parameters (up to 32 KB since CUDA 12.1) and not through the workspace: nothing is uploaded, so a call
// can be captured into a graph at any time and replayed beside other calls of the context.  A list that
// does not fit is worked off in several launches.
// ---------------------------------------------------------------------------------------------
constexpr int kParamWords = 7936;               // 31,744 bytes: with the fixed fields below the 32,764 limit
struct ParamList {
  int w[kParamWords];
};

// ---------------------------------------------------------------------------------------------
// bicache_select_tokens: per row of scores the `keep` largest, protected ends first, ties to the lowest
// index, as ascending indices.  Scores become unsigned integers in the same order; the keep-th largest is
// found digit by digit (11 bits each, largest digit first, over the bits in which the row's scores differ
// at all), then one ordered pass writes the indices.  One block per row; the row is staged in shared
// memory if it fits, else read again per pass.
// ---------------------------------------------------------------------------------------------
constexpr int kSelThreads = 1024;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelDigitBits = 11;
constexpr int kSelBins = 1 << kSelDigitBits;
constexpr int kSelStaged = 49152;               // scores of a row kept in shared memory (192 KB)

// NaN counts as -inf; -0 as +0; larger score <=> larger integer.  Never 0xffffffff.
__device__ __forceinline__ unsigned select_key(float x) {
  if (x != x) x = -INFINITY;
  const unsigned u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

struct SelectArgs {
  const float* scores;
  long long score_stride;
  int* idx;
  long long idx_stride;
  int n, keep, first, last;                     // protected: t < first, t >= n - last; first + last <= min(n, keep)
};

__global__ void __launch_bounds__(kSelThreads)
select_tokens_kernel(SelectArgs a) {
  extern __shared__ unsigned staged[];
  __shared__ int hist[kSelBins];
  __shared__ int warp_a[kSelWarps], warp_b[kSelWarps];
  __shared__ unsigned warp_lo[kSelWarps], warp_hi[kSelWarps];
  __shared__ int found_bin, found_above;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const float* row = a.scores + (long long)blockIdx.x * a.score_stride;
  int* out = a.idx + (long long)blockIdx.x * a.idx_stride;
  const bool in_smem = a.n <= kSelStaged;
  const int free_begin = a.first, free_end = a.n - a.last;       // the tokens that compete
  auto key_at = [&](int i) { return in_smem ? staged[i] : select_key(row[i]); };

  unsigned lo = 0xffffffffu, hi = 0u;
  for (int i = tid; i < a.n; i += kSelThreads) {
    const unsigned k = select_key(row[i]);
    if (in_smem) staged[i] = k;
    if (i >= free_begin && i < free_end) {
      lo = min(lo, k);
      hi = max(hi, k);
    }
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) {
    warp_lo[warp] = lo;
    warp_hi[warp] = hi;
  }
  __syncthreads();
  lo = __reduce_min_sync(0xffffffffu, warp_lo[lane]);
  hi = __reduce_max_sync(0xffffffffu, warp_hi[lane]);

  // `threshold`: the k-th largest of the competing scores, `ties`: how many equal ones are kept
  int k = a.keep - a.first - a.last;
  const int competing = free_end - free_begin;
  unsigned threshold = 0;                                          // below every key: all of them are kept
  int ties = 0;
  if (k <= 0) {
    threshold = 0xffffffffu;
  } else if (k < competing) {
    unsigned base = lo, span = hi - lo;                            // the k-th largest is in [base, base + span]
    int shift = max(0, (32 - __clz(span)) - kSelDigitBits);
    for (;;) {
      for (int b = tid; b < kSelBins; b += kSelThreads) hist[b] = 0;
      __syncthreads();
      for (int i = free_begin + tid; i < free_end; i += kSelThreads) {
        const unsigned d = key_at(i) - base;                       // below base: wraps to a large value
        if (d <= span) atomicAdd(&hist[d >> shift], 1);
      }
      __syncthreads();
      // counts from the top: thread t holds bins 2046 - 2 t and 2047 - 2 t
      const int b1 = kSelBins - 1 - 2 * tid, b0 = b1 - 1;
      const int c1 = hist[b1], c0 = hist[b0];
      int incl = c0 + c1;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      if (lane == 31) warp_a[warp] = incl;
      __syncthreads();
      const int wt = warp_a[lane];
      int below = lane < warp ? wt : 0;
      below = __reduce_add_sync(0xffffffffu, below);
      const int above1 = below + incl - c0 - c1, above0 = above1 + c1;
      if (above1 < k && k <= above1 + c1) {
        found_bin = b1;
        found_above = above1;
      } else if (above0 < k && k <= above0 + c0) {
        found_bin = b0;
        found_above = above0;
      }
      __syncthreads();
      k -= found_above;
      base += (unsigned)found_bin << shift;
      if (shift == 0) break;
      span = min(span - ((unsigned)found_bin << shift), (1u << shift) - 1u);
      shift = max(0, shift - kSelDigitBits);
    }
    threshold = base;
    ties = k;
  }

  // ordered output: every warp owns a run of the row
  const int run = (((a.n + kSelWarps - 1) / kSelWarps) + 31) & ~31;
  const int begin = min(a.n, warp * run), end = min(a.n, begin + run);
  int above = 0, equal = 0;
  for (int i0 = begin; i0 < end; i0 += 32) {
    const int i = i0 + lane;
    const bool in = i < end, prot = in && (i < free_begin || i >= free_end);
    const unsigned key = in ? key_at(i) : 0u;
    above += __popc(__ballot_sync(0xffffffffu, prot || (in && key > threshold)));
    equal += __popc(__ballot_sync(0xffffffffu, in && !prot && key == threshold));
  }
  __syncthreads();                                                  // warp_a of the last digit has been read
  if (lane == 0) {
    warp_a[warp] = above;
    warp_b[warp] = equal;
  }
  __syncthreads();
  int above_before = __reduce_add_sync(0xffffffffu, lane < warp ? warp_a[lane] : 0);
  int equal_before = __reduce_add_sync(0xffffffffu, lane < warp ? warp_b[lane] : 0);
  const unsigned lt = (1u << lane) - 1u;
  for (int i0 = begin; i0 < end; i0 += 32) {
    const int i = i0 + lane;
    const bool in = i < end, prot = in && (i < free_begin || i >= free_end);
    const unsigned key = in ? key_at(i) : 0u;
    const bool gt = prot || (in && key > threshold), eq = in && !prot && key == threshold;
    const unsigned mg = __ballot_sync(0xffffffffu, gt), me = __ballot_sync(0xffffffffu, eq);
    const int eq_rank = equal_before + __popc(me & lt);             // equal scores of lower index
    const int pos = above_before + __popc(mg & lt) + min(eq_rank, ties);
    if (gt || (eq && eq_rank < ties)) out[pos] = i;
    above_before += __popc(mg);
    equal_before += __popc(me);
  }
}

// ---------------------------------------------------------------------------------------------
// bicache_compact_prefix: token i of head j of the shorter prefix becomes token idx[layer][j][i] of the
// longer one, K and V.  A page image keeps a token's dims in two runs of 128 bytes (or one of D elements),
// and the 16-byte chunks of a run are permuted inside it, so the copy goes chunk by chunk: half a warp
// moves one token of one head (D = 128, bf16).  Unused slots of the last page become zero, as everywhere.
// An index outside the prefix leaves a zero token and raises the status word.
// ---------------------------------------------------------------------------------------------
constexpr int kCompactThreads = 256;
struct CompactArgs {
  char* pool_k;                 // first layer of the launch
  char* pool_v;
  long long layer_bytes;
  int page_bytes, num_kv_heads, chunks_per_row, swizzled;
  const int* idx;
  long long idx_layer_stride, idx_head_stride;
  int src_m, src_first, src_pages;     // pages src_first .. of the source are in the list
  int keep, dst_first, dst_pages;      // so are pages dst_first .. of the destination
  int num_layers;
  int* status;
};

__global__ void __launch_bounds__(kCompactThreads)
compact_prefix_kernel(const __grid_constant__ CompactArgs a, const __grid_constant__ ParamList list) {
  const int slots = a.dst_pages * kPageSize;
  const long long per_layer = (long long)slots * a.num_kv_heads * a.chunks_per_row;
  const long long total = per_layer * a.num_layers;
  const int row_bytes = a.chunks_per_row * 16;
  for (long long i = blockIdx.x * (long long)blockDim.x + threadIdx.x; i < total;
       i += (long long)gridDim.x * blockDim.x) {
    const int layer = (int)(i / per_layer);
    long long rem = i - layer * per_layer;
    const int c16 = (int)(rem % a.chunks_per_row); rem /= a.chunks_per_row;
    const int slot = (int)(rem % kPageSize); rem /= kPageSize;
    const int hk = (int)(rem % a.num_kv_heads);
    const int pg = (int)(rem / a.num_kv_heads);
    const int t = (a.dst_first + pg) * kPageSize + slot;
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    bool write = a.src_first == 0;                          // padding and bad indices: by the first window
    const long long lb = layer * a.layer_bytes;
    if (t < a.keep) {
      const int s = a.idx[layer * a.idx_layer_stride + hk * a.idx_head_stride + t];
      if (s < 0 || s >= a.src_m) {
        if (write) atomicCAS(a.status, kDevOk, kDevBadIndex);
      } else {
        const int sp = s / kPageSize - a.src_first;
        write = sp >= 0 && sp < a.src_pages;
        if (write) {
          const long long so = lb + ((long long)list.w[sp] * a.num_kv_heads + hk) * a.page_bytes +
                               page_chunk_offset(a.swizzled != 0, s % kPageSize, c16, row_bytes);
          k = *reinterpret_cast<const uint4*>(a.pool_k + so);
          v = *reinterpret_cast<const uint4*>(a.pool_v + so);
        }
      }
    }
    if (write) {
      const long long po = lb + ((long long)list.w[a.src_pages + pg] * a.num_kv_heads + hk) * a.page_bytes +
                           page_chunk_offset(a.swizzled != 0, slot, c16, row_bytes);
      *reinterpret_cast<uint4*>(a.pool_k + po) = k;
      *reinterpret_cast<uint4*>(a.pool_v + po) = v;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// bicache_prefix_weights.  For every cached key t of prefix g and KV head j
//   out[g][j][t] = decay in[g][j][t] + sum over the rows a and query heads h of the group
//                  exp(scale q[a][h] . k[t][j] - lse[a][h]);
// rows with an infinite lse add nothing.  The batch: groups (one per prefix), the runs of query rows that
// belong to each, and their page lists, all in the parameter list.  Row space of a group: the tokens of its
// requests one after the other, packed row p = token * G + head in the KV group, cut into row tiles.  A
// work item is one block of keys against a range of row tiles; with several ranges (splits) the items
// write partial sums and a second kernel adds them in a fixed order.
// ---------------------------------------------------------------------------------------------
struct WeightGroup {
  int m;                        // cached keys of this launch (from key0 on)
  int key0;                     // first of them in the prefix: index into the score rows
  int page_word;                // where its page list starts in the parameter words
  int seg_word;                 // where its row runs start
  int num_segs;
  int tokens;                   // rows of the group
  int key_blocks;
  int item_begin;               // first work item
  int splits, tiles_per_split;
  int part_off;                 // first partial sum (one [splits][Hkv][m] block per group)
  int pad;
  long long score_off;          // elements from the scores' base to the group's block
};
struct WeightSeg {
  long long row;                // first row of the run
  int token;                    // first token of the run in the group's numbering
  int pad;
};
constexpr int kGroupWords = sizeof(WeightGroup) / 4, kSegWords = sizeof(WeightSeg) / 4;

struct WeightArgs {
  const char* q;
  long long q_stride;           // elements between rows
  const float* lse;
  const float* in;              // nullptr: decay is 0
  float* out;
  long long head_stride;        // elements between the score rows of two KV heads
  float decay, scale;
  float* part;
  const char* pool_k;           // the layer's keys
  int page_bytes, swizzled;
  int Hq, Hkv, D;
  int num_groups, num_items;
};

__device__ __forceinline__ const WeightGroup& weight_group(const ParamList& list, int g) {
  return *reinterpret_cast<const WeightGroup*>(&list.w[g * kGroupWords]);
}
// the group of a work item: groups are few and in order
__device__ __forceinline__ int weight_group_of(const WeightArgs& a, const ParamList& list, int item) {
  int g = 0;
  while (g + 1 < a.num_groups && item >= weight_group(list, g + 1).item_begin) ++g;
  return g;
}
// row of the caller's tensors that holds token `tok` of a group
__device__ __forceinline__ long long weight_row(const ParamList& list, const WeightGroup& g, int tok) {
  const WeightSeg* s = reinterpret_cast<const WeightSeg*>(&list.w[g.seg_word]);
  int lo = 0, hi = g.num_segs - 1;                      // last run that starts at or before tok
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s[mid].token <= tok) lo = mid; else hi = mid - 1;
  }
  return s[lo].row + (tok - s[lo].token);
}

// CUDA-core form.  Block: 64 keys against tiles of 64 packed rows, each thread 4 keys x 4 rows, dims in
// shared memory as fp32 (rows padded by 4 floats: the 16-byte reads of a quarter warp fall on different
// banks).  The sums over rows are kept in fp64 per thread and added across the 16 threads of a key at the end.
constexpr int kWsKeys = 64, kWsRows = 64, kWsThreads = 256;
inline size_t weights_simt_smem(int D) { return sizeof(float) * ((size_t)(kWsKeys + kWsRows) * (D + 4) + kWsRows); }

template <typename T>
__global__ void __launch_bounds__(kWsThreads)
weights_simt_kernel(const __grid_constant__ WeightArgs a, const __grid_constant__ ParamList list) {
  using Tr = ElemTraits<T>;
  constexpr int kEsize = (int)sizeof(T), kPer = Tr::kPerChunk;
  extern __shared__ float ws_smem[];
  const int D = a.D, pitch = D + 4, chunks = D / kPer;
  float* const ks = ws_smem;
  float* const qs = ks + kWsKeys * pitch;
  float* const ls = qs + kWsRows * pitch;
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int G = a.Hq / a.Hkv;
  const WeightGroup& g = weight_group(list, weight_group_of(a, list, blockIdx.x));
  int rem = (int)blockIdx.x - g.item_begin;
  const int kb = rem % g.key_blocks; rem /= g.key_blocks;
  const int split = rem % g.splits, hk = rem / g.splits;
  const int key_begin = kb * kWsKeys;
  for (int i = tid; i < kWsKeys * chunks; i += kWsThreads) {
    const int key = i / chunks, c = i - key * chunks, t = key_begin + key;
    float f[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) f[e] = 0.f;
    if (t < g.m) {
      const char* page = a.pool_k + ((long long)list.w[g.page_word + t / kPageSize] * a.Hkv + hk) * a.page_bytes;
      Tr::unpack(*reinterpret_cast<const uint4*>(page + page_chunk_offset(a.swizzled != 0, t % kPageSize, c, D * kEsize)), f);
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) ks[key * pitch + c * kPer + e] = f[e];
  }
  double total[4] = {0.0, 0.0, 0.0, 0.0};
  const long long rows = (long long)g.tokens * G;
  const int tiles = (int)((rows + kWsRows - 1) / kWsRows);
  const int tile_begin = split * g.tiles_per_split, tile_end = min(tiles, tile_begin + g.tiles_per_split);
  for (int tile = tile_begin; tile < tile_end; ++tile) {
    __syncthreads();                                    // the last tile's rows have been used
    for (int i = tid; i < kWsRows * chunks; i += kWsThreads) {
      const int r = i / chunks, c = i - r * chunks;
      const long long p = (long long)tile * kWsRows + r;
      float f[kPer];
#pragma unroll
      for (int e = 0; e < kPer; ++e) f[e] = 0.f;
      float l = INFINITY;
      if (p < rows) {
        const int tok = (int)(p / G), h = hk * G + (int)(p - (long long)tok * G);
        const long long row = weight_row(list, g, tok);
        l = a.lse[row * a.Hq + h];
        if (!isinf(l)) Tr::unpack(*reinterpret_cast<const uint4*>(a.q + (row * a.q_stride + (long long)h * D) * kEsize + c * 16), f);
      }
#pragma unroll
      for (int e = 0; e < kPer; ++e) qs[r * pitch + c * kPer + e] = f[e];
      if (c == 0) ls[r] = l;
    }
    __syncthreads();
    float acc[4][4] = {};
    for (int d = 0; d < D; d += 4) {
      float4 kf[4], qf[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        kf[i] = *reinterpret_cast<const float4*>(&ks[(tx + 16 * i) * pitch + d]);
        qf[i] = *reinterpret_cast<const float4*>(&qs[(ty + 16 * i) * pitch + d]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          acc[i][j] = fmaf(kf[i].x, qf[j].x, acc[i][j]);
          acc[i][j] = fmaf(kf[i].y, qf[j].y, acc[i][j]);
          acc[i][j] = fmaf(kf[i].z, qf[j].z, acc[i][j]);
          acc[i][j] = fmaf(kf[i].w, qf[j].w, acc[i][j]);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float l = ls[ty + 16 * j];
      if (isinf(l)) continue;                           // masked or past the end, whatever the product is
#pragma unroll
      for (int i = 0; i < 4; ++i) total[i] += (double)expf(fmaf(a.scale, acc[i][j], -l));
    }
  }
  __syncthreads();
  double* const red = reinterpret_cast<double*>(ws_smem);          // [16][64]
#pragma unroll
  for (int i = 0; i < 4; ++i) red[ty * kWsKeys + tx + 16 * i] = total[i];
  __syncthreads();
  if (tid < kWsKeys && key_begin + tid < g.m) {
    double s = 0.0;
    for (int y = 0; y < 16; ++y) s += red[y * kWsKeys + tid];
    const int t = key_begin + tid;
    if (g.splits > 1) {
      a.part[g.part_off + ((long long)split * a.Hkv + hk) * g.m + t] = (float)s;
    } else {
      const long long o = g.score_off + hk * a.head_stride + g.key0 + t;
      a.out[o] = (float)((a.decay != 0.f ? (double)a.decay * a.in[o] : 0.0) + s);
    }
  }
}
static_assert(16 * kWsKeys * sizeof(double) <= sizeof(float) * (kWsKeys + kWsRows) * (32 + 4), "the sums are added over the tiles");

// The partial sums of the row ranges, added in order.  One thread per (KV head, key) of a group with splits.
__global__ void __launch_bounds__(256)
weights_sum_kernel(const __grid_constant__ WeightArgs a, const __grid_constant__ ParamList list) {
  const WeightGroup& g = weight_group(list, blockIdx.y);
  if (g.splits <= 1) return;
  const long long per_split = (long long)a.Hkv * g.m;
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < per_split; i += gridDim.x * 256ll) {
    const int hk = (int)(i / g.m), t = (int)(i - (long long)hk * g.m);
    double s = 0.0;
    for (int k = 0; k < g.splits; ++k) s += (double)a.part[g.part_off + k * per_split + i];
    const long long o = g.score_off + hk * a.head_stride + g.key0 + t;
    a.out[o] = (float)((a.decay != 0.f ? (double)a.decay * a.in[o] : 0.0) + s);
  }
}

}  // namespace bicache

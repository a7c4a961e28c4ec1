// Token eviction from a stored prefix: the choice of the tokens to keep, their copy into a shorter prefix,
// and the CUDA-core form of the accumulated attention weights (fp32, head dims other than 128).
#pragma once
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include "common.cuh"
#include "simt_kernels.cuh"

namespace bicache {

// ---------------------------------------------------------------------------------------------
// Lists in the kernel parameters.  Page lists and batch descriptions of these calls travel as launch
// parameters (up to 32 KB since CUDA 12.1) and not through the workspace: nothing is uploaded, so a call
// can be captured into a graph at any time and replayed beside other calls of the context.  A list that
// does not fit is worked off in several launches.  A launch costs the host about 1 us per 8 KB of
// parameters (select 4.5 us with 64 bytes, compact 8.3 us with 32 KB), so the kernels exist for lists of three lengths.
// ---------------------------------------------------------------------------------------------
constexpr int kParamWords = 7936;               // 31,744 bytes: with the fixed fields below the 32,764 limit
constexpr int kParamWordsMid = 2432, kParamWordsSmall = 896;
template <int kWords>
struct ParamList {
  int w[kWords];
};
// f(list of the shortest length that holds the first `used` words of w)
template <typename F>
inline void with_param_list(const int* w, int used, F&& f) {
  if (used <= kParamWordsSmall) f(*reinterpret_cast<const ParamList<kParamWordsSmall>*>(w));
  else if (used <= kParamWordsMid) f(*reinterpret_cast<const ParamList<kParamWordsMid>*>(w));
  else f(*reinterpret_cast<const ParamList<kParamWords>*>(w));
}

// ---------------------------------------------------------------------------------------------
// bicache_select_tokens: per row of scores the `keep` largest, protected ends first, ties to the lowest
// index, as ascending indices.  Scores become unsigned integers in the same order; the keep-th largest is
// found digit by digit (11 bits each, largest digit first, over the bits in which the row's scores differ
// at all: narrow rows spread over the bins as wide ones do) until its bin holds few enough scores to be
// ranked against one another.  Then every score becomes a bit "kept" (or, if only some of the scores equal to
// the last one are kept, two bits), a scan over the words of bits gives each its place, and the indices are
// put in order in shared memory and written out.
//
// A row is served by a cluster of 1 to 8 blocks, each with a part of it, which read one another's counts through
// distributed shared memory: several blocks make a few rows fast and let two blocks share an SM, so
// that one loads while the other counts.  Scores are read from memory once, in 16-byte loads, and stay in shared
// memory; a row too long for that is read again (from L2, as a rule) by every pass, by one block.
// The bound for many rows is the instructions per score (about 1 us for each, for 36 M scores), then memory.
// ---------------------------------------------------------------------------------------------
constexpr int kSelThreads = 512;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelDigitBits = 11;
constexpr int kSelBins = 1 << kSelDigitBits;
constexpr int kSelRanked = 256;                 // a bin of at most this many scores is ranked directly
constexpr int kSelStaged = 49152;               // scores of a block's part kept in shared memory (192 KB)
constexpr int kSelWords = kSelStaged / 32;      // bit words kept at a time
constexpr int kSelMaxCluster = 8;

// NaN counts as -inf; -0 as +0; larger score <=> larger integer.  Never 0 nor 0xffffffff.
__device__ __forceinline__ unsigned select_key(float x) {
  const unsigned u = __float_as_uint(fmaxf(x + 0.f, -INFINITY));      // the maximum of a NaN and a number is the number
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}

struct SelectArgs {
  const float* scores;
  long long score_stride;
  int* idx;
  long long idx_stride;
  int n, keep, first, last;                     // protected: t < first, t >= n - last; first + last <= min(n, keep)
};

// exclusive prefix sum of v over the block, in thread order; *total receives the sum.  Two barriers.
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  const int w = lane < kSelWarps ? warp_sums[lane] : 0;
  const int before = __reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
  *total = __reduce_add_sync(0xffffffffu, w);
  __syncthreads();                              // warp_sums may be written again
  return before + incl - v;
}

template <bool kStaged>
__global__ void __launch_bounds__(kSelThreads)
select_tokens_kernel(SelectArgs a) {
  namespace cg = cooperative_groups;
  struct Shared {                               // what the cluster's blocks read of one another
    int hist[2][kSelBins];                      // digits in turn
    unsigned lo, hi;                            // smallest and largest competing score of the part
    unsigned ranked[kSelRanked];                // scores of the last bin found in the part ...
    int num_ranked;                             // ... and how many
    int above, equal;                           // kept for sure / tied, in the part
  };
  extern __shared__ __align__(16) unsigned staged[];
  __shared__ __align__(16) Shared sh;
  __shared__ __align__(16) unsigned candidates[kSelRanked];
  __shared__ int warp_sums[kSelWarps];
  __shared__ unsigned warp_lo[kSelWarps], warp_hi[kSelWarps];
  __shared__ int found_bin, found_above, found_count;
  __shared__ unsigned found_key;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const cg::cluster_group cluster = cg::this_cluster();
  const int parts = kStaged ? (int)cluster.num_blocks() : 1, part = kStaged ? (int)cluster.block_rank() : 0;
  auto sync_parts = [&]() {
    if (parts > 1) cluster.sync(); else __syncthreads();
  };
  auto other = [&](int p) { return parts > 1 ? cluster.map_shared_rank(&sh, p) : &sh; };
  const long long row_index = blockIdx.x / parts;
  const float* __restrict__ row = a.scores + row_index * a.score_stride;
  int* out = a.idx + row_index * a.idx_stride;
  const int n = a.n, free_begin = a.first, free_end = n - a.last;      // the tokens that compete
  // The row starts `shift` scores past a 16-byte boundary.  Slot s holds token s - shift, so that 16-byte loads
  // and 16-byte shared-memory words line up; slots below `shift` and past the end are no tokens.
  const int shift = (int)((reinterpret_cast<uintptr_t>(row) >> 2) & 3);
  const int slots = n + shift, quads = (slots + 3) >> 2;
  // this block's part: whole words of 32 slots
  const int all_words = (slots + 31) >> 5, part_words = (all_words + parts - 1) / parts;
  const int quad_begin = min(quads, part * part_words * 8), quad_end = min(quads, quad_begin + part_words * 8);
  auto load_quad = [&](int v) {                                        // slots 4 v .. 4 v + 3, from memory
    float4 f;
    if (4 * v >= shift && 4 * v + 3 < slots) {
      f = *reinterpret_cast<const float4*>(row + 4 * v - shift);
    } else {
      float* e = reinterpret_cast<float*>(&f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = 4 * v + j - shift;
        e[j] = t >= 0 && t < n ? row[t] : 0.f;
      }
    }
    return make_uint4(select_key(f.x), select_key(f.y), select_key(f.z), select_key(f.w));
  };
  auto quad_at = [&](int v) { return kStaged ? reinterpret_cast<const uint4*>(staged)[v - quad_begin] : load_quad(v); };
  // competing slots; the quads that lie wholly inside take the short path
  const int slot_begin = free_begin + shift, slot_end = free_end + shift;
  auto inside = [&](int v) { return 4 * v >= slot_begin && 4 * v + 4 <= slot_end; };
  auto competes = [&](int s) { return s >= slot_begin && s < slot_end; };

  // behind the scores: the bit words
  unsigned* const bits_above = staged + (kStaged ? part_words * 32 : 0);
  unsigned* const bits_equal = bits_above + (kStaged ? part_words : kSelWords);

  for (int b = tid; b < 2 * kSelBins; b += kSelThreads) (&sh.hist[0][0])[b] = 0;
  if (tid == 0) sh.num_ranked = 0;
  unsigned lo = 0xffffffffu, hi = 0u;
  constexpr int kAhead = 4;                                            // loads in flight per thread
  for (int v0 = quad_begin + tid; v0 < quad_end; v0 += kAhead * kSelThreads) {
    uint4 k[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (v0 + j * kSelThreads < quad_end) k[j] = load_quad(v0 + j * kSelThreads);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int v = v0 + j * kSelThreads;
      if (v >= quad_end) break;
      if (kStaged) reinterpret_cast<uint4*>(staged)[v - quad_begin] = k[j];
      if (inside(v)) {
        lo = min(min(min(lo, k[j].x), k[j].y), min(k[j].z, k[j].w));
        hi = max(max(max(hi, k[j].x), k[j].y), max(k[j].z, k[j].w));
      } else {
        const unsigned e[4] = {k[j].x, k[j].y, k[j].z, k[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (competes(4 * v + i)) {
            lo = min(lo, e[i]);
            hi = max(hi, e[i]);
          }
      }
    }
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) {
    warp_lo[warp] = lo;
    warp_hi[warp] = hi;
  }
  __syncthreads();
  lo = __reduce_min_sync(0xffffffffu, warp_lo[lane % kSelWarps]);
  hi = __reduce_max_sync(0xffffffffu, warp_hi[lane % kSelWarps]);
  if (parts > 1) {
    if (tid == 0) {
      sh.lo = lo;
      sh.hi = hi;
    }
    cluster.sync();
    for (int p = 0; p < parts; ++p) {
      lo = min(lo, other(p)->lo);
      hi = max(hi, other(p)->hi);
    }
  }

  // `threshold`: the k-th largest of the competing scores; `ties` of the `equals` scores equal to it are kept
  int k = a.keep - a.first - a.last;
  unsigned threshold = 0;                                              // below every key: all of them are kept
  int ties = 0, equals = 0;
  if (k <= 0) {
    threshold = 0xffffffffu;
  } else if (k < free_end - free_begin) {
    unsigned base = lo, span = hi - lo;                                // the k-th largest is in [base, base + span]
    int digit = max(0, (32 - __clz(span)) - kSelDigitBits);
    for (int pass = 0;; ++pass) {
      int* const hist = sh.hist[pass & 1];
      for (int v = quad_begin + tid; v < quad_end; v += kSelThreads) {
        const uint4 q = quad_at(v);
        const unsigned d[4] = {q.x - base, q.y - base, q.z - base, q.w - base};   // below base: wraps to a large value
        if (inside(v)) {
          if (pass == 0) {                                             // all of them are inside the range
#pragma unroll
            for (int j = 0; j < 4; ++j) atomicAdd(&hist[d[j] >> digit], 1);
          } else if (min(min(d[0], d[1]), min(d[2], d[3])) <= span) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (d[j] <= span) atomicAdd(&hist[d[j] >> digit], 1);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (competes(4 * v + j) && d[j] <= span) atomicAdd(&hist[d[j] >> digit], 1);
        }
      }
      sync_parts();
      // every part has read the digit before this one: its bins are cleared for the next
      for (int b = tid; b < kSelBins && pass > 0; b += kSelThreads) sh.hist[(pass + 1) & 1][b] = 0;
      // counts from the top: thread t holds bins 2044 - 4 t .. 2047 - 4 t
      const int bin0 = kSelBins - 4 - 4 * tid;
      int c[4] = {0, 0, 0, 0};
      for (int p = 0; p < parts; ++p) {
        const int4 h = *reinterpret_cast<const int4*>(&other(p)->hist[pass & 1][bin0]);
        c[0] += h.x;
        c[1] += h.y;
        c[2] += h.z;
        c[3] += h.w;
      }
      int total;
      int above = block_scan(c[0] + c[1] + c[2] + c[3], warp_sums, &total);
#pragma unroll
      for (int j = 3; j >= 0; --j) {
        if (above < k && k <= above + c[j]) {
          found_bin = bin0 + j;
          found_above = above;
          found_count = c[j];
        }
        above += c[j];
      }
      __syncthreads();
      k -= found_above;
      equals = found_count;
      base += (unsigned)found_bin << digit;
      span = min(span - ((unsigned)found_bin << digit), (1u << digit) - 1u);
      if (digit == 0) {
        threshold = base;
        break;
      }
      if (equals <= kSelRanked) {
        // gather the bin's scores of all parts and rank them against one another
        for (int v = quad_begin + tid; v < quad_end; v += kSelThreads) {
          const uint4 q = quad_at(v);
          const unsigned e[4] = {q.x, q.y, q.z, q.w};
          if (min(min(q.x - base, q.y - base), min(q.z - base, q.w - base)) <= span) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (e[j] - base <= span && competes(4 * v + j)) sh.ranked[atomicAdd(&sh.num_ranked, 1)] = e[j];
          }
        }
        sync_parts();
        for (int p = 0, at = 0; p < parts; ++p) {
          const Shared* o = other(p);
          const int m = o->num_ranked;
          if (tid < m) candidates[at + tid] = o->ranked[tid];
          at += m;
        }
        __syncthreads();
        if (tid < equals) {
          const unsigned mine = candidates[tid];
          int greater = 0, same = 0;
          for (int i = 0; i < equals; ++i) {
            greater += candidates[i] > mine ? 1 : 0;
            same += candidates[i] == mine ? 1 : 0;
          }
          if (greater < k && k <= greater + same) {                    // by every thread with that score, alike
            found_key = mine;
            found_above = greater;
            found_count = same;
          }
        }
        __syncthreads();
        threshold = found_key;
        k -= found_above;
        equals = found_count;
        break;
      }
      digit = max(0, digit - kSelDigitBits);
    }
    ties = k;
  }
  const bool split = ties < equals;                                    // some of the equal scores stay, some go

  // Ordered output, at most kSelWords words at a time (one round for a staged row).  A thread turns 8 slots into
  // a byte.  Where ties are not split, "above" is all that is kept.
  int above_before = 0, equal_before = 0;                              // earlier rounds
  for (int round = quad_begin; round < quad_end || (parts > 1 && round == quad_begin); round += kSelWords * 8) {
    const int words = min(kSelWords, (quad_end - round + 7) >> 3);
    const int word_slot = round * 4;                                   // first slot of the round
    for (int byte = tid; byte < words * 4; byte += kSelThreads) {
      unsigned above = 0, equal = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int v = round + byte * 2 + i;
        if (v >= quad_end) break;
        const uint4 q = quad_at(v);
        const unsigned e[4] = {q.x, q.y, q.z, q.w};
        if (inside(v)) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            above |= e[j] > threshold ? 1u << (4 * i + j) : 0u;
            equal |= e[j] == threshold ? 1u << (4 * i + j) : 0u;
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int s = 4 * v + j;
            const bool held = s >= shift && s < slots && !competes(s);          // a protected token
            above |= held || (competes(s) && e[j] > threshold) ? 1u << (4 * i + j) : 0u;
            equal |= competes(s) && e[j] == threshold ? 1u << (4 * i + j) : 0u;
          }
        }
      }
      reinterpret_cast<unsigned char*>(bits_above)[byte] = (unsigned char)(split ? above : above | equal);
      if (split) reinterpret_cast<unsigned char*>(bits_equal)[byte] = (unsigned char)equal;
    }
    __syncthreads();
    // every thread takes a run of words: where the run starts, then token by token
    const int run = (words + kSelThreads - 1) / kSelThreads;
    const int w0 = min(words, tid * run), w1 = min(words, w0 + run);
    int n_above = 0, n_equal = 0;
    for (int i = w0; i < w1; ++i) {
      n_above += __popc(bits_above[i]);
      if (split) n_equal += __popc(bits_equal[i]);
    }
    int total_above, total_equal = 0;
    int at_above = above_before + block_scan(n_above, warp_sums, &total_above), at_equal = equal_before;
    if (split) at_equal += block_scan(n_equal, warp_sums, &total_equal);
    int part_above = 0, part_equal = 0;                                // in the parts before this one
    if (parts > 1) {
      if (tid == 0) {
        sh.above = total_above;
        sh.equal = total_equal;
      }
      cluster.sync();
      for (int p = 0; p < part; ++p) {
        part_above += other(p)->above;
        part_equal += other(p)->equal;
      }
      at_above += part_above;
      at_equal += part_equal;
    }
    // A staged row's list is put together where its scores were (they have been used) and written in order.
    const int out0 = above_before + part_above + min(equal_before + part_equal, ties);
    for (int i = w0; i < w1; ++i) {
      unsigned kept = bits_above[i];
      int at = at_above + min(at_equal, ties) - (kStaged ? out0 : 0);
      at_above += __popc(kept);
      if (split) {
        unsigned equal = bits_equal[i];
        const int here = __popc(equal);
        for (int room = max(0, ties - at_equal); here > room && __popc(equal) > room;)
          equal &= ~(0x80000000u >> __clz(equal));                     // the highest of them go
        kept |= equal;
        at_equal += here;
      }
      const int token = word_slot + i * 32 - shift;
      while (kept) {
        (kStaged ? reinterpret_cast<int*>(staged) : out)[at++] = token + __ffs(kept) - 1;
        kept &= kept - 1;
      }
    }
    above_before += total_above;
    equal_before += total_equal;
    if (kStaged) {
      __syncthreads();
      const int count = above_before + part_above + min(equal_before + part_equal, ties) - out0;
      for (int i = tid; i < count; i += kSelThreads) out[out0 + i] = (int)staged[i];
    }
    __syncthreads();                                                   // the words may be written again
  }
  if (parts > 1) cluster.sync();                                       // the others have read this block's counts
}

// Blocks per row.  More than one where a part would not leave room for a second block on the SM (20,480
// scores), and where the rows alone do not fill the GPU (down to 2048 scores a block).
inline int select_parts(long long rows, int n, int sm_count) {
  int parts = 1;
  while (parts < kSelMaxCluster && (n / parts > 20480 || (rows * parts <= sm_count && n / parts > 2048))) parts *= 2;
  return parts;
}

inline cudaError_t launch_select(const SelectArgs& a, long long rows, int sm_count, cudaStream_t stream) {
  const int parts = select_parts(rows, a.n, sm_count);
  // slots of the largest part (up to three slots before the first token, whole words)
  const int part_slots = (((a.n + 3 + 31) / 32 + parts - 1) / parts) * 32;
  if (part_slots > kSelStaged || rows * parts > 0x7fffffffLL) {
    select_tokens_kernel<false><<<(unsigned)rows, kSelThreads, 2 * kSelWords * 4, stream>>>(a);
    return cudaGetLastError();
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * parts), 1, 1);
  cfg.blockDim = dim3(kSelThreads, 1, 1);
  cfg.dynamicSmemBytes = (size_t)part_slots * 4 + part_slots / 32 * 8;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = parts;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, select_tokens_kernel<true>, a);
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

template <int kWords>
__global__ void __launch_bounds__(kCompactThreads)
compact_prefix_kernel(const __grid_constant__ CompactArgs a, const __grid_constant__ ParamList<kWords> list) {
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

__device__ __forceinline__ const WeightGroup& weight_group(const int* list, int g) {
  return *reinterpret_cast<const WeightGroup*>(&list[g * kGroupWords]);
}
// the group of a work item: groups are few and in order
__device__ __forceinline__ int weight_group_of(const WeightArgs& a, const int* list, int item) {
  int g = 0;
  while (g + 1 < a.num_groups && item >= weight_group(list, g + 1).item_begin) ++g;
  return g;
}
// row of the caller's tensors that holds token `tok` of a group
__device__ __forceinline__ long long weight_row(const int* list, const WeightGroup& g, int tok) {
  const WeightSeg* s = reinterpret_cast<const WeightSeg*>(&list[g.seg_word]);
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

template <typename T, int kWords>
__global__ void __launch_bounds__(kWsThreads)
weights_simt_kernel(const __grid_constant__ WeightArgs a, const __grid_constant__ ParamList<kWords> params) {
  const int* const list = params.w;
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
      const char* page = a.pool_k + ((long long)list[g.page_word + t / kPageSize] * a.Hkv + hk) * a.page_bytes;
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
template <int kWords>
__global__ void __launch_bounds__(256)
weights_sum_kernel(const __grid_constant__ WeightArgs a, const __grid_constant__ ParamList<kWords> params) {
  const int* const list = params.w;
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

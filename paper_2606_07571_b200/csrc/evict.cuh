// Token eviction from a stored prefix: the choice of the tokens to keep, their copy into a shorter prefix,
// and the CUDA-core form of the accumulated attention weights (fp32, head dims other than 128).
#pragma once
#include <algorithm>
#include <utility>
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include "common.cuh"
#include "simt_kernels.cuh"

namespace bicache {

// ---------------------------------------------------------------------------------------------
// Lists in the kernel parameters.  Page lists and batch descriptions of these calls travel as launch
// parameters (up to 32 KB since CUDA 12.1) and not through the workspace: nothing is uploaded, so a call
// can be captured into a graph at any time.  (Replays follow the context's other calls all the same: the
// partial sums of the weights lie in the workspace.)  A list that does not fit is worked off in several launches.  A launch costs the host about 1 us per 8 KB of
// parameters (a call of 64 bytes takes 4.5 us, one of 32 KB 8.3), so the kernels exist for lists of four lengths.
// ---------------------------------------------------------------------------------------------
constexpr int kParamWords = 7936;               // 31,744 bytes: with the fixed fields below the 32,764 limit
using ParamLengths = std::integer_sequence<int, 224, 1216, 2432, kParamWords>;
template <int kWords>
struct ParamList {
  int w[kWords];
};
// f(list of the shortest length that holds the first `used` words of w)
template <typename F, int kFirst, int... kRest>
inline void with_param_list(const int* w, int used, F&& f, std::integer_sequence<int, kFirst, kRest...>) {
  if constexpr (sizeof...(kRest) > 0) {
    if (used > kFirst) return with_param_list(w, used, f, std::integer_sequence<int, kRest...>());
  }
  f(*reinterpret_cast<const ParamList<kFirst>*>(w));
}
template <typename F>
inline void with_param_list(const int* w, int used, F&& f) {
  with_param_list(w, used, f, ParamLengths());
}
// f(std::integral_constant) for every length
template <typename F, int... kLengths>
inline void each_param_length(F&& f, std::integer_sequence<int, kLengths...>) {
  (f(std::integral_constant<int, kLengths>()), ...);
}

// ---------------------------------------------------------------------------------------------
// bicache_select_tokens: per row of scores the `keep` largest, protected ends first, ties to the lowest
// index, as ascending indices.  Scores become unsigned integers in the same order.  The keep-th largest is
// found digit by digit: 11 bits each, largest digit first, over the bits in which the row's scores differ
// at all (narrow rows spread over the bins as wide ones do).  After the first digit every thread takes a run of the
// row and keeps it as bits: what is above the digit's bin, what is inside.  Only what is inside is looked at again: its
// range (many equal scores end the search), further digits if it is much, or a list on which it is ranked once it is
// little.  Then a scan of the bits' counts gives every thread its place, and the indices go into a list that leaves
// in order.
//
// Scores are read from memory once, in 16-byte loads, and stay in shared memory: one block per row, and a
// cluster of up to 8 blocks, which read one another's counts through distributed shared memory, for rows that one
// block cannot hold.  (Clusters for shorter rows were slower, for few rows as for many: a cluster barrier costs
// about 1 us.)  A row too long for that is read again, from L2 as a rule, by every pass.
// The bound for many rows is the work on shared memory: 101 us for 896 rows of 40,001 (144 MB; one read takes 28), 29,000
// cycles a row, of which reading 7000, the first digit's counts 5000 (3 to 5 cycles for 32 of them: banks
// collide), the bits 3300, the list 4300, its way out 1500.  148 rows are a round; bringing the next round's rows into L2
// meanwhile took 13 us off.  Few rows are bound by the latency of about 12 phases between barriers: 8.9 us for 4
// rows of 16,384.
// ---------------------------------------------------------------------------------------------
constexpr int kSelThreads = 1024;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelDigitBits = 11;
constexpr int kSelBins = 1 << kSelDigitBits;
constexpr int kSelGathered = kSelBins;          // scores of the first digit's bin that are kept apart
constexpr int kSelRanked = 256;                 // at most so many are ranked directly
constexpr int kSelStaged = 49152;               // scores of a block's part kept in shared memory (192 KB)
constexpr int kSelRunQuads = 5;                 // scores / 4 of a thread's run of a row that is not staged
constexpr int kSelMaxRun = 13;                  // quads of a thread's run of a staged row, at most: 52 bits
constexpr int kSelMaxCluster = 8;
static_assert(kSelStaged / 4 <= 12 * kSelThreads, "a run and one quad more, where that makes it odd");
static_assert(kSelStaged < 65536 && 4 * kSelRunQuads * kSelThreads < 65536, "two counts in 32 bits");
static_assert(kSelBins == 2 * kSelThreads && kSelWarps == 32, "two bins to a thread, a warp over the warps' results");

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
  int rows, ahead;                              // rows that the GPU works on at a time
};

// The row starts `shift` scores past a 16-byte boundary.  Slot s holds token s - shift, so that 16-byte loads
// and 16-byte shared-memory words line up; slots below `shift` and past the end are no tokens.
struct SelectRow {
  int shift, slots, quads;
  int slot_begin, slot_end;                     // slots that compete
};
__device__ __forceinline__ SelectRow select_row(const SelectArgs& a, const float* row) {
  SelectRow r;
  r.shift = (int)((reinterpret_cast<uintptr_t>(row) >> 2) & 3);
  r.slots = a.n + r.shift;
  r.quads = (r.slots + 3) >> 2;
  r.slot_begin = a.first + r.shift;
  r.slot_end = a.n - a.last + r.shift;
  return r;
}
__device__ __forceinline__ uint4 select_load(const SelectRow& r, const float* row, int v) {       // slots 4 v .. 4 v + 3
  float4 f;
  if (4 * v >= r.shift && 4 * v + 3 < r.slots) {
    f = *reinterpret_cast<const float4*>(row + 4 * v - r.shift);
  } else {
    float* e = reinterpret_cast<float*>(&f);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int s = 4 * v + j;
      e[j] = s >= r.shift && s < r.slots ? row[s - r.shift] : 0.f;
    }
  }
  return make_uint4(select_key(f.x), select_key(f.y), select_key(f.z), select_key(f.w));
}
// a slot that does not compete is marked: protected tokens stay (largest key), other slots never do
__device__ __forceinline__ uint4 select_marked(const SelectRow& r, uint4 q, int v) {
  auto mark = [&](unsigned key, int s) {
    return s >= r.slot_begin && s < r.slot_end ? key : (s >= r.shift && s < r.slots ? 0xffffffffu : 0u);
  };
  return make_uint4(mark(q.x, 4 * v), mark(q.y, 4 * v + 1), mark(q.z, 4 * v + 2), mark(q.w, 4 * v + 3));
}
// the competing slot outside the whole quads [qa, qb) that falls to this thread, or -1
__device__ __forceinline__ int select_edge(int slot_begin, int slot_end, int qa, int qb) {
  const int t = threadIdx.x;
  if (t < 4) return slot_begin + t < min(qa * 4, slot_end) ? slot_begin + t : -1;
  if (t < 8) return slot_begin < slot_end && qb * 4 + t - 4 < slot_end ? qb * 4 + t - 4 : -1;
  return -1;
}

// exclusive prefix sum of v over the block, in thread order; *total receives the sum.  One barrier; warp_sums may be
// written again after the next.
__device__ __forceinline__ unsigned block_scan(unsigned v, unsigned* warp_sums, unsigned* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  const unsigned w = warp_sums[lane];
  const unsigned before = __reduce_add_sync(0xffffffffu, lane < warp ? w : 0u);
  *total = __reduce_add_sync(0xffffffffu, w);
  return before + incl - v;
}

// smallest lo and largest hi of the block.  One barrier; ranges may be written again after the next.
__device__ __forceinline__ void block_range(unsigned& lo, unsigned& hi, uint2* ranges) {
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if ((threadIdx.x & 31) == 0) ranges[threadIdx.x >> 5] = make_uint2(lo, hi);
  __syncthreads();
  const uint2 r = ranges[threadIdx.x & 31];
  lo = __reduce_min_sync(0xffffffffu, r.x);
  hi = __reduce_max_sync(0xffffffffu, r.y);
}

// What a thread knows of its run of up to 52 slots: bit b of the two words is slot 4 * first quad + b.
struct SelectMasks {
  unsigned above[2];                            // stays for sure
  unsigned in[2];                               // inside the range
};
__device__ __forceinline__ int mask_count(const unsigned* m) { return __popc(m[0]) + __popc(m[1]); }

__global__ void __launch_bounds__(kSelThreads)
select_tokens_kernel(SelectArgs a) {
  namespace cg = cooperative_groups;
  struct Shared {                               // what the cluster's blocks read of one another
    int hist[2][kSelBins];                      // digits in turn; the second also holds the gathered scores at first
    unsigned range[2][2];                       // smallest and largest competing score inside the range, in turn
    int num_gathered;
    int above, equal;                           // kept for sure / tied, in the part
  };
  extern __shared__ __align__(16) unsigned staged[];
  __shared__ __align__(16) Shared sh;
  __shared__ __align__(16) unsigned gathered[kSelGathered];           // all parts' scores inside the range
  __shared__ unsigned warp_sums[2][kSelWarps];                         // narrow()'s, the places'
  __shared__ uint2 ranges[kSelWarps];
  __shared__ int found_bin, found_above, found_count;
  __shared__ unsigned found_key;
  const int tid = threadIdx.x, lane = tid & 31;
  const cg::cluster_group cluster = cg::this_cluster();
  const int parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
  auto sync_parts = [&]() {
    if (parts > 1) cluster.sync(); else __syncthreads();
  };
  auto other = [&](int p) { return parts > 1 ? cluster.map_shared_rank(&sh, p) : &sh; };
  const long long row_index = blockIdx.x / parts;
  const float* __restrict__ row = a.scores + row_index * a.score_stride;
  const SelectRow r = select_row(a, row);
  const int part_quads = (r.quads + parts - 1) / parts;
  const int quad_begin = min(r.quads, part * part_quads), quad_end = min(r.quads, quad_begin + part_quads);
  uint4* const quads = reinterpret_cast<uint4*>(staged);               // quad v of the row at v - quad_begin
  // The part's competing slots [slot_begin, slot_end): whole quads [qa, qb), and up to three slots on each side,
  // one to a thread.
  const int slot_begin = max(r.slot_begin, quad_begin * 4), slot_end = min(r.slot_end, quad_end * 4);
  const int qa = (slot_begin + 3) >> 2, qb = max(qa, slot_end >> 2);
  const int edge = select_edge(slot_begin, slot_end, qa, qb);
  const unsigned edge_key = edge >= 0 ? select_key(row[edge - r.shift]) : 0u;

  unsigned lo = edge >= 0 ? edge_key : 0xffffffffu, hi = edge_key;
  constexpr int kAhead = 4;                                            // loads in flight per thread
  for (int v0 = quad_begin + tid; v0 < quad_end; v0 += kAhead * kSelThreads) {
    uint4 k[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (v0 + j * kSelThreads < quad_end) k[j] = select_load(r, row, v0 + j * kSelThreads);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int v = v0 + j * kSelThreads;
      if (v >= quad_end) break;
      const bool whole = v >= qa && v < qb;
      quads[v - quad_begin] = whole ? k[j] : select_marked(r, k[j], v);
      if (whole) {
        lo = min(min(min(lo, k[j].x), k[j].y), min(k[j].z, k[j].w));
        hi = max(max(max(hi, k[j].x), k[j].y), max(k[j].z, k[j].w));
      }
    }
  }
  reinterpret_cast<uint4*>(sh.hist)[tid] = make_uint4(0, 0, 0, 0);    // both digits: 4 * 1024 bins
  if (tid == 0) sh.num_gathered = 0;
  block_range(lo, hi, ranges);
  // The row is here; the one that this SM takes next comes into L2 while this one is worked on.
  if (part == 0 && tid == 0 && row_index + a.ahead < a.rows) {
    const uintptr_t next = reinterpret_cast<uintptr_t>(row + a.ahead * a.score_stride);
    const uintptr_t from = (next + 15) & ~(uintptr_t)15, to = (next + 4ull * a.n) & ~(uintptr_t)15;
    if (to > from)
      asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from), "r"((unsigned)(to - from)) : "memory");
  }
  if (parts > 1) {
    if (tid == 0) {
      sh.range[0][0] = lo;
      sh.range[0][1] = hi;
    }
    cluster.sync();
    const Shared* o = other(lane % parts);                             // lane p asks part p: one trip for all
    lo = __reduce_min_sync(0xffffffffu, o->range[0][0]);
    hi = __reduce_max_sync(0xffffffffu, o->range[0][1]);
  }

  // The k-th largest of the competing scores is in [base, base + span], where `inside` of them are and it is the
  // k-th from the top.  narrow(): the digit's histogram, summed over `among` parts, shortens the range.
  int k = a.keep - a.first - a.last, inside = 0, pass = 0, digit = 0;
  unsigned base = 0, span = 0;
  auto narrow = [&](int among, int buffer) {
    // counts from the top: thread t holds bins 2046 - 2 t and 2047 - 2 t
    const int bin0 = kSelBins - 2 - 2 * tid;
    int2 h = *reinterpret_cast<const int2*>(&sh.hist[buffer][bin0]);
    int c0 = h.x, c1 = h.y;
    if (among > 1) {
      int2 g[kSelMaxCluster];
#pragma unroll
      for (int p = 0; p < kSelMaxCluster; ++p)
        if (p < among && p != part) g[p] = *reinterpret_cast<const int2*>(&other(p)->hist[buffer][bin0]);
#pragma unroll
      for (int p = 0; p < kSelMaxCluster; ++p)
        if (p < among && p != part) {
          c0 += g[p].x;
          c1 += g[p].y;
        }
    }
    unsigned total;
    const int above1 = (int)block_scan((unsigned)(c0 + c1), warp_sums[0], &total), above0 = above1 + c1;
    const bool in1 = above1 < k && k <= above0, in0 = above0 < k && k <= above0 + c0;
    if (in0 || in1) {
      found_bin = in1 ? bin0 + 1 : bin0;
      found_above = in1 ? above1 : above0;
      found_count = in1 ? c1 : c0;
    }
    __syncthreads();
    k -= found_above;
    inside = found_count;
    base += (unsigned)found_bin << digit;
    span = min(span - ((unsigned)found_bin << digit), (1u << digit) - 1u);
    digit = max(0, digit - kSelDigitBits);
  };
  const bool some = k > 0 && k < a.n - a.first - a.last;               // not all, not none of those that compete
  if (some) {
    base = lo;
    span = hi - lo;
    digit = max(0, (32 - __clz(span)) - kSelDigitBits);
#pragma unroll 2
    for (int v = qa + tid; v < qb; v += kSelThreads) {                 // every score is inside the range
      const uint4 q = quads[v - quad_begin];
      atomicAdd(&sh.hist[0][(q.x - base) >> digit], 1);
      atomicAdd(&sh.hist[0][(q.y - base) >> digit], 1);
      atomicAdd(&sh.hist[0][(q.z - base) >> digit], 1);
      atomicAdd(&sh.hist[0][(q.w - base) >> digit], 1);
    }
    if (edge >= 0) atomicAdd(&sh.hist[0][(edge_key - base) >> digit], 1);
    sync_parts();
    narrow(parts, 0);
  } else {
    base = k > 0 ? 1u : 0xfffffffeu;                                   // between the marks: no score has these values
  }

  // From here on a thread has a run of slots of its own, as bits: what is above the range, what is inside.  An odd
  // number of quads, so that the runs of a quarter warp start on different banks.
  const int run = ((part_quads + kSelThreads - 1) / kSelThreads) | 1;
  const int my_quads = min(run, quad_end - quad_begin - tid * run);    // may be below 0
  const unsigned* const mine = staged + 4 * tid * run;
  SelectMasks m = {{0u, 0u}, {0u, 0u}};
  {
    const unsigned top = base + span;
#pragma unroll
    for (int i = 0; i < kSelMaxRun; ++i) {
      if (i >= my_quads) break;
      const uint4 q = reinterpret_cast<const uint4*>(mine)[i];
      const unsigned e[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int w = (4 * i + j) >> 5;
        const unsigned bit = 1u << ((4 * i + j) & 31);
        if (e[j] > top) m.above[w] |= bit;
        if (e[j] >= base) m.in[w] |= bit;
      }
    }
    m.in[0] &= ~m.above[0];
    m.in[1] &= ~m.above[1];
  }
  // f(score, word, bit) for every score of the run inside the range
  auto each_inside = [&](auto&& f) {
#pragma unroll
    for (int w = 0; w < 2; ++w)
      for (unsigned left = m.in[w]; left != 0u; left &= left - 1u) {
        const int b = __ffs((int)left) - 1;
        f(mine[32 * w + b], w, 1u << b);
      }
  };
  auto refine = [&]() {                                                // the range has become shorter
    const unsigned top = base + span;
    each_inside([&](unsigned e, int w, unsigned bit) {
      if (e > top) m.above[w] |= bit;
      if (e - base > span) m.in[w] &= ~bit;
    });
  };

  // A bin of many scores is often one of many equal ones: their smallest and largest say so, and else where
  // the next digit begins.  A bin too full to be gathered takes further digits.
  while (span > 0 && inside > k && inside > kSelRanked) {
    ++pass;
    unsigned least = 0xffffffffu, most = 0u;
    each_inside([&](unsigned e, int, unsigned) {
      least = min(least, e);
      most = max(most, e);
    });
    block_range(least, most, ranges);
    if (parts > 1) {
      if (tid == 0) {
        sh.range[pass & 1][0] = least;
        sh.range[pass & 1][1] = most;
      }
      cluster.sync();
      const Shared* o = other(lane % parts);
      least = __reduce_min_sync(0xffffffffu, o->range[pass & 1][0]);
      most = __reduce_max_sync(0xffffffffu, o->range[pass & 1][1]);
    }
    base = least;
    span = most - least;
    digit = max(0, (32 - __clz(span)) - kSelDigitBits);
    if (span == 0 || inside <= kSelGathered) break;
    each_inside([&](unsigned e, int, unsigned) { atomicAdd(&sh.hist[pass & 1][(e - base) >> digit], 1); });
    sync_parts();
    // every part has read the digit before this one: its bins are cleared for the next
    reinterpret_cast<int2*>(sh.hist[(pass + 1) & 1])[tid] = make_int2(0, 0);
    narrow(parts, pass & 1);
    refine();
  }
  if (span > 0 && inside > k) {
    // gather the scores inside; from here on every part of the cluster does the same work on the same list
    const int lists = (pass + 1) & 1, bins = pass & 1;                 // one digit's bins hold the part's list
    unsigned* const part_list = reinterpret_cast<unsigned*>(sh.hist[lists]);
    {
      const int count = mask_count(m.in);
      int at = count;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, at, o);
        if (lane >= o) at += x;
      }
      int first = 0;
      if (lane == 31 && at > 0) first = atomicAdd(&sh.num_gathered, at);
      at += __shfl_sync(0xffffffffu, first, 31) - count;
      each_inside([&](unsigned e, int, unsigned) { part_list[at++] = e; });
    }
    if (parts == 1 && tid < 4 && inside + tid < kSelGathered) part_list[inside + tid] = 0u;     // read in fours below
    sync_parts();
    unsigned* list = part_list;
    if (parts > 1) {
      const int theirs = lane < parts ? other(lane)->num_gathered : 0;
      for (int i = tid; i < kSelGathered; i += kSelThreads) {          // thread i takes the i-th of all parts' scores
        int from = -1, at = i;
#pragma unroll
        for (int p = 0; p < kSelMaxCluster; ++p) {
          const int c = __shfl_sync(0xffffffffu, theirs, p);
          if (from < 0 && at < c) from = p;
          if (from < 0) at -= c;
        }
        gathered[i] = from >= 0 ? (unsigned)other(from)->hist[lists][at] : 0u;         // past the end: below any score
      }
      list = gathered;
      __syncthreads();
    }
    const int all = inside;
    while (span > 0 && inside > k) {
      if (all <= kSelRanked) {
        if (tid < all) {
          const unsigned key = list[tid];
          int greater = 0, same = 0;
          for (int i = 0; i < all; i += 4) {
            const uint4 c = *reinterpret_cast<const uint4*>(&list[i]);
            greater += (c.x > key) + (c.y > key) + (c.z > key) + (c.w > key);
            same += (c.x == key) + (c.y == key) + (c.z == key) + (c.w == key);
          }
          if (greater < k && k <= greater + same) {                    // by every thread with that score, alike
            found_key = key;
            found_above = greater;
            found_count = same;
          }
        }
        __syncthreads();
        base = found_key;
        k -= found_above;
        inside = found_count;
        span = 0;
      } else {
        reinterpret_cast<int2*>(sh.hist[bins])[tid] = make_int2(0, 0);
        __syncthreads();
        for (int i = tid; i < all; i += kSelThreads) {
          const unsigned d = list[i] - base;
          if (d <= span) atomicAdd(&sh.hist[bins][d >> digit], 1);
        }
        __syncthreads();
        narrow(1, bins);
      }
    }
    refine();
  }

  // Kept: what is above the range, and the first k of what is inside (all of it, or equal scores).
  const int n_in = mask_count(m.in);
  unsigned total;                                                      // a part has less than 2^16 slots
  const unsigned place = block_scan((unsigned)mask_count(m.above) | (unsigned)n_in << 16, warp_sums[1], &total);
  const int part_above = (int)(total & 0xffffu), part_in = (int)(total >> 16);
  int at_above = 0, at_in = 0;                                         // of the parts before this one
  if (parts > 1) {
    if (tid == 0) {
      sh.above = part_above;
      sh.equal = part_in;
    }
    cluster.sync();
    const Shared* o = other(lane % parts);
    at_above = __reduce_add_sync(0xffffffffu, lane < part ? o->above : 0);
    at_in = __reduce_add_sync(0xffffffffu, lane < part ? o->equal : 0);
  }
  const int in_before = at_in + (int)(place >> 16);
  if (in_before >= k) {
    m.in[0] = m.in[1] = 0u;
  } else {
    for (int drop = n_in - (k - in_before); drop > 0; --drop) {        // one run of the row
      const int w = m.in[1] != 0u ? 1 : 0;                             // the last of them
      const unsigned bit = 1u << (31 - __clz((int)(w ? m.in[1] : m.in[0])));
      if (w) m.in[1] ^= bit; else m.in[0] ^= bit;
    }
  }
  // The list is put together where the scores were and leaves in order.
  int* const list = reinterpret_cast<int*>(staged);
  const int in_part = min(at_in, k);                                   // of those before the part
  int at = (int)(place & 0xffffu) + min(in_before, k) - in_part;
  const int token = (quad_begin + tid * run) * 4 - r.shift;
#pragma unroll
  for (int w = 0; w < 2; ++w)
    for (unsigned left = m.above[w] | m.in[w]; left != 0u; left &= left - 1u) list[at++] = token + 32 * w + __ffs((int)left) - 1;
  __syncthreads();
  int* const out = a.idx + row_index * a.idx_stride + at_above + in_part;
  const int count = part_above + min(at_in + part_in, k) - in_part;
#pragma unroll 4
  for (int i = tid; i < count; i += kSelThreads) out[i] = list[i];
  if (parts > 1) cluster.sync();                                       // the others have read this block's counts
}

// Rows too long to be staged: one block, which reads the row in every pass.
__global__ void __launch_bounds__(kSelThreads)
select_long_rows_kernel(SelectArgs a) {
  __shared__ __align__(16) int hist[kSelBins];
  __shared__ unsigned warp_sums[2][kSelWarps];                         // in turn, where one scan follows another
  __shared__ uint2 ranges[kSelWarps];
  __shared__ int found_bin, found_above, found_count;
  const int tid = threadIdx.x;
  const float* __restrict__ row = a.scores + blockIdx.x * a.score_stride;
  int* out = a.idx + blockIdx.x * a.idx_stride;
  const SelectRow r = select_row(a, row);
  const int qa = (r.slot_begin + 3) >> 2, qb = max(qa, r.slot_end >> 2);
  const int edge = select_edge(r.slot_begin, r.slot_end, qa, qb);
  const unsigned edge_key = edge >= 0 ? select_key(row[edge - r.shift]) : 0u;

  // The k-th largest of the competing scores is in [base, base + span], where `inside` of them are and it is the
  // k-th from the top.
  int k = a.keep - a.first - a.last, inside = a.n - a.first - a.last;
  unsigned base = 0u, span = 0xffffffffu;
  auto each_inside = [&](auto&& f) {                                   // f(score) for every one inside the range
#pragma unroll 2
    for (int v = qa + tid; v < qb; v += kSelThreads) {
      const uint4 q = select_load(r, row, v);
      const unsigned d[4] = {q.x - base, q.y - base, q.z - base, q.w - base};   // below base: wraps to a large value
      if (min(min(d[0], d[1]), min(d[2], d[3])) <= span) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (d[j] <= span) f(d[j] + base);
      }
    }
    if (edge >= 0 && edge_key - base <= span) f(edge_key);
  };
  if (k > 0 && inside > k) {
    while (span > 0 && inside > k) {
      // the range taken to what is in it (one of many equal scores becomes a range of one), then its first digit
      unsigned least = 0xffffffffu, most = 0u;
      each_inside([&](unsigned e) {
        least = min(least, e);
        most = max(most, e);
      });
      reinterpret_cast<int2*>(hist)[tid] = make_int2(0, 0);
      block_range(least, most, ranges);
      base = least;
      span = most - least;
      if (span == 0) break;
      const int digit = max(0, (32 - __clz(span)) - kSelDigitBits);
      each_inside([&](unsigned e) { atomicAdd(&hist[(e - base) >> digit], 1); });
      __syncthreads();
      // counts from the top: thread t holds bins 2046 - 2 t and 2047 - 2 t
      const int bin0 = kSelBins - 2 - 2 * tid;
      const int2 h = *reinterpret_cast<const int2*>(&hist[bin0]);
      unsigned total;
      const int above1 = (int)block_scan((unsigned)(h.x + h.y), warp_sums[0], &total), above0 = above1 + h.y;
      const bool in1 = above1 < k && k <= above0, in0 = above0 < k && k <= above0 + h.x;
      if (in0 || in1) {
        found_bin = in1 ? bin0 + 1 : bin0;
        found_above = in1 ? above1 : above0;
        found_count = in1 ? h.y : h.x;
      }
      __syncthreads();
      k -= found_above;
      inside = found_count;
      base += (unsigned)found_bin << digit;
      span = min(span - ((unsigned)found_bin << digit), (1u << digit) - 1u);
    }
  } else {
    base = k > 0 ? 1u : 0xfffffffeu;                                   // between the marks: no score has these values
    span = 0u;
  }
  // Kept: what is above the range, and the first k of what is inside (all of it, or equal scores).
  const unsigned top = base + span;
  int at_above = 0, at_in = 0, sums = 0;
  for (int round = 0; round < r.quads; round += kSelRunQuads * kSelThreads) {
    unsigned e[4 * kSelRunQuads];                                      // this thread's run
    const int v0 = round + tid * kSelRunQuads;
#pragma unroll
    for (int i = 0; i < kSelRunQuads; ++i) {
      uint4 q = make_uint4(0, 0, 0, 0);
      if (v0 + i < r.quads) q = select_marked(r, select_load(r, row, v0 + i), v0 + i);
      e[4 * i] = q.x;
      e[4 * i + 1] = q.y;
      e[4 * i + 2] = q.z;
      e[4 * i + 3] = q.w;
    }
    int n_above = 0, n_in = 0;
#pragma unroll
    for (int i = 0; i < 4 * kSelRunQuads; ++i) {
      n_above += e[i] > top ? 1 : 0;
      n_in += e[i] - base <= span ? 1 : 0;
    }
    unsigned total;                                                    // both counts in one: 20,480 scores a round
    const unsigned place = block_scan((unsigned)n_above | (unsigned)n_in << 16, warp_sums[sums], &total);
    sums ^= 1;
    int in_before = at_in + (int)(place >> 16);
    int at = at_above + (int)(place & 0xffffu) + min(in_before, k);
#pragma unroll
    for (int i = 0; i < 4 * kSelRunQuads; ++i)
      if (e[i] > top || (e[i] - base <= span && in_before++ < k)) out[at++] = v0 * 4 - r.shift + i;
    at_above += (int)(total & 0xffffu);
    at_in += (int)(total >> 16);
  }
}

// Blocks per row: as few as hold it.
inline cudaError_t launch_select(SelectArgs a, long long rows, int sm_count, cudaStream_t stream) {
  const int quads = (a.n + 3 + 3) / 4;                                 // up to three slots before the first token
  int parts = 1;
  while (parts < kSelMaxCluster && (quads + parts - 1) / parts * 4 > kSelStaged) parts *= 2;
  const int part_quads = (quads + parts - 1) / parts;
  if (part_quads * 4 > kSelStaged || rows * parts > 0x7fffffffLL) {
    select_long_rows_kernel<<<(unsigned)rows, kSelThreads, 0, stream>>>(a);
    return cudaGetLastError();
  }
  a.rows = (int)rows;
  a.ahead = std::max(1, sm_count / parts);                             // a block takes the SM's registers
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * parts), 1, 1);
  cfg.blockDim = dim3(kSelThreads, 1, 1);
  cfg.dynamicSmemBytes = (size_t)part_quads * 16;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = parts;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = parts > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, select_tokens_kernel, a);
}

// ---------------------------------------------------------------------------------------------
// bicache_compact_prefix: token i of head j of the shorter prefix becomes token idx[layer][j][i] of the
// longer one, K and V.  A page image keeps a token's dims in two runs of 128 bytes (or one of D elements),
// and the 16-byte chunks of a run are permuted inside it, so the copy goes chunk by chunk: half a warp
// moves one token of one head (D = 128, bf16), a thread the same chunk of every row it comes to.  Unused slots of the last page become zero, as everywhere.
// An index outside the prefix leaves a zero token and raises the status word.
// Bound by memory: 8192 of 16,384 tokens, 32 heads, 4 layers (1.07 GB read and written) take 169 us, 98 % of a plain
// copy's bandwidth; a single layer of 1001 tokens and 4 heads takes 2.5 us.
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
  const unsigned heads = a.num_kv_heads, dst_pages = a.dst_pages;
  const unsigned rows = kPageSize * heads * dst_pages * (unsigned)a.num_layers;      // a row: a token of a head
  const unsigned per_block = kCompactThreads / a.chunks_per_row, first = threadIdx.x / a.chunks_per_row;
  const int c16 = threadIdx.x - first * a.chunks_per_row, row_bytes = a.chunks_per_row * 16;
  if (first >= per_block) return;
  for (unsigned r = blockIdx.x * per_block + first; r < rows; r += gridDim.x * per_block) {
    const unsigned slot = r % kPageSize, page = r / kPageSize / heads, hk = r / kPageSize - page * heads;
    const unsigned layer = page / dst_pages, pg = page - layer * dst_pages;
    const int t = (a.dst_first + (int)pg) * kPageSize + (int)slot;
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    bool write = a.src_first == 0;                          // padding and bad indices: by the first window
    const long long head = layer * a.layer_bytes + (long long)hk * a.page_bytes;
    if (t < a.keep) {
      const int s = a.idx[layer * a.idx_layer_stride + hk * a.idx_head_stride + t];
      if (s < 0 || s >= a.src_m) {
        if (write) atomicCAS(a.status, kDevOk, kDevBadIndex);
      } else {
        const int sp = s / kPageSize - a.src_first;
        write = sp >= 0 && sp < a.src_pages;
        if (write) {
          const long long so = head + (long long)list.w[sp] * heads * a.page_bytes +
                               page_chunk_offset(a.swizzled != 0, s % kPageSize, c16, row_bytes);
          k = *reinterpret_cast<const uint4*>(a.pool_k + so);
          v = *reinterpret_cast<const uint4*>(a.pool_v + so);
        }
      }
    }
    if (write) {
      const long long to = head + (long long)list.w[a.src_pages + pg] * heads * a.page_bytes +
                           page_chunk_offset(a.swizzled != 0, (int)slot, c16, row_bytes);
      *reinterpret_cast<uint4*>(a.pool_k + to) = k;
      *reinterpret_cast<uint4*>(a.pool_v + to) = v;
    }
  }
}

// gather_prefix_kernel (the layer read-back) with the page list in the parameters: no copy before the launch, which
// is what a read-back of a short prefix otherwise waits for (14 us a call, 6.5 without).
template <int kWords>
__global__ void __launch_bounds__(kCompactThreads)
read_layer_kernel(const char* __restrict__ pool_k, const char* __restrict__ pool_v, char* __restrict__ dst_k,
                  char* __restrict__ dst_v, int m, int num_kv_heads, int chunks_per_row, long long dst_row_stride_bytes,
                  int page_bytes, int swizzled, const __grid_constant__ ParamList<kWords> pages) {
  const unsigned heads = num_kv_heads, rows = (unsigned)m * heads;
  const unsigned per_block = kCompactThreads / chunks_per_row, first = threadIdx.x / chunks_per_row;
  const int c16 = threadIdx.x - first * chunks_per_row, row_bytes = chunks_per_row * 16;
  if (first >= per_block) return;
  for (unsigned r = blockIdx.x * per_block + first; r < rows; r += gridDim.x * per_block) {
    const unsigned t = r / heads, hk = r - t * heads;
    const long long po = ((long long)pages.w[t / kPageSize] * heads + hk) * page_bytes +
                         page_chunk_offset(swizzled != 0, (int)(t % kPageSize), c16, row_bytes);
    const long long to = t * dst_row_stride_bytes + (long long)hk * row_bytes + c16 * 16;
    *reinterpret_cast<uint4*>(dst_k + to) = *reinterpret_cast<const uint4*>(pool_k + po);
    *reinterpret_cast<uint4*>(dst_v + to) = *reinterpret_cast<const uint4*>(pool_v + po);
  }
}
// Blocks for `rows` rows of one of the two kernels: eight rounds of resident ones at most.  (One round: 189 us for both
// kernels on 4 layers of 8192 x 32 rows where eight take 169; two rows to a thread at a time: 185 and 170.)
inline int copy_blocks(long long rows, int chunks_per_row, int sm_count) {
  const long long per_block = kCompactThreads / chunks_per_row;
  return (int)std::min<long long>((rows + per_block - 1) / per_block, 64LL * sm_count);
}

// ---------------------------------------------------------------------------------------------
// bicache_prefix_weights.  For every cached key t of prefix g and KV head j
//   out[g][j][t] = decay in[g][j][t] + sum over the rows a and query heads h of the group
//                  exp(scale q[a][h] . k[t][j] - lse[a][h]);
// rows with an infinite lse add nothing.  The batch: groups (one per prefix), the runs of query rows that
// belong to each, and their page lists, all in the parameter list.  Row space of a group: the tokens of its
// requests one after the other, packed row p = token * G + head in the KV group, cut into row tiles (of 128 rows in
// the CUDA-core form, of whole tokens in the other).  A
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
  int tiles;                    // row tiles of the group
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
  int max_item_tiles;           // row tiles of the longest item
  int tile_tokens;              // tensor-core form: tokens of a row tile (as many as give at most 128 rows)
  int boxes;                    // tensor-core form: the tensor map of q is valid
};

__device__ __forceinline__ const WeightGroup& weight_group(const int* list, int g) {
  return *reinterpret_cast<const WeightGroup*>(&list[g * kGroupWords]);
}
// the group of a work item.  They are in order; the walk is one record after the other, up to 396 of them with a
// prefix for each request.  That is cheap for a few and what such a batch waits for: 32 heads, 16 rows to a prefix, 64
// prefixes of 500 keys take 179 us, 390 of 30 keys 1663.
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

// CUDA-core form.  Block: 16 * kPerThread keys against tiles of 128 packed rows, each thread kPerThread keys x 8 rows,
// dims in shared memory as fp32 (rows padded by 4 floats: the 16-byte reads of a quarter warp fall on different
// banks).  A thread adds the exponentials of a tile's eight rows in fp32 and keeps the sums over tiles in fp64; those
// of the 16 threads of a key are added at the end.
// Bound by the fp32 products and the shared-memory reads that feed them: with 8 x 8 a step of four dims is 16 reads (64
// cycles of an SM's 128 bytes a cycle for a warp) for 256 products (64 cycles); with 4 x 8 it is 48 against 32.  So it is
// eight keys to a thread, but four where eight do not fit shared memory (head dims past 192) and where a batch has not a
// block for every SM (fp32, 4 heads of 64 dims: 2048 rows over 4096 keys 157 us with eight, 170 with four; 100 rows over
// 1000 keys 16.0 and 9.7).  The first is 27 TFLOP/s; products alone, from registers, reach 52 on this part.  With 128
// dims four would be ahead of eight there too (323 against 372 us), which the rule does not use yet.  bf16 takes as long
// as fp32 (149 us with 64 dims, 219 with 96); with head_dim 128 it takes the tensor-core form (21 us).
constexpr int kWsRows = 128, kWsThreads = 256;
constexpr int kWsAhead = 4;                             // loads of query rows a thread has on their way
constexpr int kWsEightMaxD = 192;
inline size_t weights_simt_smem(int D, int per_thread) {
  return sizeof(float) * ((size_t)(16 * per_thread + kWsRows) * (D + 4) + kWsRows);
}

__device__ __forceinline__ float exp2_approx(float x) {                  // 2 ulp; 0 below 2^-126
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <typename T, int kPerThread, int kWords>
__global__ void __launch_bounds__(kWsThreads, 2)
weights_simt_kernel(const __grid_constant__ WeightArgs a, const __grid_constant__ ParamList<kWords> params) {
  const int* const list = params.w;
  using Tr = ElemTraits<T>;
  constexpr int kEsize = (int)sizeof(T), kPer = Tr::kPerChunk, kWsKeys = 16 * kPerThread;
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
  double total[kPerThread] = {};
  const float scale_log2 = a.scale * 1.4426950408889634f;
  const long long rows = (long long)g.tokens * G;
  const int tiles = (int)((rows + kWsRows - 1) / kWsRows);
  const int tile_begin = split * g.tiles_per_split, tile_end = min(tiles, tile_begin + g.tiles_per_split);
  // a thread loads one chunk of every row it comes to
  const int per_pass = kWsThreads / chunks, first = tid / chunks, c = tid - first * chunks;
  const int load_end = first < per_pass ? kWsRows : 0;
  for (int tile = tile_begin; tile < tile_end; ++tile) {
    const long long p0 = (long long)tile * kWsRows;
    const int here = (int)min((long long)kWsRows, rows - p0);
    __syncthreads();                                    // the last tile's rows have been used
    for (int r0 = first; r0 < load_end; r0 += kWsAhead * per_pass) {
      uint4 x[kWsAhead];
      float l[kWsAhead];
#pragma unroll
      for (int u = 0; u < kWsAhead; ++u) {
        const int r = r0 + u * per_pass;
        x[u] = make_uint4(0, 0, 0, 0);
        l[u] = INFINITY;
        if (r < here) {
          const int tok = (int)((p0 + r) / G), h = hk * G + (int)(p0 + r - (long long)tok * G);
          const long long row = weight_row(list, g, tok);
          x[u] = *reinterpret_cast<const uint4*>(a.q + (row * a.q_stride + (long long)h * D) * kEsize + c * 16);
          if (c == 0) l[u] = a.lse[row * a.Hq + h];
        }
      }
#pragma unroll
      for (int u = 0; u < kWsAhead; ++u) {
        const int r = r0 + u * per_pass;
        if (r >= kWsRows) break;
        float f[kPer];
        Tr::unpack(x[u], f);
#pragma unroll
        for (int e = 0; e < kPer; ++e) qs[r * pitch + c * kPer + e] = f[e];
        if (c == 0) ls[r] = l[u];
      }
    }
    __syncthreads();
    auto sum_rows = [&](auto count) {                   // the first 16 * count rows of the tile
      constexpr int kRows = decltype(count)::value;
      float acc[kPerThread][kRows] = {};
      for (int d = 0; d < D; d += 4) {
        float4 kf[kPerThread];
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) kf[i] = *reinterpret_cast<const float4*>(&ks[(tx + 16 * i) * pitch + d]);
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
          const float4 qf = *reinterpret_cast<const float4*>(&qs[(ty + 16 * j) * pitch + d]);
#pragma unroll
          for (int i = 0; i < kPerThread; ++i) {
            acc[i][j] = fmaf(kf[i].x, qf.x, acc[i][j]);
            acc[i][j] = fmaf(kf[i].y, qf.y, acc[i][j]);
            acc[i][j] = fmaf(kf[i].z, qf.z, acc[i][j]);
            acc[i][j] = fmaf(kf[i].w, qf.w, acc[i][j]);
          }
        }
      }
      float sum[kPerThread] = {};
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        const float l = ls[ty + 16 * j];
        if (isinf(l)) continue;                         // masked or past the end, whatever the product is
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) sum[i] += exp2_approx(fmaf(scale_log2, acc[i][j], l * -1.4426950408889634f));
      }
#pragma unroll
      for (int i = 0; i < kPerThread; ++i) total[i] += (double)sum[i];
    };
    if (here <= 16) sum_rows(std::integral_constant<int, 1>());
    else if (here <= 64) sum_rows(std::integral_constant<int, 4>());
    else sum_rows(std::integral_constant<int, 8>());
  }
  __syncthreads();
  double* const red = reinterpret_cast<double*>(ws_smem);          // [16][kWsKeys]
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) red[ty * kWsKeys + tx + 16 * i] = total[i];
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
static_assert(16 * 128 * sizeof(double) <= sizeof(float) * (128 + kWsRows) * (32 + 4), "the sums are added over the tiles");

// The partial sums of the row ranges, added in order.  One thread per (KV head, key) of a group with splits.
// status: that of the kernel which wrote them, or nullptr if it has none.  Where it is raised that kernel has left some
// of them unwritten (all, if it was raised before), and the scores stay as they are.
template <int kWords>
__global__ void __launch_bounds__(256)
weights_sum_kernel(const __grid_constant__ WeightArgs a, const int* status,
                   const __grid_constant__ ParamList<kWords> params) {
  const int* const list = params.w;
  const bool complete = status == nullptr || *status == kDevOk;
  const WeightGroup& g = weight_group(list, blockIdx.y);
  if (g.splits <= 1) return;
  const long long per_split = (long long)a.Hkv * g.m;
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < per_split; i += gridDim.x * 256ll) {
    const int hk = (int)(i / g.m), t = (int)(i - (long long)hk * g.m);
    double s = 0.0;
    for (int k = 0; k < g.splits; ++k) s += (double)a.part[g.part_off + k * per_split + i];
    const long long o = g.score_off + hk * a.head_stride + g.key0 + t;
    if (complete) a.out[o] = (float)((a.decay != 0.f ? (double)a.decay * a.in[o] : 0.0) + s);
  }
}

}  // namespace bicache

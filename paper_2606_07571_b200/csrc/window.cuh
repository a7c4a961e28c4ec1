// bicache_attend_window: rows of a ragged batch attend over the cached tokens of their prefixes, under a sliding
// window and a number of first tokens that stay visible.  For a row at position p of a request whose prefix holds `len`
// tokens, token t is visible iff
//     t < len,  t <= p + right,  and  (t < sinks or t >= p - left);
//   o = sum over the visible t of softmax_t(scale q.k_t) v_t,   lse = log sum exp(scale q.k_t);
// a row that sees nothing gets o = 0, lse = -inf.
//
// This file: the batch as the kernels see it, the CUDA-core kernel (fp32, head dims other than 128), and the
// kernel that joins ranges of keys.
//
// The batch travels as launch parameters: requests, and of each the pages that some row of it sees, unless the prefix's pages
// follow one another in the pool (what an unbroken pool hands out), which the number of the first says.  A request's row
// space is its rows x the G = Hq / Hkv query heads of a KV head (packed row = row * G + head), cut into row tiles.  A row tile
// sees an interval of tokens (rows follow one another, so their windows join up) and the first tokens; its
// pages - those of the first tokens, then the interval's - are put side by side, and key tiles are cut from that
// sequence, so that the few first tokens share a tile with the window.  With few rows and many keys the key tiles are
// dealt out to several work items (splits), whose partial results the joining kernel puts together in a fixed order.
#pragma once
#include "evict.cuh"

namespace bicache {

struct WindowReq {
  long long row;                // first row of q, out and lse
  int n;                        // rows
  int pos;                      // position of the first
  int len;                      // cached tokens
  int first_page;               // of a prefix whose pages are consecutive, which needs no list; else -1
  int sink_pages;               // pages of the list that come before the gap (0: no gap)
  int gap;                      // pages left out behind them
  int page_word;                // page list in the parameter words, or among the staged pages
  int item_begin;               // first work item
  int splits, tiles_per_split;  // ranges of key tiles
  int part_off;                 // first partial result in row-heads (splits > 1)
  int row_tiles;
  int row_heads_before;         // row-heads of split requests before this one (joining kernel)
  int pad;
};
constexpr int kWindowReqWords = sizeof(WindowReq) / 4;
static_assert(sizeof(WindowReq) % 8 == 0, "8-byte aligned records");

struct WindowArgs {
  const char* q;
  char* out;
  float* lse;                   // or nullptr
  long long q_stride, out_stride;          // elements between rows
  const char *pool_k, *pool_v;  // of the layer
  const int* staged_pages;      // the page lists, if they did not fit the parameters
  long long page_stride;        // bytes of a page of all heads
  int page_bytes, swizzled;
  int Hq, Hkv, D;
  int sinks, left, right;       // left, right: -1 for no bound
  float scale;
  float *part_o, *part_lse;     // [row-head] x D, [row-head]
  int num_reqs, num_items;
};

// The last of `num` records whose start (`start` of it) is not above x.  A guess by proportion comes first, since batches are
// mostly even: every step of a search is a parameter read that waits for the one before.
template <typename R, typename F>
__device__ __forceinline__ const R& last_start(const int* list, int num, int total, int x, F&& start) {
  const R* const recs = reinterpret_cast<const R*>(list);
  int lo = 0, hi = num;
  if (num > 1) {
    const int guess = min(num - 1, (int)((long long)x * num / total));
    if (start(recs[guess]) <= x) {
      lo = guess;
      if (guess + 1 == num || start(recs[guess + 1]) > x) hi = guess + 1;
    } else {
      hi = guess;
    }
  }
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start(recs[mid]) <= x) lo = mid;
    else hi = mid;
  }
  return recs[lo];
}
// The request of a work item.
__device__ __forceinline__ const WindowReq& window_req(const WindowArgs& a, const int* list, int item) {
  return last_start<WindowReq>(list, a.num_reqs, a.num_items, item, [](const WindowReq& r) { return r.item_begin; });
}

// What a row at position p sees: tokens [first, end), and those of the first `sinks` that are below `end`.
struct WindowBounds {
  int first, end;
};
__host__ __device__ inline WindowBounds window_bounds(int sinks, int left, int right, int len, int p) {
  WindowBounds b;
  b.end = right < 0 || right >= len - p ? len : p + right + 1;       // p + right may not fit 32 bits
  b.first = left < 0 || left >= p ? 0 : p - left;
  if (b.first <= sinks) b.first = 0;
  if (b.first > b.end) b.first = b.end;
  return b;
}

// The pages that rows at positions pa .. pb see, side by side: `sink_pages` first pages, then from lo_page on; and what
// some of the rows sees, in columns of that sequence: [begin, end), and [0, sink); every row sees [all_begin, all_end).  (Windows start and end later the later
// the row, and rows that are past the cache by more than `left` see no window: if the first row does not, none does.)
struct WindowPages {
  int sink_pages, lo_page, count;
  int shift;                    // tokens left out between the two: column of token t behind the gap is t - shift
  int begin, end, sink;
  int all_begin, all_end;
};
__host__ __device__ inline WindowPages window_pages(int sinks, int left, int right, int len, int pa, int pb) {
  const WindowBounds a = window_bounds(sinks, left, right, len, pa), b = window_bounds(sinks, left, right, len, pb);
  const bool any = a.first < a.end;
  WindowPages w;
  w.sink = sinks < b.end ? sinks : b.end;
  w.sink_pages = (w.sink + kPageSize - 1) / kPageSize;
  w.lo_page = any ? a.first / kPageSize : w.sink_pages;
  const int hi_page = any ? (b.end + kPageSize - 1) / kPageSize : w.lo_page;
  if (w.lo_page <= w.sink_pages) {                                   // no gap: everything from token 0 on
    w.count = hi_page > w.sink_pages ? hi_page : w.sink_pages;
    w.sink_pages = w.lo_page = 0;
  } else {
    w.count = w.sink_pages + hi_page - w.lo_page;
  }
  w.shift = (w.lo_page - w.sink_pages) * kPageSize;
  w.begin = any ? a.first - w.shift : 0;
  w.end = any ? b.end - w.shift : 0;
  w.all_begin = b.first < b.end ? b.first - w.shift : 0;
  w.all_end = b.first < b.end ? a.end - w.shift : 0;
  return w;
}

// Columns of the page sequence that a row sees: [begin, end), and [0, sink).
struct WindowColumns {
  int begin, end, sink;
};
__device__ __forceinline__ WindowColumns window_columns(const WindowArgs& a, const WindowPages& w, int len, int p) {
  const WindowBounds b = window_bounds(a.sinks, a.left, a.right, len, p);
  WindowColumns c;
  c.begin = b.first - w.shift;
  c.end = b.end - w.shift;
  c.sink = min(a.sinks, b.end);
  if (b.first >= b.end) c.begin = c.end = 0;
  return c;
}

// One work item.
struct WindowItem {
  int hk, row0, split;          // KV head, first packed row, range of key tiles
  int tile_begin, tile_end;     // key tiles of the row tile's page sequence
  int start;                    // the tile to begin with; the others follow it, those before it come last
  WindowPages pages;
};
// The j-th tile of an item.
__device__ __forceinline__ int window_tile(int start, int begin, int end, int j) {
  const int t = start + j;
  return t < end ? t : t - (end - begin);
}
// kTile: tokens of a key tile.  Row tiles of a request have the same number of ranges; a range past a tile's end is empty.
// Row tiles go from the last, whose rows see most, to the first; neighbours are those of one KV head, which share keys in L2,
// or, with kHeadsTogether, the KV heads of one row tile, so that all long items come first.
template <int kTile, bool kHeadsTogether = false>
__device__ __forceinline__ WindowItem window_item(const WindowArgs& a, const WindowReq& r, int item, int tile_rows) {
  WindowItem it;
  const int G = a.Hq / a.Hkv;
  int at = item - r.item_begin;
  const int outer = (kHeadsTogether ? a.Hkv : r.row_tiles) * r.splits, o = at / outer;
  at -= o * outer;
  const int inner = at / r.splits, tile = r.row_tiles - 1 - (kHeadsTogether ? o : inner);
  it.hk = kHeadsTogether ? inner : o;
  it.split = at - inner * r.splits;
  it.row0 = tile * tile_rows;
  const int last = min(it.row0 + tile_rows, r.n * G) - 1;
  it.pages = window_pages(a.sinks, a.left, a.right, r.len, r.pos + it.row0 / G, r.pos + last / G);
  const int tiles = (it.pages.count * kPageSize + kTile - 1) / kTile;
  it.tile_begin = min(tiles, it.split * r.tiles_per_split);
  it.tile_end = min(tiles, it.tile_begin + r.tiles_per_split);
  // A tile that all rows see in full, else the middle of what they all see: the running maxima then start near where they
  // end.  (From the first tile on, where some rows see few keys or none, raising them cost a prompt under a window of 4096
  // with 4 first tokens a sixth of its time.)
  it.start = (it.pages.all_begin + kTile - 1) / kTile;
  if ((it.start + 1) * kTile > it.pages.all_end) it.start = (it.pages.all_begin + it.pages.all_end) / 2 / kTile;
  it.start = max(it.tile_begin, min(it.start, it.tile_end - 1));
  return it;
}
// The pool page of page `s` of an item's sequence.  (Two loads and a branch, not one load through either pointer: that would
// read the parameters by way of memory.)
__device__ __forceinline__ int window_page(const WindowArgs& a, const WindowReq& r, const int* list, const WindowPages& w, int s) {
  const int page = s < w.sink_pages ? s : s - w.sink_pages + w.lo_page;          // of the prefix
  if (r.first_page >= 0) return r.first_page + page;
  const int at = page < r.sink_pages ? page : page - r.gap;
  return a.staged_pages ? a.staged_pages[r.page_word + at] : list[r.page_word + at];
}
// The slots of page `s` of the sequence that some row of the item sees: [lo, hi), and [0, sink) besides.  What lies
// in the others must not reach a sum, not even with weight 0: it may be no number.
struct WindowSlots {
  int lo, hi, sink;
  __device__ __forceinline__ bool whole() const { return (lo <= 0 && hi >= kPageSize) || sink >= kPageSize; }
  __device__ __forceinline__ bool has(int slot) const { return (slot >= lo && slot < hi) || slot < sink; }
};
__device__ __forceinline__ WindowSlots window_slots(const WindowPages& w, int s) {
  return WindowSlots{w.begin - s * kPageSize, w.end - s * kPageSize, w.sink - s * kPageSize};
}

// Where the results of a packed row go.
struct WindowRow {
  int t, h;                     // row of the request, query head
  __device__ __forceinline__ WindowRow(const WindowArgs& a, int hk, int p) {
    const int G = a.Hq / a.Hkv;
    t = p / G;
    h = hk * G + (p - t * G);
  }
};
__device__ __forceinline__ long long window_part(const WindowArgs& a, const WindowReq& r, int split, const WindowRow& w) {
  return r.part_off + ((long long)split * r.n + w.t) * a.Hq + w.h;
}

// ---------------------------------------------------------------------------------------------
// CUDA-core kernel.  128 threads take a row tile against key tiles of 64: queries, keys and values lie in shared memory
// as fp32 (a row's end padded by 16 bytes, so that lanes on neighbouring rows read other banks).  A row tile of 64 is a grid
// of 8 x 16 threads, each with 8 rows x 4 keys of the scores (two dims to a packed product) and 8 rows x D / 16 dims of the
// output (two rows to a packed product).  A row tile of 16, for few rows, is four groups of 2 x 16 threads, each group with a quarter of the keys of a
// tile and a running softmax of its own; they are put together at the end.  All sums in fp32.  Values arrive while the scores
// are computed, the next tile's keys during the rest.
// Bound by instructions and their latency: 4500 to a warp and tile, less than half of them products, 12 warps to an SM.
// 10,334 causal fp32 rows of 4 heads of 64 dims take 1555 us (35 TFLOP/s; 256 threads with 4 rows each took 3390, products of
// the output by single rows 1670), three requests of up to 1000 rows under a window of 700 78 us.  bf16
// with 64 dims, 32 query heads over 8: 4096 causal rows 1783 us (39 TFLOP/s; 165 us with 128 dims on the tensor cores), one
// token over 16,384 keys 37 us.
// ---------------------------------------------------------------------------------------------
constexpr int kWinThreads = 128;
constexpr int kWinKeys = 64;
constexpr int kWinPer = 8;                      // rows of a thread
constexpr int kWinLanes = 16;                   // threads that share a row

inline size_t window_simt_smem(int rows, int D) {
  return sizeof(float) * ((size_t)(rows + 2 * kWinKeys) * (D + 4) + (size_t)kWinKeys * (rows + 4));
}

__device__ __forceinline__ float win_exp2(float x) {               // 2 ulp, results below 2^-126 are 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ unsigned long long win_pack(float lo, float hi) {
  unsigned long long d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ float lanes16_max(float x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float lanes16_sum(float x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// kMaxD 64 and 128: head dims of exactly that; 256: any.
constexpr int kWinAnyD = 256;
inline int window_simt_blocks(int rows, int D) {                   // that fit an SM, by shared memory and registers
  const int fit = (int)(227 * 1024 / (window_simt_smem(rows, D) + 1280));
  return std::max(1, std::min(fit, D == 64 ? 3 : 2));
}
template <typename T, int kRows, int kMaxD, int kWords>
__global__ void __launch_bounds__(kWinThreads, kMaxD == 64 ? 3 : kMaxD == 128 ? 2 : 1)
window_simt_kernel(const __grid_constant__ WindowArgs a, const __grid_constant__ ParamList<kWords> list) {
  using Tr = ElemTraits<T>;
  constexpr int kPer = Tr::kPerChunk, kEsize = (int)sizeof(T);
  constexpr int kRowGroups = kRows / kWinPer, kParts = kWinThreads / (kRowGroups * kWinLanes);   // groups over the keys
  constexpr int kPartKeys = kWinKeys / kParts, kMine = kPartKeys / kWinLanes;                    // of a group, of a thread
  constexpr int kPairs = kMaxD / (2 * kWinLanes);                  // pairs of dims of a thread
  constexpr int kPPitch = kRows + 4;
  struct PagePlace {
    long long at;                                                  // bytes from the layer's pool
    unsigned slots;                                                // those that some row of the item sees
  };
  __shared__ PagePlace places[2][kWinKeys / kPageSize];            // of a tile's pages, the next tile's beside
  extern __shared__ __align__(16) float win_smem[];
  const int D = kMaxD == kWinAnyD ? a.D : kMaxD, pitch = D + 4, chunks = D / kPer;
  float* const qs = win_smem;                                      // [kRows][pitch]
  float* const ks = qs + kRows * pitch;                            // [kWinKeys][pitch]
  float* const vs = ks + kWinKeys * pitch;
  float* const ps = vs + kWinKeys * pitch;                         // [kWinKeys][kPPitch]
  const WindowReq& r = window_req(a, list.w, blockIdx.x);
  const WindowItem it = window_item<kWinKeys, true>(a, r, blockIdx.x, kRows);
  const int G = a.Hq / a.Hkv, packed = r.n * G;
  const int tid = threadIdx.x, tx = tid % kWinLanes, ty = tid / kWinLanes % kRowGroups, part = tid / (kWinLanes * kRowGroups);

  for (int i = tid; i < kRows * chunks; i += kWinThreads) {
    const int row = i / chunks, c = i - row * chunks, p = it.row0 + row;
    float f[kPer];
    uint4 v = make_uint4(0, 0, 0, 0);
    if (p < packed) {
      const WindowRow w(a, it.hk, p);
      v = *reinterpret_cast<const uint4*>(a.q + ((r.row + w.t) * a.q_stride + (long long)w.h * D) * kEsize + c * 16);
    }
    Tr::unpack(v, f);
#pragma unroll
    for (int e = 0; e < kPer; e += 4)
      *reinterpret_cast<float4*>(&qs[row * pitch + c * kPer + e]) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
  }
  WindowColumns col[kWinPer];
#pragma unroll
  for (int i = 0; i < kWinPer; ++i) {
    const int p = it.row0 + ty * kWinPer + i;
    col[i] = WindowColumns{0, 0, 0};
    if (p < packed) col[i] = window_columns(a, it.pages, r.len, r.pos + p / G);
  }

  float m_run[kWinPer], l_run[kWinPer];
  unsigned long long acc2[kWinPer / 2][2 * kPairs];                // output, two rows to a register pair
#pragma unroll
  for (int i = 0; i < kWinPer; ++i) {
    m_run[i] = -INFINITY;
    l_run[i] = 0.f;
#pragma unroll
    for (int d = 0; d < 2 * kPairs; ++d) acc2[i / 2][d] = 0ull;
  }
  // Where a tile's pages lie, for the tiles to be staged after the next barrier.
  auto look_up = [&](int tile, PagePlace* to) {
    if (tid >= kWinKeys / kPageSize) return;
    const int s = tile * (kWinKeys / kPageSize) + tid;
    PagePlace p = PagePlace{0, 0u};
    if (s < it.pages.count) {
      const WindowSlots sl = window_slots(it.pages, s);
#pragma unroll
      for (int i = 0; i < kPageSize; ++i) p.slots |= (sl.has(i) ? 1u : 0u) << i;
      p.at = window_page(a, r, list.w, it.pages, s) * a.page_stride + (long long)it.hk * a.page_bytes;
    }
    to[tid] = p;
  };
  // One tile of keys or values; slots that no row of the item sees become zero.  fp32 is copied asynchronously.
  const int key_first = tid / chunks, c_first = tid - key_first * chunks, key_step = kWinThreads / chunks, c_step = kWinThreads - key_step * chunks;
  auto stage = [&](float* dst, const char* pool, const PagePlace* from) {
#pragma unroll 4
    for (int key = key_first, c = c_first; key < kWinKeys;) {
      const PagePlace& p = from[key / kPageSize];
      const bool has = (p.slots >> (key % kPageSize)) & 1u;
      const char* const src = has ? pool + p.at + page_chunk_offset(a.swizzled != 0, key % kPageSize, c, chunks * 16) : pool;
      float* const to = &dst[key * pitch + c * kPer];
      if constexpr (kEsize == 4) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                     ::"r"((unsigned)__cvta_generic_to_shared(to)), "l"(src), "r"(has ? 16u : 0u) : "memory");
      } else {
        float f[kPer];
        Tr::unpack(has ? *reinterpret_cast<const uint4*>(src) : make_uint4(0, 0, 0, 0), f);
#pragma unroll
        for (int e = 0; e < kPer; e += 4) *reinterpret_cast<float4*>(to + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
      }
      key += key_step;
      c += c_step;
      if (c >= chunks) {
        c -= chunks;
        ++key;
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto landed = [](bool all) {                                     // all copies of this thread, or all but the last
    if (all) asm volatile("cp.async.wait_group 0;" ::: "memory");
    else asm volatile("cp.async.wait_group 1;" ::: "memory");
  };

  const float sl2 = a.scale * 1.4426950408889634f;                 // scores are handled in the log2 domain
  const int num_tiles = it.tile_end - it.tile_begin;
  if (num_tiles > 0) {
    look_up(it.start, places[0]);
    __syncthreads();
    stage(ks, a.pool_k, places[0]);
  }
  for (int j = 0; j < num_tiles; ++j) {
    const int tile = window_tile(it.start, it.tile_begin, it.tile_end, j);
    landed(true);                                                  // the keys
    __syncthreads();                                               // ... and the last tile's values have been read
    stage(vs, a.pool_v, places[j & 1]);
    if (j + 1 < num_tiles) look_up(window_tile(it.start, it.tile_begin, it.tile_end, j + 1), places[(j + 1) & 1]);
    unsigned long long s2[kWinPer][kMine];                         // sums over even and odd dims
#pragma unroll
    for (int i = 0; i < kWinPer; ++i)
#pragma unroll
      for (int k = 0; k < kMine; ++k) s2[i][k] = 0ull;
    for (int d = 0; d < D; d += 4) {
      ulonglong2 qv[kWinPer], kv[kMine];
#pragma unroll
      for (int i = 0; i < kWinPer; ++i) qv[i] = *reinterpret_cast<const ulonglong2*>(&qs[(ty * kWinPer + i) * pitch + d]);
#pragma unroll
      for (int k = 0; k < kMine; ++k)
        kv[k] = *reinterpret_cast<const ulonglong2*>(&ks[(part * kPartKeys + tx + k * kWinLanes) * pitch + d]);
#pragma unroll
      for (int i = 0; i < kWinPer; ++i)
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
          asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(s2[i][k]) : "l"(qv[i].x), "l"(kv[k].x));
          asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(s2[i][k]) : "l"(qv[i].y), "l"(kv[k].y));
        }
    }
    __syncthreads();                                               // the keys have been read
    if (j + 1 < num_tiles) stage(ks, a.pool_k, places[(j + 1) & 1]);
    float s[kWinPer][kMine];
    const int c0 = tile * kWinKeys + part * kPartKeys;             // the group's first column
    bool whole = true;                                             // the rows see the group's keys in full
#pragma unroll
    for (int i = 0; i < kWinPer; ++i) {
      whole = whole && col[i].begin <= c0 && col[i].end >= c0 + kPartKeys;
#pragma unroll
      for (int k = 0; k < kMine; ++k)
        s[i][k] = (__uint_as_float((unsigned)s2[i][k]) + __uint_as_float((unsigned)(s2[i][k] >> 32))) * sl2;
    }
    if (!whole) {
#pragma unroll
      for (int i = 0; i < kWinPer; ++i)
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
          const int c = c0 + tx + k * kWinLanes;
          if (!((c >= col[i].begin && c < col[i].end) || c < col[i].sink)) s[i][k] = -INFINITY;
        }
    }
    float alpha[kWinPer];
#pragma unroll
    for (int i = 0; i < kWinPer; ++i) {
      float mx = s[i][0];
#pragma unroll
      for (int k = 1; k < kMine; ++k) mx = fmaxf(mx, s[i][k]);
      const float m_new = fmaxf(m_run[i], lanes16_max(mx));
      const float m_use = m_new == -INFINITY ? 0.f : m_new;        // nothing seen so far: every weight is 0
      alpha[i] = win_exp2(m_run[i] - m_use);
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < kMine; ++k) {
        s[i][k] = win_exp2(s[i][k] - m_use);
        sum += s[i][k];
      }
      l_run[i] = l_run[i] * alpha[i] + sum;                        // of this thread's keys; added up at the end
      m_run[i] = m_new;
    }
#pragma unroll
    for (int i = 0; i < kWinPer / 2; ++i) {
      const unsigned long long both = win_pack(alpha[2 * i], alpha[2 * i + 1]);
#pragma unroll
      for (int d = 0; d < 2 * kPairs; ++d) asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(acc2[i][d]) : "l"(both));
    }
#pragma unroll
    for (int k = 0; k < kMine; ++k)
#pragma unroll
      for (int i = 0; i < kWinPer; i += 4)
        *reinterpret_cast<float4*>(&ps[(part * kPartKeys + tx + k * kWinLanes) * kPPitch + ty * kWinPer + i]) =
            make_float4(s[i][k], s[i + 1][k], s[i + 2][k], s[i + 3][k]);
    landed(j + 1 == num_tiles);                                            // the values
    __syncthreads();
#pragma unroll 4
    for (int key = part * kPartKeys; key < (part + 1) * kPartKeys; ++key) {
      unsigned long long pr[kWinPer / 2];                          // the weights of two rows
#pragma unroll
      for (int i = 0; i < kWinPer / 2; i += 2) {
        const ulonglong2 p = *reinterpret_cast<const ulonglong2*>(&ps[key * kPPitch + ty * kWinPer + 2 * i]);
        pr[i] = p.x;
        pr[i + 1] = p.y;
      }
#pragma unroll
      for (int g = 0; g < kPairs; ++g) {
        const int d = (g * kWinLanes + tx) * 2;
        if (kMaxD != kWinAnyD || d < D) {
          const float2 v = *reinterpret_cast<const float2*>(&vs[key * pitch + d]);
          const unsigned long long vx = win_pack(v.x, v.x), vy = win_pack(v.y, v.y);
#pragma unroll
          for (int i = 0; i < kWinPer / 2; ++i) {
            asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc2[i][2 * g]) : "l"(pr[i]), "l"(vx));
            asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc2[i][2 * g + 1]) : "l"(pr[i]), "l"(vy));
          }
        }
      }
    }
  }

  float acc[kWinPer][2 * kPairs];
#pragma unroll
  for (int i = 0; i < kWinPer; ++i)
#pragma unroll
    for (int d = 0; d < 2 * kPairs; ++d)
      acc[i][d] = __uint_as_float((unsigned)(i & 1 ? acc2[i / 2][d] >> 32 : acc2[i / 2][d]));
#pragma unroll
  for (int i = 0; i < kWinPer; ++i) l_run[i] = lanes16_sum(l_run[i]);
  if (kParts > 1) {
    // the groups' results: accumulators where the keys were, statistics where the weights were
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWinPer; ++i) {
      const int row = ty * kWinPer + i;
      if (tx == 0) {
        ps[part * kRows + row] = m_run[i];
        ps[(kParts + part) * kRows + row] = l_run[i];
      }
#pragma unroll
      for (int g = 0; g < kPairs; ++g) {
        const int d = (g * kWinLanes + tx) * 2;
        if (kMaxD != kWinAnyD || d < D) *reinterpret_cast<float2*>(&ks[(part * kRows + row) * pitch + d]) = make_float2(acc[i][2 * g], acc[i][2 * g + 1]);
      }
    }
    __syncthreads();
    if (part != 0) return;
#pragma unroll
    for (int i = 0; i < kWinPer; ++i) {
      const int row = ty * kWinPer + i;
      float m_all = m_run[i];
#pragma unroll
      for (int o = 1; o < kParts; ++o) m_all = fmaxf(m_all, ps[o * kRows + row]);
      const float m_use = m_all == -INFINITY ? 0.f : m_all;
      float l_all = 0.f;
#pragma unroll
      for (int g = 0; g < 2 * kPairs; ++g) acc[i][g] = 0.f;
#pragma unroll
      for (int o = 0; o < kParts; ++o) {
        const float w = win_exp2(ps[o * kRows + row] - m_use);
        l_all += w * ps[(kParts + o) * kRows + row];
#pragma unroll
        for (int g = 0; g < kPairs; ++g) {
          const int d = (g * kWinLanes + tx) * 2;
          if (kMaxD != kWinAnyD || d < D) {
            const float2 v = *reinterpret_cast<const float2*>(&ks[(o * kRows + row) * pitch + d]);
            acc[i][2 * g] += w * v.x;
            acc[i][2 * g + 1] += w * v.y;
          }
        }
      }
      m_run[i] = m_all;
      l_run[i] = l_all;
    }
  }
#pragma unroll
  for (int i = 0; i < kWinPer; ++i) {
    const int p = it.row0 + ty * kWinPer + i;
    if (p >= packed) break;
    const WindowRow w(a, it.hk, p);
    const float inv = l_run[i] == 0.f ? 0.f : 1.f / l_run[i];
    const float lse = l_run[i] == 0.f ? -INFINITY : m_run[i] * 0.6931471805599453f + logf(l_run[i]);
    if (r.splits > 1) {
      const long long at = window_part(a, r, it.split, w);
      if (tx == 0) a.part_lse[at] = lse;
#pragma unroll
      for (int g = 0; g < kPairs; ++g) {
        const int d = (g * kWinLanes + tx) * 2;
        if (kMaxD != kWinAnyD || d < D) *reinterpret_cast<float2*>(a.part_o + at * D + d) = make_float2(acc[i][2 * g] * inv, acc[i][2 * g + 1] * inv);
      }
    } else {
      const long long row = r.row + w.t;
      char* const o = a.out + (row * a.out_stride + (long long)w.h * D) * kEsize;
      if (tx == 0 && a.lse) a.lse[row * a.Hq + w.h] = lse;
#pragma unroll
      for (int g = 0; g < kPairs; ++g) {
        const int d = (g * kWinLanes + tx) * 2;
        if (kMaxD != kWinAnyD || d < D) {
          Tr::store(o + d * kEsize, acc[i][2 * g] * inv);
          Tr::store(o + (d + 1) * kEsize, acc[i][2 * g + 1] * inv);
        }
      }
    }
  }
}

// Page lists that do not fit the parameters stand in the workspace, written by launches of this kernel.
template <int kWords>
__global__ void stage_pages_kernel(int* __restrict__ dst, int count, const __grid_constant__ ParamList<kWords> list) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < count) dst[i] = list.w[i];
}

// ---------------------------------------------------------------------------------------------
// Joins the ranges of a row-head: with l_s the log-sum-exp of range s and o_s its normalised result,
//   lse = log sum_s exp(l_s),  o = sum_s exp(l_s - lse) o_s,
// the ranges in ascending order.  kWarps = 1: a warp per row-head; kWarps = 8: the eight warps of a block share
// one, warp w taking ranges w, w + 8, ..; for few row-heads of many ranges.  Placed on the SMs while the kernel before
// it still runs, and waits for its end.  Latency is what it costs: 4 to 6 us, 28 row-heads of 64 ranges as 7000 of two.
// ---------------------------------------------------------------------------------------------
constexpr int kJoinWarps = 8;
constexpr int kMaxWindowSplits = 64;

template <typename T, int kWarps, int kWords>
__global__ void __launch_bounds__(kJoinWarps * 32)
window_join_kernel(const __grid_constant__ WindowArgs a, int row_heads, const int* status,
                   const __grid_constant__ ParamList<kWords> list) {
  __shared__ float red[kWarps == 1 ? 1 : kJoinWarps][kSimtMaxD];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rh = kWarps == 1 ? blockIdx.x * kJoinWarps + warp : blockIdx.x;
  if (rh >= row_heads) return;
  // a split request (those that are not split start where the next one does)
  const WindowReq& r = last_start<WindowReq>(list.w, a.num_reqs, row_heads, rh, [](const WindowReq& q) { return q.row_heads_before; });
  const int at = rh - r.row_heads_before, t = at / a.Hq, h = at - t * a.Hq;
  const long long stride = (long long)r.n * a.Hq, p0 = r.part_off + at;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // everything is requested before anything is used: the first ranges' rows, the status, the log-sum-exps
  constexpr int kStep = kWarps == 1 ? 1 : kJoinWarps;
  const int s_first = kWarps == 1 ? 0 : warp;
  float4 v[8];
  auto load = [&](int s0, int d) {
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (d < a.D && s0 + u * kStep < r.splits)
        v[u] = *reinterpret_cast<const float4*>(a.part_o + (p0 + (s0 + u * kStep) * stride) * a.D + d);
  };
  load(s_first, lane * 4);
  const int state = status ? *status : kDevOk;
  const float l0 = lane < r.splits ? a.part_lse[p0 + lane * stride] : -INFINITY;
  const float l1 = lane + 32 < r.splits ? a.part_lse[p0 + (lane + 32) * stride] : -INFINITY;
  if (state != kDevOk) return;                                     // some ranges were not computed
  const float mx = warp_max(fmaxf(l0, l1));
  const bool any = mx > -INFINITY || __any_sync(0xffffffffu, l0 != l0 || l1 != l1);      // a NaN spreads
  const float w0 = any ? expf(l0 - mx) : 0.f, w1 = any ? expf(l1 - mx) : 0.f;
  const float total = warp_sum(w0 + w1), inv = any ? 1.f / total : 0.f;
  const long long row = r.row + t;
  for (int d0 = 0; d0 < a.D; d0 += 128) {
    const int d = d0 + lane * 4;
    const bool mine = d < a.D;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = s_first; s0 < r.splits; s0 += 8 * kStep) {
      if (d0 > 0 || s0 > s_first) load(s0, d);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int s = s0 + u * kStep;
        const float w = __shfl_sync(0xffffffffu, s < 32 ? w0 : w1, s & 31);
        if (mine && s < r.splits) {
          acc.x = fmaf(w, v[u].x, acc.x);
          acc.y = fmaf(w, v[u].y, acc.y);
          acc.z = fmaf(w, v[u].z, acc.z);
          acc.w = fmaf(w, v[u].w, acc.w);
        }
      }
    }
    if (!mine) continue;
    if (kWarps == 1) {
      char* const o = a.out + (row * a.out_stride + (long long)h * a.D + d) * (int)sizeof(T);
      const float f[4] = {acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
#pragma unroll
      for (int e = 0; e < 4; ++e) ElemTraits<T>::store(o + e * (int)sizeof(T), f[e]);
    } else {
      *reinterpret_cast<float4*>(&red[warp][d]) = acc;
    }
  }
  if (kWarps > 1) {
    __syncthreads();
    for (int d = threadIdx.x; d < a.D; d += kJoinWarps * 32) {
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kJoinWarps; ++w) sum += red[w][d];
      ElemTraits<T>::store(a.out + (row * a.out_stride + (long long)h * a.D + d) * (int)sizeof(T), sum * inv);
    }
  }
  if (lane == 0 && warp == (kWarps == 1 ? warp : 0) && a.lse) a.lse[row * a.Hq + h] = any ? mx + logf(total) : -INFINITY;
}

}  // namespace bicache

// Tokens into and out of the pages of stored prefixes: keys and values of a ragged batch written at given tokens of
// their prefixes, the keys (and the queries of the same rows) rotated to their positions on the way, and the
// way back.
//
// Bound by memory: a chunk of 16 bytes is read once and written once.  The batch (runs of rows, one per request, and the
// pages they reach) travels as launch parameters, so nothing is uploaded and one launch does a layer of the whole batch,
// queries included.  Row space: the tokens of all runs one after the other; a block takes kRows of them, its
// first threads look up where each lies, and then a thread does one unit (the chunks of a head that pair up) for
// all the block's rows, as in rope_chunks_kernel.  23,000 rows of 32 heads, queries, keys and values, three position axes: 176
// us (1.13 GB, 6.4 TB/s) and 115 us back (0.76 GB, 6.6 TB/s).  16 rows: 3 us each way, a launch and three loads in turn.
#pragma once
#include "evict.cuh"
#include "rope.cuh"
#include "window.cuh"

namespace bicache {

// A run of rows and the tokens of a prefix they become.  A run that reaches the prefix's last page also clears the
// slots behind the prefix's end: the attention kernels multiply them by weight 0 and need them finite.
struct TokenRun {
  long long row;                // first row in the tensors
  int start;                    // first token of the run in the row space
  int n;                        // rows; in the row space one entry for the cleared slots may follow them
  int token;                    // first token in the prefix
  int clear;                    // the first cleared slot, as a token of the prefix
  int page_word;                // page list from the page of `token` on
  int pad;
};
constexpr int kRunWords = sizeof(TokenRun) / 4;

struct TokenArgs {
  const char *q, *k, *v;        // q: nullptr if there are no queries
  char* q_out;
  char *pool_k, *pool_v;        // of the layer
  char *k_out, *v_out;          // the way back
  long long q_stride, q_out_stride, kv_stride;      // bytes between rows
  long long page_stride;        // bytes of a page of all heads
  int Hq, Hkv;
  int head_bytes, page_bytes, swizzled;
  int pairs;                    // rotated pairs of a head (0: none)
  int q_in_place;
  int num_runs, tokens;         // runs in the list, tokens of the row space
};

// Where a token of the row space lies.
struct TokenPlace {
  long long row;                // in the tensors; -1: the slots from `slot` on are cleared
  long long page;               // bytes from the layer's pool to its page
  long long at;                 // what stands for the row in rope_position: the row, or the token
  int slot;
};
__device__ __forceinline__ TokenPlace token_place(const TokenArgs& g, const int* list, bool by_token, int t) {
  const TokenRun& r = last_start<TokenRun>(list, g.num_runs, g.tokens, t, [](const TokenRun& x) { return x.start; });
  const int i = t - r.start;
  const int token = i < r.n ? r.token + i : r.clear;
  TokenPlace p;
  p.row = i < r.n ? r.row + i : -1;
  p.page = list[r.page_word + token / kPageSize - r.token / kPageSize] * g.page_stride;
  p.at = by_token ? (long long)token : p.row;
  p.slot = token % kPageSize;
  return p;
}

template <typename T, bool kInterleaved, int kRows, typename A, int kWords>
__global__ void __launch_bounds__(kRopeThreads)
append_chunks_kernel(const __grid_constant__ A a, const __grid_constant__ TokenArgs g,
                     const __grid_constant__ ParamList<kWords> list) {
  using Tr = ElemTraits<T>;
  constexpr int kPer = Tr::kPerChunk;
  constexpr int kPairs = kInterleaved ? kPer / 2 : kPer;           // pairs of a unit
  __shared__ float4 cs[kRows][kRopeMaxPairs / 2];
  __shared__ TokenPlace place[kRows];
  const int t0 = blockIdx.x * kRows, rows = min(kRows, g.tokens - t0);
  if ((int)threadIdx.x < rows) place[threadIdx.x] = token_place(g, list.w, a.positions == nullptr, t0 + threadIdx.x);
  const int chunks = g.head_bytes / 16;
  const int turned = g.pairs / kPairs;                             // units of a head that rotate
  const int first_rest = 2 * g.pairs / kPer;                       // first chunk beyond the rotated dims
  const int rest = chunks - first_rest;
  const int per_q = g.q ? turned + (g.q_in_place ? 0 : rest) : 0, per_k = turned + rest;
  const int q_units = per_q * g.Hq, k_units = per_k * g.Hkv, units = q_units + k_units + chunks * g.Hkv;
  __syncthreads();

  // what a unit is: tensor 0 queries, 1 keys, 2 values
  auto section = [&](int u, int& which, int& h, int& c) {
    which = u < q_units ? 0 : u < q_units + k_units ? 1 : 2;
    const int v = which == 0 ? u : which == 1 ? u - q_units : u - q_units - k_units;
    const int per = which == 0 ? per_q : which == 1 ? per_k : chunks;
    h = v / per;
    c = v - h * per;
  };
  uint4 x[kRows], y[kRows];
  int which = 0, h = 0, c = 0;
  auto load = [&](int u) {
    section(u, which, h, c);
    const bool turns = which != 2 && c < turned;
    const int chunk = which == 2 || turns ? c : first_rest + c - turned;
    const char* const base = (which == 0 ? g.q : which == 1 ? g.k : g.v) + (long long)h * g.head_bytes + chunk * 16;
    const long long stride = which == 0 ? g.q_stride : g.kv_stride;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      x[i] = y[i] = make_uint4(0, 0, 0, 0);
      if (i < rows && place[i].row >= 0) {
        const char* const p = base + place[i].row * stride;
        x[i] = *reinterpret_cast<const uint4*>(p);
        if (!kInterleaved && turns) y[i] = *reinterpret_cast<const uint4*>(p + turned * 16);
      }
    }
  };
  int u = threadIdx.x;
  if (u < units) load(u);
  for (int i = threadIdx.x; i < rows * g.pairs; i += blockDim.x) {
    const int row = i / g.pairs, pair = i - row * g.pairs;
    if (place[row].row < 0) continue;
    const int unit = pair / kPairs, e = pair - unit * kPairs;
    reinterpret_cast<float2*>(&cs[row][(e >> 1) * turned + unit])[e & 1] =
        rope_cos_sin(a, rope_position(a, place[row].at, pair), a.turn[pair]);
  }
  __syncthreads();
  for (; u < units; u += blockDim.x) {
    if (u >= (int)blockDim.x) load(u);
    const bool turns = which != 2 && c < turned;
    const int chunk = which == 2 || turns ? c : first_rest + c - turned;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (i >= rows) break;
      if (which == 0 && place[i].row < 0) continue;
      if (turns) {
        float p[kPer], q[kPer];
        Tr::unpack(x[i], p);
        if (!kInterleaved) Tr::unpack(y[i], q);
        const bool data = place[i].row >= 0;                       // else zeros, and no cosines
#pragma unroll
        for (int e = 0; e < kPairs; e += 2) {
          const float4 w = data ? cs[i][(e >> 1) * turned + c] : make_float4(0.f, 0.f, 0.f, 0.f);
          if (kInterleaved) {
            const float p0 = p[2 * e], p1 = p[2 * e + 1], p2 = p[2 * e + 2], p3 = p[2 * e + 3];
            p[2 * e] = p0 * w.x - p1 * w.y;
            p[2 * e + 1] = p1 * w.x + p0 * w.y;
            p[2 * e + 2] = p2 * w.z - p3 * w.w;
            p[2 * e + 3] = p3 * w.z + p2 * w.w;
          } else {
            const float p0 = p[e], p1 = p[e + 1];
            p[e] = p0 * w.x - q[e] * w.y;
            q[e] = q[e] * w.x + p0 * w.y;
            p[e + 1] = p1 * w.z - q[e + 1] * w.w;
            q[e + 1] = q[e + 1] * w.z + p1 * w.w;
          }
        }
        x[i] = rope_pack<T>(p);
        if (!kInterleaved) y[i] = rope_pack<T>(q);
      }
      if (which == 0) {
        char* const to = g.q_out + place[i].row * g.q_out_stride + (long long)h * g.head_bytes + chunk * 16;
        *reinterpret_cast<uint4*>(to) = x[i];
        if (!kInterleaved && turns) *reinterpret_cast<uint4*>(to + turned * 16) = y[i];
      } else {
        char* const to = (which == 1 ? g.pool_k : g.pool_v) + place[i].page + (long long)h * g.page_bytes;
        const bool swz = g.swizzled != 0;
        for (int s = place[i].slot, end = place[i].row >= 0 ? s + 1 : kPageSize; s < end; ++s) {
          *reinterpret_cast<uint4*>(to + page_chunk_offset(swz, s, chunk, g.head_bytes)) = x[i];
          if (!kInterleaved && turns)
            *reinterpret_cast<uint4*>(to + page_chunk_offset(swz, s, chunk + turned, g.head_bytes)) = y[i];
        }
      }
    }
  }
}

// Any rotated width, chunk by chunk as in rope_any_kernel; kRows tokens at a time, so that a batch fills the block also
// where there are few heads.  100,000 rows of 4 KV heads, 108 of 128 dims turned, and back: 336 us, where one thread per pair
// took 720 and one token at a time 588.  What keeps it from the bandwidth (125 us) is open: the other halves from two aligned
// chunks, cosines laid out without bank conflicts and places computed once for loads and stores took 341, 363 and 363 us.
template <typename T, typename A, int kRows, int kWords>
__global__ void __launch_bounds__(kRopeThreads)
append_any_kernel(const __grid_constant__ A a, const __grid_constant__ TokenArgs g, int interleaved,
                  const __grid_constant__ ParamList<kWords> list) {
  __shared__ float2 cs[kRows][kRopeMaxPairs];
  __shared__ TokenPlace place[kRows];
  const int chunks = g.head_bytes / 16, batch = kRopeHeld * kRopeThreads / chunks * chunks;     // units of whole heads
  const int q_heads = g.q ? g.Hq : 0, per_token = chunks * (q_heads + 2 * g.Hkv);
  const bool swz = g.swizzled != 0;
  const int t0 = blockIdx.x * kRows, rows = min(kRows, g.tokens - t0), units = rows * per_token;
  if ((int)threadIdx.x < rows) place[threadIdx.x] = token_place(g, list.w, a.positions == nullptr, t0 + threadIdx.x);
  __syncthreads();
  for (int i = threadIdx.x; i < rows * g.pairs; i += kRopeThreads) {
    const int row = i / g.pairs, pair = i - row * g.pairs;
    if (place[row].row >= 0) cs[row][pair] = rope_cos_sin(a, rope_position(a, place[row].at, pair), a.turn[pair]);
  }
  __syncthreads();
  for (int u0 = 0; u0 < units; u0 += batch) {
    uint4 x[kRopeHeld];
    const int end = min(units, u0 + batch);
    auto each = [&](auto&& f) {                                    // f(held, token, 0 query 1 key 2 value, head, chunk)
#pragma unroll
      for (int i = 0; i < kRopeHeld; ++i) {
        const int u = u0 + (int)threadIdx.x + i * kRopeThreads;
        if (u >= end) continue;
        const int row = kRows == 1 ? 0 : u / per_token, v = u - row * per_token;
        const int h = v / chunks, which = h < q_heads ? 0 : h < q_heads + g.Hkv ? 1 : 2;
        f(i, row, which, h - (which == 0 ? 0 : which == 1 ? q_heads : q_heads + g.Hkv), v - h * chunks);
      }
    };
    each([&](int i, int row, int which, int h, int c) {
      const TokenPlace& pl = place[row];
      x[i] = make_uint4(0, 0, 0, 0);
      if (pl.row < 0) return;
      const char* const head = (which == 0 ? g.q + pl.row * g.q_stride : (which == 1 ? g.k : g.v) + pl.row * g.kv_stride) +
                               (long long)h * g.head_bytes;
      x[i] = which == 2 ? *reinterpret_cast<const uint4*>(head + c * 16)
                        : rope_any_chunk<T>(head, c, g.pairs, interleaved != 0, cs[row]);
    });
    __syncthreads();                                               // queries may be rotated in place
    each([&](int i, int row, int which, int h, int c) {
      const TokenPlace& pl = place[row];
      if (which == 0) {
        if (pl.row >= 0) *reinterpret_cast<uint4*>(g.q_out + pl.row * g.q_out_stride + (long long)h * g.head_bytes + c * 16) = x[i];
      } else {
        char* const to = (which == 1 ? g.pool_k : g.pool_v) + pl.page + (long long)h * g.page_bytes;
        for (int s = pl.slot, last = pl.row >= 0 ? s + 1 : kPageSize; s < last; ++s)
          *reinterpret_cast<uint4*>(to + page_chunk_offset(swz, s, c, g.head_bytes)) = x[i];
      }
    });
  }
}

// The way back: pages to rows of k_out and v_out, bit-exact.
template <int kRows, int kWords>
__global__ void __launch_bounds__(kRopeThreads)
read_tokens_kernel(const __grid_constant__ TokenArgs g, const __grid_constant__ ParamList<kWords> list) {
  __shared__ TokenPlace place[kRows];
  const int t0 = blockIdx.x * kRows, rows = min(kRows, g.tokens - t0);
  if ((int)threadIdx.x < rows) place[threadIdx.x] = token_place(g, list.w, false, t0 + threadIdx.x);
  __syncthreads();
  const int chunks = g.head_bytes / 16, units = chunks * g.Hkv;
  for (int u = threadIdx.x; u < units; u += blockDim.x) {
    const int h = u / chunks, c = u - h * chunks;
    uint4 k[kRows], v[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i)
      if (i < rows) {
        const long long from = place[i].page + (long long)h * g.page_bytes +
                               page_chunk_offset(g.swizzled != 0, place[i].slot, c, g.head_bytes);
        k[i] = *reinterpret_cast<const uint4*>(g.pool_k + from);
        v[i] = *reinterpret_cast<const uint4*>(g.pool_v + from);
      }
#pragma unroll
    for (int i = 0; i < kRows; ++i)
      if (i < rows) {
        const long long to = place[i].row * g.kv_stride + (long long)h * g.head_bytes + c * 16;
        *reinterpret_cast<uint4*>(g.k_out + to) = k[i];
        *reinterpret_cast<uint4*>(g.v_out + to) = v[i];
      }
  }
}

// Four rows to a block once that still gives every SM eight blocks, else one.
inline bool token_rows_by_four(int tokens, int sm_count) { return tokens >= 32LL * sm_count; }
inline int token_threads(int units) {
  return units >= kRopeThreads ? kRopeThreads : (units < 64 ? 64 : (units + 31) / 32 * 32);
}

template <typename T, typename A, int kWords>
cudaError_t launch_append(const A& a, const TokenArgs& g, bool interleaved, const ParamList<kWords>& list, int sm_count,
                          cudaStream_t stream) {
  constexpr int kPer = ElemTraits<T>::kPerChunk;
  if ((interleaved ? 2 * g.pairs : g.pairs) % kPer == 0) {
    const int chunks = g.head_bytes / 16, turned = g.pairs / (interleaved ? kPer / 2 : kPer);
    const int per_head = turned + chunks - 2 * g.pairs / kPer;
    const int threads = token_threads((g.q ? per_head * g.Hq : 0) + (per_head + chunks) * g.Hkv);
    const bool four = token_rows_by_four(g.tokens, sm_count);
    const unsigned blocks = four ? (unsigned)((g.tokens + 3LL) / 4) : (unsigned)g.tokens;
    if (interleaved) {
      if (four) append_chunks_kernel<T, true, 4><<<blocks, threads, 0, stream>>>(a, g, list);
      else append_chunks_kernel<T, true, 1><<<blocks, threads, 0, stream>>>(a, g, list);
    } else {
      if (four) append_chunks_kernel<T, false, 4><<<blocks, threads, 0, stream>>>(a, g, list);
      else append_chunks_kernel<T, false, 1><<<blocks, threads, 0, stream>>>(a, g, list);
    }
  } else {
    // as many tokens as make a batch, once that still gives every SM eight blocks
    const int units = g.head_bytes / 16 * ((g.q ? g.Hq : 0) + 2 * g.Hkv);
    if (units <= kRopeHeld * kRopeThreads / 4 && g.tokens >= 64LL * sm_count)
      append_any_kernel<T, A, 8><<<(unsigned)((g.tokens + 7LL) / 8), kRopeThreads, 0, stream>>>(a, g, interleaved ? 1 : 0, list);
    else
      append_any_kernel<T, A, 1><<<(unsigned)g.tokens, kRopeThreads, 0, stream>>>(a, g, interleaved ? 1 : 0, list);
  }
  return cudaGetLastError();
}

template <int kWords>
cudaError_t launch_read_tokens(const TokenArgs& g, const ParamList<kWords>& list, int sm_count, cudaStream_t stream) {
  const int threads = token_threads(g.head_bytes / 16 * g.Hkv);
  if (token_rows_by_four(g.tokens, sm_count))
    read_tokens_kernel<4><<<(unsigned)((g.tokens + 3LL) / 4), threads, 0, stream>>>(g, list);
  else
    read_tokens_kernel<1><<<(unsigned)g.tokens, threads, 0, stream>>>(g, list);
  return cudaGetLastError();
}

}  // namespace bicache

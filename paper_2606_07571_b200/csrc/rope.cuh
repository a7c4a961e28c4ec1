// Rotary positions: rows of queries and keys rotated in place or into other tensors, and the table of
// cosines and sines that the key projection into the store takes.
//
// Pair i of a row at position p turns by the angle p * f_i:
//   (a, b) -> s (a cos - b sin, b cos + a sin),   s = the attention scale (1 unless frequencies are scaled
// by a rule that has one).  The angle is kept in whole and part TURNS: f_i / (2 pi) is a 64-bit fixed-point
// fraction F_i, and p * F_i modulo 2^64 is the part of a turn, exact for every 32-bit p.  A product
// p * f_i in fp32 would be off by p 2^-24 radians (0.06 at p = 10^6), in fp64 it would cost the fp64 pipe and a
// long argument reduction; here it is one 64-bit integer multiplication.  The part of a turn is reduced to
// an eighth before it becomes fp32, so cos and sin are off by no more than about 1.2e-7.
#pragma once
#include <cuda_bf16.h>
#include "common.cuh"
#include "simt_kernels.cuh"

namespace bicache {

constexpr int kRopeMaxPairs = 128;         // head dims up to 256
constexpr int kRopeThreads = 256;

struct RopeAngles {
  unsigned long long turn[kRopeMaxPairs];  // fixed-point turns per position (2^64 = one turn)
  const int* positions;                    // device, one per row, or nullptr: position0 + row
  long long position0;
  float scale;                             // factor of cos and sin
  int pairs;
  int negate;                              // rotate backwards
};

__device__ __forceinline__ float2 rope_cos_sin(const RopeAngles& a, long long pos, unsigned long long turn) {
  // an eighth of a turn is added, so the two top bits count quarter turns and the rest, taken back to
  // [-1/8, 1/8) turn, is the argument
  const unsigned long long t = (unsigned long long)pos * turn + (1ull << 61);
  const int quarter = (int)(t >> 62);
  const long long rest = (long long)(t & ((1ull << 62) - 1)) - (1ll << 61);
  const float x = (float)(int)(rest >> 30) * 1.1641532182693481e-10f;               // half turns: 2^-33 of the integer
  // sin(pi x) / x and cos(pi x) for |x| <= 1/4 as polynomials in x^2 with the smallest largest error (by linear
  // programming: 3.3e-9 relative, 5.7e-11); 1.1e-7 in all with the fp32 roundings and that of x
  const float u = x * x;
  const float s = x * fmaf(u, fmaf(u, fmaf(u, -0.5890117345f, 2.5497609895f), -5.1677076800f), 3.1415926434f);
  const float c = fmaf(u, fmaf(u, fmaf(u, fmaf(u, 0.2313983676f, -1.3350547761f), 4.0587077773f), -4.9348021722f), 1.f);
  const float c1 = (quarter & 1) ? s : c, s1 = (quarter & 1) ? c : s;
  const float cs = (quarter == 1 || quarter == 2) ? -c1 : c1;
  const float sn = (quarter & 2) ? -s1 : s1;
  return make_float2(cs * a.scale, (a.negate ? -sn : sn) * a.scale);
}

// ---------------------------------------------------------------------------------------------
// The table [rows][pairs][2] of bicache_rope_table.  A thread keeps its pair and walks down the rows, four
// positions read ahead.  The lanes of a warp read their pairs' frequencies from as many parameter addresses, one
// after the other: few blocks, so that this is done seldom.  16,384 positions of 64 pairs (8.4 MB) take 5.5 us.
// ---------------------------------------------------------------------------------------------
constexpr int kTableRows = 4;              // rows a thread has in hand

__global__ void __launch_bounds__(kRopeThreads)
rope_table_kernel(const __grid_constant__ RopeAngles a, long long rows, float2* __restrict__ table) {
  const int per_block = kRopeThreads / a.pairs;                  // rows a block handles at a time
  const int r = (int)threadIdx.x / a.pairs, pair = (int)threadIdx.x - r * a.pairs;
  if (r >= per_block) return;
  const unsigned long long turn = a.turn[pair];
  const long long step = (long long)gridDim.x * per_block;
  for (long long row = (long long)blockIdx.x * per_block + r; row < rows; row += kTableRows * step) {
    long long pos[kTableRows];
#pragma unroll
    for (int i = 0; i < kTableRows; ++i) {
      const long long at = row + i * step;
      pos[i] = a.position0 + at;
      if (a.positions && at < rows) pos[i] = a.positions[at];
    }
#pragma unroll
    for (int i = 0; i < kTableRows; ++i) {
      const long long at = row + i * step;
      if (at < rows) table[at * a.pairs + pair] = rope_cos_sin(a, pos[i], turn);
    }
  }
}

struct RopeTensor {
  const char* in;
  char* out;
  long long in_stride, out_stride;         // bytes between rows
  int heads;                               // 0: no such tensor
};
struct RopeRows {
  RopeTensor t[2];                         // queries, keys
  long long rows;
  int head_bytes;                          // D * element size
  int in_place;                            // nothing beyond the rotated dims has to be copied
};

template <typename T> __device__ __forceinline__ uint4 rope_pack(const float* f);
template <> __device__ __forceinline__ uint4 rope_pack<float>(const float* f) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <> __device__ __forceinline__ uint4 rope_pack<__nv_bfloat16>(const float* f) {
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);      // the one rounding
    w[i] = *reinterpret_cast<const unsigned*>(&v);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// ---------------------------------------------------------------------------------------------
// Rows in 16-byte chunks, for rotated widths that fill whole chunks (half-split pairs: rot_dim / 2 a multiple of
// the chunk, interleaved pairs: rot_dim).  Bound by memory: every chunk is read and written once; 32,768 rows of 28 + 4
// heads of 128 dims (537 MB) take 80 us, a plain copy's bandwidth; 16 rows take 2.2 us, a launch.
// A block takes kRows rows and computes their cosines and sines once for all heads.  A thread owns a unit - the
// two chunks of one head whose dims pair up (half-split), one chunk (interleaved), or one chunk beyond the
// rotated dims, which is copied - and does it for all the block's rows, so the index arithmetic is paid
// once and kRows x 2 chunks are in flight; the first unit's loads are issued before the cosines and sines.
// These lie in shared memory chunk by chunk, two pairs to 16 bytes, the units of a head side by side:
// the lanes of a quarter warp read different banks.
// ---------------------------------------------------------------------------------------------
template <typename T, bool kInterleaved, int kRows>
__global__ void __launch_bounds__(kRopeThreads)
rope_chunks_kernel(const __grid_constant__ RopeAngles a, const __grid_constant__ RopeRows r) {
  using Tr = ElemTraits<T>;
  constexpr int kPer = Tr::kPerChunk;
  constexpr int kPairs = kInterleaved ? kPer / 2 : kPer;           // pairs of a unit
  __shared__ float4 cs[kRows][kRopeMaxPairs / 2];
  const int turned = a.pairs / kPairs;                             // units of a head that rotate
  const int first_rest = 2 * a.pairs / kPer;                       // first chunk beyond the rotated dims
  const int rest = r.in_place ? 0 : r.head_bytes / 16 - first_rest;
  const int per_head = turned + rest, units = per_head * (r.t[0].heads + r.t[1].heads);
  const long long row0 = (long long)blockIdx.x * kRows;
  const int rows = (int)min((long long)kRows, r.rows - row0);

  uint4 x[kRows], y[kRows];
  const char* in = nullptr;
  char* out = nullptr;
  long long in_stride = 0, out_stride = 0;
  int c = 0;                                                       // unit of the head
  auto load = [&](int u) {
    int h = u / per_head;
    c = u - h * per_head;
    const int which = h >= r.t[0].heads ? 1 : 0;
    const RopeTensor& t = r.t[which];
    h -= which ? r.t[0].heads : 0;
    const int chunk = c < turned ? c : first_rest + c - turned;
    const long long off = (long long)h * r.head_bytes + chunk * 16;
    in_stride = t.in_stride;
    out_stride = t.out_stride;
    in = t.in + row0 * in_stride + off;
    out = t.out + row0 * out_stride + off;
#pragma unroll
    for (int i = 0; i < kRows; ++i)
      if (i < rows) {
        x[i] = *reinterpret_cast<const uint4*>(in + i * in_stride);
        if (!kInterleaved && c < turned) y[i] = *reinterpret_cast<const uint4*>(in + i * in_stride + turned * 16);
      }
  };
  int u = threadIdx.x;
  if (u < units) load(u);
  for (int i = threadIdx.x; i < rows * a.pairs; i += blockDim.x) {
    const int row = i / a.pairs, pair = i - row * a.pairs;
    const long long pos = a.positions ? (long long)a.positions[row0 + row] : a.position0 + row0 + row;
    const int unit = pair / kPairs, e = pair - unit * kPairs;
    reinterpret_cast<float2*>(&cs[row][(e >> 1) * turned + unit])[e & 1] = rope_cos_sin(a, pos, a.turn[pair]);
  }
  __syncthreads();
  for (; u < units; u += blockDim.x) {
    if (u >= (int)blockDim.x) load(u);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (i >= rows) break;
      if (c < turned) {
        float p[kPer], q[kPer];
        Tr::unpack(x[i], p);
        if (!kInterleaved) Tr::unpack(y[i], q);
#pragma unroll
        for (int e = 0; e < kPairs; e += 2) {
          const float4 w = cs[i][(e >> 1) * turned + c];
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
        if (!kInterleaved) *reinterpret_cast<uint4*>(out + i * out_stride + turned * 16) = rope_pack<T>(q);
      }
      *reinterpret_cast<uint4*>(out + i * out_stride) = x[i];
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Rows, any rotated width: one thread per pair (and per dim beyond the rotated ones), element by element.
// A block takes one row at a time.
// ---------------------------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(kRopeThreads)
rope_rows_kernel(const __grid_constant__ RopeAngles a, const __grid_constant__ RopeRows r, int interleaved) {
  using Tr = ElemTraits<T>;
  constexpr int kEsize = (int)sizeof(T);
  __shared__ float2 cs[kRopeMaxPairs];
  const int dims = r.head_bytes / kEsize, rest = r.in_place ? 0 : dims - 2 * a.pairs;
  const int per_head = a.pairs + rest;
  const int units = per_head * (r.t[0].heads + r.t[1].heads);
  for (long long row = blockIdx.x; row < r.rows; row += gridDim.x) {
    const long long pos = a.positions ? (long long)a.positions[row] : a.position0 + row;
    __syncthreads();
    if ((int)threadIdx.x < a.pairs) cs[threadIdx.x] = rope_cos_sin(a, pos, a.turn[threadIdx.x]);
    __syncthreads();
    for (int u = threadIdx.x; u < units; u += kRopeThreads) {
      int h = u / per_head;
      const int i = u - h * per_head;
      const int which = h >= r.t[0].heads ? 1 : 0;
      const RopeTensor& t = r.t[which];
      h -= which ? r.t[0].heads : 0;
      const char* in = t.in + row * t.in_stride + (long long)h * r.head_bytes;
      char* out = t.out + row * t.out_stride + (long long)h * r.head_bytes;
      if (i < a.pairs) {
        const int d0 = (interleaved ? 2 * i : i) * kEsize, d1 = (interleaved ? 2 * i + 1 : i + a.pairs) * kEsize;
        const float x = Tr::load(in + d0), y = Tr::load(in + d1);
        const float2 w = cs[i];
        Tr::store(out + d0, x * w.x - y * w.y);
        Tr::store(out + d1, y * w.x + x * w.y);
      } else {
        const int d = (i + a.pairs) * kEsize;
        *reinterpret_cast<T*>(out + d) = *reinterpret_cast<const T*>(in + d);
      }
    }
  }
}

// Four rows to a block once that still gives every SM two blocks (it quarters the index arithmetic and the loads
// in flight are what hides the latency); one row to a block below that.
template <typename T>
cudaError_t launch_rope(const RopeAngles& a, const RopeRows& r, bool interleaved, int sm_count, cudaStream_t stream) {
  constexpr int kPer = ElemTraits<T>::kPerChunk;
  if ((interleaved ? 2 * a.pairs : a.pairs) % kPer == 0) {
    const int turned = a.pairs / (interleaved ? kPer / 2 : kPer);
    const int rest = r.in_place ? 0 : (r.head_bytes / 16 - 2 * a.pairs / kPer);
    const int units = (turned + rest) * (r.t[0].heads + r.t[1].heads);
    const int threads = units >= kRopeThreads ? kRopeThreads : (units < 64 ? 64 : (units + 31) / 32 * 32);
    const bool four = r.rows >= 8LL * sm_count;
    const long long blocks = four ? (r.rows + 3) / 4 : r.rows;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    if (interleaved) {
      if (four) rope_chunks_kernel<T, true, 4><<<(unsigned)blocks, threads, 0, stream>>>(a, r);
      else rope_chunks_kernel<T, true, 1><<<(unsigned)blocks, threads, 0, stream>>>(a, r);
    } else {
      if (four) rope_chunks_kernel<T, false, 4><<<(unsigned)blocks, threads, 0, stream>>>(a, r);
      else rope_chunks_kernel<T, false, 1><<<(unsigned)blocks, threads, 0, stream>>>(a, r);
    }
  } else {
    const long long blocks = r.rows < 16LL * sm_count ? r.rows : 16LL * sm_count;
    rope_rows_kernel<T><<<(unsigned)blocks, kRopeThreads, 0, stream>>>(a, r, interleaved ? 1 : 0);
  }
  return cudaGetLastError();
}

}  // namespace bicache

// Rotary positions: rows of queries and keys rotated in place or into other tensors, and the table of
// cosines and sines that the key projection into the store takes.
//
// Pair i of a row at position p turns by the angle p * f_i:
//   (a, b) -> s (a cos - b sin, b cos + a sin),   s = the attention scale (1 unless frequencies are scaled
// by a rule that has one).  The angle is kept in whole and part TURNS: f_i / (2 pi) is a 64-bit fixed-point
// fraction F_i, and p * F_i modulo 2^64 is the part of a turn, exact for every 32-bit p.  A product
// p * f_i in fp32 would be off by p 2^-24 radians (0.06 at p = 10^6), in fp64 it would cost the fp64 pipe and a
// long argument reduction; here it is one 64-bit integer multiplication.  The part of a turn is reduced to
// an eighth before it becomes fp32, so cos and sin are off by no more than about 1e-7.
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

__device__ __forceinline__ float2 rope_cos_sin(const RopeAngles& a, long long pos, int pair) {
  // an eighth of a turn is added, so the two top bits count quarter turns and the rest, taken back to
  // [-1/8, 1/8) turn, is the argument
  const unsigned long long t = (unsigned long long)pos * a.turn[pair] + (1ull << 61);
  const int quarter = (int)(t >> 62);
  const long long rest = (long long)(t & ((1ull << 62) - 1)) - (1ll << 61);
  const float half_turns = (float)(int)(rest >> 30) * 1.1641532182693481e-10f;      // 2^-33
  float s, c;
  sincospif(half_turns, &s, &c);
  const float c1 = (quarter & 1) ? s : c, s1 = (quarter & 1) ? c : s;
  const float cs = (quarter == 1 || quarter == 2) ? -c1 : c1;
  const float sn = (quarter & 2) ? -s1 : s1;
  return make_float2(cs * a.scale, (a.negate ? -sn : sn) * a.scale);
}

// ---------------------------------------------------------------------------------------------
// The table [rows][pairs][2] of bicache_rope_table: one thread per pair.
// ---------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(kRopeThreads)
rope_table_kernel(const __grid_constant__ RopeAngles a, long long rows, float2* __restrict__ table) {
  const long long total = rows * a.pairs;
  for (long long i = blockIdx.x * (long long)blockDim.x + threadIdx.x; i < total;
       i += (long long)gridDim.x * blockDim.x) {
    const long long row = i / a.pairs;
    const long long pos = a.positions ? (long long)a.positions[row] : a.position0 + row;
    table[i] = rope_cos_sin(a, pos, (int)(i - row * a.pairs));
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
// Rows, simplest form: one thread per pair (and per dim beyond the rotated ones), element by element.
// Serves every rotated width.  A block takes one row at a time; its cosines and sines are computed once
// and shared by the row's heads.
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
    if ((int)threadIdx.x < a.pairs) cs[threadIdx.x] = rope_cos_sin(a, pos, threadIdx.x);
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

}  // namespace bicache

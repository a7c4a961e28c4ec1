// Accumulated attention weights on the tensor cores (bf16, head_dim 128): for every cached key the sum over
// all query rows of exp(scale q.k - lse), see WeightGroup in evict.cuh for the batch.
//
// S^T = K Q^T: the keys are the M dimension, so a TMEM lane is one key and a thread that owns the lane sums
// over the columns (rows of queries) on its own - no shuffles, no atomics, one running sum in a register.  Two
// key tiles of 128 stay in shared memory while the row tiles of 128 stream past them; every row tile is
// gathered once per 256 keys.
//
// What bounds it: one exponential per (row, key) against 256 flops of the product.  An SM computes 16
// exponentials a cycle in the special-function unit and 8192 flops a cycle in the tensor pipe, so a 128 x 128
// tile takes 1024 cycles of the one and 512 of the other.  With few rows it is bound by reading the keys.
//
// Roles: warps 0-3 sum key tile 0, warps 4-7 key tile 1, warp 8 issues the MMAs and owns TMEM, warp 9 stages
// key tiles (pages, 4 KB bulk copies: a page already is the operand image), warps 10-13 gather the query rows
// (16-byte copies, any head grouping and row stride) with their log-sum-exps.  Key tiles have a ring of four
// slots (the next item's are fetched while this one's are used), row tiles a ring of three, S two buffers
// per key tile.  All waits are bounded as in the attention kernels.
#pragma once
#include "evict.cuh"
#include "tc_attention.cuh"

namespace bicache {
namespace wts {

using namespace tc;

constexpr int kItemKeys = 256;
constexpr int kRowTile = 128;
constexpr int kKSlots = 4, kQSlots = 3;
constexpr int kSumWarps = 8;
constexpr int kWtsThreads = 448;
constexpr unsigned kIdescNoN = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);   // as kIdescQK, N to be added

struct alignas(16) Sync {
  float neg_lse2[kQSlots][kRowTile];      // -lse log2(e) per row of the tile; -inf: the row adds nothing
  int masked[kQSlots][4];                 // per gather warp: some row of its 32 adds nothing
  unsigned long long k_full[kKSlots], k_free[kKSlots];
  unsigned long long q_full[kQSlots], q_free[kQSlots];
  unsigned long long s_full[2][2], s_free[2][2];      // [key tile][buffer]
  unsigned long long drain;
  long long wait_cycles;                  // directly before abort_flag (mbar_wait reads it)
  int abort_flag;
  unsigned tmem_base;
  int dead;
};
constexpr int kSmemBytes = 1024 + (kKSlots + kQSlots) * kTileBytes + (int)sizeof(Sync);
static_assert(kSmemBytes <= 232448, "shared memory of one CTA");

// One work item as every role derives it from the parameter list.
struct Item {
  int hk, key0, keys;                     // KV head, first key of the launch's key range, keys (1 .. 256)
  int tile_begin, tile_end, rows;         // row tiles; packed rows of the group
  int split, g;
};
__device__ __forceinline__ Item read_item(const WeightArgs& a, const int* list, int index) {
  Item it;
  it.g = weight_group_of(a, list, index);
  const WeightGroup& g = weight_group(list, it.g);
  int rem = index - g.item_begin;
  const int kb = rem % g.key_blocks;
  rem /= g.key_blocks;
  it.split = rem % g.splits;
  it.hk = rem / g.splits;
  it.key0 = kb * kItemKeys;
  it.keys = min(kItemKeys, g.m - it.key0);
  it.rows = g.tokens * (a.Hq / a.Hkv);
  const int tiles = (it.rows + kRowTile - 1) / kRowTile;
  it.tile_begin = min(tiles, it.split * g.tiles_per_split);
  it.tile_end = min(tiles, it.tile_begin + g.tiles_per_split);
  return it;
}
// columns of a row tile that are computed: its rows, to a multiple of 32
__device__ __forceinline__ int tile_cols(const Item& it, int tile) {
  return min(kRowTile, (it.rows - tile * kRowTile + 31) & ~31);
}

// A running sum with its rounding error carried along (the sums run over up to millions of rows).
struct Sum2 {
  float s, c;
  __device__ __forceinline__ void add(float x) {
    const float t = s + x, z = t - s;
    c += (s - (t - z)) + (x - z);
    s = t;
  }
  // an infinite sum has no error term (it is NaN)
  __device__ __forceinline__ double value() const { return (double)s + (isinf(s) ? 0.0 : (double)c); }
};

}  // namespace wts

template <int kWords>
__global__ void __launch_bounds__(wts::kWtsThreads, 1)
tc_weights_kernel(const __grid_constant__ WeightArgs a, const __grid_constant__ ParamList<kWords> params, int* status,
                  long long wait_cycles) {
  using namespace wts;
  const int* const list = params.w;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* const smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Sync* sy = reinterpret_cast<Sync*>(smem + (kKSlots + kQSlots) * kTileBytes);
  volatile int* abort_flag = &sy->abort_flag;
  const unsigned k_ring = smem_u32(smem), q_ring = k_ring + kKSlots * kTileBytes;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    sy->wait_cycles = wait_cycles;
    sy->dead = (*reinterpret_cast<volatile int*>(status) != 0) ? 1 : 0;
    sy->abort_flag = (sy->dead || wait_cycles < kStrictBudget) ? 1 : 0;
    for (int i = 0; i < kKSlots; ++i) {
      mbar_init(smem_u32(&sy->k_full[i]), 32);
      mbar_init(smem_u32(&sy->k_free[i]), 1);
    }
    for (int i = 0; i < kQSlots; ++i) {
      mbar_init(smem_u32(&sy->q_full[i]), 128);
      mbar_init(smem_u32(&sy->q_free[i]), 1 + kSumWarps);
    }
    for (int x = 0; x < 2; ++x)
      for (int b = 0; b < 2; ++b) {
        mbar_init(smem_u32(&sy->s_full[x][b]), 1);
        mbar_init(smem_u32(&sy->s_free[x][b]), 4);
      }
    mbar_init(smem_u32(&sy->drain), 1);
    fence_barrier_init();
  }
  if (warp == 8) {
    tmem_alloc(smem_u32(&sy->tmem_base), kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const unsigned tmem = *reinterpret_cast<volatile unsigned*>(&sy->tmem_base);
  const bool dead = *reinterpret_cast<volatile int*>(&sy->dead) != 0;

  if (warp < kSumWarps) {
    // ================================ exponentials and sums ================================
    const int x = warp >> 2;                                  // key tile
    const unsigned lane_base = (unsigned)((warp & 3) * 32) << 16;
    const float sl2 = a.scale * 1.4426950408889634f;
    const unsigned long long sl2_2 = pack2(sl2, sl2);
    bool ok = !dead;
    unsigned qt = 0, st = 0;                                  // row tiles seen; S buffers of this key tile used
    for (int item = blockIdx.x; item < a.num_items && ok; item += gridDim.x) {
      const Item it = read_item(a, list, item);
      const bool active = it.keys > x * 128;
      Sum2 total = {0.f, 0.f};
      for (int tile = it.tile_begin; tile < it.tile_end && ok; ++tile, ++qt) {
        const unsigned slot = qt % kQSlots;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->q_full[slot]), (qt / kQSlots) & 1, abort_flag));
        if (!ok) break;
        if (active) {
          const unsigned b = st & 1;
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->s_full[x][b]), (st >> 1) & 1, abort_flag));
          if (!ok) break;
          tc_fence_after();
          const int cols = tile_cols(it, tile);
          const unsigned s_addr = tmem + (x * 2 + b) * kRowTile + lane_base;
          const float* nl = sy->neg_lse2[slot];
          unsigned long long acc_a = pack2(0.f, 0.f), acc_b = acc_a;
          for (int c = 0; c < cols; c += 32) {
            unsigned r[32];
            tmem_ld32(s_addr + c, r);
            tmem_wait_ld();
            if (sy->masked[slot][c >> 5]) {
              // some rows add nothing: selected out, because a product with a key that is not finite is NaN
              float sum = 0.f;
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const float l = nl[c + i];
                const float e = ex2(fmaf(__uint_as_float(r[i]), sl2, l));
                sum += l == -INFINITY ? 0.f : e;
              }
              acc_a = add2(acc_a, pack2(sum, 0.f));
            } else {
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                const float4 l = *reinterpret_cast<const float4*>(nl + c + i);
                const unsigned long long xa =
                    fma2(pack2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), sl2_2, pack2(l.x, l.y));
                const unsigned long long xb =
                    fma2(pack2(__uint_as_float(r[i + 2]), __uint_as_float(r[i + 3])), sl2_2, pack2(l.z, l.w));
                float x0, x1, x2, x3;
                unpack2(xa, x0, x1);
                unpack2(xb, x2, x3);
                acc_a = add2(acc_a, pack2(ex2(x0), ex2(x1)));
                acc_b = add2(acc_b, pack2(ex2(x2), ex2(x3)));
              }
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&sy->s_free[x][b]));
          float s0, s1, s2, s3;
          unpack2(acc_a, s0, s1);
          unpack2(acc_b, s2, s3);
          total.add((s0 + s1) + (s2 + s3));
          ++st;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sy->q_free[slot]));
      }
      if (!ok) break;
      const WeightGroup& g = weight_group(list, it.g);
      const int t = it.key0 + x * 128 + (warp & 3) * 32 + lane;
      if (t < g.m) {
        if (g.splits > 1) {
          a.part[g.part_off + ((long long)it.split * a.Hkv + it.hk) * g.m + t] = (float)total.value();
        } else {
          const long long o = g.score_off + it.hk * a.head_stride + g.key0 + t;
          const double before = a.decay != 0.f ? (double)a.decay * (double)a.in[o] : 0.0;
          a.out[o] = (float)(before + total.value());
        }
      }
    }
    tc_fence_before();
  } else if (warp == 8) {
    // ====================================== MMA issue ======================================
    bool ok = !dead;
    unsigned qt = 0, kt = 0;                                  // row tiles and key tiles consumed
    unsigned st[2] = {0, 0};                                  // S buffers filled, per key tile
    const unsigned el = elect_one() ? 1u : 0u;
    auto kstep = [](int k) { return (unsigned long long)((k & 3) * 2 + (k >> 2) * 64); };
    for (int item = blockIdx.x; item < a.num_items && ok; item += gridDim.x) {
      const Item it = read_item(a, list, item);
      const int ktiles = it.keys > 128 ? 2 : 1;
      if (it.tile_begin >= it.tile_end) continue;             // no rows: no keys are staged either
      for (int x = 0; x < ktiles && ok; ++x)
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->k_full[(kt + x) % kKSlots]), ((kt + x) / kKSlots) & 1, abort_flag));
      for (int tile = it.tile_begin; tile < it.tile_end && ok; ++tile, ++qt) {
        const unsigned slot = qt % kQSlots;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->q_full[slot]), (qt / kQSlots) & 1, abort_flag));
        const unsigned idesc = kIdescNoN | ((unsigned)(tile_cols(it, tile) >> 3) << 17);
        const unsigned long long q_desc = make_desc(q_ring + slot * kTileBytes, 16, 2048);
        for (int x = 0; x < ktiles && ok; ++x) {
          const unsigned b = st[x] & 1;
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->s_free[x][b]), ((st[x] >> 1) & 1) ^ 1, abort_flag));
          if (!ok) break;
          tc_fence_after();
          const unsigned long long k_desc = make_desc(k_ring + ((kt + x) % kKSlots) * kTileBytes, 16, 2048);
          unsigned long long ka[8], qb[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            ka[k] = k_desc + kstep(k);
            qb[k] = q_desc + kstep(k);
          }
          mma_ss_batch8(el, tmem + (x * 2 + b) * kRowTile, ka, qb, idesc);
          mma_commit_pred(el, smem_u32(&sy->s_full[x][b]));
          ++st[x];
        }
        if (ok) mma_commit_pred(el, smem_u32(&sy->q_free[slot]));
      }
      if (ok)
        for (int x = 0; x < ktiles; ++x) mma_commit_pred(el, smem_u32(&sy->k_free[(kt + x) % kKSlots]));
      kt += ktiles;
    }
    // Whatever happened, let every MMA issued so far finish before TMEM is released.
    __syncwarp();
    if (!dead) {
      mma_commit_elect(smem_u32(&sy->drain));
      mbar_wait_issued(smem_u32(&sy->drain), 0);
    }
    __syncwarp();
  } else if (warp == 9) {
    // ====================================== key tiles ======================================
    bool ok = !dead;
    unsigned kt = 0;
    int armed[kKSlots] = {-1, -1, -1, -1};                    // the last phase armed with copies, per slot
    for (int item = blockIdx.x; item < a.num_items && ok; item += gridDim.x) {
      const Item it = read_item(a, list, item);
      if (it.tile_begin >= it.tile_end) continue;
      const WeightGroup& g = weight_group(list, it.g);
      for (int k0 = 0; k0 < it.keys && ok; k0 += 128, ++kt) {
        const unsigned slot = kt % kKSlots;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->k_free[slot]), ((kt / kKSlots) & 1) ^ 1, abort_flag));
        if (!ok) break;
        const int npages = (min(128, it.keys - k0) + kPageSize - 1) / kPageSize;
        const unsigned full = smem_u32(&sy->k_full[slot]);
        // every lane arrives, so the phase cannot complete before lane 0 has announced the bytes
        if (lane < npages)
          bulk_copy_g2s(k_ring + slot * kTileBytes + lane * kPageBytes,
                        a.pool_k + ((long long)list[g.page_word + (it.key0 + k0) / kPageSize + lane] * a.Hkv + it.hk) * kPageBytes,
                        kPageBytes, full);
        if (lane == 0)
          mbar_arrive_expect_tx(full, (unsigned)(npages * kPageBytes));
        else
          mbar_arrive(full);
        armed[slot] = (int)((kt / kKSlots) & 1);
      }
    }
    // After a give-up, bulk copies may still be in flight: wait (bounded) for the barriers armed last.
    if (!dead && (!ok || *abort_flag) && lane == 0) {
      for (int s = 0; s < kKSlots; ++s)
        if (armed[s] >= 0)
          for (unsigned n = 0; n < 4096 && !mbar_try_wait(smem_u32(&sy->k_full[s]), (unsigned)armed[s]); ++n) __nanosleep(256);
    }
  } else {
    // ====================================== query rows ======================================
    const int w = warp - 10;                                  // rows 32 w .. 32 w + 31 of every tile
    const int G = a.Hq / a.Hkv;
    const int c16 = lane & 15;
    bool ok = !dead;
    unsigned qt = 0;
    int pending = -1;                                         // slot whose copies have not been announced yet
    auto announce = [&]() {
      fence_proxy_async();
      mbar_arrive(smem_u32(&sy->q_full[pending]));
      pending = -1;
    };
    for (int item = blockIdx.x; item < a.num_items && ok; item += gridDim.x) {
      const Item it = read_item(a, list, item);
      const WeightGroup& g = weight_group(list, it.g);
      for (int tile = it.tile_begin; tile < it.tile_end && ok; ++tile, ++qt) {
        const unsigned slot = qt % kQSlots;
        // where this lane's row is, and its log-sum-exp
        const int p = tile * kRowTile + w * 32 + lane;
        long long src = 0;
        float nl = -INFINITY;
        if (p < it.rows) {
          const int tok = p / G, h = it.hk * G + (p - tok * G);
          const long long row = weight_row(list, g, tok);
          const float l = a.lse[row * a.Hq + h];
          src = (row * a.q_stride + (long long)h * 128) * 2;
          if (!isinf(l)) nl = l * -1.4426950408889634f;
        }
        const unsigned live = __ballot_sync(0xffffffffu, nl != -INFINITY);
        const unsigned q_free = smem_u32(&sy->q_free[slot]), free_parity = ((qt / kQSlots) & 1) ^ 1;
        if (pending >= 0 && !__all_sync(0xffffffffu, mbar_try_wait(q_free, free_parity))) {
          cp_async_wait<0>();                                 // the slot is not free yet: hand over what has been fetched
          announce();
        }
        ok = __all_sync(0xffffffffu, mbar_wait(q_free, free_parity, abort_flag));
        if (!ok) break;
        sy->neg_lse2[slot][w * 32 + lane] = nl;
        if (lane == 0) sy->masked[slot][w] = live != 0xffffffffu;
        if (w * 32 < tile_cols(it, tile)) {
          const unsigned dst = q_ring + slot * kTileBytes;
#pragma unroll 4
          for (int i = 0; i < 16; ++i) {
            const int r = 2 * i + (lane >> 4);
            const long long s = __shfl_sync(0xffffffffu, src, r);
            cp_async16(dst + tile_chunk_offset(w * 32 + r, c16), a.q + s + c16 * 16, (live >> r) & 1u ? 16u : 0u);
          }
        }
        cp_async_commit();
        if (pending >= 0) {
          cp_async_wait<1>();
          announce();
        }
        pending = (int)slot;
      }
    }
    cp_async_wait<0>();
    if (pending >= 0) announce();
  }

  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
  if (tid == 0 && !dead && *abort_flag) atomicCAS(status, kDevOk, kDevTimeout);
}

inline cudaError_t configure_tc_weights() {
  const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  cudaError_t e = cudaFuncSetAttribute(tc_weights_kernel<kParamWordsSmall>, attr, wts::kSmemBytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(tc_weights_kernel<kParamWordsMid>, attr, wts::kSmemBytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(tc_weights_kernel<kParamWords>, attr, wts::kSmemBytes);
  return e;
}

template <int kWords>
cudaError_t launch_tc_weights(const WeightArgs& a, const ParamList<kWords>& list, int* status, int sm_count,
                              long long wait_cycles, cudaStream_t stream) {
  if (a.num_items <= 0) return cudaSuccess;
  const int grid = a.num_items < sm_count ? a.num_items : sm_count;
  tc_weights_kernel<kWords><<<grid, wts::kWtsThreads, wts::kSmemBytes, stream>>>(
      a, list, status, wait_cycles > 0 ? wait_cycles : tc::kWaitCycles);
  return cudaGetLastError();
}

}  // namespace bicache

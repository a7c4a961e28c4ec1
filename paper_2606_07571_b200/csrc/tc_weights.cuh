// Accumulated attention weights on the tensor cores (bf16, head_dim 128): for every cached key the sum over
// all query rows of exp(scale q.k - lse), see WeightGroup in evict.cuh for the batch.
//
// S = Q K^T with 128 query rows on the TMEM lanes and 256 keys along the columns.  The keys of an item stay in
// shared memory while the row tiles stream past them.  A thread owns a row (its log-sum-exp is one register) and
// 64 of the keys, for each of which it keeps a running sum in a register; the sum over the rows of a tile, across
// the lanes, is put off until up to 48 tiles have been added, and then costs 62 shuffles for 64 keys.  (With the
// keys on the lanes the sum over rows needs no shuffles, but every log-sum-exp is a shared-memory operand of
// every thread: that form ran at 4.6 ms where this one took 4.1, 32 requests of 1024 rows and 28 heads over 16,384 keys.)
//
// What bounds it: one exponential per (row, key) against 256 flops of the product.  An SM computes 16
// exponentials a cycle in the special-function unit and 8192 flops a cycle in the tensor pipe, so a tile of 128 x
// 256 takes 2048 cycles of the one and 1024 of the other; it takes 2330 (4.2 ms, 86 % of the unit's rate).  A
// polynomial on the FMA pipe for two of every eight pairs, which is faster by itself (116 cycles against 135 for 16
// keys of four warps), gained nothing here: 4.2 ms with a register split between the roles, 5.8 without it.  Why is not
// settled.  It is not a lack of issue slots (47 % of them are used on the long prefix, the special-function unit 84 %);
// registers are short: 64 sums and 16 loaded values a thread, and the kernel spills 84 bytes at its 96.
// With few rows the kernel is bound by reading the keys.
//
// Roles: warps 0-15 exponentials and sums (warp w: lanes 32 (w & 3) .., keys 64 (w >> 2) ..), warps 16 and 17
// fetch the query rows with their log-sum-exps, warp 18 issues the MMAs and owns TMEM (two S buffers of 256 columns),
// warp 19 stages keys (pages, 4 KB bulk copies: a page already is the operand image).  A row tile is the G query heads
// of as many tokens as fit 128 rows: if its tokens are one run of rows, two TMA boxes (64 dims, G heads, the
// tokens) are the tile; a tile that spans the end of one request and the start of the next is gathered with
// 16-byte copies.  Keys have two slots of 256 (the next item's are fetched while this one's are used), row tiles a
// ring of three.  All waits are bounded as in the attention kernels.
#pragma once
#include "evict.cuh"
#include "tc_attention.cuh"

namespace bicache {
namespace wts {

using namespace tc;

constexpr int kItemKeys = 256;
constexpr int kRowTile = 128;
constexpr int kKeyBytes = kItemKeys * 128 * 2;   // 64 KB
constexpr int kKSlots = 2, kQSlots = 3;
constexpr int kSumWarps = 16;
constexpr int kRowWarp = 16, kMmaWarpW = 18, kKeyWarp = 19;
constexpr int kWtsThreads = 640;             // 20 warps: five to a scheduler, 96 registers a thread
constexpr int kGroupKeys = 4 * kItemKeys / kSumWarps;      // keys of a sum warp
constexpr int kLaneKeys = kGroupKeys / 32;                 // whose sums end in a lane
constexpr int kMaxTerms = 48;                // row tiles a thread adds before the lanes are put together
constexpr unsigned kIdescNoN = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);   // as kIdescQK, N to be added

struct alignas(16) Sync {
  float neg_lse2[kQSlots][kRowTile];      // -lse log2(e) per row of the tile; -inf: the row adds nothing
  float hop_sum[kItemKeys];               // sums on their way from one lane group to the next
  unsigned long long k_full[kKSlots], k_free[kKSlots];
  unsigned long long q_full[kQSlots], q_free[kQSlots];
  unsigned long long s_full[2], s_free[2];
  unsigned long long hop[kSumWarps / 4][4];   // [key group][lane group]: hop_sum holds the sums of lane groups >= it; 0: read
  unsigned long long drain;
  long long wait_cycles;                  // directly before abort_flag (mbar_wait reads it)
  int abort_flag;
  unsigned tmem_base;
  int dead;
};
constexpr int kSmemBytes = kKSlots * kKeyBytes + kQSlots * kTileBytes + (int)sizeof(Sync);
static_assert(kSmemBytes <= 232448, "shared memory of one CTA");

// byte offset of 16-byte chunk c16 (0..15) of row r (0..127) of a row tile: two blocks of 128 rows x 64 dims, as the TMA
// boxes write them (8-row groups 1024 bytes apart), 128-byte swizzle
__device__ __forceinline__ unsigned row_chunk_offset(int r, int c16) {
  return (unsigned)((c16 >> 3) * 16384 + r * 128 + (((c16 & 7) ^ (r & 7)) << 4));
}

// One work item as every role derives it from the parameter list.
struct Item {
  int hk, key0, keys;                     // KV head, first key of the launch's key range, keys (1 .. 256)
  int tile_begin, tile_end, tokens;       // row tiles; tokens of the group
  int split, g;
};
__device__ __forceinline__ Item read_item(const WeightArgs& a, const int* list, int index) {
  Item it;
  it.g = weight_group_of(a, list, index);
  const WeightGroup& g = weight_group(list, it.g);
  const int rem = index - g.item_begin, at = rem / g.key_blocks, kb = rem - at * g.key_blocks;
  it.hk = at;
  it.split = 0;
  if (g.splits > 1) {
    it.hk = at / g.splits;
    it.split = at - it.hk * g.splits;
  }
  it.key0 = kb * kItemKeys;
  it.keys = min(kItemKeys, g.m - it.key0);
  it.tokens = g.tokens;
  it.tile_begin = min(g.tiles, it.split * g.tiles_per_split);
  it.tile_end = min(g.tiles, it.tile_begin + g.tiles_per_split);
  return it;
}

// The items of a CTA: dealt out forth and back (0 1 2 | 2 1 0 | 0 1 2 ..), since they get shorter towards the end: over
// random batches of 2 to 8 prefixes the fullest SM has 7 % more than the mean, 10 % if every round starts with CTA 0.
struct ItemWalk {
  int item, step;
  __device__ __forceinline__ ItemWalk() : item(blockIdx.x), step(2 * (gridDim.x - blockIdx.x) - 1) {}
  __device__ __forceinline__ void next() {
    item += step;
    step = 2 * gridDim.x - step;
  }
};

// A running sum with its rounding error carried along (the sums run over up to millions of rows).
struct Sum2 {
  float s, c;
  __device__ __forceinline__ void add(float x) {
    const float t = s + x, z = t - s;
    c += (s - (t - z)) + (x - z);
    s = t;
  }
  // an infinite sum has no error term (it is NaN)
  __device__ __forceinline__ float value() const { return isinf(s) ? s : s + c; }
};

// Has the phase completed?  Unlike try_wait this does not suspend the thread.
__device__ __forceinline__ bool mbar_test(unsigned bar, unsigned parity) {
  unsigned ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// bytes to come, without an arrival
__device__ __forceinline__ void mbar_expect_tx(unsigned bar, unsigned bytes) {
  asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tmem_ld16(unsigned taddr, unsigned* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
}  // namespace wts

template <int kWords>
__global__ void __launch_bounds__(wts::kWtsThreads, 1)
tc_weights_kernel(const __grid_constant__ WeightArgs a, const __grid_constant__ CUtensorMap q_map, int* status,
                  long long wait_cycles, const __grid_constant__ ParamList<kWords> params) {
  using namespace wts;
  const int* const list = params.w;
  // No room for alignment slack: the kernel has no static shared memory, the dynamic window starts 1024-byte
  // aligned (the swizzled tiles need that), and a CTA that finds otherwise reports an error instead of computing.
  extern __shared__ __align__(1024) unsigned char smem[];
  Sync* sy = reinterpret_cast<Sync*>(smem + kKSlots * kKeyBytes + kQSlots * kTileBytes);
  volatile int* abort_flag = &sy->abort_flag;
  const unsigned k_ring = smem_u32(smem), q_ring = k_ring + kKSlots * kKeyBytes;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  // Set-up, all of it side by side: thread 0 the barriers, warp 18 TMEM, warp 19 its own barriers and the first keys,
  // every role its first item (the first reads of the parameters miss their cache), warps 16 and 17 the first
  // log-sum-exps; then one barrier for the block.
  if (tid == 0) {
    const int state = *reinterpret_cast<volatile int*>(status);
    sy->wait_cycles = wait_cycles;
    for (int i = 0; i < kQSlots; ++i) {
      mbar_init(smem_u32(&sy->q_full[i]), 64);
      mbar_init(smem_u32(&sy->q_free[i]), 1 + kSumWarps);     // the MMAs; the warps that read the log-sum-exps
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&sy->s_full[b]), 1);
      mbar_init(smem_u32(&sy->s_free[b]), kSumWarps);
    }
    for (int i = 0; i < kSumWarps; ++i) mbar_init(smem_u32(&sy->hop[i >> 2][i & 3]), 1);
    mbar_init(smem_u32(&sy->drain), 1);
    fence_barrier_init();
    if ((smem_u32(smem) & 1023u) != 0) atomicCAS(status, kDevOk, kDevInternal);
    sy->dead = state != 0 || (smem_u32(smem) & 1023u) != 0 ? 1 : 0;
    sy->abort_flag = (sy->dead || wait_cycles < kStrictBudget) ? 1 : 0;
  }
  unsigned tmem = 0;
  bool dead = false;
  auto set_up = [&]() {
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    tmem = *reinterpret_cast<volatile unsigned*>(&sy->tmem_base);
    dead = *reinterpret_cast<volatile int*>(&sy->dead) != 0;
  };

  if (warp < kSumWarps) {
    // ================================ exponentials and sums ================================
    {
      const Item it = read_item(a, list, blockIdx.x);         // only brings the parameters into their cache
      asm volatile("" ::"r"(it.hk), "r"(it.keys), "r"(it.tile_end));
    }
    set_up();
    const int lg = warp & 3, kg = warp >> 2;                  // lane group, key group
    const unsigned s_addr = tmem + kg * kGroupKeys + ((unsigned)(lg * 32) << 16);
    const float sl2 = a.scale * 1.4426950408889634f;
    const unsigned long long sl2_2 = pack2(sl2, sl2);
    bool ok = !dead;
    // lanes that have a row in every full tile (128 may not be a multiple of G); what the others add up is dropped
    const bool has_row = lg * 32 + lane < a.tile_tokens * (a.Hq / a.Hkv);
    const unsigned full = __ballot_sync(0xffffffffu, has_row);
    unsigned slot = 0, slot_parity = 0, b = 0, b_parity = 0;  // row tile ring and S buffer of the next tile
    unsigned handed = 0;                                      // items whose sums went from group to group
    const unsigned q_full0 = smem_u32(&sy->q_full[0]), q_free0 = smem_u32(&sy->q_free[0]);
    const unsigned s_full0 = smem_u32(&sy->s_full[0]), s_free0 = smem_u32(&sy->s_free[0]);
    for (ItemWalk at; at.item < a.num_items && ok; at.next()) {
      const Item it = read_item(a, list, at.item);
      const bool active = it.keys > kg * kGroupKeys;
      Sum2 total[kLaneKeys];                                  // keys kLaneKeys * lane .., over this lane group
#pragma unroll
      for (int i = 0; i < kLaneKeys; ++i) total[i] = Sum2{0.f, 0.f};
      for (int left = it.tile_end - it.tile_begin; left > 0 && ok; left -= kMaxTerms) {
        unsigned long long acc[kGroupKeys / 2];                 // keys 2 p, 2 p + 1 of the warp's
#pragma unroll
        for (int p = 0; p < kGroupKeys / 2; ++p) acc[p] = 0ull;
#pragma unroll 1
        for (int n = min(left, kMaxTerms); n > 0; --n) {
          // one vote for both waits: after a give-up the log-sum-exp read in between is any number
          bool good = mbar_wait(q_full0 + slot * 8, slot_parity, abort_flag);
          const float nl = sy->neg_lse2[slot][lg * 32 + lane];
          good = mbar_wait(s_full0 + b * 8, b_parity, abort_flag) && good;
          ok = __all_sync(0xffffffffu, good);
          if (!ok) break;
          if (lane == 0) mbar_arrive(q_free0 + slot * 8);       // the vote is behind every lane's read
          tc_fence_after();
          const bool adds = nl != -INFINITY;
          const unsigned live = __ballot_sync(0xffffffffu, adds);
          if (active && live != 0u) {
            const unsigned long long nl2 = pack2(nl, nl);
            const unsigned s_tile = s_addr + b * kItemKeys;
            // without branches inside: the compiler overlaps the end of one run of 16 keys with the start of the next
            auto sum_tile = [&](auto holes) {
#pragma unroll
              for (int c = 0; c < kGroupKeys / 16; ++c) {
                unsigned r[16];
                tmem_ld16(s_tile + c * 16, r);
                tmem_wait_ld();
                if (decltype(holes)::value) {
                  // a row that adds nothing: whatever its product is (with a key that is not finite, or from memory behind
                  // the last request), 2^-inf is 0
#pragma unroll
                  for (int i = 0; i < 16; ++i) r[i] = adds ? r[i] : 0u;
                }
#pragma unroll
                for (int p = 0; p < 8; ++p) {
                  float x0, x1;
                  unpack2(fma2(pack2(__uint_as_float(r[2 * p]), __uint_as_float(r[2 * p + 1])), sl2_2, nl2), x0, x1);
                  acc[c * 8 + p] = add2(acc[c * 8 + p], pack2(ex2(x0), ex2(x1)));
                }
              }
            };
            if (live == full) sum_tile(std::false_type()); else sum_tile(std::true_type());
          }
          tc_fence_before();
          if (lane == 0) mbar_arrive(s_free0 + b * 8);
          if (++slot == kQSlots) {
            slot = 0;
            slot_parity ^= 1;
          }
          b ^= 1;
          b_parity ^= b ^ 1;                                    // the phase changes when both buffers have been used
        }
        if (active) {
          // The lanes' sums put together: in each step a lane passes half of its keys to its partner and takes the other
          // half; lane l ends with the keys from kLaneKeys * l on.
          float v[kGroupKeys];
#pragma unroll
          for (int p = 0; p < kGroupKeys / 2; ++p) unpack2(acc[p], v[2 * p], v[2 * p + 1]);
          if (full != 0xffffffffu) {
#pragma unroll
            for (int i = 0; i < kGroupKeys; ++i) v[i] = has_row ? v[i] : 0.f;
          }
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) {
            const bool upper = (lane & o) != 0;
#pragma unroll
            for (int i = 0; i < kLaneKeys * o; ++i) {
              const float send = upper ? v[i] : v[i + kLaneKeys * o], keep = upper ? v[i + kLaneKeys * o] : v[i];
              v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
            }
          }
#pragma unroll
          for (int i = 0; i < kLaneKeys; ++i) total[i].add(v[i]);
        }
      }
      if (!ok) break;
      // Lane groups 3, 2, 1, 0 add their sums in turn; group 0 writes the result.
      if (active) {
        const int first = kg * kGroupKeys + kLaneKeys * lane;
        float sum[kLaneKeys];
#pragma unroll
        for (int i = 0; i < kLaneKeys; ++i) sum[i] = total[i].value();
        if (it.tile_begin < it.tile_end) {
          // group 3 waits for group 0 to have read the item before
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->hop[kg][(lg + 1) & 3]), (handed & 1) ^ (lg == 3 ? 1 : 0), abort_flag));
          if (!ok) break;
#pragma unroll
          for (int i = 0; i < kLaneKeys; ++i) {
            if (lg < 3) sum[i] += sy->hop_sum[first + i];
            if (lg > 0) sy->hop_sum[first + i] = sum[i];
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&sy->hop[kg][lg]));
          ++handed;
        }
        if (lg == 0) {
          const WeightGroup& g = weight_group(list, it.g);
#pragma unroll
          for (int i = 0; i < kLaneKeys; ++i) {
            const int t = it.key0 + first + i;
            if (t >= g.m) break;
            if (g.splits > 1) {
              a.part[g.part_off + ((long long)it.split * a.Hkv + it.hk) * g.m + t] = sum[i];
            } else {
              const long long o = g.score_off + it.hk * a.head_stride + g.key0 + t;
              a.out[o] = (float)((a.decay != 0.f ? (double)a.decay * (double)a.in[o] : 0.0) + (double)sum[i]);
            }
          }
        }
      }
    }
    tc_fence_before();
  } else {
    Item it = read_item(a, list, blockIdx.x);
    if (warp == kMmaWarpW) {
      // ====================================== MMA issue ======================================
      tmem_alloc(smem_u32(&sy->tmem_base), kTmemCols);
      tmem_relinquish();
      set_up();
      bool ok = !dead;
      unsigned qt = 0, kt = 0;                                // row tiles and key blocks consumed
      const unsigned el = elect_one() ? 1u : 0u;
      // a K step of 16 dims: 32 bytes inside the swizzled row; dims 64.. sit 1024 bytes further in the keys, 16 KB
      // further in a row tile
      auto kstep = [](int k) { return (unsigned long long)((k & 3) * 2 + (k >> 2) * 64); };
      auto qstep = [](int k) { return (unsigned long long)((k & 3) * 2 + (k >> 2) * 1024); };
      for (ItemWalk at; at.item < a.num_items && ok; at.next()) {
        if (at.item != blockIdx.x) it = read_item(a, list, at.item);
        if (it.tile_begin >= it.tile_end) continue;           // no rows: no keys are staged either
        const unsigned ks = kt % kKSlots;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->k_full[ks]), (kt / kKSlots) & 1, abort_flag));
        const unsigned idesc = kIdescNoN | ((unsigned)((it.keys + 15) >> 4) << 18);       // N: keys to a multiple of 16
        const unsigned long long k_desc = make_desc(k_ring + ks * kKeyBytes, 16, 2048);
        for (int tile = it.tile_begin; tile < it.tile_end && ok; ++tile, ++qt) {
          const unsigned slot = qt % kQSlots, b = qt & 1;
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->q_full[slot]), (qt / kQSlots) & 1, abort_flag));
          if (ok) ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->s_free[b]), ((qt >> 1) & 1) ^ 1, abort_flag));
          if (!ok) break;
          tc_fence_after();
          const unsigned long long q_desc = make_desc(q_ring + slot * kTileBytes, 16, 1024);
          unsigned long long qa[8], kb[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            qa[k] = q_desc + qstep(k);
            kb[k] = k_desc + kstep(k);
          }
          mma_ss_batch8(el, tmem + b * kItemKeys, qa, kb, idesc);
          mma_commit_pred(el, smem_u32(&sy->s_full[b]));
          mma_commit_pred(el, smem_u32(&sy->q_free[slot]));
        }
        if (ok) mma_commit_pred(el, smem_u32(&sy->k_free[ks]));
        ++kt;
      }
      // Whatever happened, let every MMA issued so far finish before TMEM is released.
      __syncwarp();
      if (!dead) {
        mma_commit_elect(smem_u32(&sy->drain));
        mbar_wait_issued(smem_u32(&sy->drain), 0);
      }
      __syncwarp();
    } else if (warp == kKeyWarp) {
      // ======================================== keys =========================================
      if (lane == 0) {
        for (int i = 0; i < kKSlots; ++i) {
          mbar_init(smem_u32(&sy->k_full[i]), 32);
          mbar_init(smem_u32(&sy->k_free[i]), 1);
        }
        fence_barrier_init();
      }
      __syncwarp();
      unsigned kt = 0;
      int armed[kKSlots] = {-1, -1};                          // the last phase armed with copies, per slot
      auto fetch = [&]() {
        const WeightGroup& g = weight_group(list, it.g);
        const unsigned ks = kt % kKSlots;
        const int npages = (it.keys + kPageSize - 1) / kPageSize;          // up to 16
        const unsigned full = smem_u32(&sy->k_full[ks]);
        // every lane arrives, so the phase cannot complete before lane 0 has announced the bytes
        if (lane < npages)
          bulk_copy_g2s(k_ring + ks * kKeyBytes + lane * kPageBytes,
                        a.pool_k + ((long long)list[g.page_word + it.key0 / kPageSize + lane] * a.Hkv + it.hk) * kPageBytes,
                        kPageBytes, full);
        if (lane == 0)
          mbar_arrive_expect_tx(full, (unsigned)(npages * kPageBytes));
        else
          mbar_arrive(full);
        armed[ks] = (int)((kt / kKSlots) & 1);
        ++kt;
      };
      // the first item's keys need no free slot and nobody else's barriers
      ItemWalk at;
      if (it.tile_begin < it.tile_end) fetch();
      set_up();
      bool ok = !dead;
      for (at.next(); at.item < a.num_items && ok; at.next()) {
        it = read_item(a, list, at.item);
        if (it.tile_begin >= it.tile_end) continue;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->k_free[kt % kKSlots]), ((kt / kKSlots) & 1) ^ 1, abort_flag));
        if (ok) fetch();
      }
      // After a give-up, bulk copies may still be in flight: wait (bounded) for the barriers armed last.
      if ((!ok || *abort_flag) && lane == 0) {
        for (int s = 0; s < kKSlots; ++s)
          if (armed[s] >= 0)
            for (unsigned n = 0; n < 4096 && !mbar_try_wait(smem_u32(&sy->k_full[s]), (unsigned)armed[s]); ++n) __nanosleep(256);
      }
    } else {
      // ====================================== query rows ======================================
      // Every lane looks up where its rows of a tile are and requests their log-sum-exps while the rows of the tile
      // before it are on their way, so that neither stands between two tiles' copies.
      const int w = warp - kRowWarp;                          // rows 64 w .. 64 w + 63 of every tile
      const int G = a.Hq / a.Hkv, T = a.tile_tokens;
      const int c16 = lane & 15;
      // byte offset in the tile of this lane's chunk of rows 2 j + (lane >> 4): repeats every four steps
      unsigned chunk_off[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) chunk_off[j] = row_chunk_offset(2 * j + (lane >> 4), c16);
      // token of the tile and head of the group of this lane's rows: the same in every tile
      int tok_in[2], head_in[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = w * 64 + i * 32 + lane;
        tok_in[i] = r / G;
        head_in[i] = r - tok_in[i] * G;
      }
      unsigned qt = 0;
      int boxed[kQSlots] = {-1, -1, -1};                      // the last phase armed with a box, per slot
      int pending = -1;                                       // slot whose copies have not been announced yet
      auto announce = [&]() {
        fence_proxy_async();
        mbar_arrive(smem_u32(&sy->q_full[pending]));
        pending = -1;
      };
      ItemWalk at;
      int tile = 0, tile_end = 0, tokens = 0, hk = 0, segs = 0;
      const WeightSeg* seg = nullptr;
      // the runs of rows the lane's two rows and the tile's first token are in: number, end, row of token 0
      int run[3], run_end[3];
      long long run_row[3];
      auto read_run = [&](int i, int number) {
        run[i] = number;
        run_row[i] = seg[number].row - seg[number].token;
        run_end[i] = number + 1 < segs ? seg[number + 1].token : 0x7fffffff;
      };
      auto next_item = [&]() {                                // to the next item that has row tiles
        for (; at.item < a.num_items; at.next()) {
          if (at.item != blockIdx.x) it = read_item(a, list, at.item);
          if (it.tile_begin >= it.tile_end) continue;
          const WeightGroup& g = weight_group(list, it.g);
          tile = it.tile_begin;
          tile_end = it.tile_end;
          tokens = it.tokens;
          hk = it.hk;
          segs = g.num_segs;
          seg = reinterpret_cast<const WeightSeg*>(&list[g.seg_word]);
          int lo = 0, hi = segs - 1;                          // last run that starts at or before the first token
          while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (seg[mid].token <= tile * T) lo = mid; else hi = mid - 1;
          }
#pragma unroll
          for (int i = 0; i < 3; ++i) read_run(i, lo);
          return;
        }
      };
      long long src[2], box_row = 0;
      float lse[2];
      bool one_run = false;                                   // the tile's tokens are consecutive rows
      auto look_up = [&]() {
        const int tok0 = tile * T, last = min(tokens, tok0 + T) - 1;
        while (tok0 >= run_end[2]) read_run(2, run[2] + 1);
        one_run = a.boxes && last < run_end[2];
        box_row = run_row[2] + tok0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int tok = tok0 + tok_in[i];
          src[i] = -1;
          lse[i] = INFINITY;
          if (tok_in[i] < T && tok <= last) {
            while (tok >= run_end[i]) read_run(i, run[i] + 1);
            const long long row = run_row[i] + tok;
            const int h = hk * G + head_in[i];
            src[i] = one_run ? 0 : (row * a.q_stride + (long long)h * 128) * 2;
            lse[i] = a.lse[row * a.Hq + h];
          }
        }
      };
      next_item();
      if (at.item < a.num_items) look_up();
      set_up();
      bool ok = !dead;
      while (at.item < a.num_items && ok) {
        const int box_head = hk * G, box_first = (int)box_row;
        const bool boxes = one_run;
        float row_lse[2];
        unsigned rows[2];                                     // the rows that exist
        long long from[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          row_lse[i] = lse[i];
          rows[i] = __ballot_sync(0xffffffffu, src[i] >= 0);
          from[i] = src[i];
        }
        const unsigned slot = qt % kQSlots;
        const unsigned q_free = smem_u32(&sy->q_free[slot]), free_parity = ((qt / kQSlots) & 1) ^ 1;
        const unsigned q_full = smem_u32(&sy->q_full[slot]);
        ++qt;
        if (pending >= 0 && (boxes || !__all_sync(0xffffffffu, mbar_test(q_free, free_parity)))) {
          cp_async_wait<0>();                                 // nothing more to put behind these copies yet: hand them over
          announce();
        }
        ok = __all_sync(0xffffffffu, mbar_wait(q_free, free_parity, abort_flag));
        if (!ok) break;
        const unsigned dst = q_ring + slot * kTileBytes;
        if (boxes) {
          // rows past the tile's last token come along (or as zeros, past the tensor): they add nothing
          if (lane == 0) {
            mbar_expect_tx(q_full, (unsigned)(T * G * 128));                // each warp fetches one half of the dims
            tma_load_3d(dst + w * 16384, &q_map, w * 64, box_head, box_first, q_full);
            boxed[slot] = (int)(((qt - 1) / kQSlots) & 1);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (rows[i] == 0u) continue;                      // rows that do not exist may hold anything
            const int r0 = w * 64 + i * 32;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const int r = 2 * j + (lane >> 4);
              const long long s = __shfl_sync(0xffffffffu, from[i], r);
              const bool exists = (rows[i] >> r) & 1u;
              cp_async16(dst + r0 * 128 + (j >> 2) * 1024 + chunk_off[j & 3], a.q + (exists ? s : 0) + c16 * 16,
                         exists ? 16u : 0u);
            }
          }
          cp_async_commit();
        }
        // the next tile of the item is looked up, and this one's log-sum-exps arrive, while the rows are on their way
        const bool last_tile = tile + 1 >= tile_end;
        if (!last_tile) {
          ++tile;
          look_up();
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
          sy->neg_lse2[slot][w * 64 + i * 32 + lane] = isinf(row_lse[i]) ? -INFINITY : row_lse[i] * -1.4426950408889634f;
        if (boxes) {
          __syncwarp();                                       // lane 0 has announced the bytes
          mbar_arrive(q_full);
        } else {
          if (pending >= 0) {
            cp_async_wait<1>();
            announce();
          }
          pending = (int)slot;
        }
        if (last_tile) {                                      // the next item takes longer to work out
          at.next();
          next_item();
          if (at.item < a.num_items) look_up();
        }
      }
      cp_async_wait<0>();
      if (pending >= 0) announce();
      // After a give-up, boxes may still be in flight: wait (bounded) for the barriers armed last.
      if (!dead && (!ok || *abort_flag) && lane == 0) {
        for (int s = 0; s < kQSlots; ++s)
          if (boxed[s] >= 0)
            for (unsigned n = 0; n < 4096 && !mbar_try_wait(smem_u32(&sy->q_full[s]), (unsigned)boxed[s]); ++n) __nanosleep(256);
      }
    }
  }

  __syncthreads();
  if (warp == kMmaWarpW) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
  if (tid == 0 && !dead && *abort_flag) atomicCAS(status, kDevOk, kDevTimeout);
}

inline cudaError_t configure_tc_weights() {
  const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  cudaError_t e = cudaSuccess;
  each_param_length([&](auto words) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(tc_weights_kernel<decltype(words)::value>, attr, wts::kSmemBytes);
  }, ParamLengths());
  return e;
}

template <int kWords>
cudaError_t launch_tc_weights(const WeightArgs& a, const CUtensorMap& q_map, const ParamList<kWords>& list, int* status,
                              int sm_count, long long wait_cycles, cudaStream_t stream) {
  if (a.num_items <= 0) return cudaSuccess;
  const int grid = a.num_items < sm_count ? a.num_items : sm_count;
  // the keys of the item after next wait for a whole item: about 2,500 cycles a row tile, so the default budget
  // grows with the longest item
  const long long budget = wait_cycles > 0 ? wait_cycles : tc::kWaitCycles + 20000LL * a.max_item_tiles;
  tc_weights_kernel<kWords><<<grid, wts::kWtsThreads, wts::kSmemBytes, stream>>>(a, q_map, status, budget, list);
  return cudaGetLastError();
}

}  // namespace bicache

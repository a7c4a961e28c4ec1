// Windowed attention over cached tokens on the tensor cores (bf16, head_dim 128); see window.cuh for the batch.
//
// A work item is 128 packed query rows of one KV head against a range of key tiles of 64 tokens of its page sequence.  As
// in tc_decode_kernel a CTA is small (112 KB of shared memory, 256 TMEM columns: two to an SM, so that one computes
// softmaxes while the MMAs of the other run) and S is double-buffered: S(j+1) = Q K(j+1)^T is issued before the softmax of
// tile j ends.  Roles: warps 0-3 softmax (one thread per row; they also gather the Q tile), warp 4 MMA issue and TMEM, warp
// 5 stages K tiles, warp 6 V tiles.  What the window adds:
//   - pages are looked up in the item's page sequence (first tokens, then the window's);
//   - an item begins with a tile that all its rows see (window_item), so that the running maxima hardly move;
//   - a row knows the columns it sees as an interval and a number of first columns.  A tile that some row of a warp
//     does not see in full is masked by bits, and a row that has seen nothing yet keeps -inf as its reference and 0 for it
//     in the exponent;
//   - slots that no row of the item sees may hold anything.  Their scores are masked one way or another; as values they would
//     meet weight 0, and 0 times a NaN is a NaN: a page of values with such slots comes by a copy per run of seen slots, the
//     others zeroed, where whole pages come by one bulk copy;
//   - an item that has all the keys of its rows writes the output itself, in bf16; ranges write normalised partial
//     results for window_join_kernel.
//
// What bounds it.  Few rows: reading the keys (64 tokens over caches of 700 to 16,384 keys, 1.7 GB: 260 us, 6.5 TB/s); a single
// token over 16,384 keys takes 10 us and its join 4, of which 5 are reading: starts and ends of four tiles to an item.
// Long windows: the shared-memory port, which moves 768 cycles' worth of operands for a tile that the tensor pipe computes in
// 512 (16,384 rows over as many keys that all rows see: 1219 TFLOP/s, in long runs under the power limit 1076).  Short windows: an item's start (6000 cycles until its first
// scores) and end (3500) beside 12 tiles of 1550 (two items at a time): 28 query heads, window of 500 + 201, five ragged
// requests 93 us, the tensor pipe 37 % busy.
#pragma once
#include "tc_decode.cuh"
#include "window.cuh"

namespace bicache {

template <int kWords>
__global__ void __launch_bounds__(dec::kDecThreads, 2)
tc_window_kernel(const __grid_constant__ WindowArgs a, int* status, long long wait_cycles,
                 const __grid_constant__ ParamList<kWords> params) {
  using namespace dec;
  // No room for alignment slack with two CTAs per SM: the kernel has no static shared memory, the
  // dynamic window starts 1024-byte aligned (the swizzled tiles need that), and a CTA that finds
  // otherwise reports an error instead of computing.
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* const smem = smem_raw;
  DecSync* sy = reinterpret_cast<DecSync*>(smem + kQBytes + (kKStages + kVStages) * kKvTileBytes);
  volatile int* abort_flag = &sy->abort_flag;
  const unsigned q_smem = smem_u32(smem);
  const unsigned k_ring = q_smem + kQBytes, v_ring = k_ring + kKStages * kKvTileBytes;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // the joining kernel may be placed on the SMs from now on (it waits for this grid's end)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int status_now = *reinterpret_cast<volatile int*>(status);      // arrives while the item is looked up
  const WindowReq& r = window_req(a, params.w, blockIdx.x);
  const WindowItem it = window_item<kKeys>(a, r, blockIdx.x, 128);
  const int G = a.Hq / a.Hkv;
  const int T = it.tile_end - it.tile_begin;
  const int rows = min(128, r.n * G - it.row0);                // rows of the item; the warps beyond them do nothing
  const int active = (rows + 31) >> 5;
  auto tile_of = [&](int j) { return window_tile(it.start, it.tile_begin, it.tile_end, j); };
  auto tile_pages = [&](int j) { return min(kKeys / kPageSize, it.pages.count - tile_of(j) * (kKeys / kPageSize)); };

  // Set-up, all of it side by side: warps 0-3 request the Q tile, warp 4 sets flags and barriers and fetches TMEM, warps
  // 5 and 6 set their own barriers and issue the first tiles, for which they need nobody.
  const int is_v = warp - 5;
  const int stages = is_v ? kVStages : kKStages;
  int armed[kKStages] = {-1, -1, -1};        // load warps: the last tile armed with bulk copies, per stage
  // Where lanes 0-3 find the pages of a tile.
  struct TilePage {
    const char* src;
    WindowSlots slots;
    bool bulk;                               // to be copied as a whole
  };
  auto find_tile = [&](int j) {
    TilePage p = TilePage{nullptr, WindowSlots{0, kPageSize, 0}, lane < tile_pages(j)};
    if (p.bulk) {
      const int s = tile_of(j) * (kKeys / kPageSize) + lane;
      p.src = (is_v ? a.pool_v : a.pool_k) + (long long)it.hk * a.page_bytes + window_page(a, r, params.w, it.pages, s) * a.page_stride;
      if (is_v) {
        p.slots = window_slots(it.pages, s);
        p.bulk = p.slots.whole();
      }
    }
    return p;
  };
  // One tile into its slot, which is free.
  auto load_tile = [&](int j, const TilePage& p) {
    const int b = j % stages;
    const unsigned full = smem_u32(is_v ? &sy->v_full[b] : &sy->k_full[b]);
    const unsigned dst = (is_v ? v_ring : k_ring) + b * kKvTileBytes;
    const int npages = tile_pages(j);
    const char* const src = p.src;
    const WindowSlots& slots = p.slots;
    const bool bulk = p.bulk;
    const unsigned bulks = __ballot_sync(0xffffffffu, bulk);
    if (bulk) bulk_copy_g2s(dst + lane * kPageBytes, src, kPageBytes, full);
    const unsigned pieces = ~bulks & ((1u << npages) - 1u);
    unsigned bytes = __popc(bulks) * kPageBytes;
    if (pieces != 0) bytes += copy_window_pages(dst, src, slots, pieces, full, lane);
    // every lane arrives, so the phase cannot complete before lane 0 has announced the bytes
    if (lane == 0) {
      mbar_arrive_expect_tx(full, bytes);
      armed[b] = j;
    } else {
      mbar_arrive(full);
    }
  };
  const int ahead = min(T, stages);          // tiles that find their slots free
  bool begun = false;
  bool dead;
  if (warp >= 5) {
    if (lane == 0) {
      for (int i = 0; i < stages; ++i) {
        mbar_init(smem_u32(is_v ? &sy->v_full[i] : &sy->k_full[i]), 32);
        mbar_init(smem_u32(is_v ? &sy->v_free[i] : &sy->k_free[i]), 1);
      }
      fence_barrier_init();
    }
    __syncwarp();
    asm volatile("barrier.cta.arrive 1, 224;" ::: "memory");       // the others may use the barriers
    // (one lane's answer for the warp: another CTA may raise the status at any time, and load_tile is for all lanes)
    begun = __shfl_sync(0xffffffffu, status_now, 0) == 0 && (q_smem & 1023u) == 0;
    if (begun)
      for (int j = 0; j < ahead; ++j) load_tile(j, find_tile(j));
    asm volatile("barrier.cta.sync 2, 96;" ::: "memory");          // the flags that warp 4 sets
    dead = *reinterpret_cast<volatile int*>(&sy->dead) != 0;
  } else {
    if (warp == 4) {
      if (lane == 0) {
        sy->wait_cycles = wait_cycles;
        if ((q_smem & 1023u) != 0) atomicCAS(status, kDevOk, kDevInternal);
        sy->dead = status_now != 0 || (q_smem & 1023u) != 0 ? 1 : 0;
        sy->abort_flag = (sy->dead || wait_cycles < kStrictBudget) ? 1 : 0;
        mbar_init(smem_u32(&sy->q_full), 32 * active);
        for (int i = 0; i < 2; ++i) {
          mbar_init(smem_u32(&sy->s_full[i]), 1);
          mbar_init(smem_u32(&sy->p_full[i]), 32 * active);
        }
        mbar_init(smem_u32(&sy->pv_done), 1);
        mbar_init(smem_u32(&sy->o_done), 1);
        mbar_init(smem_u32(&sy->drain), 1);
        fence_barrier_init();
      }
      __syncwarp();
      asm volatile("barrier.cta.arrive 2, 96;" ::: "memory");
      tmem_alloc(smem_u32(&sy->tmem_base), kDecTmemCols);
      tmem_relinquish();
    } else {
      if (warp < active && T > 0) {
        // The Q tile: warp w fetches rows 32 w .. 32 w + 31, lane l the 16-byte chunk (l & 15) of rows 32 w + (l >> 4) + 2 i.
        // Rows past the end stay what they are: a row of Q meets no other row's results.
        const int c16 = lane & 15, r0 = lane >> 4, here = min(32, rows - warp * 32);
        const int prow = it.row0 + warp * 32 + r0, t = prow / G;
        int jj = prow - t * G;
        // two packed rows on: two heads, and from one token's last to the next's first at most once
        const int step = G == 1 ? 0 : 2;
        const long long step_bytes = G == 1 ? 4 * a.q_stride : 512, wrap_bytes = a.q_stride * 2 - G * 256;
        const char* src = a.q + ((r.row + t) * a.q_stride + (long long)(it.hk * G + jj) * 128) * 2 + c16 * 16;
        unsigned dst[4];                             // of rows r0 + 2 i, i < 4; 8 rows on: 2048 bytes
#pragma unroll
        for (int i = 0; i < 4; ++i) dst[i] = q_smem + tile_chunk_offset(warp * 32 + r0 + 2 * i, c16);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (r0 + 2 * i < here) cp_async16(dst[i & 3] + (i >> 2) * 2048, src, 16u);
          jj += step;
          src += step_bytes;
          if (jj >= G) {
            jj -= G;
            src += wrap_bytes;
          }
        }
        cp_async_commit();
      }
    }
    tc_fence_before();
    asm volatile("barrier.cta.sync 1, 224;" ::: "memory");
    tc_fence_after();
    dead = *reinterpret_cast<volatile int*>(&sy->dead) != 0;
  }
  const unsigned tmem = warp < 5 ? *reinterpret_cast<volatile unsigned*>(&sy->tmem_base) : 0;
  const unsigned tmem_o = tmem + 128;

  if (warp < 4) {
    // ================================ softmax and epilogue =================================
    const int row = warp * 32 + lane;                        // row of the tile = TMEM lane
    const unsigned lane_base = (unsigned)(warp * 32) << 16;
    const float sl2 = a.scale * 1.4426950408889634f;         // scores are handled in the log2 domain
    float m_ref = -INFINITY, l_sum = 0.f;
    bool ok = !dead;
    if (warp < active) {
      if (T > 0) {
        cp_async_wait<0>();
        fence_proxy_async();
        if (ok) mbar_arrive(smem_u32(&sy->q_full));
      }
      // the columns this row sees, from the first tile on; a row past the end runs along unmasked and asks for nothing
      const bool mine = row < rows;
      WindowColumns col = WindowColumns{0, 0x7fffffff, 0};
      if (mine) col = window_columns(a, it.pages, r.len, r.pos + (it.row0 + row) / G);
      for (int j = 0; j < T && ok; ++j) {
        const int b = j & 1;
        const int col0 = tile_of(j) * kKeys, begin = col.begin - col0, end = col.end - col0, sink = col.sink - col0;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->s_full[b]), (j >> 1) & 1, abort_flag));
        if (!ok) break;
        tc_fence_after();
        unsigned s[64];
        tmem_ld32(tmem + b * 64 + lane_base, s);
        tmem_ld32(tmem + b * 64 + 32 + lane_base, s + 32);
        tmem_wait_ld();
        if (__any_sync(0xffffffffu, begin > 0 || end < kKeys)) {
          const unsigned lo = (low_bits(end) & ~low_bits(begin)) | low_bits(sink);
          const unsigned hi = (low_bits(end - 32) & ~low_bits(begin - 32)) | low_bits(sink - 32);
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            if (!((lo >> i) & 1u)) s[i] = 0xff800000u;             // -inf
            if (!((hi >> i) & 1u)) s[32 + i] = 0xff800000u;
          }
        }
        float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
        for (int i = 0; i < 64; i += 4) {
          mx0 = max3(mx0, __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
          mx1 = max3(mx1, __uint_as_float(s[i + 2]), __uint_as_float(s[i + 3]));
        }
        const float mx = mine ? fmaxf(mx0, mx1) * sl2 : -INFINITY;       // scale > 0
        if (j == 0) {
          m_ref = mx;
        } else if (__any_sync(0xffffffffu, mx > m_ref + 8.f)) {
          // Rare: a row's maximum exceeds the reference by more than 2^8, or it sees its first key.  O must be rescaled, and
          // S of this tile was issued before O += P V of the previous one: wait for that first.
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->pv_done), (j - 1) & 1, abort_flag));
          if (!ok) break;
          tc_fence_after();
          float alpha = 1.f;
          if (mx > m_ref + 8.f) {
            alpha = ex2(m_ref - mx);
            m_ref = mx;
          }
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            unsigned o[32];
            tmem_ld32(tmem_o + c * 32 + lane_base, o);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
            tmem_st32(tmem_o + c * 32 + lane_base, o);
          }
          tmem_wait_st();
          l_sum *= alpha;
        }
        const float neg_m = m_ref == -INFINITY ? 0.f : -m_ref;     // nothing seen so far: every weight is 0
        const unsigned long long sl2_2 = pack2(sl2, sl2), neg_m2 = pack2(neg_m, neg_m);
        unsigned long long acc_a = pack2(0.f, 0.f), acc_b = pack2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const unsigned long long xa =
              fma2(pack2(__uint_as_float(s[4 * i]), __uint_as_float(s[4 * i + 1])), sl2_2, neg_m2);
          const unsigned long long xb =
              fma2(pack2(__uint_as_float(s[4 * i + 2]), __uint_as_float(s[4 * i + 3])), sl2_2, neg_m2);
          float x0, x1, x2, x3;
          unpack2(xa, x0, x1);
          unpack2(xb, x2, x3);
          const float p0 = ex2(x0), p1 = ex2(x1), p2 = ex2(x2), p3 = ex2(x3);
          acc_a = add2(acc_a, pack2(p0, p1));
          acc_b = add2(acc_b, pack2(p2, p3));
          // What the MMA takes, as in the other attention kernels; the sum takes them unrounded.  It is the larger share of
          // the output's error: 0.0023 of its size as a root mean square, 0.0017 if only the result were rounded.
          s[2 * i] = pack_bf16(p0, p1);
          s[2 * i + 1] = pack_bf16(p2, p3);
        }
        tmem_st32(tmem + b * 64 + lane_base, s);               // P over the first 32 columns of this S
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(smem_u32(&sy->p_full[b]));
        float s0, s1, s2, s3;
        unpack2(acc_a, s0, s1);
        unpack2(acc_b, s2, s3);
        l_sum += (s0 + s1) + (s2 + s3);
      }
      // -------- epilogue: the output, or the normalised partial of this key range --------
      if (ok && T > 0) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->o_done), 0, abort_flag));
        tc_fence_after();
      }
      if (ok) {
        const WindowRow w(a, it.hk, it.row0 + (mine ? row : 0));
        const long long at = window_part(a, r, it.split, w), out_row = r.row + w.t;
        const bool whole = r.splits == 1;
        const float inv = l_sum == 0.f ? 0.f : 1.f / l_sum;
        const float lse = l_sum == 0.f ? -INFINITY : (m_ref + log2f(l_sum)) * 0.6931471805599453f;
        if (mine) {
          if (!whole) a.part_lse[at] = lse;
          else if (a.lse) a.lse[out_row * a.Hq + w.h] = lse;
        }
        // A thread holds a row (128 values).  It goes to shared memory first (the K/V rings are free by now: every tile has been
        // consumed; rows 272 bytes apart keep the 16-byte stores conflict-free), half a row at a time if it is a partial
        // result; then the warp writes whole rows.  (A bulk copy per row took 4500 cycles, this 3400.)
        unsigned char* const stage = smem + kQBytes + warp * 32 * 272;
        char* const mine_to = whole ? a.out + (out_row * a.out_stride + (long long)w.h * 128) * 2 : reinterpret_cast<char*>(a.part_o + at * 128);
        const int here = min(32, rows - warp * 32);
#pragma unroll 1
        for (int half = 0; half < (whole ? 1 : 2); ++half) {
#pragma unroll 1
          for (int c = 0; c < (whole ? 2 : 1); ++c) {
            unsigned o[64];
            if (T > 0) {
              tmem_ld32(tmem_o + (half + c) * 64 + lane_base, o);
              tmem_ld32(tmem_o + (half + c) * 64 + 32 + lane_base, o + 32);
              tmem_wait_ld();
            } else {
#pragma unroll
              for (int i = 0; i < 64; ++i) o[i] = 0u;
            }
            if (whole) {
#pragma unroll
              for (int i = 0; i < 64; i += 8) {
                uint4 v;
                v.x = pack_bf16(__uint_as_float(o[i]) * inv, __uint_as_float(o[i + 1]) * inv);
                v.y = pack_bf16(__uint_as_float(o[i + 2]) * inv, __uint_as_float(o[i + 3]) * inv);
                v.z = pack_bf16(__uint_as_float(o[i + 4]) * inv, __uint_as_float(o[i + 5]) * inv);
                v.w = pack_bf16(__uint_as_float(o[i + 6]) * inv, __uint_as_float(o[i + 7]) * inv);
                *reinterpret_cast<uint4*>(stage + lane * 272 + (c * 64 + i) * 2) = v;
              }
            } else {
#pragma unroll
              for (int i = 0; i < 64; i += 4)
                *reinterpret_cast<float4*>(stage + lane * 272 + i * 4) =
                    make_float4(__uint_as_float(o[i]) * inv, __uint_as_float(o[i + 1]) * inv,
                                __uint_as_float(o[i + 2]) * inv, __uint_as_float(o[i + 3]) * inv);
            }
          }
          __syncwarp();
          // 256 bytes a row, two rows at a time
#pragma unroll 4
          for (int i = lane >> 4; i < 32; i += 2) {
            char* const to = reinterpret_cast<char*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine_to), i));
            if (i < here)
              *reinterpret_cast<uint4*>(to + half * 256 + (lane & 15) * 16) =
                  *reinterpret_cast<const uint4*>(stage + i * 272 + (lane & 15) * 16);
          }
          __syncwarp();
        }
      }
      tc_fence_before();
    }
  } else if (warp == 4) {
    // ====================================== MMA issue ======================================
    bool ok = !dead && T > 0;
    if (ok) {
      const unsigned long long q_desc = make_desc(q_smem, 16, 2048);
      const unsigned el = elect_one() ? 1u : 0u;               // the lane that issues every MMA of this warp
      // a K step of 16 dims: 32 bytes inside the swizzled row; dims 64.. sit 1024 bytes further
      auto kstep = [](int k) { return (unsigned long long)((k & 3) * 2 + (k >> 2) * 64); };
      auto issue_s = [&](int j) {
        const int b = j & 1, ks = j % kKStages;
        bool good = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->k_full[ks]), (j / kKStages) & 1, abort_flag));
        if (!good) return false;
        tc_fence_after();
        const unsigned long long k_desc = make_desc(k_ring + ks * kKvTileBytes, 16, 2048);
        unsigned long long qa[8], kb[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          qa[k] = q_desc + kstep(k);
          kb[k] = k_desc + kstep(k);
        }
        mma_ss_batch8(el, tmem + b * 64, qa, kb, kIdescS64);
        mma_commit_pred(el, smem_u32(&sy->s_full[b]));
        mma_commit_pred(el, smem_u32(&sy->k_free[ks]));
        return true;
      };
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->q_full), 0, abort_flag));
      if (ok) ok = issue_s(0);
      for (int j = 0; j < T && ok; ++j) {
        const int b = j & 1;
        if (j + 1 < T) {
          ok = issue_s(j + 1);
          if (!ok) break;
        }
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->p_full[b]), (j >> 1) & 1, abort_flag));
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sy->v_full[b]), (j >> 1) & 1, abort_flag));
        if (!ok) break;
        tc_fence_after();
        // V is the MN-major operand: 64-dim halves 1024 bytes apart, 8-key groups 2048 bytes; a K
        // step of 16 keys is one page image (4096 bytes).  Pages past the last are skipped.
        const unsigned long long v_desc = make_desc(v_ring + b * kKvTileBytes, 1024, 2048);
        const unsigned long long vb[4] = {v_desc, v_desc + 256ull, v_desc + 512ull, v_desc + 768ull};
        mma_ts_batch4_first(el, tmem_o, tmem + b * 64, vb, kIdescPV, j > 0 ? 1u : 0u, tile_pages(j));
        mma_commit_pred(el, smem_u32(&sy->v_free[b]));
        mma_commit_pred(el, smem_u32(&sy->pv_done));
        if (j == T - 1) mma_commit_pred(el, smem_u32(&sy->o_done));
      }
      // Whatever happened, let every MMA issued so far finish before TMEM is released.
      __syncwarp();
      mma_commit_elect(smem_u32(&sy->drain));
      mbar_wait_issued(smem_u32(&sy->drain), 0);
    }
    __syncwarp();
  } else {
    // ======================================= loads ========================================
    // Warp 5 stages the K tiles, warp 6 the V tiles.
    bool ok = !dead;
    for (int j = begun ? ahead : 0; j < T && ok; ++j) {
      const TilePage p = find_tile(j);                             // while the slot is still in use
      const unsigned free_bar = smem_u32(is_v ? &sy->v_free[j % stages] : &sy->k_free[j % stages]);
      ok = __all_sync(0xffffffffu, mbar_wait(free_bar, ((j / stages) & 1) ^ 1, abort_flag));
      if (ok) load_tile(j, p);
    }
  }

  __syncthreads();
  // No copy may land after the CTA has gone.  Without a give-up all tiles have been used; after one, which is known now that
  // all roles are done, the load warps wait (bounded) for the tiles that they requested last.
  if (warp >= 5 && lane == 0 && *abort_flag) {
    for (int b = 0; b < stages; ++b)
      if (armed[b] >= 0) {
        const unsigned full = smem_u32(is_v ? &sy->v_full[b] : &sy->k_full[b]);
        for (unsigned n = 0; n < 4096 && !mbar_try_wait(full, (armed[b] / stages) & 1); ++n) __nanosleep(256);
      }
  }
  if (warp == 4) {
    tc_fence_after();
    tmem_dealloc(tmem, kDecTmemCols);
  }
  if (tid == 0 && !dead && *abort_flag) atomicCAS(status, kDevOk, kDevTimeout);
}

template <int kWords>
inline cudaError_t configure_tc_window() {
  return cudaFuncSetAttribute(tc_window_kernel<kWords>, cudaFuncAttributeMaxDynamicSharedMemorySize, dec::kDecSmemBytes);
}

template <int kWords>
inline cudaError_t launch_tc_window(const WindowArgs& a, const ParamList<kWords>& list, int* status, long long wait_cycles,
                                    cudaStream_t stream) {
  tc_window_kernel<kWords><<<(unsigned)a.num_items, dec::kDecThreads, dec::kDecSmemBytes, stream>>>(
      a, status, wait_cycles > 0 ? wait_cycles : tc::kWaitCycles, list);
  return cudaGetLastError();
}

}  // namespace bicache

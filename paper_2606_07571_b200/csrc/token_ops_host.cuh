// C ABI entry points of token eviction and rotary positions (see include/bicache.h).  Included by bicache.cu,
// behind the context and its helpers.
#pragma once
#include <cmath>

namespace {

// The calls run on the context's device; the caller's current device is put back.
struct DeviceGuard {
  int before = -1;
  explicit DeviceGuard(int device) {
    int now = -1;
    if (cudaGetDevice(&now) == cudaSuccess && now != device && cudaSetDevice(device) == cudaSuccess) before = now;
  }
  ~DeviceGuard() {
    if (before >= 0) cudaSetDevice(before);
  }
};

// No C++ exception (out of host memory) leaves a C entry point.
template <typename F>
int32_t guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return BICACHE_ERR_NOMEM;
  }
}

int cuda_status(const bicache_ctx* ctx, cudaError_t e, const char* where) {
  return e == cudaSuccess ? BICACHE_OK : fail(ctx, BICACHE_ERR_CUDA, std::string(where) + ": " + cudaGetErrorString(e));
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

// ---- accumulated weights ------------------------------------------------------------------------

// The launches of one bicache_prefix_weights call: groups are added until the parameter list is full.
// Group records grow from the front of the list, row runs and page lists from its end.
class WeightLaunches {
 public:
  WeightLaunches(bicache_ctx* ctx, const WeightArgs& args, const CUtensorMap& q_map, bool tensor, cudaStream_t stream)
      : ctx_(ctx), base_(args), q_map_(q_map), tensor_(tensor), stream_(stream) {}

  // keys [page0 * 16, min(m, (page0 + pages) * 16)) of a prefix against num_segs row runs; `first`: the call's
  // decay and input apply (else the launch adds to what an earlier one has written)
  int add(const PrefixEntry& e, const std::vector<int32_t>& pages, int page0, int num_pages, const WeightSeg* segs,
          int num_segs, int tokens, long long score_off, bool first) {
    const int need = kGroupWords + num_segs * kSegWords + ((num_pages + 1) & ~1);
    // a launch that adds to an earlier one holds one group: two parts of one prefix's rows must not meet in it
    if (groups_ > 0 && (!first || !first_ || front() + need > back_)) {
      const int st = flush();
      if (st != BICACHE_OK) return st;
    }
    first_ = first;
    WeightGroup g = WeightGroup();
    g.key0 = page0 * kPageSize;
    g.m = std::min(e.m - g.key0, num_pages * kPageSize);
    back_ -= (num_pages + 1) & ~1;                       // keeps the row runs, which follow, 8-byte aligned
    g.page_word = back_;
    std::memcpy(&list_[back_], pages.data() + page0, sizeof(int32_t) * num_pages);
    back_ -= num_segs * kSegWords;
    g.seg_word = back_;
    g.num_segs = num_segs;
    const int tok0 = num_segs ? segs[0].token : 0;
    for (int i = 0; i < num_segs; ++i) {
      WeightSeg s = segs[i];
      s.token -= tok0;
      std::memcpy(&list_[back_ + i * kSegWords], &s, sizeof(s));
    }
    g.tokens = tokens;
    g.score_off = score_off;
    std::memcpy(&list_[groups_ * kGroupWords], &g, sizeof(g));
    ++groups_;
    return BICACHE_OK;
  }

  int flush() {
    if (groups_ == 0) return BICACHE_OK;
    WeightArgs a = base_;
    if (!first_) {
      a.decay = 1.f;
      a.in = a.out;
    }
    WeightGroup* g = reinterpret_cast<WeightGroup*>(list_);
    int max_tiles = 1, max_m = 1;
    long long blocks8 = 0;                                            // CUDA-core form: 128 keys against a row tile
    for (int i = 0; i < groups_; ++i) blocks8 += (long long)((g[i].m + 127) / 128) * a.Hkv * tiles_of(g[i]);
    const int per_thread = a.D <= kWsEightMaxD && blocks8 >= ctx_->sm_count ? 8 : 4;
    const int block_keys = tensor_ ? wts::kItemKeys : 16 * per_thread;
    // long groups first: the short items of the others even out what these leave
    std::stable_sort(g, g + groups_, [&](const WeightGroup& x, const WeightGroup& y) { return tiles_of(x) > tiles_of(y); });
    for (int i = 0; i < groups_; ++i) {
      g[i].key_blocks = (g[i].m + block_keys - 1) / block_keys;
      max_tiles = std::max(max_tiles, tiles_of(g[i]));
      max_m = std::max(max_m, g[i].m);
    }
    // How many row tiles an item covers at most.  Fewer tiles make more items, which fill the SMs evenly, but every
    // item costs its start and the sum over its lanes (about two tiles, 2.5 us) and more than one range per key the
    // second kernel (about three).  Counted in tiles: the fullest SM, items being dealt out forth and back.
    const int slots = tensor_ || weights_simt_smem(a.D, per_thread) > 113 * 1024 ? ctx_->sm_count : 2 * ctx_->sm_count;
    const int choices = std::min(max_tiles, std::max(4, 128 / groups_));
    auto splits_of = [&](int tiles, int tps) { return std::max(1, (tiles + tps - 1) / tps); };
    std::vector<int> load(slots);
    int best_tps = max_tiles;
    long long best = 0x7fffffffffffffffLL;
    for (int s = 1, before = 0; s <= std::min(choices, 32); ++s) {
      const int tps = (max_tiles + s - 1) / s;
      if (tps == before) continue;
      before = tps;
      long long part = 0, even = 0;
      int at = 0;
      std::fill(load.begin(), load.end(), 0);
      for (int i = 0; i < groups_; ++i) {
        const int tiles = tiles_of(g[i]), sp = splits_of(tiles, tps), cost = (tiles + sp - 1) / sp + 2;
        const long long items = (long long)g[i].key_blocks * a.Hkv * sp;
        even += items / (2 * slots) * 2 * cost;                   // two rounds bring two items to each
        for (int left = (int)(items % (2 * slots)); left > 0; --left) {
          load[at < slots ? at : 2 * slots - 1 - at] += cost;
          at = at + 1 == 2 * slots ? 0 : at + 1;
        }
        if (sp > 1) part += (long long)sp * a.Hkv * g[i].m;
      }
      if (part > ctx_->part_capacity_rowheads * ctx_->cfg.head_dim) break;
      const long long c = even + *std::max_element(load.begin(), load.end()) + (part > 0 ? 3 : 0);
      if (c < best) {
        best = c;
        best_tps = tps;
      }
    }
    long long item = 0, part = 0;
    bool split = false;
    for (int i = 0; i < groups_; ++i) {
      const int tiles = tiles_of(g[i]);
      g[i].tiles = tiles;
      g[i].splits = splits_of(tiles, best_tps);
      g[i].tiles_per_split = (tiles + g[i].splits - 1) / g[i].splits;
      g[i].item_begin = (int)item;
      item += (long long)g[i].key_blocks * a.Hkv * g[i].splits;
      g[i].part_off = (int)part;
      if (g[i].splits > 1) {
        part += (long long)g[i].splits * a.Hkv * g[i].m;
        split = true;
      }
    }
    a.num_groups = groups_;
    a.num_items = (int)item;
    a.max_item_tiles = best_tps;
    // the records from the end follow the groups: the list is as short as what it holds
    const int gap = back_ - front();
    for (int i = 0; i < groups_; ++i) {
      g[i].page_word -= gap;
      g[i].seg_word -= gap;
    }
    std::memmove(&list_[front()], &list_[back_], sizeof(int) * (kParamWords - back_));
    cudaError_t e = cudaSuccess;
    with_param_list(list_, kParamWords - gap, [&](const auto& list) {
      constexpr int kWords = sizeof(list.w) / sizeof(int);
      if (tensor_) {
        e = launch_tc_weights(a, q_map_, list, ctx_->d_status, ctx_->sm_count, ctx_->wait_cycles, stream_);
      } else {
        const size_t smem = weights_simt_smem(a.D, per_thread);
        const bool f32 = ctx_->cfg.dtype == BICACHE_F32, eight = per_thread == 8;
        auto* const kernel = f32 ? (eight ? weights_simt_kernel<float, 8, kWords> : weights_simt_kernel<float, 4, kWords>)
                                 : (eight ? weights_simt_kernel<__nv_bfloat16, 8, kWords> : weights_simt_kernel<__nv_bfloat16, 4, kWords>);
        kernel<<<a.num_items, kWsThreads, smem, stream_>>>(a, list);
        e = cudaGetLastError();
      }
      ctx_->launches++;
      if (e == cudaSuccess && split) {
        const long long per_group = (long long)a.Hkv * max_m;
        const unsigned blocks = (unsigned)std::min<long long>((per_group + 255) / 256, 4LL * ctx_->sm_count);
        weights_sum_kernel<kWords><<<dim3(blocks, groups_), 256, 0, stream_>>>(a, tensor_ ? ctx_->d_status : nullptr, list);
        ctx_->launches++;
        e = cudaGetLastError();
      }
    });
    groups_ = 0;
    back_ = kParamWords;
    return cuda_status(ctx_, e, "prefix_weights");
  }

 private:
  int tiles_of(const WeightGroup& g) const {
    if (tensor_) return (g.tokens + base_.tile_tokens - 1) / base_.tile_tokens;
    return (int)(((long long)g.tokens * (base_.Hq / base_.Hkv) + kWsRows - 1) / kWsRows);
  }
  int front() const { return groups_ * kGroupWords; }

  bicache_ctx* ctx_;
  WeightArgs base_;
  CUtensorMap q_map_;
  bool tensor_, first_ = true;
  cudaStream_t stream_;
  int groups_ = 0, back_ = kParamWords;
  alignas(8) int list_[kParamWords];
};
static_assert(kParamWords % 2 == 0 && kGroupWords % 2 == 0 && kSegWords % 2 == 0, "8-byte aligned records");
// what one launch takes of a batch that does not fit: together less than the list
constexpr int kMaxLaunchSegs = 900, kMaxLaunchPages = 4096;
static_assert(kGroupWords + kMaxLaunchSegs * kSegWords + kMaxLaunchPages <= kParamWords, "one chunk fits a launch");

int prefix_weights_impl(bicache_ctx* ctx, int32_t layer, int32_t R, const int32_t* prefix_id, const int64_t* row_off,
                        const int32_t* seqlen, const void* q, int64_t q_row_stride, const float* lse,
                        const float* scores_in, float* scores_out, const int64_t* score_off,
                        int64_t score_head_stride, float decay, float softmax_scale, void* stream_) {
  if (!ctx) return BICACHE_ERR_INVALID;
  const bicache_config& cfg = ctx->cfg;
  if (layer < 0 || layer >= cfg.num_layers) return fail(ctx, BICACHE_ERR_INVALID, "layer out of range");
  if (R < 0) return fail(ctx, BICACHE_ERR_INVALID, "negative request count");
  if (!std::isfinite(decay) || !std::isfinite(softmax_scale))
    return fail(ctx, BICACHE_ERR_INVALID, "decay and scale must be finite");
  if (R > 0 && (!prefix_id || !row_off || !seqlen || !score_off))
    return fail(ctx, BICACHE_ERR_INVALID, "null metadata array");
  if (R > 0 && (!scores_out || (decay != 0.f && !scores_in)))
    return fail(ctx, BICACHE_ERR_INVALID, "null score pointer");
  if (!aligned16(q) || !aligned4(lse) || !aligned4(scores_in) || !aligned4(scores_out))
    return fail(ctx, BICACHE_ERR_INVALID, "misaligned tensor pointer");
  const int G = cfg.num_q_heads / cfg.num_kv_heads;
  if (R > 0 && (q_row_stride < (int64_t)cfg.num_q_heads * cfg.head_dim || (q_row_stride * ctx->esize) % 16))
    return fail(ctx, BICACHE_ERR_INVALID, "bad row stride");
  struct Run { int first, last; const PrefixEntry* e; };
  std::vector<Run> runs;
  std::vector<std::pair<int64_t, int64_t>> blocks;               // score elements [begin, end) of every prefix
  for (int i = 0; i < R; ++i) {
    if (seqlen[i] < 0 || row_off[i] < 0) return fail(ctx, BICACHE_ERR_INVALID, "negative length or offset");
    const int32_t p = prefix_id[i];
    if (p < -1) return fail(ctx, BICACHE_ERR_INVALID, "bad prefix id");
    if (p < 0) continue;
    if (seqlen[i] > 0 && (!q || !lse)) return fail(ctx, BICACHE_ERR_INVALID, "null tensor pointer");
    if (score_off[i] < 0) return fail(ctx, BICACHE_ERR_INVALID, "negative score offset");
    if (i > 0 && p == prefix_id[i - 1]) {
      if (score_off[i] != score_off[i - 1])
        return fail(ctx, BICACHE_ERR_INVALID, "requests of one prefix name different score blocks");
      runs.back().last = i;
      continue;
    }
    for (const Run& r : runs)
      if (prefix_id[r.first] == p) return fail(ctx, BICACHE_ERR_INVALID, "requests of one prefix are not contiguous");
    auto found = ctx->by_id.find(p);
    if (found == ctx->by_id.end()) return fail(ctx, BICACHE_ERR_NOTFOUND, "unknown or evicted prefix id");
    const PrefixEntry& e = *found->second;
    if (e.first_layer > layer) return fail(ctx, BICACHE_ERR_INVALID, "the prefix owns no pages in this layer");
    if (score_head_stride < e.m) return fail(ctx, BICACHE_ERR_INVALID, "score rows shorter than the prefix");
    runs.push_back(Run{i, i, &e});
    blocks.emplace_back(score_off[i], score_off[i] + (cfg.num_kv_heads - 1) * score_head_stride + e.m);
  }
  for (const Run& r : runs) {
    long long tokens = 0;
    for (int i = r.first; i <= r.last; ++i) tokens += seqlen[i];
    if (tokens > 0x7fffff00LL / G) return fail(ctx, BICACHE_ERR_INVALID, "batch too large");
  }
  std::sort(blocks.begin(), blocks.end());
  for (size_t i = 1; i < blocks.size(); ++i)
    if (blocks[i].first < blocks[i - 1].second) return fail(ctx, BICACHE_ERR_INVALID, "score blocks overlap");
  if (ctx->host_only) return fail(ctx, BICACHE_ERR_UNSUPPORTED, "host-only context has no device path");
  if (runs.empty()) return BICACHE_OK;

  DeviceGuard guard(cfg.device);
  const PoolView pool = pool_view_layer(ctx, layer);
  WeightArgs a = WeightArgs();
  a.q = static_cast<const char*>(q);
  a.q_stride = q_row_stride;
  a.lse = lse;
  a.in = decay != 0.f ? scores_in : nullptr;
  a.out = scores_out;
  a.head_stride = score_head_stride;
  a.decay = decay;
  a.scale = softmax_scale;
  a.part = ctx->d_part_o;
  a.pool_k = pool.k;
  a.page_bytes = pool.page_bytes;
  a.swizzled = pool.swizzled;
  a.Hq = cfg.num_q_heads;
  a.Hkv = cfg.num_kv_heads;
  a.D = cfg.head_dim;
  // a row tile of the tensor-core kernel holds the query heads of whole tokens
  const bool tensor = ctx->tensor_ok && ctx->path != BICACHE_PATH_SIMT && G <= wts::kRowTile;
  CUtensorMap q_map;
  std::memset(&q_map, 0, sizeof(q_map));
  if (tensor) {
    long long rows_total = 0;                                     // rows q is known to have
    for (int i = 0; i < R; ++i)
      if (prefix_id[i] >= 0 && seqlen[i] > 0) rows_total = std::max<long long>(rows_total, row_off[i] + seqlen[i]);
    a.tile_tokens = wts::kRowTile / G;
    // box coordinates are 32-bit; without boxes every row tile is gathered
    a.boxes = rows_total > 0 && rows_total < 0x7fffffffLL &&
              encode_map(&q_map, q, rows_total, cfg.num_q_heads, q_row_stride, G, a.tile_tokens);
  }
  WeightLaunches launches(ctx, a, q_map, tensor, static_cast<cudaStream_t>(stream_));
  std::vector<WeightSeg> segs;
  for (const Run& r : runs) {
    segs.clear();
    int tokens = 0;
    for (int i = r.first; i <= r.last; ++i) {
      if (seqlen[i] == 0) continue;
      segs.push_back(WeightSeg{row_off[i], tokens, 0});
      tokens += seqlen[i];
    }
    const std::vector<int32_t>& pages = pages_of(*r.e, layer);
    const int num_pages = (int)pages.size(), num_segs = (int)segs.size();
    const bool fits = kGroupWords + num_segs * kSegWords + ((num_pages + 1) & ~1) <= kParamWords;
    const int page_step = fits ? num_pages : kMaxLaunchPages, seg_step = fits ? std::max(1, num_segs) : kMaxLaunchSegs;
    for (int p0 = 0; p0 < num_pages; p0 += page_step)
      for (int s0 = 0; s0 == 0 || s0 < num_segs; s0 += seg_step) {
        const int ns = std::min(seg_step, num_segs - s0);
        const int tok_end = s0 + ns < num_segs ? segs[s0 + ns].token : tokens;
        const int st = launches.add(*r.e, pages, p0, std::min(page_step, num_pages - p0), segs.data() + s0, ns,
                                    tok_end - (ns > 0 ? segs[s0].token : 0), score_off[r.first], s0 == 0);
        if (st != BICACHE_OK) return st;
      }
  }
  return launches.flush();
}

// ---- compaction ---------------------------------------------------------------------------------

int compact_prefix_impl(bicache_ctx* ctx, int32_t src_id, int32_t dst_id, int32_t first_layer, int32_t num_layers,
                        int32_t keep, const int32_t* idx, int64_t idx_layer_stride, int64_t idx_head_stride,
                        void* stream_) {
  if (!ctx) return BICACHE_ERR_INVALID;
  const bicache_config& cfg = ctx->cfg;
  if (num_layers < 0 || first_layer < 0 || first_layer > cfg.num_layers - num_layers)
    return fail(ctx, BICACHE_ERR_INVALID, "layers out of range");
  auto fs = ctx->by_id.find(src_id), fd = ctx->by_id.find(dst_id);
  if (fs == ctx->by_id.end() || fd == ctx->by_id.end())
    return fail(ctx, BICACHE_ERR_NOTFOUND, "unknown or evicted prefix id");
  const PrefixEntry &src = *fs->second, &dst = *fd->second;
  if (src_id == dst_id) return fail(ctx, BICACHE_ERR_INVALID, "source and destination are one prefix");
  if (first_layer < src.first_layer || first_layer < dst.first_layer)
    return fail(ctx, BICACHE_ERR_INVALID, "a prefix owns no pages in the first layer");
  if (keep != dst.m) return fail(ctx, BICACHE_ERR_INVALID, "keep is not the destination's length");
  if (idx_layer_stride < 0 || idx_head_stride < 0) return fail(ctx, BICACHE_ERR_INVALID, "negative index stride");
  if ((num_layers > 0 && !idx) || !aligned4(idx)) return fail(ctx, BICACHE_ERR_INVALID, "bad index pointer");
  if (ctx->host_only) return fail(ctx, BICACHE_ERR_UNSUPPORTED, "host-only context has no device path");
  if (num_layers == 0) return BICACHE_OK;
  DeviceGuard guard(cfg.device);
  const PoolView pv = pool_view(ctx);
  CompactArgs a = CompactArgs();
  a.layer_bytes = pv.layer_bytes;
  a.page_bytes = pv.page_bytes;
  a.num_kv_heads = cfg.num_kv_heads;
  a.chunks_per_row = cfg.head_dim * ctx->esize / 16;
  a.swizzled = pv.swizzled;
  a.idx_layer_stride = idx_layer_stride;
  a.idx_head_stride = idx_head_stride;
  a.src_m = src.m;
  a.keep = dst.m;
  a.status = ctx->d_status;
  // one launch for all layers if they share page lists and places, else one per layer
  const long long max_pages = (1LL << 31) / ((long long)kPageSize * cfg.num_kv_heads);     // rows are counted in 32 bits
  const bool together = src.uniform && dst.uniform && ctx->uniform_caps &&
                        (long long)pages_of(dst, first_layer).size() * num_layers <= max_pages;
  const int step = together ? num_layers : 1;
  int list[kParamWords];
  for (int l = first_layer; l < first_layer + num_layers; l += step) {
    const std::vector<int32_t>&sp = pages_of(src, l), &dp = pages_of(dst, l);
    const int ns = (int)sp.size(), nd = (int)dp.size();
    const bool fits = ns + nd <= kParamWords;
    const int s_step = fits ? ns : kParamWords / 2;
    const int d_step = (int)std::min<long long>(fits ? nd : kParamWords / 2, max_pages);
    a.pool_k = static_cast<char*>(cfg.k_pool) + ctx->layer_off[l];
    a.pool_v = static_cast<char*>(cfg.v_pool) + ctx->layer_off[l];
    a.idx = idx + (l - first_layer) * idx_layer_stride;
    a.num_layers = step;
    for (int s0 = 0; s0 < ns; s0 += s_step)
      for (int d0 = 0; d0 < nd; d0 += d_step) {
        a.src_first = s0;
        a.src_pages = std::min(s_step, ns - s0);
        a.dst_first = d0;
        a.dst_pages = std::min(d_step, nd - d0);
        std::memcpy(list, sp.data() + s0, sizeof(int) * a.src_pages);
        std::memcpy(list + a.src_pages, dp.data() + d0, sizeof(int) * a.dst_pages);
        const int blocks = copy_blocks((long long)step * a.dst_pages * kPageSize * cfg.num_kv_heads, a.chunks_per_row, ctx->sm_count);
        with_param_list(list, a.src_pages + a.dst_pages, [&](const auto& params) {
          compact_prefix_kernel<<<blocks, kCompactThreads, 0, static_cast<cudaStream_t>(stream_)>>>(a, params);
        });
        ctx->launches++;
        const int st = cuda_status(ctx, cudaGetLastError(), "compact_prefix");
        if (st != BICACHE_OK) return st;
      }
  }
  return BICACHE_OK;
}

// ---- rotary positions ---------------------------------------------------------------------------

// Positions position0 .. position0 + rows - 1 that the angles hold: a frequency is off by up to 1.5 x 2^-64 turns, so 2^36
// positions on an angle is off by 3.5e-8 radians, which the rounding to fp32 hides; far beyond that it would not be.
bool rope_positions_ok(const int32_t* positions, int64_t position0, int64_t rows) {
  constexpr int64_t kFar = 1LL << 36;
  if (positions || rows == 0) return true;                        // 32-bit positions, or none
  return position0 >= -kFar && position0 <= kFar && rows - 1 <= kFar - position0;
}

// Frequencies to turns per position in 64-bit fixed point.
bool rope_angles(RopeAngles* a, int32_t rot_dim, const double* inv_freq, const int32_t* positions, int64_t position0,
                 float attention_scale, bool inverse) {
  if (!std::isfinite(attention_scale) || attention_scale == 0.f) return false;
  *a = RopeAngles();
  a->pairs = rot_dim / 2;
  for (int i = 0; i < a->pairs; ++i) {
    if (!(std::fabs(inv_freq[i]) <= 1048576.0)) return false;
    // |inv_freq| / (2 pi) to 2^-64 and better: the product with the leading part of 1 / (2 pi) as a sum of two
    // doubles, and the product with the rest of the constant.  The sign is put back at the end: taking a small
    // negative number modulo a turn as a double would cut it at 2^-54.
    const double f = std::fabs(inv_freq[i]), high = f * 0.15915494309189535;
    const double low = std::fma(f, 0.15915494309189535, -high) + f * -9.839338337591243e-18;
    const double part = high - std::floor(high);                  // exact; whole turns per position change nothing
    const unsigned long long turn = (unsigned long long)(part * 18446744073709551616.0) +
                                    (unsigned long long)(long long)std::nearbyint(low * 18446744073709551616.0);
    a->turn[i] = std::signbit(inv_freq[i]) ? 0ull - turn : turn;
  }
  a->positions = positions;
  a->position0 = position0;
  a->scale = inverse ? 1.f / attention_scale : attention_scale;
  if (!std::isfinite(a->scale)) return false;                     // the inverse of a subnormal scale
  a->negate = inverse ? 1 : 0;
  return true;
}

int rope_impl(bicache_ctx* ctx, int64_t rows, const int32_t* positions, int64_t position0, int32_t rot_dim,
              int32_t interleaved, int32_t inverse, const double* inv_freq, float attention_scale, const void* q,
              int64_t q_row_stride, void* q_out, int64_t q_out_row_stride, const void* k, int64_t k_row_stride,
              void* k_out, int64_t k_out_row_stride, void* stream_) {
  if (!ctx) return BICACHE_ERR_INVALID;
  const bicache_config& cfg = ctx->cfg;
  if (rows < 0) return fail(ctx, BICACHE_ERR_INVALID, "negative row count");
  if (rot_dim < 2 || rot_dim > cfg.head_dim || rot_dim % 2)
    return fail(ctx, BICACHE_ERR_INVALID, "rot_dim must be even and within the head");
  if (!inv_freq) return fail(ctx, BICACHE_ERR_INVALID, "null frequencies");
  if (!aligned4(positions)) return fail(ctx, BICACHE_ERR_INVALID, "misaligned positions");
  if (!rope_positions_ok(positions, position0, rows)) return fail(ctx, BICACHE_ERR_INVALID, "positions beyond 2^36");
  RopeAngles a;
  if (!rope_angles(&a, rot_dim, inv_freq, positions, position0, attention_scale, inverse != 0))
    return fail(ctx, BICACHE_ERR_INVALID, "a frequency that is not finite or above 2^20, or a bad scale");
  RopeRows r = RopeRows();
  r.rows = rows;
  r.head_bytes = cfg.head_dim * ctx->esize;
  r.in_place = 1;
  const void* ins[2] = {q, k};
  void* outs[2] = {q_out, k_out};
  const int64_t in_strides[2] = {q_row_stride, k_row_stride}, out_strides[2] = {q_out_row_stride, k_out_row_stride};
  const int heads[2] = {cfg.num_q_heads, cfg.num_kv_heads};
  if (rows > 0 && !q && !k && !q_out && !k_out) return fail(ctx, BICACHE_ERR_INVALID, "nothing to rotate");
  if (rows > 0 && q_out && q_out == k_out) return fail(ctx, BICACHE_ERR_INVALID, "queries and keys have one output");
  for (int i = 0; i < 2 && rows > 0; ++i) {              // no rows: an empty tensor has no address
    if (!ins[i] != !outs[i]) return fail(ctx, BICACHE_ERR_INVALID, "a tensor without its output, or the reverse");
    if (!ins[i]) continue;
    if (!aligned16(ins[i]) || !aligned16(outs[i]))
      return fail(ctx, BICACHE_ERR_INVALID, "tensor pointer not 16-byte aligned");
    const int64_t least = (int64_t)heads[i] * cfg.head_dim;
    if (in_strides[i] < least || out_strides[i] < least || (in_strides[i] * ctx->esize) % 16 ||
        (out_strides[i] * ctx->esize) % 16)
      return fail(ctx, BICACHE_ERR_INVALID, "bad row stride");
    if (ins[i] == outs[i] && in_strides[i] != out_strides[i])
      return fail(ctx, BICACHE_ERR_INVALID, "in place with two row strides");
    r.t[i].in = static_cast<const char*>(ins[i]);
    r.t[i].out = static_cast<char*>(outs[i]);
    r.t[i].in_stride = in_strides[i] * ctx->esize;
    r.t[i].out_stride = out_strides[i] * ctx->esize;
    r.t[i].heads = heads[i];
    if (ins[i] != outs[i]) r.in_place = 0;
  }
  if (ctx->host_only) return fail(ctx, BICACHE_ERR_UNSUPPORTED, "host-only context has no device path");
  if (rows == 0) return BICACHE_OK;
  DeviceGuard guard(cfg.device);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  const cudaError_t e = cfg.dtype == BICACHE_F32
                            ? launch_rope<float>(a, r, interleaved != 0, ctx->sm_count, stream)
                            : launch_rope<__nv_bfloat16>(a, r, interleaved != 0, ctx->sm_count, stream);
  ctx->launches++;
  return cuda_status(ctx, e, "rope");
}

int rope_table_impl(bicache_ctx* ctx, int64_t rows, const int32_t* positions, int64_t position0, int32_t rot_dim,
                    const double* inv_freq, float attention_scale, float* table, void* stream_) {
  if (!ctx) return BICACHE_ERR_INVALID;
  if (rows < 0) return fail(ctx, BICACHE_ERR_INVALID, "negative row count");
  if (rot_dim < 2 || rot_dim > 2 * kRopeMaxPairs || rot_dim % 2)
    return fail(ctx, BICACHE_ERR_INVALID, "rot_dim must be even, 2 to 256");
  if (!inv_freq) return fail(ctx, BICACHE_ERR_INVALID, "null frequencies");
  if ((rows > 0 && !table) || !aligned16(table) || !aligned4(positions)) return fail(ctx, BICACHE_ERR_INVALID, "bad pointer");
  if (!rope_positions_ok(positions, position0, rows)) return fail(ctx, BICACHE_ERR_INVALID, "positions beyond 2^36");
  RopeAngles a;
  if (!rope_angles(&a, rot_dim, inv_freq, positions, position0, attention_scale, false))
    return fail(ctx, BICACHE_ERR_INVALID, "a frequency that is not finite or above 2^20, or a bad scale");
  if (ctx->host_only) return fail(ctx, BICACHE_ERR_UNSUPPORTED, "host-only context has no device path");
  if (rows == 0) return BICACHE_OK;
  DeviceGuard guard(ctx->cfg.device);
  const int per_block = kRopeThreads / a.pairs;
  const int blocks = (int)std::min<long long>((rows + per_block - 1) / per_block, 2LL * ctx->sm_count);
  rope_table_kernel<<<blocks, kRopeThreads, 0, static_cast<cudaStream_t>(stream_)>>>(a, rows, reinterpret_cast<float2*>(table));
  ctx->launches++;
  return cuda_status(ctx, cudaGetLastError(), "rope_table");
}

cudaError_t configure_token_ops(bool tensor_ok) {
  cudaError_t e = cudaFuncSetAttribute(select_tokens_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelStaged * 4);
  each_param_length([&](auto words) {
    constexpr int kWords = decltype(words)::value;
    auto allow = [&](const void* kernel, int most, int per_thread) {
      if (e == cudaSuccess)
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)weights_simt_smem(most, per_thread));
    };
    allow((const void*)weights_simt_kernel<float, 8, kWords>, kWsEightMaxD, 8);
    allow((const void*)weights_simt_kernel<__nv_bfloat16, 8, kWords>, kWsEightMaxD, 8);
    allow((const void*)weights_simt_kernel<float, 4, kWords>, kSimtMaxD, 4);
    allow((const void*)weights_simt_kernel<__nv_bfloat16, 4, kWords>, kSimtMaxD, 4);
  }, ParamLengths());
  if (e == cudaSuccess && tensor_ok) e = configure_tc_weights();
  return e;
}

}  // namespace

extern "C" {

int32_t bicache_prefix_weights(bicache_ctx* ctx, int32_t layer, int32_t R, const int32_t* prefix_id,
                               const int64_t* row_off, const int32_t* seqlen, const void* q, int64_t q_row_stride,
                               const float* lse, const float* scores_in, float* scores_out,
                               const int64_t* score_off, int64_t score_head_stride, float decay,
                               float softmax_scale, void* stream) {
  return guarded([&]() {
    return prefix_weights_impl(ctx, layer, R, prefix_id, row_off, seqlen, q, q_row_stride, lse, scores_in, scores_out,
                               score_off, score_head_stride, decay, softmax_scale, stream);
  });
}

int32_t bicache_select_tokens(bicache_ctx* ctx, int64_t rows, int32_t n, const float* scores, int64_t score_row_stride,
                              int32_t keep, int32_t protect_first, int32_t protect_last, int32_t* idx_out,
                              int64_t idx_row_stride, void* stream) {
  return guarded([&]() -> int32_t {
    if (!ctx) return BICACHE_ERR_INVALID;
    if (rows < 0 || rows > 0x7fffffffLL || n < 0 || n > (1 << 30) || keep < 0 || keep > n || protect_first < 0 || protect_last < 0)
      return fail(ctx, BICACHE_ERR_INVALID, "bad row count, length, keep or protected count");
    SelectArgs a;
    a.first = std::min(protect_first, n);
    a.last = std::min(protect_last, n - a.first);
    if (keep < a.first + a.last) return fail(ctx, BICACHE_ERR_INVALID, "fewer tokens kept than protected");
    if (rows > 0 && keep > 0 && (!scores || !idx_out || !aligned4(scores) || !aligned4(idx_out)))
      return fail(ctx, BICACHE_ERR_INVALID, "bad pointer");
    if (rows > 1 && (score_row_stride < n || idx_row_stride < keep))
      return fail(ctx, BICACHE_ERR_INVALID, "bad row stride");
    if (ctx->host_only) return fail(ctx, BICACHE_ERR_UNSUPPORTED, "host-only context has no device path");
    if (rows == 0 || keep == 0) return BICACHE_OK;
    a.scores = scores;
    a.score_stride = score_row_stride;
    a.idx = idx_out;
    a.idx_stride = idx_row_stride;
    a.n = n;
    a.keep = keep;
    DeviceGuard guard(ctx->cfg.device);
    const cudaError_t e = launch_select(a, rows, ctx->sm_count, static_cast<cudaStream_t>(stream));
    ctx->launches++;
    return cuda_status(ctx, e, "select_tokens");
  });
}

int32_t bicache_compact_prefix(bicache_ctx* ctx, int32_t src_id, int32_t dst_id, int32_t first_layer,
                               int32_t num_layers, int32_t keep, const int32_t* idx, int64_t idx_layer_stride,
                               int64_t idx_head_stride, void* stream) {
  return guarded([&]() {
    return compact_prefix_impl(ctx, src_id, dst_id, first_layer, num_layers, keep, idx, idx_layer_stride, idx_head_stride, stream);
  });
}

int32_t bicache_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor,
                                 int32_t original_length, double low_turns, double high_turns, double* inv_freq) {
  const bool bands = scaling == BICACHE_ROPE_YARN || scaling == BICACHE_ROPE_BANDS;
  if (rot_dim < 2 || rot_dim > 2 * kRopeMaxPairs || rot_dim % 2 || !inv_freq || !std::isfinite(base) || base <= 1.0 ||
      scaling < BICACHE_ROPE_NONE || scaling > BICACHE_ROPE_BANDS)
    return BICACHE_ERR_INVALID;
  if (scaling != BICACHE_ROPE_NONE && (!std::isfinite(factor) || factor <= 0.0)) return BICACHE_ERR_INVALID;
  if (bands && (original_length < 1 || !std::isfinite(high_turns) || !(low_turns > 0.0) || !(high_turns > low_turns)))
    return BICACHE_ERR_INVALID;
  const double two_pi = 6.283185307179586476925286766559;
  double b = base;
  if (scaling == BICACHE_ROPE_NTK && rot_dim > 2) b = base * std::pow(factor, (double)rot_dim / (rot_dim - 2));
  // YARN: pair index at which the unscaled frequency turns `turns` times over the original length
  auto index_of = [&](double turns) {
    return rot_dim * std::log(original_length / (turns * two_pi)) / (2.0 * std::log(base));
  };
  double lo = 0.0, hi = 0.0;
  if (scaling == BICACHE_ROPE_YARN) {
    lo = std::max(std::floor(index_of(high_turns)), 0.0);
    hi = std::min(std::ceil(index_of(low_turns)), rot_dim - 1.0);
  }
  double made[kRopeMaxPairs];
  for (int32_t i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(b, -2.0 * i / rot_dim);
    if (scaling == BICACHE_ROPE_LINEAR) {
      f /= factor;
    } else if (bands) {
      double slow = (i - lo) / std::max(hi - lo, 0.001);          // the share of interpolation
      if (scaling == BICACHE_ROPE_BANDS) slow = 1.0 - (original_length * f / two_pi - low_turns) / (high_turns - low_turns);
      slow = std::min(1.0, std::max(0.0, slow));
      f = f / factor * slow + f * (1.0 - slow);
    }
    if (!std::isfinite(f)) return BICACHE_ERR_INVALID;            // a factor so small that dividing by it overflows
    made[i] = f;
  }
  std::copy(made, made + rot_dim / 2, inv_freq);
  return BICACHE_OK;
}

int32_t bicache_rope(bicache_ctx* ctx, int64_t rows, const int32_t* positions, int64_t position0, int32_t rot_dim,
                     int32_t interleaved, int32_t inverse, const double* inv_freq, float attention_scale, const void* q,
                     int64_t q_row_stride, void* q_out, int64_t q_out_row_stride, const void* k, int64_t k_row_stride,
                     void* k_out, int64_t k_out_row_stride, void* stream) {
  return guarded([&]() {
    return rope_impl(ctx, rows, positions, position0, rot_dim, interleaved, inverse, inv_freq, attention_scale, q,
                     q_row_stride, q_out, q_out_row_stride, k, k_row_stride, k_out, k_out_row_stride, stream);
  });
}

int32_t bicache_rope_table(bicache_ctx* ctx, int64_t rows, const int32_t* positions, int64_t position0, int32_t rot_dim,
                           const double* inv_freq, float attention_scale, float* table, void* stream) {
  return guarded([&]() {
    return rope_table_impl(ctx, rows, positions, position0, rot_dim, inv_freq, attention_scale, table, stream);
  });
}

}  // extern "C"

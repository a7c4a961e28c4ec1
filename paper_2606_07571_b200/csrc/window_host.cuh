// C ABI entry points of a cache that grows token by token (see include/bicache.h): tokens into and out of live prefixes,
// windowed attention over them, rotary positions with several axes.  Included by bicache.cu, behind
// token_ops_host.cuh.
#pragma once

namespace {

// ---- rotations ----------------------------------------------------------------------------------

// A rotation as the kernels take it; what is wrong with it is recorded in the context.
int rotation_angles(const bicache_ctx* ctx, const bicache_rotation* rot, int max_dim, const int32_t* positions,
                    int64_t axis_stride, int64_t rows, bool inverse, RopeAxes* a) {
  if (rot->rot_dim < 2 || rot->rot_dim > max_dim || rot->rot_dim % 2)
    return fail(ctx, BICACHE_ERR_INVALID, "rot_dim must be even and within the head");
  if (rot->num_axes < 1 || rot->num_axes > kRopeMaxAxes) return fail(ctx, BICACHE_ERR_INVALID, "1 to 4 position axes");
  if (!rot->inv_freq) return fail(ctx, BICACHE_ERR_INVALID, "null frequencies");
  if (!aligned4(positions)) return fail(ctx, BICACHE_ERR_INVALID, "misaligned positions");
  if (rot->num_axes > 1 && axis_stride < rows)
    return fail(ctx, BICACHE_ERR_INVALID, "position axes shorter than the rows");
  if (!rope_angles(a, rot->rot_dim, rot->inv_freq, positions, 0, rot->attention_scale, inverse))
    return fail(ctx, BICACHE_ERR_INVALID, "a frequency that is not finite or above 2^20, or a bad scale");
  std::fill(a->axis, a->axis + kRopeMaxPairs / 16, 0u);
  a->axis_stride = axis_stride;
  for (int i = 0; rot->pair_axis && i < a->pairs; ++i) {
    if (rot->pair_axis[i] < 0 || rot->pair_axis[i] >= rot->num_axes)
      return fail(ctx, BICACHE_ERR_INVALID, "a pair turns with an axis that is not there");
    a->axis[i >> 4] |= (unsigned)rot->pair_axis[i] << (2 * (i & 15));
  }
  return BICACHE_OK;
}

int rope_axes_impl(bicache_ctx* ctx, int64_t rows, const bicache_rotation* rot, const int32_t* positions,
                   int64_t axis_stride, int32_t inverse, const void* q, int64_t q_row_stride, void* q_out,
                   int64_t q_out_row_stride, const void* k, int64_t k_row_stride, void* k_out, int64_t k_out_row_stride,
                   void* stream) {
  if (!ctx) return BICACHE_ERR_INVALID;
  if (rows < 0) return fail(ctx, BICACHE_ERR_INVALID, "negative row count");
  if (!rot) return fail(ctx, BICACHE_ERR_INVALID, "null rotation");
  if (rows > 0 && !positions) return fail(ctx, BICACHE_ERR_INVALID, "null positions");
  RopeAxes a;
  int st = rotation_angles(ctx, rot, ctx->cfg.head_dim, positions, axis_stride, rows, inverse != 0, &a);
  if (st != BICACHE_OK) return st;
  RopeRows r;
  st = rope_tensors(ctx, rows, q, q_row_stride, q_out, q_out_row_stride, k, k_row_stride, k_out, k_out_row_stride, &r);
  return st != BICACHE_OK ? st : run_rope(ctx, a, r, rot->interleaved != 0, stream);
}

// ---- tokens in and out --------------------------------------------------------------------------

// Does a row of a tensor belong to two requests?  (Rows that are written must not.)
bool rows_overlap(int32_t R, const int64_t* row_off, const int32_t* seqlen) {
  std::vector<std::pair<int64_t, int64_t>> spans;
  spans.reserve(R);
  for (int i = 0; i < R; ++i)
    if (seqlen[i] > 0) spans.emplace_back(row_off[i], row_off[i] + seqlen[i]);
  if (!std::is_sorted(spans.begin(), spans.end())) std::sort(spans.begin(), spans.end());
  for (size_t i = 1; i < spans.size(); ++i)
    if (spans[i].first < spans[i - 1].second) return true;
  return false;
}

// Lists of three lengths; with the angles beside the longest, a launch stays below the 32,764 bytes of its parameters.
constexpr int kTokenWords = 7552;
using TokenLengths = std::integer_sequence<int, 224, 2432, kTokenWords>;
static_assert(sizeof(RopeAxes) + sizeof(TokenArgs) + 64 + 4 * kTokenWords <= 32764, "launch parameters");

// Checks of a batch of (prefix, tokens, rows) triples; *rows_end receives the end of the last row, *entries the prefixes.
int check_tokens(const bicache_ctx* ctx, int32_t layer, int32_t R, const int32_t* prefix_id, const int32_t* token_off,
                 const int64_t* row_off, const int32_t* seqlen, bool write, int64_t* rows_end,
                 std::vector<const PrefixEntry*>* entries) {
  if (layer < 0 || layer >= ctx->cfg.num_layers) return fail(ctx, BICACHE_ERR_INVALID, "layer out of range");
  if (R < 0) return fail(ctx, BICACHE_ERR_INVALID, "negative request count");
  if (R > 0 && (!prefix_id || !token_off || !row_off || !seqlen)) return fail(ctx, BICACHE_ERR_INVALID, "null metadata array");
  struct Span { int32_t id, begin, end; };
  std::vector<Span> spans;
  spans.reserve(write ? std::max(R, 0) : 0);
  entries->reserve(std::max(R, 0));
  int64_t total = 0;
  *rows_end = 0;
  for (int i = 0; i < R; ++i) {
    if (seqlen[i] < 0 || row_off[i] < 0 || token_off[i] < 0)
      return fail(ctx, BICACHE_ERR_INVALID, "negative length or offset");
    if (row_off[i] > INT64_MAX - seqlen[i]) return fail(ctx, BICACHE_ERR_INVALID, "rows beyond 2^63");
    auto found = ctx->by_id.find(prefix_id[i]);
    if (found == ctx->by_id.end()) return fail(ctx, BICACHE_ERR_NOTFOUND, "unknown or evicted prefix id");
    const PrefixEntry& e = *found->second;
    entries->push_back(&e);
    if (e.first_layer > layer) return fail(ctx, BICACHE_ERR_INVALID, "the prefix owns no pages in this layer");
    if (seqlen[i] > e.m || token_off[i] > e.m - seqlen[i])
      return fail(ctx, BICACHE_ERR_INVALID, "tokens past the end of the prefix");
    if (seqlen[i] == 0) continue;
    total += seqlen[i] + 1LL;
    *rows_end = std::max(*rows_end, row_off[i] + seqlen[i]);
    if (write) spans.push_back(Span{prefix_id[i], token_off[i], token_off[i] + seqlen[i]});
  }
  if (total > 0x7fffffffLL) return fail(ctx, BICACHE_ERR_INVALID, "batch too large");
  auto before = [](const Span& x, const Span& y) { return x.id != y.id ? x.id < y.id : x.begin < y.begin; };
  if (!std::is_sorted(spans.begin(), spans.end(), before)) std::sort(spans.begin(), spans.end(), before);
  for (size_t i = 1; i < spans.size(); ++i)
    if (spans[i].id == spans[i - 1].id && spans[i].begin < spans[i - 1].end)
      return fail(ctx, BICACHE_ERR_INVALID, "a token is written twice");
  return BICACHE_OK;
}

// The launches of one call: runs are added until the parameter list is full.  launch(list, runs, tokens) is made for
// every full list and for the rest.
template <typename F>
int token_launches(int32_t layer, const std::vector<const PrefixEntry*>& entries, const int32_t* token_off,
                   const int64_t* row_off, const int32_t* seqlen, bool write, F&& launch) {
  alignas(8) int list[kTokenWords];
  std::vector<TokenRun> runs;
  std::vector<int32_t> pages;
  int tokens = 0;
  auto flush = [&]() -> int {
    if (runs.empty()) return BICACHE_OK;
    const int words = (int)runs.size() * kRunWords;
    for (TokenRun& r : runs) r.page_word += words;
    std::memcpy(list, runs.data(), sizeof(TokenRun) * runs.size());
    std::memcpy(list + words, pages.data(), sizeof(int32_t) * pages.size());
    const int st = launch(list, words + (int)pages.size(), (int)runs.size(), tokens);
    runs.clear();
    pages.clear();
    tokens = 0;
    return st;
  };
  runs.reserve(entries.size());
  pages.reserve(2 * entries.size());
  for (size_t i = 0; i < entries.size(); ++i) {
    const PrefixEntry& e = *entries[i];
    const std::vector<int32_t>& own = pages_of(e, layer);
    for (int done = 0; done < seqlen[i];) {
      const int token = token_off[i] + done, page = token / kPageSize;
      const int room = kTokenWords - (int)(runs.size() + 1) * kRunWords - (int)pages.size();
      const int last = (token_off[i] + seqlen[i] - 1) / kPageSize;
      if (room < std::min(last - page + 1, 64)) {                    // few pages left: not worth a cut
        const int st = flush();
        if (st != BICACHE_OK) return st;
        continue;
      }
      const int take = std::min(last - page + 1, room);
      TokenRun r = TokenRun();
      r.row = row_off[i] + done;
      r.start = tokens;
      r.n = std::min(seqlen[i] - done, (page + take) * kPageSize - token);
      r.token = token;
      r.clear = e.m;
      r.page_word = (int)pages.size();
      pages.insert(pages.end(), own.begin() + page, own.begin() + page + take);
      runs.push_back(r);
      done += r.n;
      const bool ends = write && page + take == (int)own.size();     // the prefix's last page is among them
      tokens += r.n + (ends && e.m % kPageSize ? 1 : 0);
    }
  }
  return flush();
}

TokenArgs token_args(const bicache_ctx* ctx, int32_t layer) {
  const bicache_config& cfg = ctx->cfg;
  const PoolView pv = pool_view_layer(ctx, layer);
  TokenArgs g = TokenArgs();
  g.pool_k = const_cast<char*>(pv.k);
  g.pool_v = const_cast<char*>(pv.v);
  g.page_bytes = pv.page_bytes;
  g.page_stride = (long long)pv.page_bytes * cfg.num_kv_heads;
  g.swizzled = pv.swizzled;
  g.Hq = cfg.num_q_heads;
  g.Hkv = cfg.num_kv_heads;
  g.head_bytes = cfg.head_dim * ctx->esize;
  return g;
}

int append_tokens_impl(bicache_ctx* ctx, int32_t layer, int32_t R, const int32_t* prefix_id, const int32_t* token_off,
                       const int64_t* row_off, const int32_t* seqlen, const void* k, const void* v, int64_t kv_row_stride,
                       const void* q, int64_t q_row_stride, void* q_out, int64_t q_out_row_stride,
                       const bicache_rotation* rot, const int32_t* positions, int64_t axis_stride, void* stream_) {
  if (!ctx) return BICACHE_ERR_INVALID;
  const bicache_config& cfg = ctx->cfg;
  int64_t rows_end = 0;
  std::vector<const PrefixEntry*> entries;
  int st = check_tokens(ctx, layer, R, prefix_id, token_off, row_off, seqlen, true, &rows_end, &entries);
  if (st != BICACHE_OK) return st;
  const int64_t kv_least = (int64_t)cfg.num_kv_heads * cfg.head_dim, q_least = (int64_t)cfg.num_q_heads * cfg.head_dim;
  if (rows_end > 0) {
    if (!k || !v || !aligned16(k) || !aligned16(v)) return fail(ctx, BICACHE_ERR_INVALID, "bad k/v pointer");
    if (kv_row_stride < kv_least || (kv_row_stride * ctx->esize) % 16) return fail(ctx, BICACHE_ERR_INVALID, "bad row stride");
    if (!q != !q_out) return fail(ctx, BICACHE_ERR_INVALID, "queries without their output, or the reverse");
    if (q) {
      if (!rot) return fail(ctx, BICACHE_ERR_INVALID, "queries without a rotation");
      if (rows_overlap(R, row_off, seqlen)) return fail(ctx, BICACHE_ERR_INVALID, "a query row belongs to two requests");
      if (!aligned16(q) || !aligned16(q_out)) return fail(ctx, BICACHE_ERR_INVALID, "tensor pointer not 16-byte aligned");
      if (q_row_stride < q_least || q_out_row_stride < q_least || (q_row_stride * ctx->esize) % 16 ||
          (q_out_row_stride * ctx->esize) % 16)
        return fail(ctx, BICACHE_ERR_INVALID, "bad row stride");
      if (q == q_out && q_row_stride != q_out_row_stride) return fail(ctx, BICACHE_ERR_INVALID, "in place with two row strides");
      if (q_out == k || q_out == v) return fail(ctx, BICACHE_ERR_INVALID, "queries are written over keys or values");
    }
  }
  RopeAxes a = RopeAxes();
  if (rot) {
    if (rot->num_axes > 1 && rows_end > 0 && !positions) return fail(ctx, BICACHE_ERR_INVALID, "null positions");
    st = rotation_angles(ctx, rot, cfg.head_dim, positions, axis_stride, rows_end, false, &a);
    if (st != BICACHE_OK) return st;
  }
  if (ctx->host_only) return fail(ctx, BICACHE_ERR_UNSUPPORTED, "host-only context has no device path");
  if (rows_end == 0) return BICACHE_OK;
  DeviceGuard guard(cfg.device);
  TokenArgs g = token_args(ctx, layer);
  g.q = static_cast<const char*>(q);
  g.k = static_cast<const char*>(k);
  g.v = static_cast<const char*>(v);
  g.q_out = static_cast<char*>(q_out);
  g.q_stride = q_row_stride * ctx->esize;
  g.q_out_stride = q_out_row_stride * ctx->esize;
  g.kv_stride = kv_row_stride * ctx->esize;
  g.q_in_place = q == q_out ? 1 : 0;
  g.pairs = a.pairs;
  const bool interleaved = rot && rot->interleaved;
  const bool axes = rot && rot->num_axes > 1;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  return token_launches(layer, entries, token_off, row_off, seqlen, true, [&](const int* list, int words, int runs, int tokens) {
    g.num_runs = runs;
    g.tokens = tokens;
    cudaError_t e = cudaSuccess;
    with_param_list(list, words, [&](const auto& params) {
      auto typed = [&](auto zero) {
        using T = decltype(zero);
        e = axes ? launch_append<T>(a, g, interleaved, params, ctx->sm_count, stream)
                 : launch_append<T>(static_cast<const RopeAngles&>(a), g, interleaved, params, ctx->sm_count, stream);
      };
      if (cfg.dtype == BICACHE_F32) typed(0.f);
      else typed(__nv_bfloat16());
    }, TokenLengths());
    ctx->launches++;
    return cuda_status(ctx, e, "append_tokens");
  });
}

int read_tokens_impl(bicache_ctx* ctx, int32_t layer, int32_t R, const int32_t* prefix_id, const int32_t* token_off,
                     const int64_t* row_off, const int32_t* seqlen, void* k_out, void* v_out, int64_t kv_row_stride,
                     void* stream_) {
  if (!ctx) return BICACHE_ERR_INVALID;
  const bicache_config& cfg = ctx->cfg;
  int64_t rows_end = 0;
  std::vector<const PrefixEntry*> entries;
  const int st = check_tokens(ctx, layer, R, prefix_id, token_off, row_off, seqlen, false, &rows_end, &entries);
  if (st != BICACHE_OK) return st;
  if (rows_end > 0) {
    if (!k_out || !v_out || !aligned16(k_out) || !aligned16(v_out) || k_out == v_out)
      return fail(ctx, BICACHE_ERR_INVALID, "bad k/v pointer");
    if (rows_overlap(R, row_off, seqlen)) return fail(ctx, BICACHE_ERR_INVALID, "a row belongs to two requests");
    if (kv_row_stride < (int64_t)cfg.num_kv_heads * cfg.head_dim || (kv_row_stride * ctx->esize) % 16)
      return fail(ctx, BICACHE_ERR_INVALID, "bad row stride");
  }
  if (ctx->host_only) return fail(ctx, BICACHE_ERR_UNSUPPORTED, "host-only context has no device path");
  if (rows_end == 0) return BICACHE_OK;
  DeviceGuard guard(cfg.device);
  TokenArgs g = token_args(ctx, layer);
  g.k_out = static_cast<char*>(k_out);
  g.v_out = static_cast<char*>(v_out);
  g.kv_stride = kv_row_stride * ctx->esize;
  return token_launches(layer, entries, token_off, row_off, seqlen, false, [&](const int* list, int words, int runs, int tokens) {
    g.num_runs = runs;
    g.tokens = tokens;
    cudaError_t e = cudaSuccess;
    with_param_list(list, words, [&](const auto& params) {
      e = launch_read_tokens(g, params, ctx->sm_count, static_cast<cudaStream_t>(stream_));
    }, TokenLengths());
    ctx->launches++;
    return cuda_status(ctx, e, "read_tokens");
  });
}

// ---- windowed attention -------------------------------------------------------------------------

using WindowLengths = std::integer_sequence<int, 224, 2432, kParamWords>;
using WindowSimtLengths = std::integer_sequence<int, 224, kParamWords>;
static_assert(sizeof(WindowArgs) + 64 + 4 * kParamWords <= 32764, "launch parameters");

// What a kernel form takes at a time, and what its work items cost, in key tiles.
struct WindowForm {
  int tile_rows, tile_keys;
  int slots;                    // work items that run at a time
  double item_cost;             // start and end of a work item
  double join_cost;             // the joining kernel, and what it takes for a row-head of a range
  double join_row_head_cost;
  int max_splits;               // ranges of keys
  int list_words;               // what a launch's list holds
};

// The launches of one call and one kernel form.  Requests are added until the parameter list holds no more records; their
// page lists stand behind the records, or, if they are too long for that, in the workspace, where launches of
// their own write them.  (64 tokens over 31,000 pages that do not follow one another: four launches of what a list holds,
// each with its join, took 280 us, this takes 264.)
class WindowLaunches {
 public:
  WindowLaunches(bicache_ctx* ctx, const WindowArgs& args, const WindowForm& form, cudaStream_t stream)
      : ctx_(ctx), base_(args), form_(form), stream_(stream) {}
  virtual ~WindowLaunches() {}

  int add(long long row, int n, int pos, int len, const std::vector<int32_t>& pages, bool consecutive) {
    Pending p;
    p.r = WindowReq();
    p.r.row = row;
    p.r.n = n;
    p.r.pos = pos;
    p.r.len = len;
    const WindowPages w = window_pages(base_.sinks, base_.left, base_.right, len, pos, pos + n - 1);
    p.r.sink_pages = w.sink_pages;
    p.r.gap = w.lo_page - w.sink_pages;
    const int G = base_.Hq / base_.Hkv;
    p.r.row_tiles = (int)(((long long)n * G + form_.tile_rows - 1) / form_.tile_rows);
    for (int t = 0; t < p.r.row_tiles; ++t) {
      const int first = (int)((long long)t * form_.tile_rows / G);
      const int last = (int)((std::min((long long)(t + 1) * form_.tile_rows, (long long)n * G) - 1) / G);
      const int count = window_pages(base_.sinks, base_.left, base_.right, len, pos + first, pos + last).count;
      const int tiles = (count * kPageSize + form_.tile_keys - 1) / form_.tile_keys;
      p.max_tiles = std::max(p.max_tiles, tiles);
      p.sum_tiles += tiles;
    }
    p.r.first_page = consecutive ? pages[0] : -1;
    const int listed = consecutive ? 0 : w.count;
    const long long records = (long long)(pending_.size() + 1) * kWindowReqWords, all = (long long)pages_.size() + listed;
    if (records > form_.list_words || (records + all > form_.list_words && all > ctx_->cfg.num_pages)) {
      const int st = flush();                             // one request alone has no more pages than the pool
      if (st != BICACHE_OK) return st;
    }
    p.r.page_word = (int)pages_.size();
    if (listed > 0) {
      const auto behind = pages.begin() + w.sink_pages + p.r.gap;
      pages_.insert(pages_.end(), pages.begin(), pages.begin() + w.sink_pages);
      pages_.insert(pages_.end(), behind, behind + (w.count - w.sink_pages));
    }
    pending_.push_back(p);
    return BICACHE_OK;
  }

  int flush() {
    if (pending_.empty()) return BICACHE_OK;
    WindowArgs a = base_;
    cudaError_t e = cudaSuccess;
    const int words = (int)pending_.size() * kWindowReqWords;
    if (words + (long long)pages_.size() > form_.list_words) {
      a.staged_pages = ctx_->d_put_pages;
      for (size_t at = 0; at < pages_.size() && e == cudaSuccess; at += kParamWords) {
        const int count = (int)std::min<size_t>(kParamWords, pages_.size() - at);
        alignas(8) int part[kParamWords];
        std::memcpy(part, pages_.data() + at, sizeof(int) * count);
        with_param_list(part, count, [&](const auto& list) {
          stage_pages_kernel<<<(count + 255) / 256, 256, 0, stream_>>>(ctx_->d_put_pages + at, count, list);
        }, WindowSimtLengths());
        ctx_->launches++;
        e = cudaGetLastError();
      }
      if (e != cudaSuccess) return cuda_status(ctx_, e, "attend_window");
    }
    // long ones first: the short items of the others even out what these leave
    std::stable_sort(pending_.begin(), pending_.end(), [](const Pending& x, const Pending& y) { return x.max_tiles > y.max_tiles; });
    const int tps = choose_tiles_per_split();
    long long items = 0, part = 0;
    for (size_t i = 0; i < pending_.size(); ++i) {
      Pending& p = pending_[i];
      p.r.splits = splits_of(p, tps);
      p.r.tiles_per_split = std::max(1, (p.max_tiles + p.r.splits - 1) / p.r.splits);
      p.r.item_begin = (int)items;
      p.r.part_off = p.r.row_heads_before = 0;
      p.r.page_word += a.staged_pages ? 0 : words;
      items += (long long)p.r.row_tiles * a.Hkv * p.r.splits;
    }
    int row_heads = 0;
    for (Pending& p : pending_) {
      p.r.part_off = (int)part;
      p.r.row_heads_before = row_heads;
      if (p.r.splits > 1) {
        part += (long long)p.r.splits * p.r.n * a.Hq;
        row_heads += p.r.n * a.Hq;
      }
    }
    alignas(8) int list[kParamWords];
    for (size_t i = 0; i < pending_.size(); ++i) std::memcpy(list + i * kWindowReqWords, &pending_[i].r, sizeof(WindowReq));
    if (!a.staged_pages) std::memcpy(list + words, pages_.data(), sizeof(int) * pages_.size());
    const int used = words + (a.staged_pages ? 0 : (int)pages_.size());
    a.num_reqs = (int)pending_.size();
    a.num_items = (int)items;
    int most_splits = 1;
    for (const Pending& p : pending_) most_splits = std::max(most_splits, p.r.splits);
    pending_.clear();
    pages_.clear();
    if (items > 0x7fffffffLL) return fail(ctx_, BICACHE_ERR_INVALID, "batch too large");
    e = launch(a, list, used);
    ctx_->launches++;
    if (e == cudaSuccess && row_heads > 0) {
      e = join(a, list, words, row_heads, most_splits);     // needs no pages
      ctx_->launches++;
    }
    return cuda_status(ctx_, e, "attend_window");
  }

 protected:
  virtual cudaError_t launch(const WindowArgs& a, const int* list, int words) = 0;
  virtual const int* status() const { return nullptr; }      // asked by the joining kernel

  bicache_ctx* ctx_;
  WindowArgs base_;
  WindowForm form_;
  cudaStream_t stream_;

 private:
  struct Pending {
    WindowReq r;
    int max_tiles = 0;          // key tiles of a row tile, at most
    long long sum_tiles = 0;    // of all row tiles
  };
  int splits_of(const Pending& p, int tps) const {
    return std::min(form_.max_splits, std::max(1, (p.max_tiles + tps - 1) / tps));
  }
  // How many key tiles an item covers at most.  Counted in key tiles: what a slot has to do on the average, and half
  // an item at the end, or the longest item if there is no more than one to a slot.
  int choose_tiles_per_split() const {
    int max_tiles = 1;
    for (const Pending& p : pending_) max_tiles = std::max(max_tiles, p.max_tiles);
    int best_tps = max_tiles;
    double best = 1e300;
    for (int s = 1, before = 0; s <= form_.max_splits && s <= max_tiles; ++s) {
      const int tps = (max_tiles + s - 1) / s;
      if (tps == before) continue;
      before = tps;
      long long items = 0, tiles = 0, part = 0;
      for (const Pending& p : pending_) {
        const int sp = splits_of(p, tps);
        items += (long long)p.r.row_tiles * base_.Hkv * sp;
        tiles += p.sum_tiles * base_.Hkv;
        if (sp > 1) part += (long long)sp * p.r.n * base_.Hq;
      }
      if (part > ctx_->part_capacity_rowheads) break;
      if (s > 1 && items > 4LL * form_.slots) break;         // enough to even out: more would only start more often
      const double longest = tps + form_.item_cost;
      const double mean = (double)(tiles + items * form_.item_cost) / form_.slots;
      const double cost = (items <= form_.slots ? longest : std::max(longest, mean + longest / 2)) + (part > 0 ? form_.join_cost + form_.join_row_head_cost * part : 0.0);
      if (cost < best) {
        best = cost;
        best_tps = tps;
      }
    }
    return best_tps;
  }
  cudaError_t join(const WindowArgs& a, const int* list, int words, int row_heads, int most_splits) {
    cudaError_t e = cudaSuccess;
    const bool share = most_splits > 16;                     // many ranges: spread them over the block's warps
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(share ? row_heads : (row_heads + kJoinWarps - 1) / kJoinWarps), 1, 1);
    cfg.blockDim = dim3(kJoinWarps * 32, 1, 1);
    cfg.stream = stream_;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    with_param_list(list, words, [&](const auto& params) {
      constexpr int kWords = sizeof(params.w) / sizeof(int);
      auto typed = [&](auto zero) {
        using T = decltype(zero);
        e = share ? cudaLaunchKernelEx(&cfg, window_join_kernel<T, kJoinWarps, kWords>, a, row_heads, status(), params)
                  : cudaLaunchKernelEx(&cfg, window_join_kernel<T, 1, kWords>, a, row_heads, status(), params);
      };
      if (ctx_->cfg.dtype == BICACHE_F32) typed(0.f);
      else typed(__nv_bfloat16());
    }, WindowLengths());
    return e;
  }

  std::vector<Pending> pending_;
  std::vector<int32_t> pages_;
};

// f(T, rows, largest head dim) as integral constants, of the CUDA-core kernel that serves a type, row tile and head dim
template <typename F>
void with_window_simt(int dtype, int rows, int D, F&& f) {
  auto dims = [&](auto zero, auto r) {
    if (D == 64) f(zero, r, std::integral_constant<int, 64>());
    else if (D == 128) f(zero, r, std::integral_constant<int, 128>());
    else f(zero, r, std::integral_constant<int, kWinAnyD>());
  };
  auto tiles = [&](auto zero) {
    if (rows == 16) dims(zero, std::integral_constant<int, 16>());
    else dims(zero, std::integral_constant<int, 64>());
  };
  if (dtype == BICACHE_F32) tiles(0.f);
  else tiles(__nv_bfloat16());
}

class WindowSimtLaunches : public WindowLaunches {
 public:
  WindowSimtLaunches(bicache_ctx* ctx, const WindowArgs& args, int rows, cudaStream_t stream)
      : WindowLaunches(ctx, args, form_of(ctx, rows), stream) {}

 protected:
  static WindowForm form_of(const bicache_ctx* ctx, int rows) {
    return WindowForm{rows, kWinKeys, window_simt_blocks(rows, ctx->cfg.head_dim) * ctx->sm_count, 2, 2, 1e-4, kMaxWindowSplits, kParamWords};
  }
  cudaError_t launch(const WindowArgs& a, const int* list, int words) override {
    const size_t smem = window_simt_smem(form_.tile_rows, a.D);
    with_param_list(list, words, [&](const auto& params) {
      constexpr int kWords = sizeof(params.w) / sizeof(int);
      with_window_simt(ctx_->cfg.dtype, form_.tile_rows, a.D, [&](auto zero, auto rows, auto dim) {
        window_simt_kernel<decltype(zero), decltype(rows)::value, decltype(dim)::value, kWords>
            <<<(unsigned)a.num_items, kWinThreads, smem, stream_>>>(a, params);
      });
    }, WindowSimtLengths());
    return cudaGetLastError();
  }
};

class WindowTensorLaunches : public WindowLaunches {
 public:
  WindowTensorLaunches(bicache_ctx* ctx, const WindowArgs& args, cudaStream_t stream)
      : WindowLaunches(ctx, args, WindowForm{128, dec::kKeys, 2 * ctx->sm_count, 4, 5, 2e-4, kMaxWindowSplits, kParamWords}, stream) {}

 protected:
  cudaError_t launch(const WindowArgs& a, const int* list, int words) override {
    cudaError_t e = cudaSuccess;
    with_param_list(list, words, [&](const auto& params) {
      e = launch_tc_window(a, params, ctx_->d_status, ctx_->wait_cycles, stream_);
    }, WindowLengths());
    return e;
  }
  const int* status() const override { return ctx_->d_status; }
};

// Row tiles of 256: for requests with more rows than one work item of the other form takes.
class WindowTileLaunches : public WindowLaunches {
 public:
  WindowTileLaunches(bicache_ctx* ctx, const WindowArgs& args, const TcTensorMaps& maps, cudaStream_t stream)
      : WindowLaunches(ctx, args, WindowForm{kTileRows, kTileKeys, ctx->sm_count, 0, 0, 0, 1, kWindowTileWords}, stream), maps_(maps) {}

 protected:
  cudaError_t launch(const WindowArgs& a, const int* list, int words) override {
    TensorArgs t = TensorArgs();
    t.q = a.q;
    t.out = a.out;
    t.lse = a.lse;
    t.q_stride = a.q_stride;
    t.out_stride = a.out_stride;
    t.Hq = a.Hq;
    t.Hkv = a.Hkv;
    t.D = a.D;
    t.scale = a.scale;
    cudaError_t e = cudaSuccess;
    with_param_list(list, words, [&](const auto& params) {
      constexpr int kWords = sizeof(params.w) / sizeof(int);
      e = launch_tc_window_tiles(WindowBatch<kWords>{a, params}, t, ctx_->d_status, ctx_->sm_count, maps_, ctx_->wait_cycles, stream_);
    }, WindowTileLengths());
    return e;
  }

 private:
  TcTensorMaps maps_;
};

int attend_window_impl(bicache_ctx* ctx, int32_t layer, int32_t R, const int32_t* prefix_id, const int32_t* cached_len,
                       const int32_t* query_pos, const int64_t* row_off, const int32_t* seqlen, const void* q,
                       int64_t q_row_stride, void* out, int64_t out_row_stride, float* lse_out, int32_t sinks,
                       int32_t left, int32_t right, float softmax_scale, void* stream_) {
  if (!ctx) return BICACHE_ERR_INVALID;
  const bicache_config& cfg = ctx->cfg;
  if (layer < 0 || layer >= cfg.num_layers) return fail(ctx, BICACHE_ERR_INVALID, "layer out of range");
  if (R < 0) return fail(ctx, BICACHE_ERR_INVALID, "negative request count");
  if (sinks < 0 || left < -1 || right < -1) return fail(ctx, BICACHE_ERR_INVALID, "negative window");
  if (!std::isfinite(softmax_scale)) return fail(ctx, BICACHE_ERR_INVALID, "the scale must be finite");
  if (R > 0 && (!prefix_id || !cached_len || !query_pos || !row_off || !seqlen))
    return fail(ctx, BICACHE_ERR_INVALID, "null metadata array");
  int64_t total = 0;
  std::vector<const PrefixEntry*> entries(std::max(R, 0), nullptr);
  for (int i = 0; i < R; ++i) {
    if (seqlen[i] < 0 || row_off[i] < 0 || query_pos[i] < 0 || cached_len[i] < 0)
      return fail(ctx, BICACHE_ERR_INVALID, "negative length, offset or position");
    if (row_off[i] > INT64_MAX - seqlen[i]) return fail(ctx, BICACHE_ERR_INVALID, "rows beyond 2^63");
    if (query_pos[i] > 0x7fffffff - seqlen[i]) return fail(ctx, BICACHE_ERR_INVALID, "positions beyond 2^31");
    total += seqlen[i];
    if (prefix_id[i] < -1) return fail(ctx, BICACHE_ERR_INVALID, "bad prefix id");
    if (prefix_id[i] < 0) {
      if (cached_len[i] > 0) return fail(ctx, BICACHE_ERR_INVALID, "cached tokens without a prefix");
      continue;
    }
    auto found = ctx->by_id.find(prefix_id[i]);
    if (found == ctx->by_id.end()) return fail(ctx, BICACHE_ERR_NOTFOUND, "unknown or evicted prefix id");
    if (found->second->first_layer > layer) return fail(ctx, BICACHE_ERR_INVALID, "the prefix owns no pages in this layer");
    entries[i] = &*found->second;
    if (cached_len[i] > found->second->m) return fail(ctx, BICACHE_ERR_INVALID, "more cached tokens than the prefix holds");
  }
  const int G = cfg.num_q_heads / cfg.num_kv_heads;
  if (total > 0x7fffff00LL / G) return fail(ctx, BICACHE_ERR_INVALID, "batch too large");
  if (total > 0) {
    if (!q || !out || !aligned16(q) || !aligned16(out) || !aligned4(lse_out))
      return fail(ctx, BICACHE_ERR_INVALID, "bad tensor pointer");
    if (q == out) return fail(ctx, BICACHE_ERR_INVALID, "the output must not be the queries");
    if (rows_overlap(R, row_off, seqlen)) return fail(ctx, BICACHE_ERR_INVALID, "a row belongs to two requests");
    const int64_t least = (int64_t)cfg.num_q_heads * cfg.head_dim;
    if (q_row_stride < least || out_row_stride < least || (q_row_stride * ctx->esize) % 16 || (out_row_stride * ctx->esize) % 16)
      return fail(ctx, BICACHE_ERR_INVALID, "bad row stride");
  }
  if (ctx->host_only) return fail(ctx, BICACHE_ERR_UNSUPPORTED, "host-only context has no device path");
  if (total == 0) return BICACHE_OK;
  DeviceGuard guard(cfg.device);
  const PoolView pool = pool_view_layer(ctx, layer);
  WindowArgs a = WindowArgs();
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse_out;
  a.q_stride = q_row_stride;
  a.out_stride = out_row_stride;
  a.pool_k = pool.k;
  a.pool_v = pool.v;
  a.page_bytes = pool.page_bytes;
  a.page_stride = (long long)pool.page_bytes * cfg.num_kv_heads;
  a.swizzled = pool.swizzled;
  a.Hq = cfg.num_q_heads;
  a.Hkv = cfg.num_kv_heads;
  a.D = cfg.head_dim;
  a.sinks = sinks;
  a.left = left;
  a.right = right;
  a.scale = softmax_scale;
  a.part_o = ctx->d_part_o;
  a.part_lse = ctx->d_part_lse;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  static const std::vector<int32_t> no_pages;
  // the requests of one kernel form after the other
  auto run = [&](WindowLaunches& launches, auto&& takes) -> int {
    for (int i = 0; i < R; ++i) {
      if (seqlen[i] == 0 || !takes(seqlen[i])) continue;
      const PrefixEntry* const e = entries[i];
      const int st = launches.add(row_off[i], seqlen[i], query_pos[i], cached_len[i], e ? pages_of(*e, layer) : no_pages,
                                  e && e->consecutive);
      if (st != BICACHE_OK) return st;
    }
    return launches.flush();
  };
  // the tensor-core kernel takes the row maximum before scaling, which needs a positive scale
  if (ctx->tensor_ok && ctx->path != BICACHE_PATH_SIMT && softmax_scale > 0.f) {
    // Requests with more than 128 packed rows go through the kernel with row tiles of 256, which shares every key tile
    // between two tiles of 128 rows, if there are three of them to an SM and the query heads of a KV head divide 128 (else
    // one warp gathers the query tiles, and short items wait for it); it does not split the keys.  Both sides, 256 first, in
    // turn in one process, runs of 3 calls / of 40, where long ones meet the power limit; us:
    //   32 heads, 16,384 rows: all keys 3276, 3609 / 3752, 4086; window 4096 844, 884 / 893, 893, with 4 first tokens 863, 897
    //   / 1000, 998; window 1024 327, 324 / 315, 319.  8 KV heads, 16,384 rows, window 4096: 784, 847 / 920, 946.
    //   few tiles, 32 heads over 8192 keys: 3.0 tiles to an SM, all keys 366, 368 / 356, 361, window 2048 168, 153 / 161, 146,
    //   window 512 81, 68 / 77, 65; 1.1 to an SM, all keys 240, 143 / 235, 138.
    //   28 heads over 4: 16,384 rows, window 4096 737, 737 / 864, 801, window 1024 305, 267 / 296, 255; five ragged requests,
    //   window 500 + 201 94, 80 / 90, 76.
    // So it pays for long windows; calls with three to five tiles to an SM under a window of 2048 or less would be 10 to
    // 20 % faster in the other form.
    long long tiles = 0, rows_total = 0;
    for (int i = 0; i < R; ++i) {
      if (seqlen[i] > 0) rows_total = std::max<long long>(rows_total, row_off[i] + seqlen[i]);     // an empty one's row says nothing
      if ((long long)seqlen[i] * G > 128) tiles += ((long long)seqlen[i] * G + kTileRows - 1) / kTileRows * cfg.num_kv_heads;
    }
    TcTensorMaps maps;
    std::memset(&maps, 0, sizeof(maps));
    maps.q_tma = (128 % G == 0) ? 1 : 0;
    maps.o_tma = (32 % G == 0) ? 1 : 0;
    const bool by_256 = tiles >= 3LL * ctx->sm_count && maps.q_tma && rows_total < 0x7fffffffLL &&              // box coordinates are 32-bit
                        encode_map(&maps.q, q, rows_total, cfg.num_q_heads, q_row_stride, maps.q_tma ? G : 1, maps.q_tma ? 128 / G : 128) &&
                        encode_map(&maps.o, out, rows_total, cfg.num_q_heads, out_row_stride, maps.o_tma ? G : 1, maps.o_tma ? 32 / G : 32);
    ctx->last_kernel = by_256 ? BICACHE_KERNEL_TENSOR : BICACHE_KERNEL_KEY_RANGES;
    if (by_256) {
      WindowTileLaunches launches(ctx, a, maps, stream);
      const int st = run(launches, [&](int n) { return (long long)n * G > 128; });
      if (st != BICACHE_OK) return st;
    }
    WindowTensorLaunches launches(ctx, a, stream);
    return run(launches, [&](int n) { return !by_256 || (long long)n * G <= 128; });
  }
  ctx->last_kernel = BICACHE_KERNEL_SIMT;
  // A row tile of 16 where that holds a request's rows of a KV head, else of 64; of 16 for all if the call has no more than
  // two tiles of 64 rows x 64 keys to an SM: 113 rows of 4 heads over as many keys take 14 us so and 23 with tiles of 64, a
  // call with 2.1 tiles to an SM 27 and 23.
  long long steps = 0;
  for (int i = 0; i < R; ++i)
    if (seqlen[i] > 0)
      steps += ((long long)seqlen[i] * G + 63) / 64 * cfg.num_kv_heads *
               (1 + window_pages(sinks, left, right, cached_len[i], query_pos[i], query_pos[i] + seqlen[i] - 1).count * kPageSize / kWinKeys);
  const bool small = steps <= 2LL * ctx->sm_count;
  WindowSimtLaunches few(ctx, a, 16, stream), many(ctx, a, 64, stream);
  const int st = run(few, [&](int n) { return small || (long long)n * G <= 16; });
  return st != BICACHE_OK ? st : run(many, [&](int n) { return !small && (long long)n * G > 16; });
}

cudaError_t configure_window(const bicache_config& cfg, bool tensor_ok) {
  cudaError_t e = cudaSuccess;
  each_param_length([&](auto words) {
    constexpr int kWords = decltype(words)::value;
    for (int rows : {16, 64})
      with_window_simt(cfg.dtype, rows, cfg.head_dim, [&](auto zero, auto r, auto dim) {
        if (e == cudaSuccess)
          e = cudaFuncSetAttribute(window_simt_kernel<decltype(zero), decltype(r)::value, decltype(dim)::value, kWords>,
                                   cudaFuncAttributeMaxDynamicSharedMemorySize, (int)window_simt_smem(rows, decltype(dim)::value));
      });
  }, WindowSimtLengths());
  if (tensor_ok)
    each_param_length([&](auto words) {
      if (e == cudaSuccess) e = configure_tc_window<decltype(words)::value>();
    }, WindowLengths());
  return e;
}

}  // namespace

extern "C" {

int32_t bicache_append_tokens(bicache_ctx* ctx, int32_t layer, int32_t R, const int32_t* prefix_id,
                              const int32_t* token_off, const int64_t* row_off, const int32_t* seqlen, const void* k,
                              const void* v, int64_t kv_row_stride, const void* q, int64_t q_row_stride, void* q_out,
                              int64_t q_out_row_stride, const bicache_rotation* rotation, const int32_t* positions,
                              int64_t position_axis_stride, void* stream) {
  return guarded([&]() {
    return append_tokens_impl(ctx, layer, R, prefix_id, token_off, row_off, seqlen, k, v, kv_row_stride, q, q_row_stride,
                              q_out, q_out_row_stride, rotation, positions, position_axis_stride, stream);
  });
}

int32_t bicache_read_tokens(bicache_ctx* ctx, int32_t layer, int32_t R, const int32_t* prefix_id,
                            const int32_t* token_off, const int64_t* row_off, const int32_t* seqlen, void* k_out,
                            void* v_out, int64_t kv_row_stride, void* stream) {
  return guarded([&]() {
    return read_tokens_impl(ctx, layer, R, prefix_id, token_off, row_off, seqlen, k_out, v_out, kv_row_stride, stream);
  });
}

int32_t bicache_attend_window(bicache_ctx* ctx, int32_t layer, int32_t R, const int32_t* prefix_id,
                              const int32_t* cached_len, const int32_t* query_pos, const int64_t* row_off,
                              const int32_t* seqlen, const void* q, int64_t q_row_stride, void* out,
                              int64_t out_row_stride, float* lse_out, int32_t sinks, int32_t left, int32_t right,
                              float softmax_scale, void* stream) {
  return guarded([&]() {
    return attend_window_impl(ctx, layer, R, prefix_id, cached_len, query_pos, row_off, seqlen, q, q_row_stride, out,
                              out_row_stride, lse_out, sinks, left, right, softmax_scale, stream);
  });
}

int32_t bicache_rope_axes(bicache_ctx* ctx, int64_t rows, const bicache_rotation* rotation, const int32_t* positions,
                          int64_t position_axis_stride, int32_t inverse, const void* q, int64_t q_row_stride, void* q_out,
                          int64_t q_out_row_stride, const void* k, int64_t k_row_stride, void* k_out,
                          int64_t k_out_row_stride, void* stream) {
  return guarded([&]() {
    return rope_axes_impl(ctx, rows, rotation, positions, position_axis_stride, inverse, q, q_row_stride, q_out,
                          q_out_row_stride, k, k_row_stride, k_out, k_out_row_stride, stream);
  });
}

int32_t bicache_rope_axes_table(bicache_ctx* ctx, int64_t rows, const bicache_rotation* rotation,
                                const int32_t* positions, int64_t position_axis_stride, float* table, void* stream) {
  return guarded([&]() -> int32_t {
    if (!ctx) return BICACHE_ERR_INVALID;
    if (rows < 0) return fail(ctx, BICACHE_ERR_INVALID, "negative row count");
    if (!rotation) return fail(ctx, BICACHE_ERR_INVALID, "null rotation");
    if (rows > 0 && (!positions || !table)) return fail(ctx, BICACHE_ERR_INVALID, "null pointer");
    if (!aligned16(table)) return fail(ctx, BICACHE_ERR_INVALID, "table not 16-byte aligned");
    RopeAxes a;
    const int st = rotation_angles(ctx, rotation, 2 * kRopeMaxPairs, positions, position_axis_stride, rows, false, &a);
    return st != BICACHE_OK ? st : run_rope_table(ctx, a, rows, table, stream);
  });
}

}  // extern "C"

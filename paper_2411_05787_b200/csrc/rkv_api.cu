// C ABI of librkv: argument validation, workspace, tensor maps, launches.
#include <math.h>
#include <string.h>

#include <mutex>
#include <new>
#include <utility>

#include "rkv_internal.h"

namespace {

using rkv::AttnParams;
using rkv::CacheDev;
using rkv::QuantDev;
using rkv::ScoreParams;
using rkv::SelectParams;

rkv::EncodeTiledFn g_encode = nullptr;
// kernel attributes (dynamic shared-memory sizes) are set per device, once
constexpr int kMaxDevices = 64;
bool g_prepared[kMaxDevices] = {};
std::mutex g_prepare_mu;

bool config_ok(const rkv_config* c, rkv_status* why) {
  if (c == nullptr) { *why = RKV_ERR_INVALID_ARG; return false; }
  if (c->n_seq < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->max_len < 1 || c->max_small < 1 ||
      c->n_q_heads % c->n_kv_heads != 0) { *why = RKV_ERR_INVALID_ARG; return false; }
  if (c->head_dim != rkv::kHeadDim || c->n_q_heads / c->n_kv_heads > rkv::kMaxGroup ||
      c->agg < RKV_AGG_MAX || c->agg > RKV_AGG_FIRST || c->pool_kernel < 1 || c->pool_kernel > 31 ||
      c->pool_kernel % 2 == 0 ||
      (int64_t)c->max_len > (int64_t)rkv::kSelectCluster * rkv::kSelectMaxKeysPerCta ||
      (int64_t)c->n_seq * c->n_kv_heads > 65535 * 8) { *why = RKV_ERR_UNSUPPORTED; return false; }
  if (!(c->softmax_scale >= 0.f) || isinf(c->softmax_scale)) { *why = RKV_ERR_INVALID_ARG; return false; }
  return true;
}

int splits_for(const rkv_config* c) {
  int s = (c->max_len + rkv::kTile - 1) / rkv::kTile;
  return s < rkv::kMaxSplits ? (s < 1 ? 1 : s) : rkv::kMaxSplits;
}

struct WsLayout { size_t partials, ml_t, tickets, len_tickets, win_keys, keys, hist, anchor, counts, logits, status, total; int64_t logit_stride; };

WsLayout ws_layout(const rkv_config* c) {
  WsLayout w;
  const size_t bg = (size_t)c->n_seq * c->n_kv_heads;
  const int group = c->n_q_heads / c->n_kv_heads;
  auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
  w.logit_stride = ((int64_t)c->max_len + 63) & ~int64_t(63);
  size_t off = 0;
  w.partials = off; off = up(off + bg * splits_for(c) * rkv::PartialLayout::kFloats * sizeof(float));
  w.ml_t = off;     off = up(off + bg * 16 * (size_t)splits_for(c) * sizeof(float));
  w.tickets = off;  off = up(off + bg * sizeof(int32_t));
  w.len_tickets = off; off = up(off + (size_t)c->n_seq * sizeof(int32_t));
  w.win_keys = off; off = up(off + bg * (size_t)c->max_small * sizeof(uint32_t));
  w.keys = off;     off = up(off + bg * (size_t)w.logit_stride * sizeof(uint32_t));
  w.hist = off;     off = up(off + bg * (size_t)rkv::kSelectBins * sizeof(uint32_t));
  w.anchor = off;   off = up(off + bg * sizeof(int32_t));
  w.counts = off;   off = up(off + bg * sizeof(int32_t));
  const int gp = group <= 4 ? 4 : 8;   // position-major logits, padded to a vector width
  w.logits = off;   off = up(off + bg * gp * (size_t)w.logit_stride * sizeof(float));
  w.status = off;   off = up(off + sizeof(int32_t));
  w.total = off;
  return w;
}

rkv_status cuda_fail(rkv_ctx* ctx, cudaError_t e, const char* where) {
  if (ctx) ctx->last_error = std::string(where) + ": " + cudaGetErrorString(e);
  return RKV_ERR_CUDA;
}

bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15) == 0; }   // NULL counts as aligned
bool cache_ok(const rkv_cache* c) {
  return c && c->k && c->v && c->row_offset && c->cap && c->len && c->n_rows > 0 && c->n_rows < (int64_t(1) << 31) &&
         (reinterpret_cast<uintptr_t>(c->k) & 15) == 0 && (reinterpret_cast<uintptr_t>(c->v) & 15) == 0;
}

// Brackets one kernel launch with events when profiling is on.
struct LaunchScope {
  rkv_ctx* ctx; cudaStream_t st; int kind; cudaEvent_t stop = nullptr;
  static cudaEvent_t get(rkv_ctx* c) {
    cudaEvent_t e = nullptr;
    if (!c->event_pool.empty()) { e = c->event_pool.back(); c->event_pool.pop_back(); return e; }
    if (cudaEventCreate(&e) != cudaSuccess) return nullptr;
    return e;
  }
  LaunchScope(rkv_ctx* c, cudaStream_t s, int k) : ctx(c), st(s), kind(k) {
    if (!ctx->profiling) return;
    cudaEvent_t start = get(ctx);
    stop = get(ctx);
    if (start == nullptr || stop == nullptr) { stop = nullptr; return; }
    cudaEventRecord(start, st);
    ctx->timed.push_back({kind, start, stop});
  }
  ~LaunchScope() { if (stop != nullptr) cudaEventRecord(stop, st); }
};

CacheDev dev_of(const rkv_cache* c) { return CacheDev{c->k, c->v, c->row_offset, c->cap, c->len}; }

QuantDev dev_of(const rkv_quant_cache* c) {
  return QuantDev{static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->k_scale, c->v_scale,
                  c->row_offset, c->cap, c->len, c->n_rows};
}
bool quant_ok(const rkv_quant_cache* c) {
  return c && c->k && c->v && c->k_scale && c->v_scale && c->row_offset && c->cap && c->len && c->n_rows > 0 &&
         c->n_rows < (int64_t(1) << 31) && c->n_rows % rkv::kQuantBlock == 0 && aligned16(c->k) && aligned16(c->v) &&
         (reinterpret_cast<uintptr_t>(c->k_scale) & 3) == 0 && (reinterpret_cast<uintptr_t>(c->v_scale) & 3) == 0;
}
bool paged_ok(const rkv_ctx* ctx, const rkv_paged_cache* c) {
  return c && c->k && c->v && c->table && c->len && (c->page == 16 || c->page == 32 || c->page == 64 || c->page == 128) &&
         c->n_pages > 0 && c->n_pages < (int64_t(1) << 31) &&
         c->n_pages * c->page < ((int64_t(1) << 31) + ctx->cfg.n_kv_heads - 1) / ctx->cfg.n_kv_heads && c->table_stride > 0 &&
         aligned16(c->k) && aligned16(c->v) && aligned16(c->k_min) && aligned16(c->k_max) &&
         (c->k_min == nullptr) == (c->k_max == nullptr);
}
rkv::PagedDev dev_of(const rkv_ctx* ctx, const rkv_paged_cache* c) {
  return rkv::PagedDev{c->k, c->v, c->k_min, c->k_max, c->table, c->len, c->n_pages,
                       c->page == 16 ? 4 : c->page == 32 ? 5 : c->page == 64 ? 6 : 7, c->table_stride, ctx->cfg.n_kv_heads};
}
// What the score pass and the selection read of a cache: its sizes (the rows' pointer is its identity there).
rkv_cache sizes_of(const rkv_quant_cache* c) { return rkv_cache{c->k, c->v, c->n_rows, c->row_offset, c->cap, c->len}; }
// The 8-bit calls launch on the context's device only.
bool on_device(const rkv_ctx* ctx) {
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && dev == ctx->device;
}

// [n_rows][128] bf16 as {64 channels, row, half}: one box = 64 rows x both halves, 128-byte swizzle.
// quant: [n_rows][128] codes, one box = 128 rows.  paged_box: the rows of a pool of pages, one box = this many of them, of
// both 64-channel halves or of one.
rkv_status tensor_map(rkv_ctx* ctx, void* base, int64_t n_rows, CUtensorMap* out, bool quant = false, int paged_box = 0,
                      int halves = 2) {
  // the map depends on nothing else
  const std::pair<uint64_t, int64_t> key(reinterpret_cast<uint64_t>(base),
                                         quant ? -n_rows : n_rows + ((int64_t)(paged_box * halves) << 32) + ((int64_t)halves << 48));
  auto it = ctx->tmaps.find(key);
  if (it != ctx->tmaps.end()) { *out = it->second; return RKV_OK; }
  if (g_encode == nullptr) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
    if (e != cudaSuccess || fn == nullptr || qres != cudaDriverEntryPointSuccess)
      return cuda_fail(ctx, e == cudaSuccess ? cudaErrorUnknown : e, "cudaGetDriverEntryPoint(cuTensorMapEncodeTiled)");
    g_encode = reinterpret_cast<rkv::EncodeTiledFn>(fn);
  }
  CUtensorMap tm;
  CUresult r = quant           ? rkv::encode_quant_map(g_encode, base, n_rows, &tm)
               : paged_box > 0 ? rkv::encode_paged_map(g_encode, base, n_rows, paged_box, halves, &tm)
                               : rkv::encode_cache_map(g_encode, base, n_rows, &tm);
  if (r != CUDA_SUCCESS) {
    ctx->last_error = "cuTensorMapEncodeTiled failed with CUresult " + std::to_string((int)r);
    return RKV_ERR_CUDA;
  }
  if (ctx->tmaps.size() > 8192) ctx->tmaps.clear();
  ctx->tmaps.emplace(key, tm);
  *out = tm;
  return RKV_OK;
}

// Positions per CTA.  Full step: one balanced wave over 2 CTAs per SM when that keeps chunks moderate,
// otherwise fixed 2048-position chunks over several waves (ragged batches then balance by count).
// Small step: the work is tiny and latency-bound, so chunks of at least 256 positions keep the
// number of partials that the last CTA has to fold small.
int choose_chunk(const rkv_ctx* ctx, int n_max, bool full, int* grid_x) {
  const int bg = ctx->cfg.n_seq * ctx->cfg.n_kv_heads;
  const int slots = 2 * ctx->sm_count;
  int splits = slots / bg;
  if (splits < 1) splits = 1;
  if (splits > ctx->max_splits) splits = ctx->max_splits;
  int chunk = (n_max + splits - 1) / splits;
  if (chunk > 4096) chunk = 2048;
  const int floor_chunk = full ? rkv::kTile : ctx->small_min_chunk;
  if (chunk < floor_chunk) chunk = floor_chunk;
  chunk = (chunk + 15) & ~15;
  int gx = (n_max + chunk - 1) / chunk;
  while (gx > ctx->max_splits) {  // keep the partial buffer's bound
    chunk *= 2;
    gx = (n_max + chunk - 1) / chunk;
  }
  *grid_x = gx < 1 ? 1 : gx;
  return chunk;
}

// Longest small cache that the clustered partial step takes (8 CTAs x 1024 positions).
constexpr int kClusterMaxLen = 8192;

// From how many (sequences x KV heads x shared positions) on these are attended by one pass for all.  Every sequence by itself
// / together, us, with 200 positions of their own behind the prefix (* what is taken):
//   prefix                      1024           4096          16384
//    8 x 8 heads of 4     *7.2 / 14.8    *14.2 / 16.7   46.2 / *25.5
//   32 x 8 heads of 4    *17.0 / 22.0    48.1 / *25.5  156.3 / *32.9
//   64 x 4 heads of 7    *17.5 / 24.6    48.0 / *28.0  157.1 / *39.2
//   64 x 1 head  of 8     *7.3 / 20.0   *14.3 / 21.7    45.4 / *26.0
//    4 x 8 heads of 4     *6.5 / 13.8    *10.2 / 15.7    28.4 / *23.1
constexpr int kSharedMin = 1 << 19;

struct AppendArgs {
  const void* k_new; const void* v_new; const rkv_cache* full;
  const int32_t* evict_order; int32_t* evict_count; const int32_t* k_small; int max_evict;   // all null / 0: the cache grows
};

bool cluster_eligible(const rkv_ctx* ctx, int n_max) { return ctx->small_cluster != 0 && n_max <= kClusterMaxLen; }

rkv_status run_attention(rkv_ctx* ctx, const void* q, const rkv_cache* cache, const int32_t* active, void* out,
                         int n_max, int limit, bool logits, cudaStream_t st, int* chunk_out, int* gx_out,
                         const AppendArgs* app = nullptr, bool score_only = false) {
  if (!aligned16(q) || !aligned16(out) || (app != nullptr && (!aligned16(app->k_new) || !aligned16(app->v_new))))
    return RKV_ERR_INVALID_ARG;   // the kernels read and write these 16 bytes at a time
  CUtensorMap tm_k, tm_v;
  rkv_status s = tensor_map(ctx, cache->k, cache->n_rows, &tm_k);
  if (s != RKV_OK) return s;
  s = tensor_map(ctx, cache->v, cache->n_rows, &tm_v);
  if (s != RKV_OK) return s;
  AttnParams p;
  memset(&p, 0, sizeof(p));
  int gx = 1;
  const bool cluster = !logits && cluster_eligible(ctx, n_max);
  if (cluster) {   // 1, 2, 4 or 8 CTAs per (sequence, KV head), whole tiles each
    const int tiles = (n_max + rkv::kTile - 1) / rkv::kTile;
    gx = tiles >= 5 ? 8 : tiles >= 3 ? 4 : tiles >= 2 ? 2 : 1;
    // with many (sequence, KV head) pairs one wave of CTAs is enough: fewer, longer CTAs per pair spend a smaller
    // share of their time on the exchange inside the cluster
    const int bg = ctx->cfg.n_seq * ctx->cfg.n_kv_heads;
    while (gx > 1 && (int64_t)gx * bg > 2 * ctx->sm_count) gx >>= 1;
    p.chunk = ((tiles + gx - 1) / gx) * rkv::kTile;
  } else {
    p.chunk = choose_chunk(ctx, n_max, logits, &gx);
  }
  // Streaming forms: the head's tiles are dealt out to the gx CTAs in turn; the partial slots in use are then
  // min(tiles, gx), which is what the consumers of (chunk, gx) compute when they are told chunk = one tile.
  p.interleave = (logits && ctx->interleave) ? 1 : 0;
  if (chunk_out) *chunk_out = p.interleave ? rkv::kTile : p.chunk;
  if (gx_out) *gx_out = gx;
  p.q = q;
  p.row_offset = cache->row_offset;
  p.cap = cache->cap;
  p.len = cache->len;
  p.active = active;
  p.out = out;
  p.partials = ctx->partials;
  p.tickets = ctx->tickets;
  p.ml_t = ctx->ml_t;
  p.logits = logits ? ctx->logits : nullptr;
  p.hist = ctx->hist;
  p.anchor = ctx->anchor;
  p.status = ctx->status;
  p.logit_stride = ctx->logit_stride;
  p.n_q_heads = ctx->cfg.n_q_heads;
  p.n_kv_heads = ctx->cfg.n_kv_heads;
  p.group = ctx->group;
  p.gp = ctx->gp;
  p.max_splits = ctx->max_splits;
  p.max_len = limit;
  p.scale = ctx->cfg.softmax_scale;
  // without a mask: a cluster per head always has work; a streaming grid has when it serves a single sequence
  p.spec = (active == nullptr && (cluster || (logits && ctx->cfg.n_seq == 1))) ? 1 : 0;
  // Early cache read: only when the launch before this one on the stream leaves the attended cache alone (a
  // gather or an append into it forbids it; so does an unknown history).
  p.early = (cluster && p.spec != 0 && ctx->early_read && rkv::early_read_safe(st, cache)) ? 1 : 0;
  // The streaming pass does the same with its first tiles: all stages of its ring, or - when the launch before it
  // is the short merge kernel of the previous pass, whose few loads would queue behind them - one tile.
  if (logits && p.spec != 0 && ctx->early_read && rkv::early_read_safe(st, cache))
    p.early = rkv::last_launch_was_fold(st) ? 1 : rkv::kStages;
  if (app != nullptr) {   // the clustered partial step and the full step's attention pass can take the append with them
    if (!cluster && !(logits && !score_only)) return RKV_ERR_INVALID_ARG;
    p.k_new = app->k_new;
    p.v_new = app->v_new;
    p.small_k = cache->k;
    p.small_v = cache->v;
    p.small_len = cache->len;
    p.len_tickets = ctx->len_tickets;
    p.has_full = app->full != nullptr;
    p.evict_order = app->evict_order;
    p.evict_count = app->evict_count;
    p.k_small = app->k_small;
    p.max_evict = app->max_evict;
    if (app->full != nullptr) {
      p.full_k = app->full->k;
      p.full_v = app->full->v;
      p.full_row_offset = app->full->row_offset;
      p.full_cap = app->full->cap;
      p.full_len = app->full->len;
    }
  }
  cudaError_t e;
  {
    LaunchScope scope(ctx, st, logits ? RKV_KERNEL_ATTN_FULL : RKV_KERNEL_ATTN_SMALL);
    // few clusters (half the SMs or fewer): the wide form of the clustered kernel, one CTA per SM
    const bool wide = cluster && (int64_t)gx * ctx->cfg.n_kv_heads * ctx->cfg.n_seq * 2 <= ctx->sm_count;
    e = cluster      ? rkv::launch_attention_cluster(p, tm_k, tm_v, ctx->cfg.n_seq, gx, app != nullptr, wide, st)
        : score_only ? rkv::launch_attention_scores(p, tm_k, tm_v, ctx->cfg.n_seq, gx, st)
                     : rkv::launch_attention(p, tm_k, tm_v, ctx->cfg.n_seq, gx, logits, st, app != nullptr);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "attention launch");
  ctx->launches += 1;
  rkv::note_launch(st, app != nullptr ? cache : nullptr, app != nullptr ? app->full : nullptr);
  return RKV_OK;
}

// The pass over the 8-bit cache, in one of three forms (all write the same workspace):
//   splits    one sequence: its tiles of 128 positions are dealt out in turn to as many CTAs per KV head as fit one wave
//             (two to an SM); a fold launch - or the score pass - finishes the output
//   cluster   1, 2, 4 or 8 CTAs per (sequence, KV head) are a cluster and finish the output themselves.  For one sequence
//             up to 2048 positions (8 KV heads, cluster against splits: 4.1 / 5.0 us at 1000, 4.85 / 5.1 at 2048, 6.6 / 6.05 at
//             4096, 9.9 / 7.1 at 8192), for a batch while no CTA can get more than 8 tiles
//   balanced  longer batches: equal runs of tiles across heads and sequences, then its own fold
// Which of the two is faster for a batch depends on how its lengths differ, which only the device knows, and on how much
// of the chip the clusters fill; the bound of 8 tiles a CTA goes by neither.  Cluster against balanced in us (attention
// alone, 4 queries a head; ragged: spread evenly below the largest; * the form that is taken):
//   tiles a CTA (few heads)          2              4              8             16
//   positions                      2048           4096           8192          16384
//   2 x 4 heads, one length    *5.1 /  6.8    *6.9 /  8.7   *10.2 /  9.4    17.0 / *13.4
//                    ragged    *5.0 /  6.1    *6.8 /  7.4   *10.1 /  9.2    16.8 / *10.9
//   2 x 1 head,  one length    *4.9 /  6.7    *6.7 /  7.8   *10.0 /  8.4    16.6 / *10.3
//                    ragged    *4.8 /  6.1    *6.6 /  6.9    *9.9 /  7.3    16.5 /  *9.2
//   8 x 8 heads, one length    *8.8 / 13.0   *14.0 / 17.8    23.7 / *27.3   42.6 / *46.1
//                    ragged    *7.9 / 10.7   *12.8 / 14.4    21.2 / *20.1   38.3 / *32.2
//   tiles a CTA (8 x 8)              4              8             16             32
// So at 8 tiles a CTA clusters that leave most of the chip empty lose 8 to 36 % to the balanced form, and from 16 on it
// loses 8 to 15 % to them on a full batch of one length, for not waiting for the longest sequence of a ragged one.
constexpr int kQuantClusterMaxLen = 2048, kQuantClusterMaxTiles = 8;
struct QuantPass { int gx; bool finished; const int32_t* counts; };   // what the second half has to know

rkv_status run_quant_attention(rkv_ctx* ctx, const void* q, const rkv_quant_cache* cache, const int32_t* active,
                               void* out, int n_max, bool logits, bool fold_out, cudaStream_t st, QuantPass* pass) {
  if (!aligned16(q) || !aligned16(out)) return RKV_ERR_INVALID_ARG;
  CUtensorMap tm_k, tm_v;
  rkv_status s = tensor_map(ctx, cache->k, cache->n_rows, &tm_k, true);
  if (s != RKV_OK) return s;
  s = tensor_map(ctx, cache->v, cache->n_rows, &tm_v, true);
  if (s != RKV_OK) return s;
  const int n_seq = ctx->cfg.n_seq;
  const int64_t bg = (int64_t)n_seq * ctx->cfg.n_kv_heads, slots = 2 * ctx->sm_count;
  const int tiles = (n_max + rkv::kQuantTile - 1) / rkv::kQuantTile;
  int gx = (int)(slots / bg);
  if (gx > ctx->max_splits) gx = ctx->max_splits;
  if (gx > tiles) gx = tiles;
  if (gx < 1) gx = 1;
  const int cluster_gx = gx >= 8 ? 8 : gx >= 4 ? 4 : gx >= 2 ? 2 : 1;
  const int64_t most = bg * tiles;   // tiles there can be
  const int64_t runs = most < slots ? most : slots;
  const bool balanced = n_seq > 1 && tiles > kQuantClusterMaxTiles * cluster_gx && n_seq <= rkv::kQuantMaxSeq &&
                        (most + bg) * (slots + 1) < (int64_t(1) << 32);   // (the kernel cuts the runs in 32 bits)
  const bool cluster = !balanced && (n_seq > 1 || n_max <= kQuantClusterMaxLen || gx <= 8);
  if (cluster) gx = cluster_gx;
  rkv::QuantAttnParams p;
  memset(&p, 0, sizeof(p));
  p.q = q;
  p.k_scale = cache->k_scale;
  p.v_scale = cache->v_scale;
  p.row_offset = cache->row_offset;
  p.cap = cache->cap;
  p.len = cache->len;
  p.active = active;
  p.out = out;
  p.partials = ctx->partials;
  p.ml_t = ctx->ml_t;
  p.logits = logits ? ctx->logits : nullptr;
  p.hist = ctx->hist;
  p.counts = ctx->split_counts;
  p.status = ctx->status;
  p.n_rows = cache->n_rows;
  p.logit_stride = ctx->logit_stride;
  p.n_seq = n_seq;
  p.n_q_heads = ctx->cfg.n_q_heads;
  p.n_kv_heads = ctx->cfg.n_kv_heads;
  p.group = ctx->group;
  p.gp = ctx->gp;
  p.max_splits = ctx->max_splits;
  p.max_len = n_max;
  p.scale = ctx->cfg.softmax_scale;
  p.spec = (active == nullptr && !balanced) ? 1 : 0;
  // as in the bf16 pass: one tile ahead of the wait behind the short merge kernel, the whole ring behind others
  if (p.spec != 0 && ctx->early_read && rkv::early_read_safe(st, cache)) p.early = rkv::last_launch_was_fold(st) ? 1 : 2;
  cudaError_t e;
  {
    LaunchScope scope(ctx, st, RKV_KERNEL_ATTN_FULL);
    if (balanced) {
      e = rkv::launch_quant_balanced(p, tm_k, tm_v, (int)runs, st);
    } else {
      e = rkv::launch_quant_attention(p, tm_k, tm_v, n_seq, gx, cluster, gx * bg <= slots, st);
    }
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "8-bit attention launch");
  ctx->launches += 1;
  rkv::note_launch(st, nullptr, nullptr);
  *pass = {balanced ? ctx->max_splits : gx, cluster || balanced || fold_out, balanced ? ctx->split_counts : nullptr};
  if (cluster || (!balanced && !fold_out)) return RKV_OK;
  {
    LaunchScope scope(ctx, st, RKV_KERNEL_FOLD);
    e = balanced ? rkv::launch_quant_fold(p, st)
                 : rkv::launch_fold(ctx->partials, ctx->ml_t, cache->len, cache->cap, active, out, n_seq, ctx->cfg.n_q_heads,
                                    ctx->cfg.n_kv_heads, rkv::kQuantTile, ctx->max_splits, n_max, gx, st);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "fold launch");
  ctx->launches += 1;
  rkv::note_launch(st, nullptr, nullptr, true);
  return RKV_OK;
}

}  // namespace

namespace rkv {
bool g_use_pdl = true;

namespace {
struct ByteRange { uintptr_t lo, hi; };
std::mutex g_writes_mu;
struct LastLaunch { std::vector<ByteRange> writes; bool fold = false; };
std::map<cudaStream_t, LastLaunch> g_writes;   // per stream: the library's last launch
bool g_writes_lost = false;   // the record was dropped once: a stream without an entry is then unknown, not clean
constexpr size_t kMaxTrackedStreams = 1024;
void add_ranges(std::vector<ByteRange>* v, const rkv_cache* c) {
  if (c == nullptr || c->k == nullptr || c->v == nullptr) return;
  const uintptr_t bytes = (uintptr_t)c->n_rows * kHeadDim * 2;
  v->push_back({reinterpret_cast<uintptr_t>(c->k), reinterpret_cast<uintptr_t>(c->k) + bytes});
  v->push_back({reinterpret_cast<uintptr_t>(c->v), reinterpret_cast<uintptr_t>(c->v) + bytes});
}
void add_ranges(std::vector<ByteRange>* v, const rkv_quant_cache* c) {   // (scales are read behind the wait in any case)
  for (const void* rows : {c->k, c->v})
    v->push_back({reinterpret_cast<uintptr_t>(rows), reinterpret_cast<uintptr_t>(rows) + (uintptr_t)c->n_rows * kHeadDim});
}
}  // namespace

static LastLaunch& new_launch(cudaStream_t st, bool fold) {   // (the lock is held)
  if (g_writes.size() >= kMaxTrackedStreams && g_writes.find(st) == g_writes.end()) {
    g_writes.clear();
    g_writes_lost = true;
  }
  LastLaunch& v = g_writes[st];
  v.fold = fold;
  v.writes.clear();
  return v;
}

void note_launch(cudaStream_t st, const rkv_cache* a, const rkv_cache* b, bool fold) {
  std::lock_guard<std::mutex> lock(g_writes_mu);
  LastLaunch& v = new_launch(st, fold);
  add_ranges(&v.writes, a);
  add_ranges(&v.writes, b);
}

void note_quant_store(cudaStream_t st, const rkv_quant_cache* c) {
  std::lock_guard<std::mutex> lock(g_writes_mu);
  add_ranges(&new_launch(st, false).writes, c);
}

void note_rows(cudaStream_t st, std::initializer_list<std::pair<const void*, size_t>> writes) {
  std::lock_guard<std::mutex> lock(g_writes_mu);
  LastLaunch& v = new_launch(st, false);
  for (const auto& w : writes)
    if (w.first != nullptr) v.writes.push_back({reinterpret_cast<uintptr_t>(w.first), reinterpret_cast<uintptr_t>(w.first) + w.second});
}

bool last_launch_was_fold(cudaStream_t st) {
  std::lock_guard<std::mutex> lock(g_writes_mu);
  auto it = g_writes.find(st);
  return it != g_writes.end() && it->second.fold;
}

template <typename Cache>
static bool last_launch_spares(cudaStream_t st, const Cache* c) {
  std::lock_guard<std::mutex> lock(g_writes_mu);
  auto it = g_writes.find(st);
  if (it == g_writes.end()) return !g_writes_lost;   // never launched here: whatever runs before is not ours and
                                                     // therefore complete before a kernel of ours starts
  std::vector<ByteRange> mine;
  add_ranges(&mine, c);
  for (const ByteRange& w : it->second.writes)
    for (const ByteRange& r : mine)
      if (w.lo < r.hi && r.lo < w.hi) return false;
  return true;
}
bool early_read_safe(cudaStream_t st, const rkv_cache* c) { return last_launch_spares(st, c); }
bool early_read_safe(cudaStream_t st, const rkv_quant_cache* c) { return last_launch_spares(st, c); }
}  // namespace rkv

extern "C" {

size_t rkv_workspace_bytes(const rkv_config* cfg) {
  rkv_status why;
  if (!config_ok(cfg, &why)) return 0;
  return ws_layout(cfg).total;
}

rkv_status rkv_create(const rkv_config* cfg, rkv_ctx** out) {
  if (out == nullptr) return RKV_ERR_INVALID_ARG;
  *out = nullptr;
  rkv_status why;
  if (!config_ok(cfg, &why)) return why;
  rkv_ctx* ctx = new (std::nothrow) rkv_ctx();
  if (ctx == nullptr) return RKV_ERR_WORKSPACE;
  ctx->cfg = *cfg;
  if (ctx->cfg.softmax_scale == 0.f) ctx->cfg.softmax_scale = 1.0f / sqrtf((float)cfg->head_dim);
  ctx->group = cfg->n_q_heads / cfg->n_kv_heads;
  ctx->max_splits = splits_for(cfg);
  ctx->launches = 0;
  ctx->profiling = false;
  ctx->small_min_chunk = 256;
  ctx->small_cluster = 1;
  ctx->early_read = 1;
  ctx->interleave = 1;
  ctx->select_keys_per_cta = 4096;
  ctx->score_slice = 0;
  ctx->shared_min = kSharedMin;
  ctx->gp = ctx->group <= 4 ? 4 : 8;
  ctx->workspace = nullptr;
  cudaError_t e = cudaGetDevice(&ctx->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&ctx->sm_count, cudaDevAttrMultiProcessorCount, ctx->device);
  if (e != cudaSuccess) { delete ctx; return RKV_ERR_CUDA; }
  if (ctx->device < 0 || ctx->device >= kMaxDevices) { delete ctx; return RKV_ERR_UNSUPPORTED; }
  {
    std::lock_guard<std::mutex> lock(g_prepare_mu);
    if (!g_prepared[ctx->device]) {
      e = rkv::prepare_attention();
      if (e == cudaSuccess) e = rkv::prepare_select();
      if (e == cudaSuccess) e = rkv::prepare_quant_attention();
      if (e == cudaSuccess) e = rkv::prepare_page_select();
      if (e == cudaSuccess) e = rkv::prepare_paged_attention();
      if (e == cudaSuccess) e = rkv::prepare_prefix_attention();
      if (e != cudaSuccess) { delete ctx; return RKV_ERR_CUDA; }
      g_prepared[ctx->device] = true;
    }
  }
  const WsLayout w = ws_layout(cfg);
  e = cudaMalloc(reinterpret_cast<void**>(&ctx->workspace), w.total);
  if (e != cudaSuccess) { delete ctx; return RKV_ERR_WORKSPACE; }
  e = cudaMemset(ctx->workspace, 0, w.total);
  if (e != cudaSuccess) { cudaFree(ctx->workspace); delete ctx; return RKV_ERR_CUDA; }
  ctx->workspace_bytes = w.total;
  ctx->partials = reinterpret_cast<float*>(ctx->workspace + w.partials);
  ctx->ml_t = reinterpret_cast<float*>(ctx->workspace + w.ml_t);
  ctx->tickets = reinterpret_cast<int32_t*>(ctx->workspace + w.tickets);
  ctx->len_tickets = reinterpret_cast<int32_t*>(ctx->workspace + w.len_tickets);
  ctx->win_keys = reinterpret_cast<uint32_t*>(ctx->workspace + w.win_keys);
  ctx->keys = reinterpret_cast<uint32_t*>(ctx->workspace + w.keys);
  ctx->hist = reinterpret_cast<uint32_t*>(ctx->workspace + w.hist);   // zeroed with the rest of the workspace above
  ctx->anchor = reinterpret_cast<int32_t*>(ctx->workspace + w.anchor);
  ctx->split_counts = reinterpret_cast<int32_t*>(ctx->workspace + w.counts);
  ctx->pending_keys.valid = false;
  ctx->pending_full.valid = false;
  ctx->logits = reinterpret_cast<float*>(ctx->workspace + w.logits);
  ctx->status = reinterpret_cast<int32_t*>(ctx->workspace + w.status);
  ctx->logit_stride = w.logit_stride;
  *out = ctx;
  return RKV_OK;
}

rkv_status rkv_destroy(rkv_ctx* ctx) {
  if (ctx == nullptr) return RKV_ERR_INVALID_ARG;
  cudaError_t e = cudaSuccess;
  if (ctx->workspace) e = cudaFree(ctx->workspace);
  for (auto& t : ctx->timed) { cudaEventDestroy(t.start); cudaEventDestroy(t.stop); }
  for (auto ev : ctx->event_pool) cudaEventDestroy(ev);
  delete ctx;
  return e == cudaSuccess ? RKV_OK : RKV_ERR_CUDA;
}

// First half of the full step: attention over the full cache, logits and softmax statistics to the workspace.
// fold_out: a second kernel finishes out from the partials right away (otherwise the selection kernel does).
static rkv_status full_attention_part(rkv_ctx* ctx, const void* q, const rkv_cache* full, const int32_t* active,
                                      void* out, int32_t max_len_hint, cudaStream_t st, bool score_only,
                                      bool fold_out, const AppendArgs* app = nullptr) {
  if (!ctx || !q || !cache_ok(full) || (!out && !score_only)) return RKV_ERR_INVALID_ARG;
  int n_max = max_len_hint == 0 ? ctx->cfg.max_len : max_len_hint;
  if (n_max < 1 || n_max > ctx->cfg.max_len) return RKV_ERR_INVALID_ARG;
  int chunk = 0, gx = 1;
  ctx->pending_full.valid = false;
  ctx->pending_keys.valid = false;   // the logits those keys came from are about to be overwritten
  rkv_status s = run_attention(ctx, q, full, active, out, n_max, n_max, true, st, &chunk, &gx, app, score_only);
  if (s != RKV_OK) return s;
  if (fold_out && !score_only) {
    cudaError_t e;
    {
      LaunchScope scope(ctx, st, RKV_KERNEL_FOLD);
      e = rkv::launch_fold(ctx->partials, ctx->ml_t, full->len, full->cap, active, out, ctx->cfg.n_seq,
                           ctx->cfg.n_q_heads, ctx->cfg.n_kv_heads, chunk, ctx->max_splits, n_max, gx, st);
    }
    if (e != cudaSuccess) return cuda_fail(ctx, e, "fold launch");
    ctx->launches += 1;
    rkv::note_launch(st, nullptr, nullptr, true);
  }
  ctx->pending_full = {true, chunk, gx, n_max, full->k, active, nullptr, false};
  return RKV_OK;
}

// Second half: scores and top-K from what the first half left in the workspace; folds out unless it is NULL.
// stage: both launches (the score pass, then the selection), or one of them - rkv_score_keys launches the score pass
// alone and leaves a record for the rkv_select_topk that launches the selection alone.
enum SelectStage { kStageBoth, kStageScore, kStageSelect };
static rkv_status select_part(rkv_ctx* ctx, const void* q, const rkv_cache* full, const int32_t* k_small,
                              int32_t k_max, const int32_t* active, void* out, float* scores, int64_t score_stride,
                              int32_t* topk_idx, void* q_last_full, cudaStream_t st, SelectStage stage = kStageBoth) {
  if (!ctx || !cache_ok(full) || !k_small || (!topk_idx && stage != kStageScore) ||
      (q_last_full != nullptr && q == nullptr))
    return RKV_ERR_INVALID_ARG;
  if (k_max < 1 || k_max > ctx->cfg.max_small) return RKV_ERR_INVALID_ARG;
  int n_max, chunk, gx;
  const int32_t* counts = nullptr;
  const bool quant = stage == kStageSelect ? ctx->pending_keys.quant : ctx->pending_full.quant;   // an 8-bit cache's pass
  if (stage == kStageSelect) {
    if (!ctx->pending_keys.valid || ctx->pending_keys.k_max != k_max) return RKV_ERR_INVALID_ARG;
    n_max = ctx->pending_keys.n_max;
    chunk = gx = 0;                 // (geometry of the attention pass: the score pass has used it)
    ctx->pending_keys.valid = false;
  } else {
    if (!ctx->pending_full.valid) return RKV_ERR_INVALID_ARG;   // no attention pass to take the logits from
    n_max = ctx->pending_full.n_max, chunk = ctx->pending_full.chunk, gx = ctx->pending_full.gx;
    counts = ctx->pending_full.counts;
    if (scores != nullptr && score_stride < n_max) return RKV_ERR_INVALID_ARG;
    ctx->pending_full.valid = false;
    ctx->pending_keys.valid = false;
  }
  // two launches: the score pass over all positions (keys, scores, histogram; folds out[] when asked to), then
  // the selection proper, one small cluster per (sequence, KV head)
  const int bg = ctx->cfg.n_seq * ctx->cfg.n_kv_heads;
  ScoreParams cp;
  memset(&cp, 0, sizeof(cp));
  cp.logits = ctx->logits;
  cp.partials = ctx->partials;
  cp.ml_t = ctx->ml_t;
  cp.q = q;
  cp.out = out;
  cp.q_last_full = q_last_full;
  cp.cap = full->cap;
  cp.len = full->len;
  cp.k_small = k_small;
  cp.active = active;
  cp.scores = scores;
  cp.keys = ctx->keys;
  cp.hist = ctx->hist;
  cp.anchor = ctx->anchor;
  cp.status = ctx->status;
  cp.logit_stride = ctx->logit_stride;
  cp.score_stride = score_stride;
  cp.n_q_heads = ctx->cfg.n_q_heads;
  cp.n_kv_heads = ctx->cfg.n_kv_heads;
  cp.group = ctx->group;
  cp.agg = ctx->cfg.agg;
  cp.k_max = k_max;
  cp.max_len = n_max;
  cp.slice = rkv::score_slice_for(n_max, bg, ctx->sm_count);
  if (cp.slice < ctx->score_slice) cp.slice = ctx->score_slice;   // the option is a floor
  cp.n_slices = (n_max + cp.slice - 1) / cp.slice;
  cp.chunk = chunk;
  cp.max_splits = ctx->max_splits;
  cp.grid_splits = gx;
  cp.split_counts = counts;
  cp.pool_half = (ctx->cfg.pool_kernel - 1) / 2;
  cp.row_offset = full->row_offset;
  cp.quant_rows = quant ? full->n_rows : 0;
  SelectParams sp;
  memset(&sp, 0, sizeof(sp));
  sp.keys = ctx->keys;
  sp.hist = ctx->hist;
  sp.anchor = ctx->anchor;
  sp.cap = full->cap;
  sp.len = full->len;
  sp.k_small = k_small;
  sp.active = active;
  sp.topk_idx = topk_idx;
  sp.win_keys = ctx->win_keys;
  sp.win_stride = ctx->cfg.max_small;
  sp.logit_stride = ctx->logit_stride;
  sp.n_kv_heads = ctx->cfg.n_kv_heads;
  sp.k_max = k_max;
  sp.max_len = n_max;
  const int cluster = rkv::select_cluster_for(n_max, ctx->select_keys_per_cta);
  sp.keys_per_thread = rkv::select_keys_per_thread(n_max, cluster);
  sp.per_fixed = ctx->cfg.n_seq == 1 ? 1 : 0;
  sp.row_offset = full->row_offset;
  sp.quant_rows = quant ? full->n_rows : 0;
  cudaError_t e;
  if (stage != kStageSelect) {
    {
      LaunchScope scope(ctx, st, RKV_KERNEL_SCORE);
      e = rkv::launch_score(cp, ctx->cfg.n_seq, st);
    }
    if (e != cudaSuccess) return cuda_fail(ctx, e, "score launch");
    ctx->launches += 1;
    if (stage == kStageScore) {
      ctx->pending_keys = {true, n_max, k_max, full->k, active, quant};
      rkv::note_launch(st, nullptr, nullptr);
      return RKV_OK;
    }
  }
  {
    LaunchScope scope(ctx, st, RKV_KERNEL_SELECT);
    e = rkv::launch_select(sp, ctx->cfg.n_seq, cluster, st);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "select launch");
  ctx->launches += 1;
  rkv::note_launch(st, nullptr, nullptr);
  return RKV_OK;
}

static rkv_status full_step_impl(rkv_ctx* ctx, const void* q, const rkv_cache* full, const int32_t* k_small,
                                 int32_t k_max, const int32_t* active, void* out, float* scores, int64_t score_stride,
                                 int32_t* topk_idx, void* q_last_full, int32_t max_len_hint, void* stream,
                                 bool score_only) {
  // everything the second half would reject is rejected before the first half launches
  if (!ctx || !q || !cache_ok(full) || !k_small || (!out && !score_only) || !topk_idx) return RKV_ERR_INVALID_ARG;
  if (k_max < 1 || k_max > ctx->cfg.max_small) return RKV_ERR_INVALID_ARG;
  const int n_max = max_len_hint == 0 ? ctx->cfg.max_len : max_len_hint;
  if (n_max < 1 || n_max > ctx->cfg.max_len) return RKV_ERR_INVALID_ARG;
  if (scores != nullptr && score_stride < n_max) return RKV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  rkv_status s = full_attention_part(ctx, q, full, active, out, max_len_hint, st, score_only, false);
  if (s != RKV_OK) return s;
  return select_part(ctx, q, full, k_small, k_max, active, out, scores, score_stride, topk_idx, q_last_full, st);
}

// The 8-bit cache's first half: as full_attention_part.  Without kept logits there is nothing for a second half.
// fold_out: finish out here in every form; otherwise *finished says whether the score pass has to.
static rkv_status quant_attention_part(rkv_ctx* ctx, const void* q, const rkv_quant_cache* full, const int32_t* active,
                                       void* out, int32_t max_len_hint, bool logits, bool fold_out, cudaStream_t st,
                                       bool* finished) {
  if (!ctx || !q || !quant_ok(full) || !out || !on_device(ctx)) return RKV_ERR_INVALID_ARG;
  const int n_max = max_len_hint == 0 ? ctx->cfg.max_len : max_len_hint;
  if (n_max < 1 || n_max > ctx->cfg.max_len) return RKV_ERR_INVALID_ARG;
  ctx->pending_full.valid = false;
  ctx->pending_keys.valid = false;
  QuantPass pass;
  rkv_status s = run_quant_attention(ctx, q, full, active, out, n_max, logits, fold_out, st, &pass);
  if (s != RKV_OK) return s;
  if (logits) ctx->pending_full = {true, rkv::kQuantTile, pass.gx, n_max, full->k, active, pass.counts, true};
  *finished = pass.finished;
  return RKV_OK;
}

rkv_status rkv_quant_full_attention(rkv_ctx* ctx, const void* q, const rkv_quant_cache* full, const int32_t* active,
                                    void* out, int32_t keep_logits, int32_t max_len_hint, void* stream) {
  bool finished = false;
  return quant_attention_part(ctx, q, full, active, out, max_len_hint, keep_logits != 0, true,
                              static_cast<cudaStream_t>(stream), &finished);
}

rkv_status rkv_quant_full_step(rkv_ctx* ctx, const void* q, const rkv_quant_cache* full, const int32_t* k_small,
                               int32_t k_max, const int32_t* active, void* out, float* scores, int64_t score_stride,
                               int32_t* topk_idx, void* q_last_full, int32_t max_len_hint, void* stream) {
  // everything the second half would reject is rejected before the first half launches
  if (!ctx || !q || !quant_ok(full) || !k_small || !out || !topk_idx) return RKV_ERR_INVALID_ARG;
  if (k_max < 1 || k_max > ctx->cfg.max_small) return RKV_ERR_INVALID_ARG;
  const int n_max = max_len_hint == 0 ? ctx->cfg.max_len : max_len_hint;
  if (n_max < 1 || n_max > ctx->cfg.max_len) return RKV_ERR_INVALID_ARG;
  if (scores != nullptr && score_stride < n_max) return RKV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  bool finished = false;   // the output is complete; otherwise the score pass folds it
  rkv_status s = quant_attention_part(ctx, q, full, active, out, max_len_hint, true, false, st, &finished);
  if (s != RKV_OK) return s;
  const rkv_cache sizes = sizes_of(full);
  return select_part(ctx, q, &sizes, k_small, k_max, active, finished ? nullptr : out, scores, score_stride, topk_idx, q_last_full, st);
}

rkv_status rkv_quant_score_keys(rkv_ctx* ctx, const void* q, const rkv_quant_cache* full, const int32_t* k_small,
                                int32_t k_max, const int32_t* active, float* scores, int64_t score_stride,
                                void* q_last_full, void* stream) {
  if (!ctx || !quant_ok(full) || !on_device(ctx)) return RKV_ERR_INVALID_ARG;
  const rkv_cache sizes = sizes_of(full);
  return rkv_score_keys(ctx, q, &sizes, k_small, k_max, active, scores, score_stride, q_last_full, stream);
}

rkv_status rkv_quant_select_topk(rkv_ctx* ctx, const void* q, const rkv_quant_cache* full, const int32_t* k_small,
                                 int32_t k_max, const int32_t* active, float* scores, int64_t score_stride,
                                 int32_t* topk_idx, void* q_last_full, void* stream) {
  if (!ctx || !quant_ok(full) || !on_device(ctx)) return RKV_ERR_INVALID_ARG;
  const rkv_cache sizes = sizes_of(full);
  return rkv_select_topk(ctx, q, &sizes, k_small, k_max, active, scores, score_stride, topk_idx, q_last_full, stream);
}

rkv_status rkv_quant_store(rkv_ctx* ctx, const void* k_new, int64_t k_seq_stride, int64_t k_tok_stride,
                           const void* v_new, int64_t v_seq_stride, int64_t v_tok_stride, int32_t n_tok,
                           const int32_t* start, const int32_t* count, const rkv_quant_cache* full, void* stream) {
  if (!ctx || !k_new || !v_new || !quant_ok(full) || !on_device(ctx)) return RKV_ERR_INVALID_ARG;
  if (!aligned16(k_new) || !aligned16(v_new) || ((k_seq_stride | k_tok_stride | v_seq_stride | v_tok_stride) & 7) != 0)
    return RKV_ERR_INVALID_ARG;   // the kernel reads 16 bytes at a time
  if (n_tok < 1) return RKV_ERR_INVALID_ARG;
  const rkv::QuantNew rows = {k_new, v_new, k_seq_stride, k_tok_stride, v_seq_stride, v_tok_stride, n_tok};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  {
    LaunchScope scope(ctx, st, RKV_KERNEL_APPEND);
    e = rkv::launch_quant_store(rows, start, count, dev_of(full), ctx->cfg.n_seq, ctx->cfg.n_kv_heads,
                                ctx->len_tickets, ctx->status, st);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "8-bit store launch");
  ctx->launches += 1;
  rkv::note_quant_store(st, full);
  return RKV_OK;
}

rkv_status rkv_quant_gather_small(rkv_ctx* ctx, const int32_t* topk_idx, const int32_t* k_small, int32_t k_max,
                                  const rkv_quant_cache* full, const rkv_cache* small_cache, const int32_t* active,
                                  void* stream) {
  if (!ctx || !topk_idx || !k_small || !quant_ok(full) || !cache_ok(small_cache) || !on_device(ctx))
    return RKV_ERR_INVALID_ARG;
  if (k_max < 1 || k_max > ctx->cfg.max_small) return RKV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  {
    LaunchScope scope(ctx, st, RKV_KERNEL_GATHER);
    e = rkv::launch_quant_gather(topk_idx, k_small, k_max, dev_of(full), dev_of(small_cache), small_cache->n_rows, active,
                                 ctx->cfg.n_seq, ctx->cfg.n_kv_heads, ctx->status, st);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "8-bit gather launch");
  ctx->launches += 1;
  rkv::note_launch(st, small_cache, nullptr);
  return RKV_OK;
}

rkv_status rkv_rope_frequencies(const rkv_rope_config* c, uint64_t* freqs, float* amplitude) {
  if (!c || !freqs || !amplitude) return RKV_ERR_INVALID_ARG;
  if (c->rot_dim < 16 || c->rot_dim > rkv::kHeadDim || c->rot_dim % 16 != 0 || c->scaling < RKV_ROPE_NONE ||
      c->scaling > RKV_ROPE_RAMP)
    return RKV_ERR_UNSUPPORTED;
  const bool scaled = c->scaling != RKV_ROPE_NONE;
  if (!(c->theta > 1.0) || isinf(c->theta) || (scaled && (!(c->factor >= 1.0) || isinf(c->factor))))
    return RKV_ERR_INVALID_ARG;
  if (c->scaling >= RKV_ROPE_BANDS && c->trained_len < 1) return RKV_ERR_INVALID_ARG;
  if (c->scaling == RKV_ROPE_BANDS && !(c->low > 0.0 && c->low < c->high)) return RKV_ERR_INVALID_ARG;
  if (c->scaling == RKV_ROPE_RAMP && !(c->slow > 0.0 && c->slow < c->fast)) return RKV_ERR_INVALID_ARG;
  constexpr long double kTwoPi = 6.283185307179586476925286766559L;
  const long double factor = scaled ? c->factor : 1.0L, ln_theta = logl((long double)c->theta);
  double first = 0.0, last = 0.0;
  if (c->scaling == RKV_ROPE_RAMP) {   // the pairs that turn `fast` and `slow` times over the trained length
    auto at = [&](double turns) {
      return (double)(c->rot_dim * logl(c->trained_len / (turns * kTwoPi)) / (2.0L * ln_theta));
    };
    first = fmax(floor(at(c->fast)), 0.0);
    last = fmin(ceil(at(c->slow)), (double)(c->rot_dim - 1));
  }
  for (int i = 0; i < c->rot_dim / 2; ++i) {
    const long double w = expl(-2.0L * i / c->rot_dim * ln_theta);
    long double stretched = 1.0L;      // share of w / factor
    if (!scaled) {
      stretched = 0.0L;
    } else if (c->scaling == RKV_ROPE_BANDS) {
      const long double turns = c->trained_len * w / kTwoPi;
      const long double kept = turns >= c->high ? 1.0L : turns <= c->low ? 0.0L : (turns - c->low) / ((long double)c->high - c->low);
      stretched = 1.0L - kept;
    } else if (c->scaling == RKV_ROPE_RAMP) {
      stretched = fmin(fmax((i - first) / fmax(last - first, 0.001), 0.0), 1.0);
    }
    const long double f = (w * (1.0L - stretched) + w / factor * stretched) / kTwoPi;   // < 0.16 turns per position
    freqs[i] = (uint64_t)roundl(ldexpl(f, 64));
  }
  *amplitude = c->scaling == RKV_ROPE_RAMP ? (float)(0.1L * logl(factor) + 1.0L) : 1.0f;
  return RKV_OK;
}

rkv_status rkv_rope(rkv_ctx* ctx, const void* qkv, int32_t is_bf16, int64_t tok_stride, const int32_t* pos,
                    int32_t n_tok, int32_t n_q, int32_t n_kv, const uint64_t* freqs, int32_t rot_dim, int32_t layout,
                    float amplitude, void* q, void* k, void* v, void* stream) {
  if (!ctx || !qkv || !pos || !freqs || !q || !k || n_tok < 1 || n_q < 1 || n_kv < 1 || n_q > (1 << 16) ||
      n_kv > (1 << 16) || !on_device(ctx))
    return RKV_ERR_INVALID_ARG;
  if (rot_dim < 16 || rot_dim > rkv::kHeadDim || rot_dim % 16 != 0 || (layout != RKV_ROPE_HALF && layout != RKV_ROPE_INTERLEAVED))
    return RKV_ERR_UNSUPPORTED;
  if (!aligned16(qkv) || !aligned16(q) || !aligned16(k) || !aligned16(v) || (tok_stride * (is_bf16 ? 2 : 4)) % 16 != 0 ||
      (reinterpret_cast<uintptr_t>(freqs) & 7) != 0)
    return RKV_ERR_INVALID_ARG;   // the kernel reads and writes 16 bytes at a time
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  {
    LaunchScope scope(ctx, st, RKV_KERNEL_ROPE);
    e = rkv::launch_rope(qkv, is_bf16 != 0, tok_stride, pos, n_tok, n_q, n_kv, freqs,
                         rot_dim, layout == RKV_ROPE_INTERLEAVED, amplitude, q, k, v, st);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "rotary launch");
  ctx->launches += 1;
  // with one KV head the outputs can be a cache's own rows
  const size_t q_bytes = (size_t)n_tok * n_q * rkv::kHeadDim * 2, kv_bytes = (size_t)n_tok * n_kv * rkv::kHeadDim * 2;
  rkv::note_rows(st, {{q, q_bytes}, {k, kv_bytes}, {v, kv_bytes}});
  return RKV_OK;
}

// ------------------------------------------------------------------------------------------------------ the paged cache
rkv_status rkv_paged_append(rkv_ctx* ctx, const void* qkv, int32_t is_bf16, int64_t seq_stride, int64_t tok_stride,
                            int32_t n_tok, const int32_t* start, const int32_t* count, const uint64_t* freqs,
                            int32_t rot_dim, int32_t layout, float amplitude, const rkv_paged_cache* cache, void* q,
                            void* stream) {
  if (!ctx || !qkv || !q || n_tok < 1 || !paged_ok(ctx, cache) || !on_device(ctx)) return RKV_ERR_INVALID_ARG;
  if (freqs != nullptr && (rot_dim < 16 || rot_dim > rkv::kHeadDim || rot_dim % 16 != 0 ||
                           (layout != RKV_ROPE_HALF && layout != RKV_ROPE_INTERLEAVED)))
    return RKV_ERR_UNSUPPORTED;
  const int64_t size = is_bf16 ? 2 : 4;
  if (!aligned16(qkv) || !aligned16(q) || (seq_stride * size) % 16 != 0 || (tok_stride * size) % 16 != 0 ||
      (reinterpret_cast<uintptr_t>(freqs) & 7) != 0)
    return RKV_ERR_INVALID_ARG;   // the kernel reads and writes 16 bytes at a time
  rkv::PagedAppendParams p;
  memset(&p, 0, sizeof(p));
  p.c = dev_of(ctx, cache);
  p.qkv = qkv;
  p.seq_stride = seq_stride;
  p.tok_stride = tok_stride;
  p.start = start;
  p.count = count;
  p.freqs = reinterpret_cast<const unsigned long long*>(freqs);
  p.q = q;
  p.tickets = ctx->len_tickets;
  p.status = ctx->status;
  p.n_tok = n_tok;
  p.n_q_heads = ctx->cfg.n_q_heads;
  p.rot = freqs != nullptr ? rot_dim : 0;
  p.amp = amplitude;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  {
    LaunchScope scope(ctx, st, RKV_KERNEL_APPEND);
    e = rkv::launch_paged_append(p, is_bf16 != 0, freqs != nullptr && layout == RKV_ROPE_INTERLEAVED, ctx->cfg.n_seq,
                                 ctx->sm_count, st);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "paged append launch");
  ctx->launches += 1;
  // (a pool, or the queries, may lie in memory that another cache's calls read early)
  const size_t pool = (size_t)cache->n_pages * ctx->cfg.n_kv_heads * cache->page * rkv::kHeadDim * 2;
  const size_t bounds = pool / cache->page, q_bytes = (size_t)ctx->cfg.n_seq * n_tok * ctx->cfg.n_q_heads * rkv::kHeadDim * 2;
  rkv::note_rows(st, {{cache->k, pool}, {cache->v, pool}, {cache->k_min, bounds}, {cache->k_max, bounds}, {q, q_bytes}});
  return RKV_OK;
}

// The pass over pages, in one of three forms:
//   splits    a head's tiles are dealt out in turn to as many CTAs per KV head as fit one wave (two to an SM), a fold finishes
//   cluster   1, 2, 4 or 8 CTAs per (sequence, KV head) are a cluster and finish the output themselves
//   balanced  longer batches, and what sequences hold behind a shared prefix (whose partials have to be folded in any case):
//             equal runs of tiles across heads and sequences, then the fold
// A cluster has at most eight CTAs and a wave of them is not always full, so it is for so many tiles a CTA:
//   one sequence 16; batches whose CTAs fill their waves to four fifths 32, and 64 of listed pages, where sequences differ less in
//   what they attend; other batches 8.
// Cluster / otherwise, us (sequences x heads x group, positions; ragged: lengths from 0 to that; one cache again and again; * what
// is taken):
//   1 x 8 x 4   1024  *4.3 / 6.5   4096 *6.4 / 8.6   8192 *8.8 / 9.7   12000 11.3 / *10.6   16384 14.2 / *11.9
//   4 x 8 x 4   8192 *23.1 / 24.3, ragged *16.5 / 18.6     32768 79.8 / *81.2, ragged 28.2 / *30.4
//   8 x 8 x 4   4096 *22.8 / 24.5, ragged *15.8 / 17.3     16384 80.2 / *83.4, ragged 44.0 / *37.7
//  16 x 4 x 7   8192 *42.6 / 46.3, ragged *27.1 / 28.9     32768 156.3 / *160.1, ragged 85.3 / *71.7
//  64 x 8 x 4   2048 *78.9 / 84.8, ragged *46.6 / 47.2      8192 293.9 / *311.2, ragged 169.4 / *156.3
//   listed, with its selection: 8 x 8 x 4, 4096 of 32768 *35.7 / 38.9, ragged *27.3 / 34.2
//                              64 x 8 x 4, 4096 of 8192 *170.6 / 184.4, ragged *136.1 / 137.2
// Wide CTAs (one to an SM) pay where all clusters are resident at once: eight-CTA clusters find room for 14 on 148 SMs.  Wide /
// narrow: 14 heads, 4096 positions *6.5 / 7.6; 16 heads 12.2 / *8.3; 2 x 8 heads, 2048 of 32768 listed 19.3 / *14.3.
struct PagedForm { bool cluster, wide; int gx; };
static PagedForm paged_form(const rkv_ctx* ctx, int first_slot, int most, bool listed) {
  const int64_t bg = (int64_t)ctx->cfg.n_seq * ctx->cfg.n_kv_heads, slots = 2 * ctx->sm_count;
  const int tiles = (most + rkv::kTile - 1) / rkv::kTile, room = ctx->max_splits - first_slot;
  int gx = (int)(slots / bg);
  if (gx > room) gx = room;
  if (gx > tiles) gx = tiles;
  if (gx < 1) gx = 1;
  const int cluster_gx = gx >= 8 ? 8 : gx >= 4 ? 4 : gx >= 2 ? 2 : 1;
  const int64_t ctas = cluster_gx * bg, waves = (ctas + slots - 1) / slots;
  const int limit = 5 * ctas >= 4 * waves * slots ? (listed ? 64 : 32) : ctx->cfg.n_seq == 1 ? 16 : 8;
  const bool cluster = first_slot == 0 && tiles <= limit * cluster_gx;
  return {cluster, cluster && 5 * ctas <= 4 * ctx->sm_count, cluster ? cluster_gx : gx};
}

static rkv_status run_paged_attention(rkv_ctx* ctx, rkv::PagedAttnParams& p, const rkv_paged_cache* cache, int most,
                                      int kind, cudaStream_t st) {
  CUtensorMap tm_k, tm_v;
  const int64_t rows = cache->n_pages * ctx->cfg.n_kv_heads * cache->page;
  const int box = cache->page < rkv::kTile ? cache->page : rkv::kTile;
  rkv_status s = tensor_map(ctx, cache->k, rows, &tm_k, false, box);
  if (s != RKV_OK) return s;
  s = tensor_map(ctx, cache->v, rows, &tm_v, false, box);
  if (s != RKV_OK) return s;
  const int64_t bg = (int64_t)ctx->cfg.n_seq * ctx->cfg.n_kv_heads, slots = 2 * ctx->sm_count;
  const PagedForm form = paged_form(ctx, p.first_slot, most, p.page_idx != nullptr);
  const bool cluster = form.cluster;
  const int gx = form.gx;
  // tiles that there can be: behind a shared prefix a sequence may be shorter than that, but not as long in all
  const int64_t units = bg * ((p.max_len + rkv::kTile - 1) / rkv::kTile + 1);
  const bool balanced = !cluster && ctx->cfg.n_seq > 1 && ctx->cfg.n_seq <= rkv::kBalancedMaxSeq &&
                        units * (slots + 1) < (int64_t(1) << 32);   // (the kernel cuts the runs in 32 bits)
  p.counts = balanced ? ctx->split_counts : nullptr;
  cudaError_t e;
  {
    LaunchScope scope(ctx, st, kind);
    e = balanced ? rkv::launch_paged_balanced(p, tm_k, tm_v, (int)(units < slots ? units : slots), st)
                 : rkv::launch_paged_attention(p, tm_k, tm_v, ctx->cfg.n_seq, gx, cluster, form.wide, st);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "paged attention launch");
  ctx->launches += 1;
  rkv::note_launch(st, nullptr, nullptr);
  if (cluster) return RKV_OK;
  {
    LaunchScope scope(ctx, st, RKV_KERNEL_FOLD);
    e = rkv::launch_paged_fold(p, ctx->cfg.n_seq, gx, st);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "fold launch");
  ctx->launches += 1;
  rkv::note_launch(st, nullptr, nullptr, true);
  return RKV_OK;
}

static rkv::PagedAttnParams paged_params(const rkv_ctx* ctx, const rkv_paged_cache* cache, const void* q,
                                         const int32_t* active, void* out, int n_max) {
  rkv::PagedAttnParams p;
  memset(&p, 0, sizeof(p));
  p.c = dev_of(ctx, cache);
  p.q = q;
  p.active = active;
  p.out = out;
  p.partials = ctx->partials;
  p.ml_t = ctx->ml_t;
  p.status = ctx->status;
  p.n_seq = ctx->cfg.n_seq;
  p.n_q_heads = ctx->cfg.n_q_heads;
  p.group = ctx->group;
  p.max_splits = ctx->max_splits;
  p.max_len = n_max;
  p.scale = ctx->cfg.softmax_scale;
  return p;
}

rkv_status rkv_paged_attention(rkv_ctx* ctx, const void* q, const rkv_paged_cache* cache, const int32_t* active,
                               const int32_t* shared, int32_t n_shared, void* out, int32_t max_len_hint, void* stream) {
  if (!ctx || !q || !out || !paged_ok(ctx, cache) || !on_device(ctx) || !aligned16(q) || !aligned16(out))
    return RKV_ERR_INVALID_ARG;
  const int n_max = max_len_hint == 0 ? ctx->cfg.max_len : max_len_hint;
  if (n_max < 1 || n_max > ctx->cfg.max_len || n_shared < 0 || (shared == nullptr) != (n_shared == 0))
    return RKV_ERR_INVALID_ARG;
  ctx->pending_full.valid = false;   // its partials and logits are about to be overwritten
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  rkv::PagedAttnParams p = paged_params(ctx, cache, q, active, out, n_max);
  const int64_t from = (int64_t)n_shared * cache->page;
  // A batch of one shares with nobody; there has to be a slot for the shared positions beside the sequences' own; and the pass
  // over them, a pass over the sequences' own and the fold take about 11 us whatever there is to do.
  if (from == 0 || from > n_max || ctx->cfg.n_seq == 1 || ctx->max_splits < 2 ||
      from * ctx->cfg.n_seq * ctx->cfg.n_kv_heads < ctx->shared_min)
    return run_paged_attention(ctx, p, cache, n_max, RKV_KERNEL_ATTN_FULL, st);
  rkv::PrefixAttnParams x;
  memset(&x, 0, sizeof(x));
  x.c = p.c;
  x.q = q;
  x.shared = shared;
  x.partials = ctx->partials;
  x.ml_t = ctx->ml_t;
  x.status = ctx->status;
  x.n_rows = cache->n_pages * ctx->cfg.n_kv_heads * cache->page;
  x.n_shared = n_shared;
  x.n_seq = ctx->cfg.n_seq;
  x.n_q_heads = ctx->cfg.n_q_heads;
  x.group = ctx->group;
  x.max_splits = ctx->max_splits;
  x.scale = ctx->cfg.softmax_scale;
  CUtensorMap tm_k, tm_v;
  const int box = cache->page < rkv::kPrefixTile ? cache->page : rkv::kPrefixTile;
  rkv_status s = tensor_map(ctx, cache->k, x.n_rows, &tm_k, false, box, 1);
  if (s != RKV_OK) return s;
  s = tensor_map(ctx, cache->v, x.n_rows, &tm_v, false, box, 1);
  if (s != RKV_OK) return s;
  // one wave of CTAs, one to an SM
  const int tiles = (int)((from + rkv::kPrefixTile - 1) / rkv::kPrefixTile);
  const int blocks = (ctx->cfg.n_seq * ctx->group + 255) / 256 * ctx->cfg.n_kv_heads;
  int splits = ctx->sm_count / blocks;
  if (splits > tiles) splits = tiles;
  if (splits > ctx->max_splits / 2) splits = ctx->max_splits / 2;
  if (splits < 1) splits = 1;
  cudaError_t e;
  {
    LaunchScope scope(ctx, st, RKV_KERNEL_ATTN_FULL);
    e = rkv::launch_prefix_attention(x, tm_k, tm_v, splits, st);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "shared attention launch");
  ctx->launches += 1;
  rkv::note_launch(st, nullptr, nullptr);
  p.from = (int)from;
  p.first_slot = splits;
  return run_paged_attention(ctx, p, cache, n_max > from ? n_max - (int)from : 1, RKV_KERNEL_ATTN_FULL, st);
}

rkv_status rkv_paged_sparse_attention(rkv_ctx* ctx, const void* q, const rkv_paged_cache* cache, const int32_t* active,
                                      int32_t top_pages, int32_t first_pages, int32_t last_pages, int32_t* page_idx,
                                      void* out, int32_t max_len_hint, void* stream) {
  if (!ctx || !q || !out || !page_idx || !paged_ok(ctx, cache) || !cache->k_min || !on_device(ctx) || !aligned16(q) ||
      !aligned16(out) || top_pages < 1 || first_pages < 0 || last_pages < 0)
    return RKV_ERR_INVALID_ARG;
  const int n_max = max_len_hint == 0 ? ctx->cfg.max_len : max_len_hint;
  if (n_max < 1 || n_max > ctx->cfg.max_len) return RKV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ctx->pending_full.valid = false;
  int most = (n_max - 1) / cache->page + 1;
  if (most > cache->table_stride) most = cache->table_stride;
  rkv::PageSelectParams sp;
  memset(&sp, 0, sizeof(sp));
  sp.c = dev_of(ctx, cache);
  sp.q = q;
  sp.active = active;
  sp.keys = reinterpret_cast<uint64_t*>(ctx->logits);       // (8 bytes a page of 16 positions or more, of 16 or more a position)
  sp.key_stride = ctx->logit_stride * ctx->gp / 2;
  sp.page_idx = page_idx;
  sp.status = ctx->status;
  sp.n_q_heads = ctx->cfg.n_q_heads;
  sp.group = ctx->group;
  sp.top = top_pages;
  sp.first = first_pages;
  sp.last = last_pages;
  sp.max_len = n_max;
  cudaError_t e;
  {
    LaunchScope scope(ctx, st, RKV_KERNEL_SELECT);
    e = rkv::launch_page_scores(sp, ctx->cfg.n_seq, most, st);
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "page score launch");
  ctx->launches += 1;
  rkv::note_launch(st, nullptr, nullptr);
  rkv::PagedAttnParams p = paged_params(ctx, cache, q, active, out, n_max);
  p.page_idx = page_idx;
  p.top = top_pages;
  const int taken = top_pages < most ? top_pages : most;
  if (paged_form(ctx, 0, taken * cache->page, true).cluster && most <= rkv::kMaxPickFrom && taken <= rkv::kMaxPicked) {
    p.keys = sp.keys;
    p.key_stride = sp.key_stride;
    p.first = first_pages;
    p.last = last_pages;
  } else {
    {
      LaunchScope scope(ctx, st, RKV_KERNEL_SELECT);
      e = rkv::launch_page_select(sp, ctx->cfg.n_seq, most, st);
    }
    if (e != cudaSuccess) return cuda_fail(ctx, e, "page selection launch");
    ctx->launches += 1;
    rkv::note_launch(st, nullptr, nullptr);
  }
  return run_paged_attention(ctx, p, cache, taken * cache->page, RKV_KERNEL_ATTN_SMALL, st);
}

rkv_status rkv_full_step(rkv_ctx* ctx, const void* q, const rkv_cache* full, const int32_t* k_small, int32_t k_max,
                         const int32_t* active, void* out, float* scores, int64_t score_stride, int32_t* topk_idx,
                         void* q_last_full, int32_t max_len_hint, void* stream) {
  return full_step_impl(ctx, q, full, k_small, k_max, active, out, scores, score_stride, topk_idx, q_last_full,
                        max_len_hint, stream, false);
}

rkv_status rkv_score_step(rkv_ctx* ctx, const void* q, const rkv_cache* full, const int32_t* k_small, int32_t k_max,
                          const int32_t* active, float* scores, int64_t score_stride, int32_t* topk_idx,
                          void* q_last_full, int32_t max_len_hint, void* stream) {
  return full_step_impl(ctx, q, full, k_small, k_max, active, nullptr, scores, score_stride, topk_idx, q_last_full,
                        max_len_hint, stream, true);
}

rkv_status rkv_full_attention(rkv_ctx* ctx, const void* q, const rkv_cache* full, const int32_t* active, void* out,
                              int32_t max_len_hint, void* stream) {
  return full_attention_part(ctx, q, full, active, out, max_len_hint, static_cast<cudaStream_t>(stream), false, true);
}

rkv_status rkv_append_full_attention(rkv_ctx* ctx, const void* q, const void* k_new, const void* v_new,
                                     const rkv_cache* full, const int32_t* active, void* out, int32_t max_len_hint,
                                     void* stream) {
  if (!k_new || !v_new) return RKV_ERR_INVALID_ARG;
  const AppendArgs app = {k_new, v_new, nullptr, nullptr, nullptr, nullptr, 0};   // one cache: the attended one
  return full_attention_part(ctx, q, full, active, out, max_len_hint, static_cast<cudaStream_t>(stream), false, true,
                             &app);
}

rkv_status rkv_select_topk(rkv_ctx* ctx, const void* q, const rkv_cache* full, const int32_t* k_small, int32_t k_max,
                           const int32_t* active, float* scores, int64_t score_stride, int32_t* topk_idx,
                           void* q_last_full, void* stream) {
  if (ctx != nullptr && ctx->pending_keys.valid) {   // rkv_score_keys has run: the selection alone is left
    if (full == nullptr || ctx->pending_keys.full_k != full->k || ctx->pending_keys.active != active ||
        scores != nullptr || q_last_full != nullptr)
      return RKV_ERR_INVALID_ARG;   // (scores and q_last_full are outputs of the score pass)
    return select_part(ctx, q, full, k_small, k_max, active, nullptr, nullptr, 0, topk_idx, nullptr,
                       static_cast<cudaStream_t>(stream), kStageSelect);
  }
  if (ctx != nullptr && ctx->pending_full.valid && full != nullptr &&
      (ctx->pending_full.full_k != full->k || ctx->pending_full.active != active))
    return RKV_ERR_INVALID_ARG;   // not the cache / mask of the attention pass it completes
  return select_part(ctx, q, full, k_small, k_max, active, nullptr, scores, score_stride, topk_idx, q_last_full,
                     static_cast<cudaStream_t>(stream));
}

rkv_status rkv_score_keys(rkv_ctx* ctx, const void* q, const rkv_cache* full, const int32_t* k_small, int32_t k_max,
                          const int32_t* active, float* scores, int64_t score_stride, void* q_last_full,
                          void* stream) {
  if (ctx != nullptr && ctx->pending_full.valid && full != nullptr &&
      (ctx->pending_full.full_k != full->k || ctx->pending_full.active != active))
    return RKV_ERR_INVALID_ARG;   // not the cache / mask of the attention pass it completes
  return select_part(ctx, q, full, k_small, k_max, active, nullptr, scores, score_stride, nullptr, q_last_full,
                     static_cast<cudaStream_t>(stream), kStageScore);
}

rkv_status rkv_gather_small(rkv_ctx* ctx, const int32_t* topk_idx, const int32_t* k_small, int32_t k_max,
                            const rkv_cache* full, const rkv_cache* small_cache, const int32_t* active,
                            void* stream) {
  if (!ctx || !topk_idx || !k_small || !cache_ok(full) || !cache_ok(small_cache)) return RKV_ERR_INVALID_ARG;
  if (k_max < 1 || k_max > ctx->cfg.max_small) return RKV_ERR_INVALID_ARG;
  cudaError_t e;
  {
    LaunchScope scope(ctx, static_cast<cudaStream_t>(stream), RKV_KERNEL_GATHER);
    e = rkv::launch_gather(topk_idx, k_small, k_max, dev_of(full), dev_of(small_cache), active, ctx->cfg.n_seq,
                           ctx->cfg.n_kv_heads, ctx->status, static_cast<cudaStream_t>(stream));
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "gather launch");
  ctx->launches += 1;
  rkv::note_launch(static_cast<cudaStream_t>(stream), small_cache, nullptr);
  return RKV_OK;
}

rkv_status rkv_small_step(rkv_ctx* ctx, const void* q, const rkv_cache* small_cache, const int32_t* active,
                          void* out, int32_t max_len_hint, void* stream) {
  if (!ctx || !q || !cache_ok(small_cache) || !out) return RKV_ERR_INVALID_ARG;
  int n_max = max_len_hint == 0 ? ctx->cfg.max_small : max_len_hint;
  if (n_max < 1 || n_max > ctx->cfg.max_small) return RKV_ERR_INVALID_ARG;
  return run_attention(ctx, q, small_cache, active, out, n_max, n_max, false, static_cast<cudaStream_t>(stream),
                       nullptr, nullptr);
}

rkv_status rkv_append_small_step(rkv_ctx* ctx, const void* q, const void* k_new, const void* v_new,
                                 const rkv_cache* full, const rkv_cache* small_cache, const int32_t* active,
                                 void* out, int32_t max_len_hint, void* stream) {
  if (!ctx || !q || !k_new || !v_new || !cache_ok(small_cache) || !out) return RKV_ERR_INVALID_ARG;
  if (full != nullptr && !cache_ok(full)) return RKV_ERR_INVALID_ARG;
  int n_max = max_len_hint == 0 ? ctx->cfg.max_small : max_len_hint;
  if (n_max < 1 || n_max > ctx->cfg.max_small) return RKV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (cluster_eligible(ctx, n_max)) {   // one launch: the attention kernel appends
    const AppendArgs app = {k_new, v_new, full, nullptr, nullptr, nullptr, 0};
    return run_attention(ctx, q, small_cache, active, out, n_max, n_max, false, st, nullptr, nullptr, &app);
  }
  rkv_status s = rkv_append(ctx, k_new, v_new, full, small_cache, stream);
  if (s != RKV_OK) return s;
  return run_attention(ctx, q, small_cache, active, out, n_max, n_max, false, st, nullptr, nullptr);
}

// Largest small cache whose eviction order one block can sort in shared memory.
constexpr int kEvictMaxK = 4096;

rkv_status rkv_gather_small_evict(rkv_ctx* ctx, const int32_t* topk_idx, const int32_t* k_small, int32_t k_max,
                                  const rkv_cache* full, const rkv_cache* small_cache, const int32_t* active,
                                  int32_t* evict_order, int32_t* evict_count, int32_t max_evict, void* stream) {
  if (!evict_order || !evict_count || max_evict < 1 || max_evict > kEvictMaxK) return RKV_ERR_INVALID_ARG;
  if (k_max > kEvictMaxK) return RKV_ERR_UNSUPPORTED;
  rkv_status s = rkv_gather_small(ctx, topk_idx, k_small, k_max, full, small_cache, active, stream);
  if (s != RKV_OK) return s;
  cudaError_t e;
  {
    LaunchScope scope(ctx, static_cast<cudaStream_t>(stream), RKV_KERNEL_GATHER);
    e = rkv::launch_evict_order(ctx->win_keys, ctx->cfg.max_small, k_small, k_max, full->len, active, evict_order,
                                evict_count, max_evict, ctx->cfg.n_seq, ctx->cfg.n_kv_heads,
                                static_cast<cudaStream_t>(stream));
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "eviction-order launch");
  ctx->launches += 1;
  rkv::note_launch(static_cast<cudaStream_t>(stream), nullptr, nullptr);
  return RKV_OK;
}

rkv_status rkv_append_small_step_evict(rkv_ctx* ctx, const void* q, const void* k_new, const void* v_new,
                                       const rkv_cache* full, const rkv_cache* small_cache, const int32_t* k_small,
                                       const int32_t* active, void* out, const int32_t* evict_order,
                                       int32_t* evict_count, int32_t max_evict, int32_t max_len_hint, void* stream) {
  if (!ctx || !q || !k_new || !v_new || !cache_ok(small_cache) || !out || !k_small || !evict_order || !evict_count)
    return RKV_ERR_INVALID_ARG;
  if (full != nullptr && !cache_ok(full)) return RKV_ERR_INVALID_ARG;
  if (max_evict < 1 || max_evict > kEvictMaxK) return RKV_ERR_INVALID_ARG;
  int n_max = max_len_hint == 0 ? ctx->cfg.max_small : max_len_hint;
  if (n_max < 1 || n_max > ctx->cfg.max_small) return RKV_ERR_INVALID_ARG;
  if (!cluster_eligible(ctx, n_max)) return RKV_ERR_UNSUPPORTED;   // the evicting append lives in the clustered kernel
  const AppendArgs app = {k_new, v_new, full, evict_order, evict_count, k_small, max_evict};
  return run_attention(ctx, q, small_cache, active, out, n_max, n_max, false, static_cast<cudaStream_t>(stream), nullptr,
                       nullptr, &app);
}

rkv_status rkv_append(rkv_ctx* ctx, const void* k_new, const void* v_new, const rkv_cache* full,
                      const rkv_cache* small_cache, void* stream) {
  if (!ctx || !k_new || !v_new || (full == nullptr && small_cache == nullptr)) return RKV_ERR_INVALID_ARG;
  if ((full && !cache_ok(full)) || (small_cache && !cache_ok(small_cache))) return RKV_ERR_INVALID_ARG;
  CacheDev none = {nullptr, nullptr, nullptr, nullptr, nullptr};
  cudaError_t e;
  {
    LaunchScope scope(ctx, static_cast<cudaStream_t>(stream), RKV_KERNEL_APPEND);
    e = rkv::launch_append(k_new, v_new, full ? dev_of(full) : none, small_cache ? dev_of(small_cache) : none,
                           full != nullptr, small_cache != nullptr, ctx->cfg.n_seq, ctx->cfg.n_kv_heads, ctx->status,
                           static_cast<cudaStream_t>(stream));
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "append launch");
  ctx->launches += 1;
  rkv::note_launch(static_cast<cudaStream_t>(stream), full, small_cache);
  return RKV_OK;
}

rkv_status rkv_should_refresh(rkv_ctx* ctx, const void* q_now, const void* q_last_full, float threshold,
                              int32_t* flag, int32_t* keep, float* sim, void* stream) {
  if (!ctx || !q_now || !q_last_full || !flag) return RKV_ERR_INVALID_ARG;
  cudaError_t e;
  {
    LaunchScope scope(ctx, static_cast<cudaStream_t>(stream), RKV_KERNEL_TRIGGER);
    e = rkv::launch_trigger(q_now, q_last_full, threshold, flag, keep, sim, ctx->cfg.n_seq, ctx->cfg.n_q_heads,
                            static_cast<cudaStream_t>(stream));
  }
  if (e != cudaSuccess) return cuda_fail(ctx, e, "trigger launch");
  ctx->launches += 1;
  rkv::note_launch(static_cast<cudaStream_t>(stream), nullptr, nullptr);
  return RKV_OK;
}

rkv_status rkv_get_device_status(rkv_ctx* ctx, int32_t* host_bits, void* stream) {
  if (!ctx || !host_bits) return RKV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t bits = 0;
  cudaError_t e = cudaMemcpyAsync(&bits, ctx->status, sizeof(bits), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaMemsetAsync(ctx->status, 0, sizeof(int32_t), st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return cuda_fail(ctx, e, "status read");
  *host_bits = bits;
  return bits == 0 ? RKV_OK : RKV_ERR_DEVICE_CHECK;
}

const char* rkv_status_string(rkv_status s) {
  switch (s) {
    case RKV_OK: return "ok";
    case RKV_ERR_INVALID_ARG: return "invalid argument";
    case RKV_ERR_UNSUPPORTED: return "unsupported configuration";
    case RKV_ERR_WORKSPACE: return "workspace allocation failed";
    case RKV_ERR_CUDA: return "CUDA error";
    case RKV_ERR_DEVICE_CHECK: return "device-side check failed";
  }
  return "unknown status";
}

const char* rkv_last_cuda_error(const rkv_ctx* ctx) { return ctx ? ctx->last_error.c_str() : ""; }

int64_t rkv_launch_count(const rkv_ctx* ctx) { return ctx ? ctx->launches : 0; }

rkv_status rkv_set_option(rkv_ctx* ctx, int32_t option, int32_t value) {
  if (!ctx) return RKV_ERR_INVALID_ARG;
  switch (option) {
    case RKV_OPT_SMALL_MIN_CHUNK:
      if (value < rkv::kTile || value > (1 << 20)) return RKV_ERR_INVALID_ARG;
      ctx->small_min_chunk = value;
      return RKV_OK;
    case RKV_OPT_SMALL_CLUSTER:
      ctx->small_cluster = value != 0;
      return RKV_OK;
    case RKV_OPT_DEPENDENT_LAUNCH:
      rkv::g_use_pdl = value != 0;
      return RKV_OK;
    case RKV_OPT_EARLY_CACHE_READ:
      ctx->early_read = value != 0;
      return RKV_OK;
    case RKV_OPT_INTERLEAVE_TILES:
      ctx->interleave = value != 0;
      return RKV_OK;
    case RKV_OPT_SELECT_KEYS_PER_CTA:
      if (value < 512 || value > rkv::kSelectMaxKeysPerCta) return RKV_ERR_INVALID_ARG;
      ctx->select_keys_per_cta = value;
      return RKV_OK;
    case RKV_OPT_SCORE_SLICE:
      if (value != 0 && value != 1024 && value != 2048 && value != 4096 && value != rkv::kSelectMaxSlice)
        return RKV_ERR_INVALID_ARG;
      ctx->score_slice = value;
      return RKV_OK;
    case RKV_OPT_SHARED_MIN:
      if (value < 0) return RKV_ERR_INVALID_ARG;
      ctx->shared_min = value;
      return RKV_OK;
    default:
      return RKV_ERR_INVALID_ARG;
  }
}

rkv_status rkv_get_option(const rkv_ctx* ctx, int32_t option, int32_t* value) {
  if (!ctx || !value) return RKV_ERR_INVALID_ARG;
  switch (option) {
    case RKV_OPT_SMALL_MIN_CHUNK: *value = ctx->small_min_chunk; return RKV_OK;
    case RKV_OPT_SMALL_CLUSTER: *value = ctx->small_cluster; return RKV_OK;
    case RKV_OPT_DEPENDENT_LAUNCH: *value = rkv::g_use_pdl ? 1 : 0; return RKV_OK;
    case RKV_OPT_EARLY_CACHE_READ: *value = ctx->early_read; return RKV_OK;
    case RKV_OPT_INTERLEAVE_TILES: *value = ctx->interleave; return RKV_OK;
    case RKV_OPT_SELECT_KEYS_PER_CTA: *value = ctx->select_keys_per_cta; return RKV_OK;
    case RKV_OPT_SCORE_SLICE: *value = ctx->score_slice; return RKV_OK;
    case RKV_OPT_SHARED_MIN: *value = ctx->shared_min; return RKV_OK;
    default: return RKV_ERR_INVALID_ARG;
  }
}

rkv_status rkv_set_profiling(rkv_ctx* ctx, int32_t on) {
  if (!ctx) return RKV_ERR_INVALID_ARG;
  ctx->profiling = on != 0;
  return RKV_OK;
}

rkv_status rkv_get_profile(rkv_ctx* ctx, double* total_us, int64_t* launches) {
  if (!ctx || !total_us || !launches) return RKV_ERR_INVALID_ARG;
  for (int i = 0; i < RKV_KERNEL_KINDS; ++i) { total_us[i] = 0.0; launches[i] = 0; }
  for (auto& t : ctx->timed) {
    cudaError_t e = cudaEventSynchronize(t.stop);
    float ms = 0.f;
    if (e == cudaSuccess) e = cudaEventElapsedTime(&ms, t.start, t.stop);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "profile read");
    total_us[t.kind] += 1000.0 * ms;
    launches[t.kind] += 1;
    ctx->event_pool.push_back(t.start);
    ctx->event_pool.push_back(t.stop);
  }
  ctx->timed.clear();
  return RKV_OK;
}

}  // extern "C"

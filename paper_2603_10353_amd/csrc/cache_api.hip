// C-ABI entry points of the 8-bit key/value cache: argument checks and dispatch to the kernel launchers.
#include <cmath>
#include <cstring>

#include "cache_common.h"

namespace shplb {
namespace {

bool misaligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) & (to - 1); }

int32_t check_cache(const shplb_cache* c, CacheArgs* a) {
  if (!c) return SHPLB_E_NULL;
  if (c->n_seq < 1 || c->n_kv_heads < 1 || c->max_pages < 1 || c->n_pages < 1) return SHPLB_E_SHAPE;
  if (int64_t(c->n_seq) * c->n_kv_heads > SHPLB_MAX_SEQ_HEADS || c->max_pages > SHPLB_MAX_BLOCKS) return SHPLB_E_UNSUPPORTED;
  if (c->head_dim != kHeadDim || (c->block != 64 && c->block != 128)) return SHPLB_E_UNSUPPORTED;
  if (c->format != SHPLB_CACHE_E4M3 && c->format != SHPLB_CACHE_INT8) return SHPLB_E_UNSUPPORTED;
  if (!c->k_pages || !c->v_pages || !c->k_scale || !c->v_scale || !c->page_table || !c->lens) return SHPLB_E_NULL;
  if (misaligned(c->k_pages, 16) || misaligned(c->v_pages, 16) || misaligned(c->k_scale, 4) || misaligned(c->v_scale, 4) ||
      misaligned(c->page_table, 4) || misaligned(c->lens, 4))
    return SHPLB_E_SHAPE;
  *a = CacheArgs{c->n_seq, c->n_kv_heads, c->max_pages, c->n_pages, c->block == 64 ? 6 : 7, c->format,
                 static_cast<uint8_t*>(c->k_pages), static_cast<uint8_t*>(c->v_pages), c->k_scale, c->v_scale, c->page_table, c->lens};
  return SHPLB_OK;
}

// n_heads, stride_t, stride_h: those of the tensors that the call takes.
int32_t check_step(const shplb_cache* c, const shplb_step* t, int32_t n_heads, int64_t stride_t, int64_t stride_h, StepArgs* a) {
  if (!t) return SHPLB_E_NULL;
  if (t->n_tokens < 0 || t->max_tokens < 0 || misaligned(t->cu_tokens, 4)) return SHPLB_E_SHAPE;
  if (!t->cu_tokens && int64_t(c->n_seq) * t->max_tokens != t->n_tokens) return SHPLB_E_SHAPE;
  if (stride_h < kHeadDim || stride_t < stride_h || stride_t / n_heads < stride_h || (stride_t | stride_h) & 7) return SHPLB_E_SHAPE;
  if (stride_t >= int64_t(1) << 24) return SHPLB_E_UNSUPPORTED;
  *a = StepArgs{t->n_tokens, t->max_tokens, t->cu_tokens, stride_t, stride_h};
  return SHPLB_OK;
}

// The query side of a step: heads in groups, and the most rows that a KV head has.
int32_t check_queries(const shplb_cache* c, const shplb_step* t, HeadGroups* g, int64_t* most_rows) {
  if (!t) return SHPLB_E_NULL;
  if (t->n_q_heads < 1 || t->max_tokens < 0) return SHPLB_E_SHAPE;
  if (!(t->softmax_scale >= 0.0f) || !std::isfinite(t->softmax_scale)) return SHPLB_E_SHAPE;
  std::memset(g, 0, sizeof(*g));
  int most = 0;
  if (!t->kv_head_of) {
    if (t->n_q_heads % c->n_kv_heads) return SHPLB_E_SHAPE;
    most = g->group = t->n_q_heads / c->n_kv_heads;
  } else {
    if (t->n_q_heads > SHPLB_MAX_MAPPED_HEADS || c->n_kv_heads > SHPLB_MAX_MAPPED_HEADS) return SHPLB_E_UNSUPPORTED;
    g->mapped = 1;
    for (int h = 0; h < t->n_q_heads; ++h)
      if (t->kv_head_of[h] < 0 || t->kv_head_of[h] >= c->n_kv_heads) return SHPLB_E_SHAPE;
    int at = 0;
    for (int kv = 0; kv < c->n_kv_heads; ++kv) {
      g->begin[kv] = uint16_t(at);
      for (int h = 0; h < t->n_q_heads; ++h)
        if (t->kv_head_of[h] == kv) g->head[at++] = uint8_t(h);
      g->begin[kv + 1] = uint16_t(at);
      most = at - g->begin[kv] > most ? at - g->begin[kv] : most;
    }
  }
  *most_rows = int64_t(most) * t->max_tokens;
  if (t->n_q_heads > SHPLB_MAX_SEQ_HEADS || *most_rows > (1 << 24)) return SHPLB_E_UNSUPPORTED;
  // places in the list of all units are 32-bit numbers, and a grid, whose threads are, has workgroups of 256 for every tile
  const int rows = cache_attn_rows(*most_rows);
  const int64_t tiles = *most_rows > rows ? (*most_rows + rows - 1) / rows : 1, items = int64_t(c->n_seq) * c->n_kv_heads * tiles;
  if (items >= int64_t(1) << 24 || items * (int64_t(c->max_pages) * c->block / 64 + kCacheMostStart) >= int64_t(1) << 30) return SHPLB_E_UNSUPPORTED;
  return SHPLB_OK;
}

int64_t align256(int64_t x) { return (x + 255) & ~int64_t(255); }

struct AttnLayout {
  int64_t part_o, part_ml, begun, stats, total, tiles;
};
AttnLayout attn_layout(const shplb_cache* c, const shplb_step* t, int64_t most_rows) {
  AttnLayout w;
  const int rows = cache_attn_rows(most_rows);
  w.tiles = most_rows > rows ? (most_rows + rows - 1) / rows : 1;
  int64_t off = 0;
  w.part_o = off; off += align256(kCacheSlotRows * kHeadDim * 4);
  w.part_ml = off; off += align256(kCacheSlotRows * 2 * 4);
  w.begun = off; off += align256(int64_t(c->n_seq) * c->n_kv_heads * w.tiles * 8);
  w.stats = off; off += align256(int64_t(t->n_tokens) * t->n_q_heads * 8);
  w.total = off;
  return w;
}

// Tensors and workspace of an attention call that has rows.
struct AttnPlace {
  const void* q;
  void* out;
  float* lse;
  void* workspace;
};
int32_t place_attn(const AttnPlace& at, const shplb_step* step, const AttnLayout& w, CacheAttnArgs* a) {
  if (!at.q || !at.out || !at.workspace) return SHPLB_E_NULL;
  if (at.q == at.out || misaligned(at.q, 16) || misaligned(at.out, 16) || misaligned(at.workspace, 256) || misaligned(at.lse, 4)) return SHPLB_E_SHAPE;
  char* ws = static_cast<char*>(at.workspace);
  a->tiles = int32_t(w.tiles);
  a->n_q_heads = step->n_q_heads;
  a->scale_log2 = (step->softmax_scale > 0.0f ? step->softmax_scale : 1.0f / std::sqrt(float(kHeadDim))) * 1.4426950408889634f;
  a->q = static_cast<const uint16_t*>(at.q);
  a->out = static_cast<uint16_t*>(at.out);
  a->lse = at.lse;
  a->part_o = reinterpret_cast<float*>(ws + w.part_o);
  a->part_ml = reinterpret_cast<float*>(ws + w.part_ml);
  a->begun = reinterpret_cast<int32_t*>(ws + w.begun);
  a->stats = reinterpret_cast<float*>(ws + w.stats);
  return SHPLB_OK;
}

// What windows add to the arguments: sizes that no position reaches are as good as 2^30.
int32_t check_window(const shplb_cache* c, int32_t max_tokens, int32_t n_sink, int32_t window, int64_t most_rows, CacheView* v) {
  if (n_sink < 0 || window < 1) return SHPLB_E_BUDGET;
  constexpr int32_t kMost = 1 << 30;
  *v = CacheView{};
  v->window = window < kMost ? window : kMost;
  v->n_sink = n_sink < kMost ? n_sink : kMost;
  // a tile has the rows of cache_attn_rows() tokens at most, and sees window + tokens - 1 positions beside the first ones
  const int64_t tokens = max_tokens < cache_attn_rows(most_rows) ? max_tokens : cache_attn_rows(most_rows), most = int64_t(v->window) + (tokens > 0 ? tokens : 1) - 1;
  const int64_t units = (int64_t(v->n_sink) + 63) / 64 + (most + 62) / 64 + 1, all = int64_t(c->max_pages) * c->block / 64;
  v->most_units = int32_t(units < all ? units : all);
  return SHPLB_OK;
}

// A call on sequences with prefixes: its arguments, without the tensors.
struct SharedArgs {
  CacheAttnArgs own, pre;
  int64_t most_rows, most_listed;  // (of units in the prefixes' list)
  int32_t rows_pre;                // rows of an item of the prefixes' list
  AttnLayout w;                    // of the own tokens' part; the prefixes' one lies behind it
  int64_t part_o, part_ml, begun, whole_o[2], whole_ml[2], total;
};
int32_t check_shared(const shplb_cache* prefix, const shplb_cache* cache, const shplb_step* step, SharedArgs* x) {
  if (int32_t st = check_cache(prefix, &x->pre.c)) return st;
  if (int32_t st = check_cache(cache, &x->own.c)) return st;
  if (prefix->n_kv_heads != cache->n_kv_heads || prefix->format != cache->format) return SHPLB_E_SHAPE;
  if (int32_t st = check_queries(cache, step, &x->own.groups, &x->most_rows)) return st;
  if (int32_t st = check_step(cache, step, step->n_q_heads, step->q_stride_t, step->q_stride_h, &x->own.t)) return st;
  // the rows of a KV head, all of which may have the same prefix
  const int64_t most_heads = step->max_tokens > 0 ? x->most_rows / step->max_tokens : 1, rows = int64_t(step->n_tokens) * most_heads;
  if (rows > 1 << 24) return SHPLB_E_UNSUPPORTED;
  x->rows_pre = prefix_attn_rows(rows / prefix->n_seq, int64_t(prefix->n_seq) * prefix->n_kv_heads, int64_t(prefix->max_pages) * prefix->block);
  const int64_t items = (rows / x->rows_pre + prefix->n_seq) * prefix->n_kv_heads;
  x->most_listed = items * (int64_t(prefix->max_pages) * prefix->block / 64 + kCacheMostStart);
  if (items >= int64_t(1) << 24 || x->most_listed >= int64_t(1) << 30) return SHPLB_E_UNSUPPORTED;
  x->w = attn_layout(cache, step, x->most_rows);
  int64_t off = x->w.total;
  x->part_o = off; off += align256(prefix_slot_rows(x->rows_pre) * kHeadDim * 4);
  x->part_ml = off; off += align256(prefix_slot_rows(x->rows_pre) * 2 * 4);
  const int64_t all = int64_t(step->n_tokens) * step->n_q_heads;
  x->begun = off; off += align256(all * 8);
  for (int y = 0; y < 2; ++y) {
    x->whole_o[y] = off; off += align256(all * kHeadDim * 4);
    x->whole_ml[y] = off; off += align256(all * 8);
  }
  x->total = off;
  return SHPLB_OK;
}

}  // namespace
}  // namespace shplb

using namespace shplb;

extern "C" {

int32_t shplb_cache_append(const shplb_cache* cache, const shplb_step* step, const void* k, const void* v, void* stream) {
  CacheArgs c;
  StepArgs t;
  if (int32_t st = check_cache(cache, &c)) return st;
  if (int32_t st = check_step(cache, step, cache->n_kv_heads, step ? step->kv_stride_t : 0, step ? step->kv_stride_h : 0, &t)) return st;
  if (t.n_tokens == 0 || t.max_tokens == 0) return SHPLB_OK;
  if (!k || !v) return SHPLB_E_NULL;
  if (misaligned(k, 16) || misaligned(v, 16)) return SHPLB_E_SHAPE;
  return launch_cache_append(c, t, k, v, static_cast<hipStream_t>(stream));
}

int32_t shplb_cache_load(const shplb_cache* cache, const shplb_step* step, void* k_out, void* v_out, void* stream) {
  CacheArgs c;
  StepArgs t;
  if (int32_t st = check_cache(cache, &c)) return st;
  if (int32_t st = check_step(cache, step, cache->n_kv_heads, step ? step->kv_stride_t : 0, step ? step->kv_stride_h : 0, &t)) return st;
  if (t.n_tokens == 0 || t.max_tokens == 0) return SHPLB_OK;
  if (!k_out || !v_out) return SHPLB_E_NULL;
  if (misaligned(k_out, 16) || misaligned(v_out, 16)) return SHPLB_E_SHAPE;
  return launch_cache_load(c, t, k_out, v_out, static_cast<hipStream_t>(stream));
}

int32_t shplb_cache_attn_workspace_bytes(const shplb_cache* cache, const shplb_step* step, int64_t* bytes_out) {
  if (!bytes_out) return SHPLB_E_NULL;
  CacheArgs c;
  StepArgs t;
  HeadGroups g;
  int64_t most_rows;
  if (int32_t st = check_cache(cache, &c)) return st;
  if (int32_t st = check_queries(cache, step, &g, &most_rows)) return st;
  if (int32_t st = check_step(cache, step, step->n_q_heads, step->q_stride_t, step->q_stride_h, &t)) return st;
  *bytes_out = attn_layout(cache, step, most_rows).total;
  return SHPLB_OK;
}

int32_t shplb_cache_attn(const shplb_cache* cache, const shplb_step* step, const void* q, void* out, float* lse_out,
                         const float* weight_in, float* weight_out, void* workspace, void* stream) {
  CacheAttnArgs a{};
  int64_t most_rows;
  if (int32_t st = check_cache(cache, &a.c)) return st;
  if (int32_t st = check_queries(cache, step, &a.groups, &most_rows)) return st;
  if (int32_t st = check_step(cache, step, step->n_q_heads, step->q_stride_t, step->q_stride_h, &a.t)) return st;
  if (a.t.max_tokens == 0) a.t.n_tokens = 0;
  if (weight_in && !weight_out) return SHPLB_E_NULL;
  if (a.t.n_tokens == 0 && !weight_out) return SHPLB_OK;
  if ((a.t.n_tokens > 0 && (!q || !out)) || !workspace) return SHPLB_E_NULL;
  if ((q && q == out) || misaligned(q, 16) || misaligned(out, 16) || misaligned(workspace, 256) || misaligned(lse_out, 4) || misaligned(weight_in, 4) ||
      misaligned(weight_out, 4))
    return SHPLB_E_SHAPE;
  const int32_t n_wg = persistent_workgroups();   // two per compute unit
  if (n_wg < 0) return n_wg;
  const AttnLayout w = attn_layout(cache, step, most_rows);
  a.tiles = int32_t(w.tiles);
  char* ws = static_cast<char*>(workspace);
  a.n_q_heads = step->n_q_heads;
  a.scale_log2 = (step->softmax_scale > 0.0f ? step->softmax_scale : 1.0f / std::sqrt(float(kHeadDim))) * 1.4426950408889634f;
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse_out;
  a.weight_in = weight_in;
  a.weight_out = weight_out;
  a.part_o = reinterpret_cast<float*>(ws + w.part_o);
  a.part_ml = reinterpret_cast<float*>(ws + w.part_ml);
  a.begun = reinterpret_cast<int32_t*>(ws + w.begun);
  a.stats = reinterpret_cast<float*>(ws + w.stats);
  return launch_cache_attn(a, int32_t(most_rows), n_wg / 2, static_cast<hipStream_t>(stream));
}

int32_t shplb_cache_attn_window_workspace_bytes(const shplb_cache* cache, const shplb_step* step, int32_t n_sink, int32_t window, int64_t* bytes_out) {
  if (n_sink < 0 || window < 1) return SHPLB_E_BUDGET;
  return shplb_cache_attn_workspace_bytes(cache, step, bytes_out);
}

int32_t shplb_cache_attn_window(const shplb_cache* cache, const shplb_step* step, int32_t n_sink, int32_t window, const void* q, void* out,
                                float* lse_out, void* workspace, void* stream) {
  CacheAttnArgs a{};
  int64_t most_rows;
  if (int32_t st = check_cache(cache, &a.c)) return st;
  if (int32_t st = check_queries(cache, step, &a.groups, &most_rows)) return st;
  if (int32_t st = check_step(cache, step, step->n_q_heads, step->q_stride_t, step->q_stride_h, &a.t)) return st;
  if (int32_t st = check_window(cache, step->max_tokens, n_sink, window, most_rows, &a.view)) return st;
  if (a.t.n_tokens == 0 || a.t.max_tokens == 0) return SHPLB_OK;
  AttnPlace at{q, out, lse_out, workspace};
  if (int32_t st = place_attn(at, step, attn_layout(cache, step, most_rows), &a)) return st;
  const int32_t n_wg = persistent_workgroups();
  if (n_wg < 0) return n_wg;
  return launch_cache_attn_window(a, int32_t(most_rows), n_wg / 2, static_cast<hipStream_t>(stream));
}

int32_t shplb_cache_attn_shared_workspace_bytes(const shplb_cache* prefix, const shplb_cache* cache, const shplb_step* step, int64_t* bytes_out) {
  if (!bytes_out) return SHPLB_E_NULL;
  SharedArgs x{};
  if (int32_t st = check_shared(prefix, cache, step, &x)) return st;
  *bytes_out = x.total;
  return SHPLB_OK;
}

int32_t shplb_cache_attn_shared(const shplb_cache* prefix, const int32_t* cu_prefix, const shplb_cache* cache, const shplb_step* step, const void* q,
                                void* out, float* lse_out, void* workspace, void* stream) {
  SharedArgs x{};
  if (int32_t st = check_shared(prefix, cache, step, &x)) return st;
  if (x.own.t.n_tokens == 0 || x.own.t.max_tokens == 0) return SHPLB_OK;
  if (!cu_prefix) return SHPLB_E_NULL;
  if (misaligned(cu_prefix, 4)) return SHPLB_E_SHAPE;
  AttnPlace at{q, out, lse_out, workspace};
  if (int32_t st = place_attn(at, step, x.w, &x.own)) return st;
  const int32_t n_wg = persistent_workgroups();
  if (n_wg < 0) return n_wg;
  const CacheArgs prefixes = x.pre.c;
  x.pre = x.own;
  x.pre.c = prefixes;
  x.pre.view.groups = cu_prefix;
  x.pre.view.members = cache->n_seq;
  x.pre.view.most_listed = int32_t(x.most_listed);
  char* ws = static_cast<char*>(workspace);
  x.pre.part_o = reinterpret_cast<float*>(ws + x.part_o);
  x.pre.part_ml = reinterpret_cast<float*>(ws + x.part_ml);
  x.pre.begun = reinterpret_cast<int32_t*>(ws + x.begun);
  for (int y = 0; y < 2; ++y) {
    CacheView& v = y == 0 ? x.own.view : x.pre.view;
    v.whole_o = reinterpret_cast<float*>(ws + x.whole_o[y]);
    v.whole_ml = reinterpret_cast<float*>(ws + x.whole_ml[y]);
  }
  return launch_cache_attn_shared(x.own, x.pre, int32_t(x.most_rows), x.rows_pre, n_wg / 2, static_cast<hipStream_t>(stream));
}

int32_t shplb_cache_evict_workspace_bytes(const shplb_cache* cache, int64_t* bytes_out) {
  if (!bytes_out) return SHPLB_E_NULL;
  CacheArgs c;
  if (int32_t st = check_cache(cache, &c)) return st;
  *bytes_out = cache_evict_workspace(c);
  return SHPLB_OK;
}

int32_t shplb_cache_evict(const shplb_cache* cache, const float* weight, const int32_t* keep, int32_t n_sink, int32_t n_recent,
                          const shplb_cache* to, float* weight_out, int32_t* kept_out, void* workspace, void* stream) {
  CacheArgs c, d;
  if (int32_t st = check_cache(cache, &c)) return st;
  if (int32_t st = check_cache(to, &d)) return st;
  if (n_sink < 0 || n_recent < 0) return SHPLB_E_BUDGET;
  if (c.n_seq != d.n_seq || c.n_kv_heads != d.n_kv_heads || c.format != d.format || c.table == d.table) return SHPLB_E_SHAPE;
  if (!weight || !keep || !weight_out || !kept_out || !workspace) return SHPLB_E_NULL;
  if (misaligned(weight, 4) || misaligned(keep, 4) || misaligned(weight_out, 4) || misaligned(kept_out, 4) || misaligned(workspace, 256))
    return SHPLB_E_SHAPE;
  if (int64_t(d.n_seq) * d.n_kv_heads * d.max_pages >= int64_t(1) << 23) return SHPLB_E_UNSUPPORTED;
  // heads are worked on side by side: what one writes is nothing that another reads, or writes in another meaning
  const void* arrays[] = {d.lens, weight_out, kept_out, workspace, weight, keep, c.lens, c.table, d.table};
  for (int written = 0; written < 4; ++written)
    for (int other = written + 1; other < 9; ++other)
      if (arrays[written] == arrays[other]) return SHPLB_E_SHAPE;
  return launch_cache_evict(c, weight, keep, n_sink, n_recent, d, weight_out, kept_out, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"

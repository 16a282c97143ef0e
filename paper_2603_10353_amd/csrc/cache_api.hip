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
  CacheAttnArgs a;
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

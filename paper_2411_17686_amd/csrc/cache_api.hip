// C-ABI layer of the decoder's cache and its attention: argument checks and launches.  Host code only.
#include <algorithm>
#include <cmath>

#include "attend.hpp"
#include "checks.hpp"
#include "share.hpp"

using namespace ficoco;

namespace {

// paged: with a cache (its heads), else dense keys and values; shapes: of a plan, which needs no tensors
const char* attention_fault(const ficoco_attention& a, int heads, int d_head, bool paged, int* code, bool shapes = false) {
  *code = FICOCO_EINVAL;
  if (a.B < 0 || a.n_q < 0 || a.H < 1 || heads < 1) return "a size is negative, or there are no heads";
  if (a.H % heads != 0) return "H is not a multiple of the key / value heads";
  if (a.d_head != d_head) return "d_head is not that of the cache";
  if (a.window < 0 || a.sinks < 0 || a.max_len < 0) return "window, sinks or max_len is negative";
  if (!shapes && (!(a.scale > 0.0f) || !std::isfinite(a.scale))) return "scale must be positive and finite";
  if (!paged && a.n_k < 0) return "a size is negative";
  const int64_t st[4][3] = {{a.q_stride_b, a.q_stride_h, a.q_stride_n}, {a.o_stride_b, a.o_stride_h, a.o_stride_n},
                            {a.k_stride_b, a.k_stride_h, a.k_stride_n}, {a.v_stride_b, a.v_stride_h, a.v_stride_n}};
  for (int i = 0; i < (shapes ? 0 : paged ? 2 : 4); ++i)
    if (st[i][0] < 0 || st[i][1] < 0 || st[i][2] < 0) return "a stride is negative";
  if (!shapes && a.B > 0 && a.n_q > 0) {
    if (!a.Q || !a.O || (!paged && a.n_k > 0 && (!a.K || !a.V))) return "a pointer is NULL";
    if (((uintptr_t)a.Q | (uintptr_t)a.O | (paged ? 0 : (uintptr_t)a.K | (uintptr_t)a.V)) & 1) return "a tensor is not aligned to its elements";
    const size_t out = extent(a.B, a.H, a.n_q, a.o_stride_b, a.o_stride_h, a.o_stride_n, d_head, 2);
    if (ranges_overlap(a.O, out, a.Q, extent(a.B, a.H, a.n_q, a.q_stride_b, a.q_stride_h, a.q_stride_n, d_head, 2)) ||
        (!paged && (ranges_overlap(a.O, out, a.K, extent(a.B, heads, a.n_k, a.k_stride_b, a.k_stride_h, a.k_stride_n, d_head, 2)) ||
                    ranges_overlap(a.O, out, a.V, extent(a.B, heads, a.n_k, a.v_stride_b, a.v_stride_h, a.v_stride_n, d_head, 2)))))
      return "O overlaps an input (outputs may not alias inputs)";
  }
  *code = FICOCO_EUNSUPPORTED;
  if (d_head != 64 && d_head != 128) return "d_head must be 64 or 128";
  if ((int64_t)a.n_q * (a.H / heads) > 0x3fffffff) return "more than 2^30 rows of one key / value head";
  if ((__int128)a.B * a.H * a.n_q > kMaxRows) return "2^31 rows or more in one call";      // (three times 2^31 pass 64 bits)
  if (!paged && a.n_k > kMaxTokens) return "more than 2^30 keys";
  *code = FICOCO_EINVAL;
  if (!shapes && rows_collide(d_head, {{{a.o_stride_b, a.B}, {a.o_stride_h, a.H}, {a.o_stride_n, a.n_q}}})) return "rows of O overlap";
  *code = FICOCO_OK;
  return nullptr;
}

int64_t most_keys(const ficoco_cache& c, const ficoco_attention& a) {
  const int64_t room = (int64_t)c.max_pages * c.page_size;
  return a.max_len > 0 ? std::min<int64_t>(room, a.max_len) : room;
}

AttendArgs arguments(const ficoco_attention& a, int heads, const AttendPlan& pl, char* ws) {
  AttendArgs x{};
  x.Q = (const bf16_t*)a.Q;
  x.q_sb = a.q_stride_b; x.q_sh = a.q_stride_h; x.q_sn = a.q_stride_n;
  x.O = (bf16_t*)a.O;
  x.o_sb = a.o_stride_b; x.o_sh = a.o_stride_h; x.o_sn = a.o_stride_n;
  x.seq = a.seq; x.q_len = a.q_len; x.k_len = a.k_len; x.q_start = a.q_start;
  x.B = a.B; x.H_kv = heads; x.group = a.H / heads; x.n_q = a.n_q; x.n_k = a.n_k;
  x.by_heads = Divisor(heads); x.by_group = Divisor(a.H / heads); x.by_splits = Divisor(pl.splits); x.by_all = Divisor((int64_t)a.B * heads);
  x.splits = pl.splits; x.row_tiles = pl.row_tiles; x.part_rows = pl.row_tiles * pl.rows;
  x.scale_log2e = a.scale * 1.44269504088896340736f;
  x.window = a.window; x.sinks = a.sinks;
  x.K = (const bf16_t*)a.K; x.V = (const bf16_t*)a.V;
  x.k_sb = a.k_stride_b; x.k_sh = a.k_stride_h; x.k_sn = a.k_stride_n;
  x.v_sb = a.v_stride_b; x.v_sh = a.v_stride_h; x.v_sn = a.v_stride_n;
  x.part_ms = (float2*)(ws + pl.part_ms);
  x.part_o = (float*)(ws + pl.part_o);
  return x;
}

// The pages of a layer.
void layer_pages(AttendArgs& x, const ficoco_cache& c, int32_t layer) {
  const int64_t blocks = (int64_t)layer * c.n_pages * c.heads;
  x.k = (const uint8_t*)c.k + blocks * c.page_size * c.d_head;
  x.v = (const uint8_t*)c.v + blocks * c.page_size * c.d_head;
  x.k_exp = c.k_exp + blocks;
  x.v_exp = c.v_exp + blocks;
  x.table = c.table; x.len = c.len;
  x.n_pages = c.n_pages; x.n_seqs = c.n_seqs; x.max_pages = c.max_pages;
  x.page_shift = __builtin_ctz((unsigned)c.page_size);
}

// ---- sequences that share pages -------------------------------------------------------------------------------
const char* share_fault(const ficoco_cache& c, const ficoco_attention& a, bool shapes, SharePlan* pl, int* code) {
  if (const char* why = attention_fault(a, c.heads, c.d_head, true, code, shapes)) return why;
  *code = FICOCO_EUNSUPPORTED;
  if (a.B > kMaxCall) return "more than 1024 sequences in a call";
  // (six times the rows, and the pieces of a tile: see share_plan())
  if (8 * (int64_t)a.B * a.n_q * (a.H / c.heads) + 2048 * kTileRows > kMaxRows) return "too many rows in one call";
  *pl = share_plan(c, a);
  if ((int64_t)pl->items * c.heads * kTileThreads > kMaxThreads || (int64_t)a.B * a.H * a.n_q * (a.d_head / 4) * 8 > kMaxThreads) return "too many rows in one call";
  *code = FICOCO_OK;
  return nullptr;
}

ShareArgs share_arguments(const ficoco_cache& c, const ficoco_attention& a, const SharePlan& pl, void* plan, char* ws) {
  ShareArgs s{};
  AttendPlan none{};
  none.splits = 1;
  none.part_ms = pl.part_ms; none.part_o = pl.part_o;
  s.a = arguments(a, c.heads, none, ws);
  layer_pages(s.a, c, 0);
  // what the plan's numbers depend on
  uint64_t mark = 0x9e3779b97f4a7c15ull;
  for (const int64_t x : {(int64_t)a.B, (int64_t)a.H, (int64_t)c.heads, (int64_t)a.n_q, (int64_t)a.d_head, (int64_t)a.window, (int64_t)a.sinks, (int64_t)a.max_len, (int64_t)c.page_size, (int64_t)c.n_pages,
                          (int64_t)c.n_seqs, (int64_t)c.max_pages, (int64_t)pl.items, (int64_t)pl.pieces})
    mark = (mark ^ (uint64_t)x) * 0x100000001b3ull + (mark >> 29);
  s.mark = mark;
  s.plan = (char*)plan;
  s.by_rows = Divisor((int64_t)a.n_q * (a.H / c.heads));
  s.own_tile = pl.own_tile; s.pieces = pl.pieces; s.items = pl.items;
  s.d_head = a.d_head;
  s.entries = pl.entries; s.members = pl.members; s.owners = pl.owners; s.items_at = pl.items_at;
  return s;
}

}  // namespace

extern "C" {

int ficoco_cache_reserve(ficoco_ctx* ctx, const ficoco_cache* c, int32_t n, const int32_t* seq, const int32_t* n_new, int32_t n_each,
                         int32_t* start, void* stream) {
  const char* fn = "ficoco_cache_reserve";
  int rc = begin(ctx, c, fn);
  if (rc == FICOCO_OK) rc = check_count(ctx, *c, n, fn);
  if (rc != FICOCO_OK || n == 0) return rc;
  if (!start) return fail(ctx, FICOCO_EINVAL, fn, "start is NULL");
  if (!n_new && n_each < 0) return fail(ctx, FICOCO_EINVAL, fn, "n_each is negative");
  launch_cache_reserve(*c, n, seq, n_new, n_each, start, (hipStream_t)stream);
  return finish(ctx, fn);
}

int ficoco_cache_append(ficoco_ctx* ctx, const ficoco_cache* c, int32_t layer, const ficoco_tokens* t, void* stream) {
  const char* fn = "ficoco_cache_append";
  int rc = begin(ctx, c, fn);
  if (rc == FICOCO_OK) rc = check_tokens(ctx, *c, layer, t, true, fn);
  if (rc != FICOCO_OK || t->n == 0 || t->n_max == 0) return rc;
  launch_cache_append(*c, layer, *t, (hipStream_t)stream);
  return finish(ctx, fn);
}

int ficoco_cache_read(ficoco_ctx* ctx, const ficoco_cache* c, int32_t layer, const ficoco_tokens* t, void* stream) {
  const char* fn = "ficoco_cache_read";
  int rc = begin(ctx, c, fn);
  if (rc == FICOCO_OK) rc = check_tokens(ctx, *c, layer, t, false, fn);
  if (rc != FICOCO_OK || t->n == 0 || t->n_max == 0) return rc;
  launch_cache_read(*c, layer, *t, (hipStream_t)stream);
  return finish(ctx, fn);
}

int ficoco_cache_fork(ficoco_ctx* ctx, const ficoco_cache* c, int32_t n, const int32_t* src, const int32_t* dst, int32_t whole, int32_t* done,
                      void* stream) {
  const char* fn = "ficoco_cache_fork";
  int rc = begin(ctx, c, fn);
  if (rc == FICOCO_OK) rc = check_count(ctx, *c, n, fn);
  if (rc != FICOCO_OK || n == 0) return rc;
  if (!src || !dst || !done) return fail(ctx, FICOCO_EINVAL, fn, "a pointer is NULL");
  if ((int64_t)c->layers * c->heads > kMaxGridY) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "more than 65535 heads in all layers");
  launch_cache_fork(*c, n, src, dst, whole != 0, done, (hipStream_t)stream);
  return finish(ctx, fn);
}

int ficoco_cache_workspace_bytes(const ficoco_cache* c, int32_t n, size_t* out_bytes) {
  if (!c || !out_bytes || n < 0 || n > kMaxCall) return FICOCO_EINVAL;
  int code;
  if (cache_fault(*c, &code)) return code;
  if (too_many_pages(*c, n)) return FICOCO_EUNSUPPORTED;
  *out_bytes = std::max<size_t>(256, compact_workspace(*c, n));
  return FICOCO_OK;
}

int ficoco_cache_compact(ficoco_ctx* ctx, const ficoco_cache* c, int32_t layer_begin, int32_t n_layers, int32_t n, const int32_t* src,
                         const int32_t* dst, int32_t vis_begin, int32_t N, int32_t n_keep, const int32_t* keep_idx, int32_t* done, void* ws,
                         size_t ws_bytes, void* stream) {
  const char* fn = "ficoco_cache_compact";
  int rc = begin(ctx, c, fn);
  if (rc == FICOCO_OK) rc = check_count(ctx, *c, n, fn);
  if (rc != FICOCO_OK) return rc;
  if (layer_begin < 0 || n_layers < 0 || (int64_t)layer_begin + n_layers > c->layers) return fail(ctx, FICOCO_EINVAL, fn, "no such layers");
  if (vis_begin < 0 || N < 0 || n_keep < 0 || n_keep > N || (int64_t)vis_begin + N > 0x7fffffff)
    return fail(ctx, FICOCO_EINVAL, fn, "vis_begin, N or n_keep is out of range");
  if (n == 0) return FICOCO_OK;
  if (!src || !dst || !done || (n_keep > 0 && !keep_idx)) return fail(ctx, FICOCO_EINVAL, fn, "a pointer is NULL");
  if ((int64_t)n_layers * c->heads > kMaxGridY) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "more than 65535 heads in all layers");
  if (!ws || ((uintptr_t)ws & 255)) return fail(ctx, FICOCO_EINVAL, fn, "workspace is NULL or not 256-byte aligned");
  if (ws_bytes < compact_workspace(*c, n)) return fail(ctx, FICOCO_ENOMEM, fn, "workspace smaller than ficoco_cache_workspace_bytes()");
  if (reaches_into(*c, ws, compact_workspace(*c, n)) || ranges_overlap(ws, compact_workspace(*c, n), keep_idx, (size_t)n * n_keep * sizeof(int32_t)))
    return fail(ctx, FICOCO_EINVAL, fn, "the workspace overlaps the cache or keep_idx");
  launch_cache_compact(*c, layer_begin, n_layers, n, src, dst, vis_begin, N, n_keep, keep_idx, done, (char*)ws, (hipStream_t)stream);
  return finish(ctx, fn);
}

int ficoco_cache_free(ficoco_ctx* ctx, const ficoco_cache* c, int32_t n, const int32_t* seq, void* stream) {
  const char* fn = "ficoco_cache_free";
  const int rc = begin(ctx, c, fn);
  if (rc != FICOCO_OK) return rc;
  if (n < 0) return fail(ctx, FICOCO_EINVAL, fn, "n is negative");
  if (n == 0) return FICOCO_OK;
  if ((int64_t)n * kMoveThreads > kMaxThreads) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "more than 2^24 sequences in a call");
  launch_cache_free(*c, n, seq, (hipStream_t)stream);
  return finish(ctx, fn);
}

int ficoco_cache_attention_workspace_bytes(const ficoco_cache* c, const ficoco_attention* a, size_t* out_bytes) {
  if (!c || !a || !out_bytes) return FICOCO_EINVAL;
  int code;
  if (cache_fault(*c, &code) || attention_fault(*a, c->heads, c->d_head, true, &code)) return code;
  *out_bytes = attend_plan(*a, c->heads, most_keys(*c, *a), true).total;
  return FICOCO_OK;
}

int ficoco_cache_attention(ficoco_ctx* ctx, const ficoco_cache* c, int32_t layer, const ficoco_attention* a, void* ws, size_t ws_bytes, void* stream) {
  const char* fn = "ficoco_cache_attention";
  const int rc = begin(ctx, c, fn);
  if (rc != FICOCO_OK) return rc;
  if (!a) return fail(ctx, FICOCO_EINVAL, fn, "attention is NULL");
  if (layer < 0 || layer >= c->layers) return fail(ctx, FICOCO_EINVAL, fn, "no such layer");
  int code;
  if (const char* why = attention_fault(*a, c->heads, c->d_head, true, &code)) return fail(ctx, code, fn, why);
  if (a->B == 0 || a->n_q == 0) return FICOCO_OK;
  const AttendPlan pl = attend_plan(*a, c->heads, most_keys(*c, *a), true);
  if (!ws || ((uintptr_t)ws & 255)) return fail(ctx, FICOCO_EINVAL, fn, "workspace is NULL or not 256-byte aligned");
  if (ws_bytes < pl.total) return fail(ctx, FICOCO_ENOMEM, fn, "workspace smaller than ficoco_cache_attention_workspace_bytes()");
  const size_t out = extent(a->B, a->H, a->n_q, a->o_stride_b, a->o_stride_h, a->o_stride_n, a->d_head, 2);
  if (ranges_overlap(a->O, out, ws, pl.total) ||
      ranges_overlap(a->Q, extent(a->B, a->H, a->n_q, a->q_stride_b, a->q_stride_h, a->q_stride_n, a->d_head, 2), ws, pl.total))
    return fail(ctx, FICOCO_EINVAL, fn, "Q or O overlaps the workspace");
  if (reaches_into(*c, a->O, out) || reaches_into(*c, ws, pl.total)) return fail(ctx, FICOCO_EINVAL, fn, "O or the workspace overlaps the cache");
  if ((int64_t)a->B * c->heads * pl.row_tiles * pl.splits * kTileThreads > kMaxThreads)
    return fail(ctx, FICOCO_EUNSUPPORTED, fn, "too many rows in one call");
  AttendArgs x = arguments(*a, c->heads, pl, (char*)ws);
  layer_pages(x, *c, layer);
  if (pl.few) launch_few_rows(x, a->d_head, (hipStream_t)stream);
  else launch_page_rows(x, a->d_head, (hipStream_t)stream);
  if (pl.splits > 1) launch_join_rows(x, a->d_head, (hipStream_t)stream);
  return finish(ctx, fn);
}

int ficoco_cache_share_bytes(const ficoco_cache* c, const ficoco_attention* a, size_t* plan_bytes, size_t* ws_bytes) {
  if (!c || !a || !plan_bytes || !ws_bytes) return FICOCO_EINVAL;
  int code;
  SharePlan pl;
  if (cache_fault(*c, &code) || share_fault(*c, *a, true, &pl, &code)) return code;
  *plan_bytes = pl.bytes;
  *ws_bytes = pl.ws_bytes;
  return FICOCO_OK;
}

int ficoco_cache_share(ficoco_ctx* ctx, const ficoco_cache* c, const ficoco_attention* a, const int32_t* group, int32_t always, void* plan, size_t plan_bytes, void* stream) {
  const char* fn = "ficoco_cache_share";
  const int rc = begin(ctx, c, fn);
  if (rc != FICOCO_OK) return rc;
  if (!a) return fail(ctx, FICOCO_EINVAL, fn, "attention is NULL");
  int code;
  SharePlan pl;
  if (const char* why = share_fault(*c, *a, true, &pl, &code)) return fail(ctx, code, fn, why);
  if (a->B == 0 || a->n_q == 0) return FICOCO_OK;
  if (!plan || ((uintptr_t)plan & 255)) return fail(ctx, FICOCO_EINVAL, fn, "plan is NULL or not 256-byte aligned");
  if (plan_bytes < pl.bytes) return fail(ctx, FICOCO_ENOMEM, fn, "plan smaller than ficoco_cache_share_bytes()");
  if (reaches_into(*c, plan, pl.bytes)) return fail(ctx, FICOCO_EINVAL, fn, "the plan overlaps the cache");
  for (const int32_t* p : {group, a->seq, a->q_len, a->k_len, a->q_start})
    if (ranges_overlap(p, (size_t)a->B * sizeof(int32_t), plan, pl.bytes)) return fail(ctx, FICOCO_EINVAL, fn, "the plan overlaps an input");
  ShareArgs s = share_arguments(*c, *a, pl, plan, nullptr);
  s.group = group;
  s.always = always != 0;
  launch_share(s, (hipStream_t)stream);
  return finish(ctx, fn);
}

int ficoco_cache_shared_attention(ficoco_ctx* ctx, const ficoco_cache* c, int32_t layer, const ficoco_attention* a, const void* plan, size_t plan_bytes, void* ws, size_t ws_bytes,
                                  void* stream) {
  const char* fn = "ficoco_cache_shared_attention";
  const int rc = begin(ctx, c, fn);
  if (rc != FICOCO_OK) return rc;
  if (!a) return fail(ctx, FICOCO_EINVAL, fn, "attention is NULL");
  if (layer < 0 || layer >= c->layers) return fail(ctx, FICOCO_EINVAL, fn, "no such layer");
  int code;
  SharePlan pl;
  if (const char* why = share_fault(*c, *a, false, &pl, &code)) return fail(ctx, code, fn, why);
  if (a->B == 0 || a->n_q == 0) return FICOCO_OK;
  if (!plan || ((uintptr_t)plan & 255)) return fail(ctx, FICOCO_EINVAL, fn, "plan is NULL or not 256-byte aligned");
  if (plan_bytes < pl.bytes) return fail(ctx, FICOCO_ENOMEM, fn, "plan smaller than ficoco_cache_share_bytes()");
  if (!ws || ((uintptr_t)ws & 255)) return fail(ctx, FICOCO_EINVAL, fn, "workspace is NULL or not 256-byte aligned");
  if (ws_bytes < pl.ws_bytes) return fail(ctx, FICOCO_ENOMEM, fn, "workspace smaller than ficoco_cache_share_bytes()");
  const size_t out = extent(a->B, a->H, a->n_q, a->o_stride_b, a->o_stride_h, a->o_stride_n, a->d_head, 2);
  const size_t in = extent(a->B, a->H, a->n_q, a->q_stride_b, a->q_stride_h, a->q_stride_n, a->d_head, 2);
  if (ranges_overlap(a->O, out, ws, pl.ws_bytes) || ranges_overlap(a->Q, in, ws, pl.ws_bytes) || ranges_overlap(plan, pl.bytes, ws, pl.ws_bytes) ||
      ranges_overlap(a->O, out, plan, pl.bytes))
    return fail(ctx, FICOCO_EINVAL, fn, "Q, O, the plan and the workspace overlap");
  if (reaches_into(*c, a->O, out) || reaches_into(*c, ws, pl.ws_bytes)) return fail(ctx, FICOCO_EINVAL, fn, "O or the workspace overlaps the cache");
  ShareArgs s = share_arguments(*c, *a, pl, (void*)plan, (char*)ws);
  layer_pages(s.a, *c, layer);
  launch_share_rows(s, a->d_head, (hipStream_t)stream);
  return finish(ctx, fn);
}

int ficoco_window_attention(ficoco_ctx* ctx, const ficoco_attention* a, void* stream) {
  const char* fn = "ficoco_window_attention";
  if (!ctx) return FICOCO_EINVAL;
  if (!a) return fail(ctx, FICOCO_EINVAL, fn, "attention is NULL");
  const int rc = check_device(ctx, fn);
  if (rc != FICOCO_OK) return rc;
  int code;
  if (const char* why = attention_fault(*a, a->H_kv, a->d_head, false, &code)) return fail(ctx, code, fn, why);
  if (a->B == 0 || a->n_q == 0) return FICOCO_OK;
  const AttendPlan pl = attend_plan(*a, a->H_kv, a->n_k, false);
  if ((int64_t)a->B * a->H_kv * pl.row_tiles * kTileThreads > kMaxThreads) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "too many rows in one call");
  launch_dense_rows(arguments(*a, a->H_kv, pl, nullptr), a->d_head, (hipStream_t)stream);
  return finish(ctx, fn);
}

}  // extern "C"

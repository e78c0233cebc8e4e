// C-ABI layer of the decoder's cache and its attention: argument checks and launches.  Host code only.
#include <algorithm>
#include <array>
#include <cmath>
#include <utility>

#include "attend.hpp"
#include "ctx.hpp"

using namespace ficoco;

namespace {

constexpr int64_t kMaxGridY = 65535, kMaxRows = 0x7fffffff;
constexpr int64_t kMaxThreads = 0xffffffff;      // of a launch, along one axis
constexpr int64_t kMaxTokens = 1 << 30;      // (a block behind the last token, too, is named by 32 bits)

// Whether rows of d elements may share elements: none do where every stride steps over all that the smaller ones span.
bool rows_collide(int64_t d, std::array<std::pair<int64_t, int64_t>, 3> dims) {      // (stride, extent)
  std::sort(dims.begin(), dims.end());
  for (const auto& [stride, extent] : dims) {
    if (extent <= 1) continue;
    if (stride < d) return true;
    d += stride * (extent - 1);
  }
  return false;
}

// What is wrong with the description of a cache, or nullptr; *code its status.
const char* cache_fault(const ficoco_cache& c, int* code) {
  *code = FICOCO_EINVAL;
  if (c.layers < 1 || c.n_pages < 1 || c.heads < 1 || c.n_seqs < 1 || c.max_pages < 1) return "a size of the cache is not positive";
  if (!c.k || !c.v || !c.k_exp || !c.v_exp || !c.table || !c.len || !c.refs) return "a pointer of the cache is NULL";
  if (((uintptr_t)c.k | (uintptr_t)c.v) & 15) return "pages must be 16-byte aligned";
  if (((uintptr_t)c.table | (uintptr_t)c.len | (uintptr_t)c.refs) & 3) return "table, len and refs must be 4-byte aligned";
  *code = FICOCO_EUNSUPPORTED;
  if (c.page_size != 16 && c.page_size != 32 && c.page_size != 64 && c.page_size != 128) return "page_size must be 16, 32, 64 or 128";
  if (c.d_head != 64 && c.d_head != 128) return "d_head must be 64 or 128";
  if (c.n_seqs > kMaxSlots) return "more than 8192 slots";
  if ((int64_t)c.max_pages * c.page_size > kMaxTokens) return "a row of the table holds more than 2^30 tokens";
  if (c.heads > kMaxGridY) return "too many heads";
  *code = FICOCO_OK;
  return nullptr;
}

// The pages that a call can ask for are counted in 32 bits.
bool too_many_pages(const ficoco_cache& c, int32_t n) { return (int64_t)n * c.max_pages > 0x7fffffff; }

int begin(ficoco_ctx* ctx, const ficoco_cache* c, const char* fn) {
  if (!ctx) return FICOCO_EINVAL;
  if (!c) return fail(ctx, FICOCO_EINVAL, fn, "cache is NULL");
  const int dev_rc = check_device(ctx, fn);
  if (dev_rc != FICOCO_OK) return dev_rc;
  int code;
  const char* why = cache_fault(*c, &code);
  return why ? fail(ctx, code, fn, why) : FICOCO_OK;
}

int check_count(ficoco_ctx* ctx, const ficoco_cache& c, int32_t n, const char* fn) {
  if (n < 0) return fail(ctx, FICOCO_EINVAL, fn, "n is negative");
  if (n > kMaxCall) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "more than 1024 sequences in a call");
  if (too_many_pages(c, n)) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "the rows of the table of a call have room for 2^31 pages or more");
  return FICOCO_OK;
}

// Bytes from a tensor's first to its last element.
size_t extent(int64_t b, int64_t h, int64_t n, int64_t sb, int64_t sh, int64_t sn, int64_t d, size_t es) {
  return b > 0 && h > 0 && n > 0 ? (size_t)((b - 1) * sb + (h - 1) * sh + (n - 1) * sn + d) * es : 0;
}
size_t pool_bytes(const ficoco_cache& c) {
  return (size_t)c.layers * c.n_pages * c.heads * c.page_size * c.d_head;
}
// Whether [p, p + n) shares bytes with an array of the cache.
bool reaches_into(const ficoco_cache& c, const void* p, size_t n) {
  const size_t exps = (size_t)c.layers * c.n_pages * c.heads;
  return ranges_overlap(p, n, c.k, pool_bytes(c)) || ranges_overlap(p, n, c.v, pool_bytes(c)) || ranges_overlap(p, n, c.k_exp, exps) ||
         ranges_overlap(p, n, c.v_exp, exps) || ranges_overlap(p, n, c.table, (size_t)c.n_seqs * c.max_pages * sizeof(int32_t)) ||
         ranges_overlap(p, n, c.len, (size_t)c.n_seqs * sizeof(int32_t)) || ranges_overlap(p, n, c.refs, (size_t)c.n_pages * sizeof(int32_t));
}

int check_tokens(ficoco_ctx* ctx, const ficoco_cache& c, int32_t layer, const ficoco_tokens* t, bool write, const char* fn) {
  if (!t) return fail(ctx, FICOCO_EINVAL, fn, "tokens is NULL");
  if (layer < 0 || layer >= c.layers) return fail(ctx, FICOCO_EINVAL, fn, "no such layer");
  if (t->n < 0 || t->n_max < 0) return fail(ctx, FICOCO_EINVAL, fn, "n or n_max is negative");
  if (t->dtype != FICOCO_F32 && t->dtype != FICOCO_BF16) return fail(ctx, FICOCO_EINVAL, fn, "unknown dtype");
  if (t->n == 0 || t->n_max == 0) return FICOCO_OK;
  if (write ? !t->K || !t->V || !t->start : !t->K && !t->V) return fail(ctx, FICOCO_EINVAL, fn, "a pointer is NULL");
  const uintptr_t align = t->dtype == FICOCO_BF16 ? 1 : 3;
  if (((uintptr_t)t->K | (uintptr_t)t->V) & align) return fail(ctx, FICOCO_EINVAL, fn, "K or V is not aligned to its elements");
  if (t->n_max > kMaxTokens) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "more than 2^30 tokens of a sequence");
  if (2 * (int64_t)t->n > kMaxGridY) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "more than 32767 sequences in a call");
  if (token_threads(c, t->n_max, write) > kMaxThreads) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "n_max takes more than 2^32 threads");
  if (t->k_stride_b < 0 || t->k_stride_h < 0 || t->k_stride_n < 0 || t->v_stride_b < 0 || t->v_stride_h < 0 || t->v_stride_n < 0)
    return fail(ctx, FICOCO_EINVAL, fn, "a stride is negative");
  if (!write) {
    if ((t->K && rows_collide(c.d_head, {{{t->k_stride_b, t->n}, {t->k_stride_h, c.heads}, {t->k_stride_n, t->n_max}}})) ||
        (t->V && rows_collide(c.d_head, {{{t->v_stride_b, t->n}, {t->v_stride_h, c.heads}, {t->v_stride_n, t->n_max}}})) || t->K == t->V)
      return fail(ctx, FICOCO_EINVAL, fn, "rows that are written overlap");
    const size_t es = t->dtype == FICOCO_BF16 ? 2 : 4;
    if (reaches_into(c, t->K, extent(t->n, c.heads, t->n_max, t->k_stride_b, t->k_stride_h, t->k_stride_n, c.d_head, es)) ||
        reaches_into(c, t->V, extent(t->n, c.heads, t->n_max, t->v_stride_b, t->v_stride_h, t->v_stride_n, c.d_head, es)))
      return fail(ctx, FICOCO_EINVAL, fn, "K or V overlaps the cache");
  }
  return FICOCO_OK;
}

// paged: with a cache (its heads), else dense keys and values
const char* attention_fault(const ficoco_attention& a, int heads, int d_head, bool paged, int* code) {
  *code = FICOCO_EINVAL;
  if (a.B < 0 || a.n_q < 0 || a.H < 1 || heads < 1) return "a size is negative, or there are no heads";
  if (a.H % heads != 0) return "H is not a multiple of the key / value heads";
  if (a.d_head != d_head) return "d_head is not that of the cache";
  if (a.window < 0 || a.sinks < 0 || a.max_len < 0) return "window, sinks or max_len is negative";
  if (!(a.scale > 0.0f) || !std::isfinite(a.scale)) return "scale must be positive and finite";
  if (!paged && a.n_k < 0) return "a size is negative";
  const int64_t st[4][3] = {{a.q_stride_b, a.q_stride_h, a.q_stride_n}, {a.o_stride_b, a.o_stride_h, a.o_stride_n},
                            {a.k_stride_b, a.k_stride_h, a.k_stride_n}, {a.v_stride_b, a.v_stride_h, a.v_stride_n}};
  for (int i = 0; i < (paged ? 2 : 4); ++i)
    if (st[i][0] < 0 || st[i][1] < 0 || st[i][2] < 0) return "a stride is negative";
  if (a.B > 0 && a.n_q > 0) {
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
  if (rows_collide(d_head, {{{a.o_stride_b, a.B}, {a.o_stride_h, a.H}, {a.o_stride_n, a.n_q}}})) return "rows of O overlap";
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
  const int64_t blocks = (int64_t)layer * c->n_pages * c->heads;
  x.k = (const uint8_t*)c->k + blocks * c->page_size * c->d_head;
  x.v = (const uint8_t*)c->v + blocks * c->page_size * c->d_head;
  x.k_exp = c->k_exp + blocks;
  x.v_exp = c->v_exp + blocks;
  x.table = c->table; x.len = c->len;
  x.n_pages = c->n_pages; x.n_seqs = c->n_seqs; x.max_pages = c->max_pages;
  x.page_shift = __builtin_ctz((unsigned)c->page_size);
  if (pl.few) launch_few_rows(x, a->d_head, (hipStream_t)stream);
  else launch_page_rows(x, a->d_head, (hipStream_t)stream);
  if (pl.splits > 1) launch_join_rows(x, a->d_head, (hipStream_t)stream);
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

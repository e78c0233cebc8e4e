// Checks of arguments that the entry points around the cache share.  Host code only.
#pragma once
#include <algorithm>
#include <array>
#include <utility>

#include "cache.hpp"
#include "ctx.hpp"

namespace ficoco {

constexpr int64_t kMaxGridY = 65535, kMaxRows = 0x7fffffff;
constexpr int64_t kMaxThreads = 0xffffffff;      // of a launch, along one axis
constexpr int64_t kMaxTokens = 1 << 30;      // (a block behind the last token, too, is named by 32 bits)

// Whether rows of d elements may share elements: none do where every stride steps over all that the smaller ones span.
inline bool rows_collide(int64_t d, std::array<std::pair<int64_t, int64_t>, 3> dims) {      // (stride, extent)
  std::sort(dims.begin(), dims.end());
  for (const auto& [stride, extent] : dims) {
    if (extent <= 1) continue;
    if (stride < d) return true;
    d += stride * (extent - 1);
  }
  return false;
}

// What is wrong with the description of a cache, or nullptr; *code its status.
inline const char* cache_fault(const ficoco_cache& c, int* code) {
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
inline bool too_many_pages(const ficoco_cache& c, int32_t n) { return (int64_t)n * c.max_pages > 0x7fffffff; }

inline int begin(ficoco_ctx* ctx, const ficoco_cache* c, const char* fn) {
  if (!ctx) return FICOCO_EINVAL;
  if (!c) return fail(ctx, FICOCO_EINVAL, fn, "cache is NULL");
  const int dev_rc = check_device(ctx, fn);
  if (dev_rc != FICOCO_OK) return dev_rc;
  int code;
  const char* why = cache_fault(*c, &code);
  return why ? fail(ctx, code, fn, why) : FICOCO_OK;
}

inline int check_count(ficoco_ctx* ctx, const ficoco_cache& c, int32_t n, const char* fn) {
  if (n < 0) return fail(ctx, FICOCO_EINVAL, fn, "n is negative");
  if (n > kMaxCall) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "more than 1024 sequences in a call");
  if (too_many_pages(c, n)) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "the rows of the table of a call have room for 2^31 pages or more");
  return FICOCO_OK;
}

// Bytes from a tensor's first to its last element.
inline size_t extent(int64_t b, int64_t h, int64_t n, int64_t sb, int64_t sh, int64_t sn, int64_t d, size_t es) {
  return b > 0 && h > 0 && n > 0 ? (size_t)((b - 1) * sb + (h - 1) * sh + (n - 1) * sn + d) * es : 0;
}
inline size_t pool_bytes(const ficoco_cache& c) {
  return (size_t)c.layers * c.n_pages * c.heads * c.page_size * c.d_head;
}
// Whether [p, p + n) shares bytes with an array of the cache.
inline bool reaches_into(const ficoco_cache& c, const void* p, size_t n) {
  const size_t exps = (size_t)c.layers * c.n_pages * c.heads;
  return ranges_overlap(p, n, c.k, pool_bytes(c)) || ranges_overlap(p, n, c.v, pool_bytes(c)) || ranges_overlap(p, n, c.k_exp, exps) ||
         ranges_overlap(p, n, c.v_exp, exps) || ranges_overlap(p, n, c.table, (size_t)c.n_seqs * c.max_pages * sizeof(int32_t)) ||
         ranges_overlap(p, n, c.len, (size_t)c.n_seqs * sizeof(int32_t)) || ranges_overlap(p, n, c.refs, (size_t)c.n_pages * sizeof(int32_t));
}

inline int check_tokens(ficoco_ctx* ctx, const ficoco_cache& c, int32_t layer, const ficoco_tokens* t, bool write, const char* fn) {
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

}  // namespace ficoco

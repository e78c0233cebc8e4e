// C-ABI layer of the rotation: argument checks and launches.  Host code only.
#include <cmath>
#include <initializer_list>

#include "checks.hpp"
#include "rotary.hpp"

using namespace ficoco;

namespace {

// Elements of a [B][H][n][d] tensor, in bytes.
struct Span3 {
  uintptr_t p;
  int64_t extent[3], stride[3], row;
  bool empty() const { return !p || extent[0] <= 0 || extent[1] <= 0 || extent[2] <= 0; }
  int64_t bytes() const {
    return row + (extent[0] - 1) * stride[0] + (extent[1] - 1) * stride[1] + (extent[2] - 1) * stride[2];
  }
};
Span3 span3(const void* p, int64_t b, int64_t h, int64_t n, int64_t sb, int64_t sh, int64_t sn, int64_t d, int64_t es) {
  return Span3{(uintptr_t)p, {b, h, n}, {sb * es, sh * es, sn * es}, d * es};
}
// Bytes that a tensor takes of a period: of its strides, those that are not whole periods.
int64_t in_period(const Span3& x, int64_t period) {
  int64_t n = x.row;
  for (int i = 0; i < 3; ++i)
    if (x.extent[i] > 1 && x.stride[i] % period != 0) n += (x.extent[i] - 1) * x.stride[i];
  return n;
}
// Whether two tensors may share bytes.  None are shared where their ranges do not meet, or where both repeat with one period and lie in
// different parts of it (views of one packed projection).
bool may_meet(const Span3& x, const Span3& y) {
  if (x.empty() || y.empty() || !ranges_overlap((const void*)x.p, (size_t)x.bytes(), (const void*)y.p, (size_t)y.bytes())) return false;
  for (int i = 0; i < 3; ++i) {
    const int64_t period = x.stride[i];
    if (x.extent[i] <= 1 || period <= 0) continue;
    const int64_t nx = in_period(x, period), ny = in_period(y, period);
    const int64_t apart = (int64_t)(y.p >= x.p ? (y.p - x.p) % (uint64_t)period : (period - (int64_t)((x.p - y.p) % (uint64_t)period)) % period);
    if (nx <= period && ny <= period && apart >= nx && apart + ny <= period) return false;
  }
  return true;
}
bool same(const Span3& x, const Span3& y) {
  if (x.p != y.p || x.row != y.row) return false;
  for (int i = 0; i < 3; ++i)
    if (x.extent[i] != y.extent[i] || (x.extent[i] > 1 && x.stride[i] != y.stride[i])) return false;
  return true;
}

constexpr int kMaxHead = 512;
constexpr int64_t kMaxHeads = 0x3fffffff;      // of a call (a lane counts them in 32 bits, and beyond the last one)

const char* rotary_fault(const ficoco_rotary& r) {
  if (r.d_head < 1) return "d_head is not positive";
  if (r.rot_dim < 0 || r.rot_dim % 2 != 0 || r.rot_begin < 0 || (int64_t)r.rot_begin + r.rot_dim > r.d_head) return "the rotated features are no even part of a head";
  if (r.layout != FICOCO_ROTARY_HALVES && r.layout != FICOCO_ROTARY_PAIRS) return "unknown layout";
  if (r.norm != FICOCO_NORM_NONE && r.norm != FICOCO_NORM_RMS && r.norm != FICOCO_NORM_LAYER) return "unknown norm";
  if (r.weight_dtype != FICOCO_F32 && r.weight_dtype != FICOCO_BF16) return "unknown weight_dtype";
  if (r.norm != FICOCO_NORM_NONE && (!(r.eps >= 0.0f) || !std::isfinite(r.eps))) return "eps must be finite and not negative";
  if (r.rot_dim > 0 && (!r.turns || ((uintptr_t)r.turns & 7))) return "turns is NULL or not 8-byte aligned";
  if (r.rot_dim > 0 && !std::isfinite(r.amplitude)) return "amplitude must be finite";
  if (r.norm == FICOCO_NORM_NONE && (r.q_weight || r.k_weight || r.q_bias || r.k_bias)) return "weights or biases without a norm";
  const uintptr_t align = r.weight_dtype == FICOCO_F32 ? 3 : 1;
  if (((uintptr_t)r.q_weight | (uintptr_t)r.k_weight | (uintptr_t)r.q_bias | (uintptr_t)r.k_bias) & align) return "a weight or bias is not aligned to its elements";
  return nullptr;
}

// What is wrong with the positions of a call.
const char* positions_fault(const ficoco_rotation& x) {
  if (!x.pos) return nullptr;
  if (x.axes < 1 || x.axes > 256) return "axes must be 1 .. 256";
  if (x.pos_stride_axis < 0 || x.pos_stride_b < 0) return "a stride is negative";
  if ((uintptr_t)x.pos & 3) return "pos must be 4-byte aligned";
  return nullptr;
}

HeadRows queries(const ficoco_rotation& x) {
  return HeadRows{x.Q, x.Q_out, x.q_stride_b, x.q_stride_h, x.q_stride_n, x.qo_stride_b, x.qo_stride_h, x.qo_stride_n, x.Q ? x.H : 0};
}

// What is wrong with one tensor of B x n tokens and its output.
const char* rows_fault(int64_t B, int64_t n, int64_t heads, int64_t d, const HeadRows& x, int dtype, int out_dtype) {
  if (!x.out) return "an output is NULL";
  if (heads < 1) return "there are no heads";
  const uintptr_t align = dtype == FICOCO_BF16 ? 1 : 3, out_align = out_dtype == FICOCO_BF16 ? 1 : 3;
  if (((uintptr_t)x.x & align) || ((uintptr_t)x.out & out_align)) return "a tensor is not aligned to its elements";
  if (x.sb < 0 || x.sh < 0 || x.sn < 0 || x.ob < 0 || x.oh < 0 || x.on < 0) return "a stride is negative";
  if (rows_collide(d, {{{x.ob, B}, {x.oh, heads}, {x.on, n}}})) return "rows that are written overlap";
  return nullptr;
}

Span3 source(const HeadRows& x, int64_t B, int64_t n, int64_t d, int dtype) {
  return span3(x.x, B, x.heads, n, x.sb, x.sh, x.sn, d, dtype == FICOCO_BF16 ? 2 : 4);
}
Span3 target(const HeadRows& x, int64_t B, int64_t n, int64_t d, int dtype) {
  return span3(x.out, B, x.heads, n, x.ob, x.oh, x.on, d, dtype == FICOCO_BF16 ? 2 : 4);
}

// Whether rows that are written may be among what else a call reads: positions, lengths and slots (`lists`, of B each), frequencies and weights.
bool into_inputs(const ficoco_rotary& r, const ficoco_rotation& x, int64_t B, int64_t n, std::initializer_list<const void*> lists, int64_t q_heads, int64_t k_heads, const Span3& out) {
  if (out.empty()) return false;
  auto meets = [&](const void* p, int64_t bytes) { return p && bytes > 0 && ranges_overlap(p, (size_t)bytes, (const void*)out.p, (size_t)out.bytes()); };
  for (const void* p : lists)
    if (meets(p, B * 4)) return true;
  const int64_t row = (int64_t)r.d_head * (r.weight_dtype == FICOCO_F32 ? 4 : 2), q_row = r.per_head ? q_heads * row : row, k_row = r.per_head ? k_heads * row : row;
  return meets(x.pos, ((x.axes - 1) * x.pos_stride_axis + (B - 1) * x.pos_stride_b + n) * 4) || meets(r.turns, (int64_t)r.rot_dim * 4) || meets(r.axis, r.rot_dim / 2) ||
         meets(r.q_weight, q_row) || meets(r.q_bias, q_row) || meets(r.k_weight, k_row) || meets(r.k_bias, k_row);
}

}  // namespace

extern "C" {

int ficoco_rotate(ficoco_ctx* ctx, const ficoco_rotary* r, const ficoco_rotation* x, void* stream) {
  const char* fn = "ficoco_rotate";
  if (!ctx) return FICOCO_EINVAL;
  if (!r || !x) return fail(ctx, FICOCO_EINVAL, fn, "rotary or rotation is NULL");
  const int rc = check_device(ctx, fn);
  if (rc != FICOCO_OK) return rc;
  if (const char* why = rotary_fault(*r)) return fail(ctx, FICOCO_EINVAL, fn, why);
  if (const char* why = positions_fault(*x)) return fail(ctx, FICOCO_EINVAL, fn, why);
  if (r->d_head > kMaxHead) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "d_head is more than 512");
  if (x->B < 0 || x->n < 0) return fail(ctx, FICOCO_EINVAL, fn, "a size is negative");
  if ((x->dtype != FICOCO_F32 && x->dtype != FICOCO_BF16) || (x->out_dtype != FICOCO_F32 && x->out_dtype != FICOCO_BF16))
    return fail(ctx, FICOCO_EINVAL, fn, "unknown dtype");
  if (x->B == 0 || x->n == 0) return FICOCO_OK;
  if (!x->Q && !x->K) return fail(ctx, FICOCO_EINVAL, fn, "Q and K are both NULL");
  if ((int64_t)(x->Q ? x->H : 0) + (x->K ? x->H_kv : 0) > kMaxHeads) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "too many heads");
  RotateArgs a{};
  a.r = rotary_args(*r, *x);
  a.q = queries(*x);
  a.k = HeadRows{x->K, x->K_out, x->k_stride_b, x->k_stride_h, x->k_stride_n, x->ko_stride_b, x->ko_stride_h, x->ko_stride_n, x->K ? x->H_kv : 0};
  a.B = x->B; a.n = x->n;
  a.n_rows = x->n_rows;
  for (const HeadRows* h : {&a.q, &a.k})
    if (h->x)
      if (const char* why = rows_fault(x->B, x->n, h->heads, r->d_head, *h, x->dtype, x->out_dtype)) return fail(ctx, FICOCO_EINVAL, fn, why);
  const Span3 q = source(a.q, x->B, x->n, r->d_head, x->dtype), k = source(a.k, x->B, x->n, r->d_head, x->dtype);
  const Span3 qo = target(a.q, x->B, x->n, r->d_head, x->out_dtype), ko = target(a.k, x->B, x->n, r->d_head, x->out_dtype);
  const bool one_type = x->dtype == x->out_dtype;
  if ((!(one_type && same(q, qo)) && may_meet(q, qo)) || (!(one_type && same(k, ko)) && may_meet(k, ko)) || may_meet(qo, k) || may_meet(ko, q) || may_meet(qo, ko))
    return fail(ctx, FICOCO_EINVAL, fn, "an output shares elements with another tensor");
  for (const Span3& out : {qo, ko})
    if (into_inputs(*r, *x, x->B, x->n, {x->start, x->n_rows}, a.q.heads, a.k.heads, out)) return fail(ctx, FICOCO_EINVAL, fn, "an output overlaps positions, lengths, frequencies or weights");
  if (rotate_threads(a, x->dtype, x->out_dtype) > kMaxRows - 256) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "too many rows in one call");
  launch_rotate(a, x->dtype, x->out_dtype, (hipStream_t)stream);
  return finish(ctx, fn);
}

int ficoco_cache_append_rotated(ficoco_ctx* ctx, const ficoco_cache* c, int32_t layer, const ficoco_rotary* r, const ficoco_tokens* t,
                                const ficoco_rotation* x, void* stream) {
  const char* fn = "ficoco_cache_append_rotated";
  int rc = begin(ctx, c, fn);
  if (rc == FICOCO_OK) rc = check_tokens(ctx, *c, layer, t, true, fn);
  if (rc != FICOCO_OK) return rc;
  if (!r || !x) return fail(ctx, FICOCO_EINVAL, fn, "rotary or rotation is NULL");
  if (const char* why = rotary_fault(*r)) return fail(ctx, FICOCO_EINVAL, fn, why);
  if (const char* why = positions_fault(*x)) return fail(ctx, FICOCO_EINVAL, fn, why);
  if (r->d_head != c->d_head) return fail(ctx, FICOCO_EINVAL, fn, "d_head is not that of the cache");
  if (r->rot_begin % 8 != 0 || r->rot_dim % 16 != 0) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "rot_begin must be a multiple of 8 and rot_dim of 16");
  if (x->Q && (x->dtype != t->dtype || (x->out_dtype != FICOCO_F32 && x->out_dtype != FICOCO_BF16)))
    return fail(ctx, FICOCO_EINVAL, fn, "Q must have the type of K, Q_out a known one");
  if (t->n == 0 || t->n_max == 0) return FICOCO_OK;
  if (x->Q && x->H > kMaxHeads) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "too many heads");
  RotateArgs a{};
  a.r = rotary_args(*r, *x);
  a.r.start = nullptr;
  a.q = queries(*x);
  a.B = t->n; a.n = t->n_max;
  a.n_rows = t->n_new;
  a.seq = t->seq; a.first = t->start; a.n_seqs = c->n_seqs;
  if (x->Q) {
    if (const char* why = rows_fault(t->n, t->n_max, x->H, r->d_head, a.q, x->dtype, x->out_dtype)) return fail(ctx, FICOCO_EINVAL, fn, why);
    const int64_t d = r->d_head, es = t->dtype == FICOCO_BF16 ? 2 : 4;
    const Span3 q = source(a.q, t->n, t->n_max, d, x->dtype), qo = target(a.q, t->n, t->n_max, d, x->out_dtype);
    const Span3 k = span3(t->K, t->n, c->heads, t->n_max, t->k_stride_b, t->k_stride_h, t->k_stride_n, d, es);
    const Span3 v = span3(t->V, t->n, c->heads, t->n_max, t->v_stride_b, t->v_stride_h, t->v_stride_n, d, es);
    if ((!(x->dtype == x->out_dtype && same(q, qo)) && may_meet(q, qo)) || may_meet(qo, k) || may_meet(qo, v))
      return fail(ctx, FICOCO_EINVAL, fn, "Q_out shares elements with another tensor");
    if (into_inputs(*r, *x, t->n, t->n_max, {t->seq, t->start, t->n_new}, x->H, c->heads, qo)) return fail(ctx, FICOCO_EINVAL, fn, "Q_out overlaps positions, lengths, frequencies or weights");
    if (reaches_into(*c, x->Q_out, (size_t)qo.bytes())) return fail(ctx, FICOCO_EINVAL, fn, "Q_out overlaps the cache");
    if (rotate_threads(a, x->dtype, x->out_dtype) > kMaxRows - 256) return fail(ctx, FICOCO_EUNSUPPORTED, fn, "too many rows in one call");
  }
  launch_append_rotated(*c, layer, *t, a, x->out_dtype, (hipStream_t)stream);
  return finish(ctx, fn);
}

}  // extern "C"

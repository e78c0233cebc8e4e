// Norm and rotation of queries and keys, and the frequencies that it goes by.
#include <cmath>

#include "rotary.hpp"

namespace ficoco {
namespace {

constexpr int kRotateThreads = 256;

// How rows are laid over lanes: 2^shift lanes a row, `per_token` items a token, HPT heads an item (per_token apart).
struct RowShape { int shift, per_token; };

// A lane holds NS slots of a head (slot_of()) and turns them in HPT heads by the same angles.  All loads of a lane are on their way before the angles are formed.
//
// Bound by memory.
template <typename T, typename TO, int W, int NS, int HPT>
__global__ __launch_bounds__(kRotateThreads) void rotate_kernel(RotateArgs a, RowShape shape) {
  const uint32_t at = blockIdx.x * kRotateThreads + threadIdx.x, item = at >> shape.shift, token = item / (uint32_t)shape.per_token;
  const int lanes = 1 << shape.shift, i = at & (lanes - 1), h0 = item - token * shape.per_token, b = token / (uint32_t)a.n;
  const int t = token - (uint32_t)b * a.n;
  if (b >= a.B) return;
  int rows = a.n;
  if (a.n_rows) rows = a.n_rows[b] < rows ? a.n_rows[b] : rows;
  bool there = t < rows;
  int64_t own = t;
  if (a.first) {
    const int s = a.seq ? a.seq[b] : b, first = a.first[b];
    there &= s >= 0 && s < a.n_seqs && first >= 0;
    own += first;
  } else if (a.r.start) {
    own += a.r.start[b];
  }
  Slot<W> slot[NS];
#pragma unroll
  for (int k = 0; k < NS; ++k) slot[k] = slot_of<W>(a.r, i + k * lanes);
  const int heads = a.q.heads + a.k.heads;
  float v[HPT][NS][2 * W];
#pragma unroll
  for (int j = 0; j < HPT; ++j) {
    const int h = h0 + j * shape.per_token;
    const bool key = h >= a.q.heads;
    const HeadRows& x = key ? a.k : a.q;
    const T* p = (const T*)x.x + (int64_t)b * x.sb + (int64_t)(key ? h - a.q.heads : h) * x.sh + (int64_t)t * x.sn;
#pragma unroll
    for (int k = 0; k < NS; ++k) {
#pragma unroll
      for (int e = 0; e < 2 * W; ++e) v[j][k][e] = 0.0f;
      if (there && h < heads) {
        if (slot[k].a >= 0) load_chunk<W>(p + slot[k].a, v[j][k]);
        if (slot[k].b >= 0) load_chunk<W>(p + slot[k].b, v[j][k] + W);
      }
    }
  }
  if (!there) return;                                      // (all lanes of a row)
  Angles<W> angle[NS];
  const Place place = place_of(a.r, b, t, own);
#pragma unroll
  for (int k = 0; k < NS; ++k) angles_of<W>(a.r, slot[k], place, angle[k]);
#pragma unroll
  for (int j = 0; j < HPT; ++j) {
    const int h = h0 + j * shape.per_token;
    if (h >= heads) break;
    const bool key = h >= a.q.heads;
    const HeadRows& x = key ? a.k : a.q;
    const int hh = key ? h - a.q.heads : h;
    normalise<W, NS>(a.r, slot, lanes, key ? a.r.k_weight : a.r.q_weight, key ? a.r.k_bias : a.r.q_bias, hh, v[j]);
    TO* p = (TO*)x.out + (int64_t)b * x.ob + (int64_t)hh * x.oh + (int64_t)t * x.on;
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      turn<W>(a.r, slot[k], angle[k], v[j][k]);
      if (slot[k].a >= 0) store_chunk<W>(p + slot[k].a, v[j][k]);
      if (slot[k].b >= 0) store_chunk<W>(p + slot[k].b, v[j][k] + W);
    }
  }
}

// The widest chunk that the rotated features begin and end with.
int chunk_width(const RotaryArgs& r) {
  for (int w = 8; w > 1; w /= 2)
    if (r.d % w == 0 && r.begin % w == 0 && r.rot % (2 * w) == 0) return w;
  return 1;
}
RowShape shape_of(const RotateArgs& a, int width, int hpt) {
  const int slots = slots_of(a.r.d, a.r.rot, width);
  int shift = 0;
  while (shift < 6 && 1 << shift < slots) ++shift;
  const int heads = a.q.heads + a.k.heads;
  return RowShape{shift, (heads + hpt - 1) / hpt};
}
// Several heads a lane where there are rows enough to fill the chip that way.
int heads_a_lane(const RotateArgs& a) { return (int64_t)a.B * a.n * (a.q.heads + a.k.heads) * a.r.d >= 1 << 23 ? 4 : 1; }

template <typename T, typename TO, int W, int NS>
void launch_rows(const RotateArgs& a, hipStream_t s) {
  const int hpt = heads_a_lane(a);
  const RowShape shape = shape_of(a, W, hpt);
  const dim3 grid((unsigned)(((((int64_t)a.B * a.n * shape.per_token) << shape.shift) + kRotateThreads - 1) / kRotateThreads));
  if (hpt == 4) hipLaunchKernelGGL((rotate_kernel<T, TO, W, NS, 4>), grid, dim3(kRotateThreads), 0, s, a, shape);
  else hipLaunchKernelGGL((rotate_kernel<T, TO, W, NS, 1>), grid, dim3(kRotateThreads), 0, s, a, shape);
}
template <typename T, typename TO>
void launch_width(const RotateArgs& a, hipStream_t s) {
  switch (chunk_width(a.r)) {
    case 8: launch_rows<T, TO, 8, 1>(a, s); break;
    case 4: launch_rows<T, TO, 4, 1>(a, s); break;
    case 2: launch_rows<T, TO, 2, 2>(a, s); break;
    default: launch_rows<T, TO, 1, 4>(a, s); break;
  }
}

}  // namespace

RotaryArgs rotary_args(const ficoco_rotary& r, const ficoco_rotation& x) {
  RotaryArgs y{};
  y.turns = r.turns;
  y.axis = r.axis;
  y.pos = x.pos;
  y.pos_sa = x.pos_stride_axis; y.pos_sb = x.pos_stride_b;
  y.start = x.start;
  y.q_weight = r.q_weight; y.k_weight = r.k_weight; y.q_bias = r.q_bias; y.k_bias = r.k_bias;
  y.axes = x.axes; y.d = r.d_head; y.begin = r.rot_begin; y.rot = r.rot_dim;
  y.pairs = r.layout == FICOCO_ROTARY_PAIRS; y.norm = r.norm; y.weight_f32 = r.weight_dtype == FICOCO_F32; y.per_head = r.per_head != 0;
  y.eps = r.eps; y.amplitude = r.amplitude; y.inv_d = 1.0f / (float)r.d_head;
  return y;
}

int64_t rotate_threads(const RotateArgs& a) {
  const RowShape shape = shape_of(a, chunk_width(a.r), heads_a_lane(a));
  const __int128 n = ((__int128)a.B * a.n * shape.per_token) << shape.shift;
  return n > INT64_MAX ? INT64_MAX : (int64_t)n;
}

void launch_rotate(const RotateArgs& a, int dtype, int out_dtype, hipStream_t s) {
  if (dtype == FICOCO_BF16) {
    if (out_dtype == FICOCO_BF16) launch_width<bf16_t, bf16_t>(a, s); else launch_width<bf16_t, float>(a, s);
  } else {
    if (out_dtype == FICOCO_BF16) launch_width<float, bf16_t>(a, s); else launch_width<float, float>(a, s);
  }
}

}  // namespace ficoco

extern "C" int ficoco_rotary_turns(const ficoco_frequencies* f, uint64_t* turns) {
  if (!f || f->rot_dim < 0 || f->rot_dim % 2 != 0 || f->rot_dim > 512 || (f->rot_dim > 0 && !turns)) return FICOCO_EINVAL;
  if (!(f->base > 0.0) || !std::isfinite(f->base) || !(f->factor > 0.0) || !std::isfinite(f->factor) || !(f->length >= 0.0) || !std::isfinite(f->length)) return FICOCO_EINVAL;
  if (f->length > 0.0 && !(std::isfinite(f->low) && std::isfinite(f->high) && f->low < f->high)) return FICOCO_EINVAL;
  const long double two_pi = 6.283185307179586476925286766559005768L;
  for (int i = 0; i < f->rot_dim / 2; ++i) {
    if (f->divisors && !(std::isfinite(f->divisors[i]) && f->divisors[i] != 0.0)) return FICOCO_EINVAL;
  }
  for (int i = 0; i < f->rot_dim / 2; ++i) {
    long double w = powl((long double)f->base, -2.0L * i / f->rot_dim) / (f->divisors ? (long double)f->divisors[i] : 1.0L);
    long double keep = 0.0L;
    if (f->length > 0.0) {
      keep = (f->length * w / two_pi - f->low) / ((long double)f->high - f->low);
      keep = keep < 0.0L ? 0.0L : keep > 1.0L ? 1.0L : keep;
    }
    w *= keep + (1.0L - keep) / f->factor;
    long double part = w / two_pi;
    part -= floorl(part);                                  // positions are whole: whole turns of a frequency do not count
    part *= 18446744073709551616.0L;
    turns[i] = part >= 18446744073709551615.5L || !(part >= 0.0L) ? 0 : (uint64_t)(part + 0.5L);
  }
  return FICOCO_OK;
}

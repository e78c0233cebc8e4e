// Norm and rotation of queries and keys, and the frequencies that it goes by.
#include <algorithm>
#include <cmath>

#include "rotary.hpp"

namespace ficoco {
namespace {

constexpr int kRotateThreads = 256;

enum NormForm { kNoNorm, kPlainNorm, kAnyNorm };      // (none; root mean square without a bias; whatever the call says)

// How rows are laid over lanes: `lanes` lanes a row, items of up to `heads` heads of one token, q_items of queries and k_items of keys.
struct RowShape {
  int lanes, heads, q_items, k_items;
  Divisor by_lanes, by_items, by_rows;
};

// A lane holds NS slots of a head (slot_of()) and turns them by the same angles in all heads of its item, each read and written once.
//
// Many rows are bound by memory: 32768 tokens, 32 heads of 128 features of which half turn, 537 MB of bfloat16, 104 us (5.1 TB/s, what a copy of 1 GiB reaches); a norm and
// sines by three axes cost a little: 8 ragged prompts of up to 2979 tokens, 40 heads of 128, 356 MB, 79 us (4.5 TB/s).  Single precision by chunks of four: 576 patches of 16 images, 32 heads of 80,
// 189 MB, 44 us (4.3 TB/s).  A few tokens take 3 to 5 us, a launch and two loads one after the other.
template <typename T, typename TO, int W, int NS, NormForm NORM>
__global__ __launch_bounds__(kRotateThreads) void rotate_kernel(RotateArgs a, RowShape shape) {
  // Heads of a lane whose loads are on their way together: two (the 537 MB above 104 us, by one 108, by four 102; 2 prompts of 4100 tokens in single precision with a norm 36 us, 39 and 38), but one
  // where a norm has more to do for each byte and registers for more wavefronts count (the 356 MB above 79 us, by two 82; 16720 tokens, 20 heads of 72, a root mean square 30 and 32, a mean taken out 38 and 42).  (The next heads' loads before these heads are done: 113 us and 99.)
  constexpr int kAtOnce = NORM != kNoNorm && sizeof(T) == 2 ? 1 : 2;
  const int at = blockIdx.x * kRotateThreads + threadIdx.x, all = shape.by_lanes.of(at), token = shape.by_items.of(all), b = shape.by_rows.of(token);
  const int i = at - all * shape.lanes, t = token - b * a.n, in = all - token * (shape.q_items + shape.k_items);
  if (b >= a.B) return;
  const bool key = in >= shape.q_items;
  const HeadRows& x = key ? a.k : a.q;
  const int first = key ? in - shape.q_items : in, step = key ? shape.k_items : shape.q_items;      // heads first, first + step ..
  int rows = a.n;
  if (a.n_rows) rows = a.n_rows[b] < rows ? a.n_rows[b] : rows;
  bool there = t < rows;
  int64_t own = t;
  if (a.first) {
    const int s = a.seq ? a.seq[b] : b, from = a.first[b];
    there &= s >= 0 && s < a.n_seqs && from >= 0;
    own += from;
  } else if (a.r.start) {
    own += a.r.start[b];
  }
  if (!there) return;                                      // (all lanes of a row)
  Slot<W> slot[NS];
#pragma unroll
  for (int k = 0; k < NS; ++k) slot[k] = slot_of<W>(a.r, i + k * shape.lanes);
  Angles<W> angle[NS];
  Weights<W, NS> weights;
  const void *weight = key ? a.r.k_weight : a.r.q_weight, *bias = key ? a.r.k_bias : a.r.q_bias;
  const T* from = (const T*)x.x + (int64_t)b * x.sb + (int64_t)t * x.sn;
  TO* to = (TO*)x.out + (int64_t)b * x.ob + (int64_t)t * x.on;
  for (int h0 = first; h0 < x.heads; h0 += kAtOnce * step) {
    Raw<T, W> raw[kAtOnce][NS][2];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int h = h0 + j * step;
      if (h < x.heads) {
        const T* p = from + (int64_t)h * x.sh;
#pragma unroll
        for (int k = 0; k < NS; ++k) {
          if (slot[k].a >= 0) __builtin_memcpy(&raw[j][k][0], p + slot[k].a, sizeof(raw[j][k][0]));
          if (slot[k].b >= 0) __builtin_memcpy(&raw[j][k][1], p + slot[k].b, sizeof(raw[j][k][1]));
        }
      }
    }
    if (h0 == first) {
      const Place place = place_of(a.r, b, t, own);
#pragma unroll
      for (int k = 0; k < NS; ++k) angles_of<W>(a.r, slot[k], place, angle[k]);
      if (NORM != kNoNorm && !a.r.per_head) weights_of<W, NS>(a.r, slot, weight, bias, 0, weights);
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int h = h0 + j * step;
      if (h >= x.heads) break;
      float v[NS][2 * W];
#pragma unroll
      for (int k = 0; k < NS; ++k) {
#pragma unroll
        for (int e = 0; e < 2 * W; ++e) v[k][e] = 0.0f;
        if (slot[k].a >= 0) widen<W>(raw[j][k][0], v[k]);
        if (slot[k].b >= 0) widen<W>(raw[j][k][1], v[k] + W);
      }
      if (NORM != kNoNorm && (NORM == kPlainNorm || a.r.norm != FICOCO_NORM_NONE)) {
        if (a.r.per_head) weights_of<W, NS>(a.r, slot, weight, bias, h, weights);
        normalise<W, NS, NORM == kPlainNorm>(a.r, slot, shape.lanes, weights, v);
      }
      TO* p = to + (int64_t)h * x.oh;
#pragma unroll
      for (int k = 0; k < NS; ++k) {
        turn<W>(a.r, slot[k], angle[k], v[k]);
        if (slot[k].a >= 0) store_chunk<W>(p + slot[k].a, v[k]);
        if (slot[k].b >= 0) store_chunk<W>(p + slot[k].b, v[k] + W);
      }
    }
  }
}

// The widest chunk that the rotated features begin and end with, of 16 bytes at most: lanes next to each other then load what lies next to each other (16 images'
// patches, heads of 80 in single precision: by chunks of eight 55 us, of four 44).
int chunk_width(const RotaryArgs& r, int most) {
  for (int w = most; w > 1; w /= 2)
    if (r.d % w == 0 && r.begin % w == 0 && r.rot % (2 * w) == 0) return w;
  return 1;
}
RowShape shape_of(const RotateArgs& a, int width) {
  const int slots = std::max(1, slots_of(a.r.d, a.r.rot, width));
  RowShape s{};
  // A norm is a sum over lanes of one wavefront, a power of two of them; without one a row takes what lanes it needs.
  s.lanes = slots;
  if (a.r.norm != FICOCO_NORM_NONE || slots > kWave)
    for (s.lanes = 1; s.lanes < kWave && s.lanes < slots;) s.lanes *= 2;
  // Items of four heads share their angles, where there are rows enough to fill the chip that way: 40 heads of 128 with a norm, 400 tokens 6.9 us, by items of one head 5.2, 800 tokens 7.7 and 8.3,
  // 20000 tokens 80 and 130; 32 heads of 64 in single precision, 800 tokens 5.0 and 4.9, 1600 tokens 6.3 and 7.2.  (The 537 MB of rotate_kernel() by items of two 102 us, of four 104, of eight 109; its 356 MB by eight 79 as by four.)
  const int64_t q_heads = a.q.heads, k_heads = a.k.heads;      // (as many as 32 bits hold: what follows asks for more)
  s.heads = (__int128)a.B * a.n * (q_heads + k_heads) * a.r.d >= 3 << 20 ? 4 : 1;
  s.q_items = (int)((q_heads + s.heads - 1) / s.heads);
  s.k_items = (int)((k_heads + s.heads - 1) / s.heads);
  s.by_lanes = Divisor(s.lanes);
  s.by_items = Divisor((int64_t)s.q_items + s.k_items);
  s.by_rows = Divisor(a.n);
  return s;
}

template <typename T, typename TO, int W, int NS, NormForm NORM>
void launch_rows(const RotateArgs& a, hipStream_t s) {
  const RowShape shape = shape_of(a, W);
  const int64_t threads = (int64_t)a.B * a.n * (shape.q_items + shape.k_items) * shape.lanes;
  hipLaunchKernelGGL((rotate_kernel<T, TO, W, NS, NORM>), dim3((unsigned)((threads + kRotateThreads - 1) / kRotateThreads)), dim3(kRotateThreads), 0, s, a, shape);
}
template <typename T, typename TO, int W>
void launch_norm(const RotateArgs& a, hipStream_t s) {
  if (a.r.norm == FICOCO_NORM_NONE) launch_rows<T, TO, W, 1, kNoNorm>(a, s);
  else if (a.r.norm == FICOCO_NORM_RMS && !a.r.q_bias && !a.r.k_bias) launch_rows<T, TO, W, 1, kPlainNorm>(a, s);
  else launch_rows<T, TO, W, 1, kAnyNorm>(a, s);
}
// A slot a lane; several where there are more slots than a wavefront has lanes, of chunks of two beyond 256 features, of one beyond 128 (always room for several: 16 heads of 72 of which 36 turn, 35810 tokens of
// bfloat16, 87 us instead of 44; of 66, 30000 tokens, 223 instead of 53).  Without a norm chunks of one, too, go by the form that has none, two heads at once (the 66 features 38 us, by the general form, one head at
// once for a norm's sake, 53; 96 of which 50 turn 51 and 86); several slots a lane are better off with the general one (300 features, 15000 tokens, 122, by two heads at once 137; 201 of which 50 turn 165 and 261).
template <typename T, typename TO>
void launch_width(const RotateArgs& a, hipStream_t s) {
  constexpr int most = sizeof(T) == 2 && sizeof(TO) == 2 ? 8 : 4;
  const int width = chunk_width(a.r, most);
  const bool one = slots_of(a.r.d, a.r.rot, width) <= kWave;
  switch (width) {
    case 8: if constexpr (most == 8) launch_norm<T, TO, 8>(a, s); break;
    case 4: launch_norm<T, TO, 4>(a, s); break;
    case 2: if (one) launch_norm<T, TO, 2>(a, s); else launch_rows<T, TO, 2, 2, kAnyNorm>(a, s); break;
    default:
      if (!one) launch_rows<T, TO, 1, 4, kAnyNorm>(a, s);
      else if (a.r.norm == FICOCO_NORM_NONE) launch_rows<T, TO, 1, 1, kNoNorm>(a, s);
      else launch_rows<T, TO, 1, 1, kAnyNorm>(a, s);
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

int64_t rotate_threads(const RotateArgs& a, int dtype, int out_dtype) {
  const RowShape s = shape_of(a, chunk_width(a.r, dtype == FICOCO_BF16 && out_dtype == FICOCO_BF16 ? 8 : 4));
  const __int128 n = (__int128)a.B * a.n * ((int64_t)s.q_items + s.k_items) * s.lanes;
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

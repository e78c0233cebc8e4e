// Norm and rotation of queries and keys: what the kernel of dense rows (rotary.hip) and those that write into pages (rotary_cache.hip) share.
#pragma once
#include <type_traits>

#include "cache.hpp"

namespace ficoco {

struct RotaryArgs {
  const uint64_t* turns;
  const uint8_t* axis;
  const int32_t* pos;
  int64_t pos_sa, pos_sb;
  const int32_t* start;
  const void *q_weight, *k_weight, *q_bias, *k_bias;
  int axes, d, begin, rot, pairs, norm, weight_f32, per_head;      // pairs: neighbours turn together, else the two halves
  float eps, amplitude, inv_d;
};
RotaryArgs rotary_args(const ficoco_rotary& r, const ficoco_rotation& x);

// A head's features as slots of two chunks of W: the two chunks of a slot hold W pairs that turn together (halves: features W i of either half; neighbours: 2 W
// features in a row), and behind these slots come the features that do not turn, in their order, two chunks each.
template <int W>
struct Slot {
  int a, b;            // first features of the chunks, -1: no such chunk
  int turn;            // first frequency, -1: not turned
};
template <int W>
__device__ __forceinline__ Slot<W> slot_of(const RotaryArgs& r, int i) {
  const int turned = r.rot / (2 * W);
  if (i < turned) {
    const int a = r.begin + (r.pairs ? 2 * W : W) * i;
    return Slot<W>{a, r.pairs ? a + W : a + r.rot / 2, W * i};
  }
  const int rest = r.d - r.rot, at = 2 * W * (i - turned);
  auto place = [&](int f) { return f >= rest ? -1 : f < r.begin ? f : f + r.rot; };
  return Slot<W>{place(at), place(at + W), -1};
}
inline int slots_of(int d, int rot, int w) { return rot / (2 * w) + ((d - rot) / w + 1) / 2; }

// Where token t of sequence b stands: on every axis there where positions are given, else `own`.
struct Place {
  const int32_t* pos;
  int64_t own, step;
};
__device__ __forceinline__ Place place_of(const RotaryArgs& r, int b, int64_t t, int64_t own) {
  return Place{r.pos ? r.pos + (int64_t)b * r.pos_sb + t : nullptr, own, r.pos_sa};
}

// sin and cos of `angle` turns / 2^32, times `amplitude`: a quarter turn by its two top bits (rounded), the rest |x| <= pi / 4 by the first terms of their series (what is left
// out is below 2^-29).
__device__ __forceinline__ void sin_cos(uint32_t angle, float amplitude, float& s, float& c) {
  const uint32_t q = angle + 0x20000000u;
  const float x = (float)(int32_t)(angle - (q & 0xc0000000u)) * 1.46291807926715968105e-9f, y = x * x;      // 2 pi / 2^32
  float u = fmaf(y, 2.7557319224e-6f, -1.9841269841e-4f);
  u = fmaf(y, u, 8.3333333333e-3f);
  u = fmaf(y, u, -1.6666666667e-1f);
  u = fmaf(x * y, u, x);
  float v = fmaf(y, -2.7557319224e-7f, 2.4801587302e-5f);
  v = fmaf(y, v, -1.3888888889e-3f);
  v = fmaf(y, v, 4.1666666667e-2f);
  v = fmaf(y, v, -0.5f);
  v = fmaf(y, v, 1.0f);
  const bool odd = q & 0x40000000u;
  s = (odd ? v : u) * __uint_as_float(__float_as_uint(amplitude) ^ (q & 0x80000000u));
  c = (odd ? u : v) * __uint_as_float(__float_as_uint(amplitude) ^ ((q ^ q << 1) & 0x80000000u));
}

// The fraction of a turn, in 2^-32, of `turns` at position p, -2^31 <= p < 2^32: bits 32 .. 63 of their product.
__device__ __forceinline__ uint32_t turned_by(int64_t p, uint64_t turns) {
  const uint32_t low = (uint32_t)turns;
  return (uint32_t)p * (uint32_t)(turns >> 32) + __umulhi((uint32_t)p, low) - (low & (uint32_t)(p >> 63));
}
constexpr int kFewAxes = 4;
template <int W>
struct Angles { float s[W], c[W]; };
template <int W>
__device__ __forceinline__ void angles_of(const RotaryArgs& r, const Slot<W>& slot, const Place& p, Angles<W>& x) {
  if (slot.turn < 0) return;
  uint64_t turns[W];
  __builtin_memcpy(turns, r.turns + slot.turn, sizeof(turns));
  if (!p.pos || r.axes == 1 || !r.axis) {
    const int64_t at = p.pos ? (int64_t)p.pos[0] : p.own;
#pragma unroll
    for (int i = 0; i < W; ++i) sin_cos(turned_by(at, turns[i]), r.amplitude, x.s[i], x.c[i]);
  } else {
    uint64_t axis = 0;
    __builtin_memcpy(&axis, r.axis + slot.turn, W);
    int32_t at[W];
    if (r.axes <= kFewAxes) {                              // (uniform: a load for each axis, not for each pair)
      int32_t on[kFewAxes];
#pragma unroll
      for (int k = 0; k < kFewAxes; ++k) on[k] = p.pos[(k < r.axes ? k : 0) * p.step];
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const uint32_t which = (uint32_t)(axis >> 8 * i) & 255;
        at[i] = on[0];
#pragma unroll
        for (int k = 1; k < kFewAxes; ++k) at[i] = which == (uint32_t)k ? on[k] : at[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const int on = (int)(axis >> 8 * i) & 255;
        at[i] = p.pos[(on < r.axes ? on : 0) * p.step];
      }
    }
#pragma unroll
    for (int i = 0; i < W; ++i) sin_cos(turned_by(at[i], turns[i]), r.amplitude, x.s[i], x.c[i]);
  }
}
template <int W>
__device__ __forceinline__ void turn(const RotaryArgs& r, const Slot<W>& slot, const Angles<W>& x, float (&v)[2 * W]) {
  if (slot.turn < 0) return;
  if (r.pairs) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float a = v[2 * i], b = v[2 * i + 1];
      v[2 * i] = fmaf(a, x.c[i], -(b * x.s[i]));
      v[2 * i + 1] = fmaf(b, x.c[i], a * x.s[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float a = v[i], b = v[W + i];
      v[i] = fmaf(a, x.c[i], -(b * x.s[i]));
      v[W + i] = fmaf(b, x.c[i], a * x.s[i]);
    }
  }
}

// A chunk as it comes out of memory, in whole words where it has any: the compiler otherwise gives every half word a register of its own.
template <typename T, int W>
struct Raw {
  static constexpr int WORDS = W * (int)sizeof(T) / 4;
  typename std::conditional<WORDS == 0, uint16_t, uint32_t>::type x[WORDS == 0 ? W : WORDS];
};
template <int W>
__device__ __forceinline__ void widen(const Raw<bf16_t, W>& r, float* x) {
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if constexpr (W == 1) x[i] = __uint_as_float((uint32_t)r.x[i] << 16);
    else x[i] = __uint_as_float(i % 2 ? r.x[i / 2] & 0xffff0000u : r.x[i / 2] << 16);
  }
}
template <int W>
__device__ __forceinline__ void widen(const Raw<float, W>& r, float* x) {
#pragma unroll
  for (int i = 0; i < W; ++i) x[i] = __uint_as_float(r.x[i]);
}
template <int W, typename T>
__device__ __forceinline__ void load_chunk(const T* p, float* x) {
  Raw<T, W> r;
  __builtin_memcpy(&r, p, sizeof(r));
  widen<W>(r, x);
}
template <int W>
__device__ __forceinline__ void store_chunk(float* p, const float* x) { __builtin_memcpy(p, x, W * sizeof(float)); }
template <int W>
__device__ __forceinline__ void store_chunk(bf16_t* p, const float* x) {
  __bf16 h[W];
#pragma unroll
  for (int i = 0; i < W; ++i) h[i] = (__bf16)x[i];
  __builtin_memcpy(p, h, sizeof(h));
}
template <int W>
__device__ __forceinline__ void load_weights(const void* w, int f32, int64_t at, float* x) {
  if (f32) load_chunk<W>((const float*)w + at, x);
  else load_chunk<W>((const bf16_t*)w + at, x);
}

// Sum over `lanes` (a power of two) neighbouring lanes.
__device__ __forceinline__ float group_sum(float v, int lanes) {
  if (lanes > 1) v += dpp_move<0xB1>(v);
  if (lanes > 2) v += dpp_move<0x4E>(v);
  if (lanes > 4) v += dpp_move<0x141>(v);
  if (lanes > 8) v += dpp_move<0x140>(v);
  if (lanes > 16) v += __shfl_xor(v, 16);
  if (lanes > 32) v += __shfl_xor(v, 32);
  return v;
}

// Weights and biases of a lane's slots; those of chunks that do not exist do not matter.
template <int W, int NS>
struct Weights { float w[NS][2 * W], o[NS][2 * W]; };
template <int W, int NS>
__device__ __forceinline__ void weights_of(const RotaryArgs& r, const Slot<W> (&slot)[NS], const void* weight, const void* bias, int h, Weights<W, NS>& x) {
  const int64_t at = r.per_head ? (int64_t)h * r.d : 0;
#pragma unroll
  for (int k = 0; k < NS; ++k) {
#pragma unroll
    for (int i = 0; i < 2 * W; ++i) {
      x.w[k][i] = 1.0f;
      x.o[k][i] = 0.0f;
    }
    if (weight) {
      if (slot[k].a >= 0) load_weights<W>(weight, r.weight_f32, at + slot[k].a, x.w[k]);
      if (slot[k].b >= 0) load_weights<W>(weight, r.weight_f32, at + slot[k].b, x.w[k] + W);
    }
    if (bias) {
      if (slot[k].a >= 0) load_weights<W>(bias, r.weight_f32, at + slot[k].a, x.o[k]);
      if (slot[k].b >= 0) load_weights<W>(bias, r.weight_f32, at + slot[k].b, x.o[k] + W);
    }
  }
}

// The sum of f(v) over the chunks of a slot.  Chunks of 8 are added as the two slots of 4 that they consist of, so that the sum over a row is the same number
// for either width.
template <int W, typename F>
__device__ __forceinline__ float slot_sum(bool halves, const float (&v)[2 * W], F f) {
#pragma clang fp contract(off)
  float s = 0.0f;
  if constexpr (W == 8) {
    float z = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s = f(i < 4 ? v[i] : halves ? v[4 + i] : v[i], s);
      z = f(i < 4 ? (halves ? v[4 + i] : v[8 + i]) : v[8 + i], z);
    }
    return s + z;
  } else {
#pragma unroll
    for (int i = 0; i < 2 * W; ++i) s = f(v[i], s);
    return s;
  }
}

// The norm of a head's row in NS slots a lane, `lanes` lanes; chunks that do not exist hold zeros.  PLAIN: a root mean square without a bias, decided by the caller.
template <int W, int NS, bool PLAIN = false>
__device__ __forceinline__ void normalise(const RotaryArgs& r, const Slot<W> (&slot)[NS], int lanes, const Weights<W, NS>& x, float (&v)[NS][2 * W]) {
#pragma clang fp contract(off)      // (a row gives the same numbers in every kernel that normalises it)
  if (!PLAIN && r.norm == FICOCO_NORM_LAYER) {
    float mean = 0.0f;
#pragma unroll
    for (int k = 0; k < NS; ++k) mean += slot_sum<W>(slot[k].turn >= 0 && !r.pairs, v[k], [](float a, float s) { return a + s; });
    mean = group_sum(mean, lanes) * r.inv_d;
#pragma unroll
    for (int k = 0; k < NS; ++k) {
#pragma unroll
      for (int i = 0; i < 2 * W; ++i) v[k][i] = (i < W ? slot[k].a : slot[k].b) >= 0 ? v[k][i] - mean : 0.0f;
    }
  }
  float square = 0.0f;
#pragma unroll
  for (int k = 0; k < NS; ++k) square += slot_sum<W>(slot[k].turn >= 0 && !r.pairs, v[k], [](float a, float s) { return fmaf(a, a, s); });
  const float inv = 1.0f / sqrtf(fmaf(group_sum(square, lanes), r.inv_d, r.eps));
#pragma unroll
  for (int k = 0; k < NS; ++k) {
#pragma unroll
    for (int i = 0; i < 2 * W; ++i) v[k][i] = PLAIN ? v[k][i] * inv * x.w[k][i] : fmaf(v[k][i] * inv, x.w[k][i], x.o[k][i]);
  }
}

struct HeadRows {       // queries or keys of a call
  const void* x;
  void* out;
  int64_t sb, sh, sn, ob, oh, on;
  int heads;
};
struct RotateArgs {
  RotaryArgs r;
  HeadRows q, k;
  int B, n;
  const int32_t *n_rows;
  // of an append: rows of entries that it leaves out are left out
  const int32_t *seq, *first;
  int n_seqs;
};
void launch_rotate(const RotateArgs& a, int dtype, int out_dtype, hipStream_t s);
int64_t rotate_threads(const RotateArgs& a, int dtype, int out_dtype);
void launch_append_rotated(const ficoco_cache& c, int layer, const ficoco_tokens& t, const RotateArgs& q, int out_dtype, hipStream_t s);

}  // namespace ficoco

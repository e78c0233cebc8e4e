// New tokens from their projection into the pages of the cache: keys normalised and rotated on the way, queries beside them.
#include "rotary.hpp"

namespace ficoco {
namespace {

// to_e4m3() of values that are numbers and stay within the largest one.
__device__ __forceinline__ uint2 numbers_to_e4m3(const float (&x)[8], float inv) {
  int a = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
  a = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, a, true);
  int b = __builtin_amdgcn_cvt_pk_fp8_f32(x[4] * inv, x[5] * inv, 0, false);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(x[6] * inv, x[7] * inv, b, true);
  return uint2{(uint32_t)a, (uint32_t)b};
}

// One workgroup per touched page, head, sequence and K / V, as cache_append_kernel (cache.hip); a lane holds the two chunks of a slot of a key, so that
// pairs that turn together are in one lane and a key's norm takes D / 16 lanes.
//
// 8 ragged prompts of up to 2979 tokens, 8 heads of 128, three axes, 107 MB: 41 us (2.6 TB/s), some 9 of them for the sines, which every head forms again (values alone: 27 for as many bytes, as fast as memory
// gives them).  Two heads a workgroup, or four one after the other with one set of angles, take more registers or wait more often: 54 and 50 us, where this took 43; angles in front of the
// page 44; a workgroup of 512 threads with one row each 44, registers for two wavefronts more a SIMD 50.
template <typename T, int GPT>
__global__ __launch_bounds__(kMoveThreads) void append_rotated_kernel(ficoco_cache c, int64_t layer_pages, RotaryArgs r, TokenSide ks, TokenSide vs, int n_max,
                                                                      const int32_t* __restrict__ seq, const int32_t* __restrict__ start,
                                                                      const int32_t* __restrict__ n_new) {
  __shared__ float scratch[kMoveThreads / kWave];
  const bool key = !(blockIdx.z & 1);
  const int b = blockIdx.z >> 1, h = blockIdx.y, shift = __builtin_ctz(c.page_size), P = 1 << shift, row_shift = __builtin_ctz(c.d_head / 16);
  const TokenSide& side = key ? ks : vs;
  const Span sp = span_of(c, b, n_max, seq, start, n_new);
  const int64_t at = (sp.first >> shift) + (int64_t)blockIdx.x, pos0 = at << shift;
  if (sp.first < 0 || pos0 >= sp.stop || at >= c.max_pages) return;
  const T* x = (const T*)side.x + (int64_t)b * side.sb + (int64_t)h * side.sh;
  const int i16 = threadIdx.x & ((1 << row_shift) - 1);    // (the same for all of a thread's rows)
  Slot<8> slot[1] = {Slot<8>{16 * i16, 16 * i16 + 8, -1}};
  if (key) slot[0] = slot_of<8>(r, i16);
  float v[GPT][1][16];
#pragma unroll
  for (int j = 0; j < GPT; ++j) {
    const int row = (threadIdx.x + j * kMoveThreads) >> row_shift;
    const int64_t pos = pos0 + row;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[j][0][i] = 0.0f;
    if (row < P && pos >= sp.first && pos < sp.stop) {
      const T* from = x + (pos - sp.first) * side.sn;
      load_chunk<8>(from + slot[0].a, v[j][0]);
      load_chunk<8>(from + slot[0].b, v[j][0] + 8);
    }
  }
  const int page = c.table[(int64_t)sp.slot * c.max_pages + at];
  if (!page_ok(c, page)) return;
  const int64_t block = (layer_pages + page) * c.heads + h;
  uint8_t* pool = side.pool + block * P * c.d_head;
  const int old = pos0 < sp.first ? side.exps[block] : 0;
  if (key) {                                               // (uniform)
#pragma unroll
    for (int j = 0; j < GPT; ++j) {
      const int64_t pos = pos0 + ((threadIdx.x + j * kMoveThreads) >> row_shift);
      if (r.norm != FICOCO_NORM_NONE) {
        Weights<8, 1> weights;
        weights_of<8, 1>(r, slot, r.k_weight, r.k_bias, h, weights);
        normalise<8, 1>(r, slot, 1 << row_shift, weights, v[j]);
      }
      if (pos >= sp.first && pos < sp.stop) {
        Angles<8> angle;
        angles_of<8>(r, slot[0], place_of(r, b, pos - sp.first, pos), angle);
        turn<8>(r, slot[0], angle, v[j][0]);
      }
    }
  }
  // Magnitudes as whole numbers, in their order; those from infinity's on do not count, and a wavefront that has any looks at each value for itself.
  uint32_t most = 0;
  float top = 0.0f;
#pragma unroll
  for (int j = 0; j < GPT; ++j) {
    const int row = (threadIdx.x + j * kMoveThreads) >> row_shift;
    const int64_t pos = pos0 + row;
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(v[j][0][i]) & 0x7fffffffu);
    if (row < P && pos >= sp.first && pos < sp.stop) most = max(most, m);       // (a bias makes something of rows that are not there)
  }
  const bool numbers = __all(most < 0x7f800000u);
  if (numbers) {
    top = __uint_as_float(most);
  } else {
#pragma unroll
    for (int j = 0; j < GPT; ++j) {
      const int row = (threadIdx.x + j * kMoveThreads) >> row_shift;
      const int64_t pos = pos0 + row;
      const bool fresh = row < P && pos >= sp.first && pos < sp.stop;
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, fresh ? finite_magnitude(v[j][0][i]) : 0.0f);
    }
  }
  int e = block_exponent(block_max(top, scratch));
  e = e > old ? e : old;
  const float inv = exp_inverse(e);
  __syncthreads();                                         // the byte is read before it is written
#pragma unroll
  for (int j = 0; j < GPT; ++j) {
    const int row = (threadIdx.x + j * kMoveThreads) >> row_shift;
    const int64_t pos = pos0 + row;
    if (row >= P || pos >= sp.stop) continue;
    uint2* to_a = (uint2*)(pool + row * c.d_head + slot[0].a);
    uint2* to_b = (uint2*)(pool + row * c.d_head + slot[0].b);
    float(&a)[8] = *(float(*)[8])v[j][0];
    float(&z)[8] = *(float(*)[8])(v[j][0] + 8);
    if (pos < sp.first) {
      if (e == old) continue;
      from_e4m3(*to_a, exp_scale(old), a);
      from_e4m3(*to_b, exp_scale(old), z);
    } else if (numbers && e != kExpTop) {                  // (uniform) no value is beyond the block's largest number
      *to_a = numbers_to_e4m3(a, inv);
      *to_b = numbers_to_e4m3(z, inv);
      continue;
    } else if (e == kExpTop) {
      keep_finite(a);
      keep_finite(z);
    }
    *to_a = to_e4m3(a, inv);
    *to_b = to_e4m3(z, inv);
  }
  if (threadIdx.x == 0) side.exps[block] = (uint8_t)e;
}

// One token a sequence, queries, keys and values of all heads in one launch: D / 16 lanes a row, the queries first, then the keys, then the values.  Where a
// new token raises its block's exponent, the wavefront rewrites the older tokens together, 4 KB on their way at once.
//
// A launch and four loads one after the other, 6 us for 48 sequences, 32 heads on 8 of 128 with a norm, and what has to be rewritten: over the 64 steps of a page, where 3 % of the tokens have
// values four times as large, 7.9 us on average and 13 at most.  Sequences are next to each other, not heads: a large token raises the blocks of all of its heads, which are
// of different wavefronts then (heads next to each other, 13.7 us on average and 41 at most).
template <typename T, typename TO, int D>
__global__ __launch_bounds__(kMoveThreads) void append_rotated_token_kernel(ficoco_cache c, int64_t layer_pages, RotateArgs a, TokenSide ks, TokenSide vs, int items,
                                                                            const int32_t* __restrict__ seq, const int32_t* __restrict__ start,
                                                                            const int32_t* __restrict__ n_new) {
  constexpr int L = D / 16;
  const int item = (blockIdx.x * kMoveThreads + threadIdx.x) / L, i16 = threadIdx.x % L, lane = threadIdx.x % kWave;
  const int n_query = a.B * a.q.heads, n_key = a.B * c.heads;
  const bool there = item < items, query = item < n_query, value = item >= n_query + n_key;
  const int in = query ? item : value ? item - n_query - n_key : item - n_query;
  const int h = there ? in / a.B : 0, b = there ? in - h * a.B : 0;
  const TokenSide& side = value ? vs : ks;
  const Span sp = span_of(c, b, 1, seq, start, n_new);
  const bool live = there && sp.first >= 0;
  const int shift = __builtin_ctz(c.page_size), place = sp.first & ((1 << shift) - 1), at = sp.first >> shift;
  Slot<8> slot[1] = {Slot<8>{16 * i16, 16 * i16 + 8, -1}};
  if (!value) slot[0] = slot_of<8>(a.r, i16);
  float v[1][16] = {};
  if (live) {
    const T* x = query ? (const T*)a.q.x + (int64_t)b * a.q.sb + (int64_t)h * a.q.sh : (const T*)side.x + (int64_t)b * side.sb + (int64_t)h * side.sh;
    load_chunk<8>(x + slot[0].a, v[0]);
    load_chunk<8>(x + slot[0].b, v[0] + 8);
  }
  const int page = live && !query && at < c.max_pages ? c.table[(int64_t)sp.slot * c.max_pages + at] : -1;
  const bool ok = page_ok(c, page);
  const int64_t block = ok ? (layer_pages + page) * c.heads + h : 0;
  const int old = ok && place > 0 ? side.exps[block] : 0;
  if (!value) {
    if (a.r.norm != FICOCO_NORM_NONE) {
      Weights<8, 1> weights;
      weights_of<8, 1>(a.r, slot, query ? a.r.q_weight : a.r.k_weight, query ? a.r.q_bias : a.r.k_bias, h, weights);
      normalise<8, 1>(a.r, slot, L, weights, v);
    }
    if (live) {
      Angles<8> angle;
      angles_of<8>(a.r, slot[0], place_of(a.r, b, 0, sp.first), angle);
      turn<8>(a.r, slot[0], angle, v[0]);
    }
  }
  if (query && live) {
    TO* out = (TO*)a.q.out + (int64_t)b * a.q.ob + (int64_t)h * a.q.oh;
    store_chunk<8>(out + slot[0].a, v[0]);
    store_chunk<8>(out + slot[0].b, v[0] + 8);
  }
  float top = 0.0f;
#pragma unroll
  for (int j = 0; j < 16; ++j) top = fmaxf(top, finite_magnitude(v[0][j]));
  top = fmaxf(top, dpp_move<0xB1>(top));
  top = fmaxf(top, dpp_move<0x4E>(top));
  if constexpr (L == 8) top = fmaxf(top, dpp_move<0x141>(top));
  int e = block_exponent(top);
  e = e > old ? e : old;
  uint8_t* pool = side.pool + (block << shift) * D;
  if (ok) {
    float(&x)[8] = *(float(*)[8])v[0];
    float(&y)[8] = *(float(*)[8])(v[0] + 8);
    if (e == kExpTop) {
      keep_finite(x);
      keep_finite(y);
    }
    const float inv = exp_inverse(e);
    *(uint2*)(pool + place * D + slot[0].a) = to_e4m3(x, inv);
    *(uint2*)(pool + place * D + slot[0].b) = to_e4m3(y, inv);
    if (e != old && i16 == 0) side.exps[block] = (uint8_t)e;   // (the lanes of a row read the byte in one instruction, before)
  }
  uint64_t rising = __ballot(ok && e != old && place > 0 && i16 == 0);
  while (rising) {                                         // (uniform)
    const int from = __builtin_ctzll(rising);
    rising &= rising - 1;
    const uint64_t where = (uint64_t)pool;
    uint8_t* p = (uint8_t*)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(where >> 32), from) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)where, from));
    const float scale = exp_scale(__builtin_amdgcn_readlane(old, from)), inv = exp_inverse(__builtin_amdgcn_readlane(e, from));
    const int pieces = __builtin_amdgcn_readlane(place, from) * (D / 16);
    for (int base = 0; base < pieces; base += 4 * kWave) {
      uint4 q[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int at = base + k * kWave + lane;
        if (at < pieces) q[k] = *(const uint4*)(p + 16 * at);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int at = base + k * kWave + lane;
        if (at >= pieces) continue;
        float x[8], y[8];
        from_e4m3(uint2{q[k].x, q[k].y}, scale, x);
        from_e4m3(uint2{q[k].z, q[k].w}, scale, y);
        const uint2 u = to_e4m3(x, inv), w = to_e4m3(y, inv);
        *(uint4*)(p + 16 * at) = uint4{u.x, u.y, w.x, w.y};
      }
    }
  }
}

template <typename T, typename TO>
void launch_tokens(const ficoco_cache& c, int64_t lp, const TokenSide& k, const TokenSide& v, const RotateArgs& a, int items, const ficoco_tokens& t, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)items * (c.d_head / 16) + kMoveThreads - 1) / kMoveThreads));
  if (c.d_head == 128) hipLaunchKernelGGL((append_rotated_token_kernel<T, TO, 128>), grid, dim3(kMoveThreads), 0, s, c, lp, a, k, v, items, t.seq, t.start, t.n_new);
  else hipLaunchKernelGGL((append_rotated_token_kernel<T, TO, 64>), grid, dim3(kMoveThreads), 0, s, c, lp, a, k, v, items, t.seq, t.start, t.n_new);
}

template <typename T>
void launch_append(const ficoco_cache& c, int layer, const ficoco_tokens& t, const RotateArgs& a, int out_dtype, hipStream_t s) {
  const TokenSide k = side_of(t, c, false), v = side_of(t, c, true);
  const int64_t lp = (int64_t)layer * c.n_pages;
  const int64_t items = (int64_t)t.n * ((int64_t)a.q.heads + 2 * (int64_t)c.heads);
  if (t.n_max == 1 && items <= 0x7fffffff / 16) {
    if (out_dtype == FICOCO_BF16) launch_tokens<T, bf16_t>(c, lp, k, v, a, (int)items, t, s); else launch_tokens<T, float>(c, lp, k, v, a, (int)items, t, s);
    return;
  }
  if (a.q.heads > 0) launch_rotate(a, t.dtype, out_dtype, s);
  const dim3 grid(append_pages(c, t.n_max), c.heads, 2 * t.n);
  const int groups = c.page_size * c.d_head / 16;
  if (groups <= 256) hipLaunchKernelGGL((append_rotated_kernel<T, 1>), grid, dim3(groups), 0, s, c, lp, a.r, k, v, t.n_max, t.seq, t.start, t.n_new);
  else if (groups <= 512) hipLaunchKernelGGL((append_rotated_kernel<T, 2>), grid, dim3(kMoveThreads), 0, s, c, lp, a.r, k, v, t.n_max, t.seq, t.start, t.n_new);
  else hipLaunchKernelGGL((append_rotated_kernel<T, 4>), grid, dim3(kMoveThreads), 0, s, c, lp, a.r, k, v, t.n_max, t.seq, t.start, t.n_new);
}

}  // namespace

void launch_append_rotated(const ficoco_cache& c, int layer, const ficoco_tokens& t, const RotateArgs& a, int out_dtype, hipStream_t s) {
  if (t.dtype == FICOCO_BF16) launch_append<bf16_t>(c, layer, t, a, out_dtype, s); else launch_append<float>(c, layer, t, a, out_dtype, s);
}

}  // namespace ficoco

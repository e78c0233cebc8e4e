// Internal declarations of the decoder's key / value cache: pages of 8 bits (cache.hip) and the attention that reads
// them (cache_attn.hip, tile_attn.hip).
#pragma once
#include "common.hpp"

namespace ficoco {

constexpr int kMaxSlots = 8192;      // slots of a cache (their owners in a call are kept in LDS)
constexpr int kMaxCall = 1024;       // sequences of a call that hands out pages: one thread each
constexpr int kMoveThreads = 256;    // of a workgroup that moves tokens or pages
constexpr int kExpBias = 127, kExpMin = 17;
constexpr float kE4m3Max = 448.0f;
constexpr int kExpTop = 247;         // byte of the largest floats: 2^120, in units of which they lie below 256
constexpr float kTopFinite = 240.0f * 0x1p120f;      // the largest E4M3 number of such a block that is read back as a finite one

// Workspace of a compaction: {first new page, pages, tokens, -} of every sequence, then the rows of the table before it.
inline size_t compact_workspace(const ficoco_cache& c, int n) {
  return ((size_t)n * 4 * sizeof(int32_t) + (size_t)n * c.max_pages * sizeof(int32_t) + 255) / 256 * 256;
}

// Threads of an append (write) or a read along the tokens of a sequence.
inline int append_pages(const ficoco_cache& c, int n_max) { return (n_max + c.page_size - 2) / c.page_size + 1; }
inline int64_t token_threads(const ficoco_cache& c, int n_max, bool write) {
  const int rows = kMoveThreads / (c.d_head / 8), pieces = c.page_size * c.d_head / 16;
  return write ? (int64_t)append_pages(c, n_max) * (pieces < kMoveThreads ? pieces : kMoveThreads) : ((int64_t)n_max + rows - 1) / rows * kMoveThreads;
}

void launch_cache_reserve(const ficoco_cache& c, int n, const int32_t* seq, const int32_t* n_new, int n_each, int32_t* start, hipStream_t s);
void launch_cache_append(const ficoco_cache& c, int layer, const ficoco_tokens& t, hipStream_t s);
void launch_cache_read(const ficoco_cache& c, int layer, const ficoco_tokens& t, hipStream_t s);
void launch_cache_fork(const ficoco_cache& c, int n, const int32_t* src, const int32_t* dst, bool whole, int32_t* done, hipStream_t s);
void launch_cache_compact(const ficoco_cache& c, int layer_begin, int n_layers, int n, const int32_t* src, const int32_t* dst, int vis_begin, int N,
                          int n_keep, const int32_t* keep_idx, int32_t* done, char* ws, hipStream_t s);
void launch_cache_free(const ficoco_cache& c, int n, const int32_t* seq, hipStream_t s);

// ---- blocks of 8 bits -----------------------------------------------------------------------------------------
// 2^(byte - 127) and its inverse as floats (byte in 1 .. 253)
__device__ __forceinline__ float exp_scale(int byte) { return __uint_as_float((uint32_t)byte << 23); }
__device__ __forceinline__ float exp_inverse(int byte) { return __uint_as_float((uint32_t)(2 * kExpBias - byte) << 23); }

// The exponent byte of a block whose largest magnitude is amax >= 0 (finite): the smallest k with amax <= 448 * 2^k = 1.75 * 2^(k + 8).
__device__ __forceinline__ int block_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < kExpMin ? kExpMin : e;      // (denormals and zero read as e = -8 or -7: the least byte)
}
__device__ __forceinline__ float finite_magnitude(float x) {
  const float a = fabsf(x);
  return a <= 3.402823466e38f ? a : 0.0f;        // (false for NaN too)
}

// Values of a block with byte kExpTop: finite ones from 248 * 2^120 on would be rounded to 2^128, which is read back as infinity.
__device__ __forceinline__ void keep_finite(float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(x[i]);
    x[i] = a > kTopFinite && a <= 3.402823466e38f ? copysignf(kTopFinite, x[i]) : x[i];
  }
}

// Eight values to E4M3, times `inv`: beyond the largest number the largest; NaN becomes the positive NaN (the conversion's own does not
// keep to one sign: NaN goes through it as 448, the number below).
__device__ __forceinline__ uint2 to_e4m3(const float (&x)[8], float inv) {
  float y[8];
  uint32_t nan[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float p = x[i] * inv;
    y[i] = fmaxf(fminf(p, kE4m3Max), -kE4m3Max);
    nan[i / 4] |= p == p ? 0u : 0x7fu << 8 * (i % 4);
  }
  int a = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  a = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], a, true);
  int b = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], b, true);
  return uint2{(uint32_t)a | nan[0], (uint32_t)b | nan[1]};
}
__device__ __forceinline__ void from_e4m3(uint2 q, float scale, float (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int w = (int)(h ? q.y : q.x);
    x[4 * h + 0] = __builtin_amdgcn_cvt_f32_fp8(w, 0) * scale;
    x[4 * h + 1] = __builtin_amdgcn_cvt_f32_fp8(w, 1) * scale;
    x[4 * h + 2] = __builtin_amdgcn_cvt_f32_fp8(w, 2) * scale;
    x[4 * h + 3] = __builtin_amdgcn_cvt_f32_fp8(w, 3) * scale;
  }
}

}  // namespace ficoco

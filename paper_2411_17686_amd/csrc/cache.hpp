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

// n / d without a division: m = floor(2^(31 + l) / d) + 1 with 2^l >= d, and n m / 2^(31 + l) is above n / d by less than 1 / d for n < 2^31.
struct Divisor {
  uint32_t d, m, s;
  Divisor() = default;
  explicit Divisor(int64_t by) : d((uint32_t)by), m(0), s(0) {
    int l = 0;
    while ((int64_t)1 << l < by) ++l;
    if (l > 0) {
      m = (uint32_t)(((uint64_t)1 << (31 + l)) / (uint64_t)by + 1);
      s = (uint32_t)(l - 1);
    }
  }
  __device__ __forceinline__ int of(int n) const { return d == 1 ? n : (int)(__umulhi((uint32_t)n, m) >> s); }
};

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


// ---- tokens in and out of blocks ----------------------------------------------------------------------------
__device__ __forceinline__ bool slot_ok(const ficoco_cache& c, int s) { return s >= 0 && s < c.n_seqs; }
__device__ __forceinline__ bool page_ok(const ficoco_cache& c, int p) { return p >= 0 && p < c.n_pages; }
__device__ __forceinline__ int pages_of(const ficoco_cache& c, int64_t tokens) { return (int)((tokens + c.page_size - 1) / c.page_size); }

__device__ __forceinline__ void load8f(const bf16_t* p, float (&x)[8]) {
  uint4 r;
  __builtin_memcpy(&r, p, 16);
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8f(const float* p, float (&x)[8]) { __builtin_memcpy(x, p, 32); }
__device__ __forceinline__ void store8f(float* p, const float (&x)[8]) { __builtin_memcpy(p, x, 32); }
__device__ __forceinline__ void store8f(bf16_t* p, const float (&x)[8]) {      // (exact: three mantissa bits)
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xffff0000u);
  __builtin_memcpy(p, w, 16);
}

struct TokenSide {       // K or V of a call
  const void* x;
  int64_t sb, sh, sn;
  uint8_t* pool;
  uint8_t* exps;
};

__device__ __forceinline__ float block_max(float v, float* scratch) {
  v = wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
  const int nw = blockDim.x / kWave;
  __syncthreads();
  if (threadIdx.x % kWave == 0) scratch[threadIdx.x / kWave] = v;
  __syncthreads();
  for (int w = 0; w < nw; ++w) v = fmaxf(v, scratch[w]);
  return v;
}

// What a call writes to one sequence: positions [first, stop) of slot `slot`, none where first < 0.
struct Span { int slot, first; int64_t stop; };
__device__ __forceinline__ Span span_of(const ficoco_cache& c, int b, int n_max, const int32_t* seq, const int32_t* start, const int32_t* n_new) {
  const int s = seq ? seq[b] : b, first = start[b];
  int n = n_new ? n_new[b] : n_max;
  n = n < n_max ? n : n_max;
  return slot_ok(c, s) && first >= 0 && n > 0 ? Span{s, first, (int64_t)first + n} : Span{0, -1, -1};
}

inline TokenSide side_of(const ficoco_tokens& t, const ficoco_cache& c, bool v) {
  return v ? TokenSide{t.V, t.v_stride_b, t.v_stride_h, t.v_stride_n, (uint8_t*)c.v, c.v_exp}
           : TokenSide{t.K, t.k_stride_b, t.k_stride_h, t.k_stride_n, (uint8_t*)c.k, c.k_exp};
}

}  // namespace ficoco

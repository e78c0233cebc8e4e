// What the attention kernels share: the rows of a workgroup, which keys they see, and the parts of a result whose
// keys are cut over several workgroups.
#pragma once
#include "cache.hpp"

namespace ficoco {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

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

// A key / value head serves `group` query heads; their rows are taken together, row r = query r / group of head
// r % group, so that a block's keys are read once for all of them.
struct AttendArgs {
  const bf16_t* Q;
  int64_t q_sb, q_sh, q_sn;
  bf16_t* O;
  int64_t o_sb, o_sh, o_sn;
  const int32_t *seq, *q_len, *k_len, *q_start;
  int B, H_kv, group, n_q, n_k, splits, row_tiles;
  Divisor by_heads, by_group, by_splits, by_all;       // H_kv, group, splits, B * H_kv
  float scale_log2e;
  int window, sinks;
  // pages of the layer
  const uint8_t *k, *v, *k_exp, *v_exp;
  const int32_t *table, *len;
  int n_pages, n_seqs, max_pages, page_shift;
  // dense keys and values
  const bf16_t *K, *V;
  int64_t k_sb, k_sh, k_sn, v_sb, v_sh, v_sn;
  // parts of cut rows: [B * H_kv][splits][rows] of (maximum, sum) and of sums of values
  float2* part_ms;
  float* part_o;
  int part_rows;                      // row_tiles * rows of a workgroup
};

constexpr float kNoLogit = -3.402823466e38f;     // maximum of a row that has seen nothing (a finite one: differences stay numbers)

// What the rows of one sequence see.
struct Sight {
  int first;        // position of query 0
  int queries;      // that count
  int keys;         // keys there are
};
template <bool PAGED>
__device__ __forceinline__ Sight sight_of(const AttendArgs& a, int b, int& slot) {
  Sight s;
  slot = b;
  if constexpr (PAGED) {
    slot = a.seq ? a.seq[b] : b;
    const bool ok = slot >= 0 && slot < a.n_seqs;
    slot = ok ? slot : 0;
    s.keys = ok ? a.len[slot] : 0;
    const int64_t room = (int64_t)a.max_pages << a.page_shift;
    s.keys = s.keys < room ? s.keys : (int)room;
  } else {
    s.keys = a.n_k;
  }
  if (a.k_len) s.keys = a.k_len[b] < s.keys ? a.k_len[b] : s.keys;
  s.keys = s.keys > 0 ? s.keys : 0;
  s.queries = a.q_len && a.q_len[b] < a.n_q ? a.q_len[b] : a.n_q;
  s.first = a.q_start ? a.q_start[b] : s.keys - s.queries;
  return s;
}

// Blocks of KEYS keys that queries at positions lo .. hi of a sequence see: `head` blocks from key 0 on (the first tokens),
// then the blocks from `near` on.
template <int KEYS>
struct Blocks {
  int head, near, count;
  int near_key, first_keys;       // keys below near_key are seen by no row unless they are below first_keys
  int end;                        // keys behind the last one seen
  __device__ __forceinline__ Blocks(const AttendArgs& a, const Sight& s, int lo, int hi) {
    end = hi < s.keys ? hi + 1 : s.keys;
    end = end > 0 ? end : 0;
    near_key = a.window > 0 && lo >= a.window ? lo - a.window + 1 : 0;
    near_key = near_key < end ? near_key : end;
    first_keys = a.sinks < near_key ? a.sinks : near_key;
    near = near_key / KEYS;
    head = (first_keys + KEYS - 1) / KEYS;
    head = head < near ? head : near;
    count = head + (end + KEYS - 1) / KEYS - near;
  }
  __device__ __forceinline__ int block(int i) const { return i < head ? i : near + (i - head); }
};

// The keys that one row sees: [lo, lo + span], and those below `first`.
struct RowSight {
  int lo, first;
  uint32_t span;
  RowSight() = default;
  __device__ __forceinline__ RowSight(const AttendArgs& a, int pos, int keys) {
    const int hi = pos < keys ? pos : keys - 1;
    const int64_t from = a.window > 0 ? (int64_t)pos - a.window + 1 : 0;
    lo = from > 0 ? (int)from : 0;
    first = a.window > 0 ? (a.sinks < hi + 1 ? a.sinks : hi + 1) : 0;
    span = (uint32_t)(hi - lo);
    if (hi < lo) {                       // nothing but first keys: a range that holds no key there can be
      lo = 0x7fffffff;
      span = 0;
    }
  }
  __device__ __forceinline__ bool sees(int key) const { return (uint32_t)(key - lo) <= span; }
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)a, (__bf16)b});
}
// Four E4M3 numbers times a power of two as four bfloat16 (exact).
__device__ __forceinline__ uint2 widen_e4m3(uint32_t q, float scale) {
  return uint2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale, true))};
}

constexpr int kTileWaves = 4, kTileThreads = kTileWaves * kWave;
constexpr int kTileRows = 32 * kTileWaves;   // rows of a workgroup where there are many
constexpr int kTileKeys = 64;                // keys of its step
constexpr float kSlack = 8.0f;               // (units of log2) growth of a row's maximum that is put up with

// (fmaxf() would first bring either argument into canonical form, an instruction more for each)
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
__device__ __forceinline__ float halves_max(float v) { return fmaxf(v, __shfl_xor(v, 32)); }

// The 32 rows of a wavefront, out of the lanes that hold them (a row in two lanes, four features at a time) through 64 * D bytes of
// LDS of its own, so that lanes next to each other store 16 bytes next to each other: with 8 bytes a lane and two lanes a row the
// stores of a workgroup took 1.6 us.  to(row, piece): where piece (16 bytes) of row 0 .. 31 goes, null for nowhere.
template <int D, typename F>
__device__ __forceinline__ void rows_out(const f32x16_t (&o)[D / 32], float inv, uint8_t* lds, F to) {
  constexpr int CH = D / 8;
  const int lane = threadIdx.x % kWave, row = lane % 32, half = lane / 32;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(uint2*)(lds + row * 2 * D + ((4 * i + j) ^ (row & (CH - 1))) * 16 + half * 8) =
          uint2{pack_bf16(o[i][4 * j] * inv, o[i][4 * j + 1] * inv), pack_bf16(o[i][4 * j + 2] * inv, o[i][4 * j + 3] * inv)};
  }
#pragma unroll
  for (int k = 0; k < CH / 2; ++k) {
    const int r = (k * kWave + lane) / CH, c = lane % CH;
    const uint4 x = *(const uint4*)(lds + r * 2 * D + (c ^ (r & (CH - 1))) * 16);
    if (void* p = to(r, c)) __builtin_memcpy(p, &x, 16);
  }
}
// The same in single precision, half of the features at a time; pieces 0 .. D / 4 - 1.
template <int D, typename F>
__device__ __forceinline__ void float_rows_out(const f32x16_t (&o)[D / 32], uint8_t* lds, F to) {
  constexpr int CH = D / 8, DH = D / 64;
  const int lane = threadIdx.x % kWave, row = lane % 32, half = lane / 32;
#pragma unroll
  for (int part = 0; part < 2; ++part) {
#pragma unroll
    for (int i = 0; i < DH; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x16_t& x = o[part * DH + i];
        *(f32x4_t*)(lds + row * 2 * D + ((8 * i + 2 * j + half) ^ (row & (CH - 1))) * 16) = f32x4_t{x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]};
      }
    }
#pragma unroll
    for (int k = 0; k < CH / 2; ++k) {
      const int r = (k * kWave + lane) / CH, c = lane % CH;
      const uint4 x = *(const uint4*)(lds + r * 2 * D + (c ^ (r & (CH - 1))) * 16);
      if (void* p = to(r, part * CH + c)) __builtin_memcpy(p, &x, 16);
    }
  }
}

// Between products and a branch behind which their results are read.  A result may be read a number of instructions after the product
// at the earliest; the compiler keeps to that inside a block, but not everywhere across a branch (seen with ROCm 7.2: copies
// of the last two registers of a 32 x 32 result in the block behind a branch, three instructions later, got what was there before).
__device__ __forceinline__ void products_settle() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// How the keys of a call are cut: few workgroups otherwise leave compute units idle.
struct AttendPlan {
  bool few;            // single tokens (cache_attn.hip), else tiles of 128 rows (page_attn.hip; dense: tile_attn.hip)
  int rows;            // rows of a workgroup
  int row_tiles, splits;
  size_t part_ms, part_o, total;
};
AttendPlan attend_plan(const ficoco_attention& a, int heads, int64_t max_keys, bool paged);

void launch_few_rows(const AttendArgs& a, int d_head, hipStream_t s);
void launch_page_rows(const AttendArgs& a, int d_head, hipStream_t s);
void launch_dense_rows(const AttendArgs& a, int d_head, hipStream_t s);
void launch_join_rows(const AttendArgs& a, int d_head, hipStream_t s);

}  // namespace ficoco

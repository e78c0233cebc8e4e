// Attention of dense prompts, with or without a window.
#include <algorithm>

#include "attend.hpp"

namespace ficoco {
namespace {

typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4_t* lds_i16x4_t;

// Rows of keys and values in LDS, in bfloat16, 16-byte chunks; chunk c of a row lies at c ^ swizzle.  A key row is read 16 bytes a lane
// by 16 rows at once, a value row by groups of 16 lanes, two groups four keys x 32 features at once: these put either on all 64 banks.
template <int D> __device__ __forceinline__ int key_swizzle(int row) { return D == 128 ? row & 15 : row >> 1 & 7; }
template <int D> __device__ __forceinline__ int value_swizzle(int row) { return D == 128 ? (row & 3) << 2 : (row & 2) << 1; }

enum TileSource {
  kDenseDirect,      // 16-byte aligned rows: straight into LDS
  kDense             // any other: through registers
};
template <int D> struct TileRaw { uint4 x[D / 32]; };       // a thread's share of a step's keys or values

// One pass with a running maximum and sum, 128 rows a workgroup, 32 a wavefront, 64 keys a step.  32 x 32 x 16 products:
//   S^T[key][row] = K Q^T, the queries in registers; a lane holds 32 logits of one row
//   O^T[feature][row] += V^T P^T, the contraction in the order in which the lanes hold the weights; V^T out of LDS by transposing reads
// A step's weights are formed beside the products of the next step's logits: exponentials and products of one wavefront otherwise take
// turns.  So keys are in LDS a step ahead of the values; either in two buffers, what comes next on its way while a step is computed.
//
// Bound by LDS, out of which four SIMDs at their full rate would take 128 bytes a cycle, all it gives, while the loads write to it, and by the matrix cores at the
// clock that they leave (1.9 GHz): 16384 tokens, window of 4096, 32 heads of 128 on 8: 920 .. 960 us on different cards, 1.00 .. 1.05 PFLOP/s of
// products (a large library product reaches 1.2); without its loads it would take 714, without exponentials 843 (where it takes 920).  Two prompts of 675 tokens,
// 32 heads: 19 .. 20 us, of which 5 before the first step.  Weights are rounded to bfloat16 for the second product, as in few_rows_kernel (cache_attn.hip).
template <int D, TileSource SRC>
__global__ __launch_bounds__(kTileThreads, 2) void tile_rows_kernel(AttendArgs a) {
  constexpr int DT = D / 32, KS = D / 16, CH = D / 8;
  constexpr int NL = D / 32;                       // 16-byte loads of a thread
  // (four arrays, chosen at compile time: the compiler then knows that loads into one do not concern reads of another)
  __shared__ __align__(16) bf16_t sk0[kTileKeys * D], sk1[kTileKeys * D], sv0[kTileKeys * D], sv1[kTileKeys * D];
  const int tid = threadIdx.x, lane = tid % kWave, wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int c32 = lane % 32, half = lane / 32;
  // The last rows of all heads first, as they see most keys; heads whose number is a multiple of 8 stay on their XCD.  (Head after head, an eighth of the
  // workgroups to an XCD: two prompts of 675 tokens 23.4 us instead of 20.0, three of up to 7745 with 28 heads on 4 809 instead of 550, of 4096 with heads of 64
  // 61 instead of 57, one of 16384 the same.)
  const int back = a.by_all.of(blockIdx.x), bh = blockIdx.x - back * a.B * a.H_kv, b = a.by_heads.of(bh), h = bh - b * a.H_kv, tile = a.row_tiles - 1 - back;
  int slot;
  const Sight s = sight_of<false>(a, b, slot);
  const int rows = s.queries * a.group, row0 = tile * kTileRows;
  if (s.queries <= 0 || row0 >= rows) return;
  auto pos_of = [&](int r) { return s.first + a.by_group.of(r < rows ? r : rows - 1); };
  const Blocks<kTileKeys> blocks(a, s.keys, pos_of(row0), pos_of(row0 + kTileRows - 1));
  const int begin = 0, end = blocks.count;

  const int r = row0 + 32 * wv + c32, my_r = r < rows ? r : rows - 1;
  const int t = a.by_group.of(my_r), g = my_r - t * a.group, pos = s.first + t;
  const int lo = pos_of(row0 + 32 * wv), hi = pos_of(row0 + 32 * wv + 31);      // positions of the wavefront
  bf16x8_t qf[KS];
  f32x16_t o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x16_t{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
  float top = kNoLogit, sum = 0.0f;

  auto wanted = [&](int key) { return key < blocks.end && (key >= blocks.near_key || key < blocks.first_keys); };

  // ---- straight into LDS: a wavefront's load fills 64 chunks in a row.  Rows that no query of the workgroup sees become zeros (places
  // behind the end of their buffer): their weights are zero, and zero times what memory happens to hold may be NaN.
  // (Buffer loads: behind a global load into LDS the compiler waits for all reads of LDS at once.)
  const int d_row = 64 / CH * wv + lane / CH;                                   // rows of load j: d_row + RJ * j
  constexpr int RJ = 64 * kTileWaves / CH;
  auto rows_at = [&](const bf16_t* base, int64_t sn, int step) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(base + (int64_t)blocks.block(step) * kTileKeys * sn), 0, step < end ? 0x7fffffff : 0, 0x00027000);
  };
  auto hidden_rows = [&](int step) {               // bit j: the row of load j is hidden
    const int key0 = blocks.block(step) * kTileKeys;
    int hidden = 0;
    if (!(key0 + kTileKeys <= blocks.end && (key0 >= blocks.near_key || key0 + kTileKeys <= blocks.first_keys))) {
#pragma unroll
      for (int j = 0; j < NL; ++j) hidden |= (wanted(key0 + d_row + RJ * j) ? 0 : 1) << j;
    }
    return hidden;
  };
  const int k_bytes = (int)a.k_sn * 2, v_bytes = (int)a.v_sn * 2;               // (64 rows lie within 2^30 bytes: launch_dense_rows)
  const int k_off = d_row * k_bytes + (lane % CH ^ key_swizzle<D>(d_row)) * 16, v_off = d_row * v_bytes + (lane % CH ^ value_swizzle<D>(d_row)) * 16;
  auto direct = [&](__amdgpu_buffer_rsrc_t from, int hidden, bf16_t* to, int off, int row_bytes, int j) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(to + (j * kTileWaves + wv) * 64 * 8), 16,
                                             off + (int)((uint32_t)hidden << (31 - j) & 0x80000000u), RJ * j * row_bytes, 0, 0);
  };

  // ---- through registers
  // (load j: row my_row + RJ * j, for which the swizzles are the same, so that one address serves all; addresses of their own cost heads of 128 ten
  // spilled registers, 1319 us instead of 1158 for 16384 tokens)
  const int my_row = tid / CH, my_chunk = tid % CH;
  static_assert(RJ % 16 == 0, "swizzles look at four bits of a row at most");
  auto load_dense = [&](TileRaw<D>& raw, const bf16_t* base, int64_t sn, int step) {
    const int key0 = blocks.block(step) * kTileKeys + my_row;
    const bf16_t* from = base + (int64_t)key0 * sn + 8 * my_chunk;
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      raw.x[j] = uint4{0, 0, 0, 0};
      if (step < end && wanted(key0 + RJ * j)) __builtin_memcpy(&raw.x[j], from + j * RJ * sn, 16);
    }
  };
  const bf16_t* Kb = a.K + (int64_t)b * a.k_sb + (int64_t)h * a.k_sh;
  const bf16_t* Vb = a.V + (int64_t)b * a.v_sb + (int64_t)h * a.v_sh;
  auto load_k = [&](TileRaw<D>& raw, bf16_t* to, int step) {
    if constexpr (SRC == kDense) {
      load_dense(raw, Kb, a.k_sn, step);
    } else {
      const __amdgpu_buffer_rsrc_t from = rows_at(Kb, a.k_sn, step);
      const int hidden = hidden_rows(step);
#pragma unroll
      for (int j = 0; j < NL; ++j) direct(from, hidden, to, k_off, k_bytes, j);
    }
  };
  auto load_v = [&](TileRaw<D>& raw, bf16_t* to, int step) {
    if constexpr (SRC == kDense) {
      load_dense(raw, Vb, a.v_sn, step);
    } else {
      const __amdgpu_buffer_rsrc_t from = rows_at(Vb, a.v_sn, step);
      const int hidden = hidden_rows(step);
#pragma unroll
      for (int j = 0; j < NL; ++j) direct(from, hidden, to, v_off, v_bytes, j);
    }
  };
  auto store = [&](const TileRaw<D>& raw, bf16_t* to, bool keys) {
    if constexpr (SRC != kDenseDirect) {
      uint4* r = (uint4*)to + my_row * CH + (my_chunk ^ (keys ? key_swizzle<D>(my_row) : value_swizzle<D>(my_row)));
#pragma unroll
      for (int j = 0; j < NL; ++j) r[j * RJ * CH] = raw.x[j];
    }
  };
  auto arrived = [&]() {
    if constexpr (SRC == kDenseDirect) __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0)
    __syncthreads();
  };

  const int k_swizzle = key_swizzle<D>(c32);
  auto logits = [&](f32x16_t (&S)[2]) {            // of the first step
    const bf16_t* k0 = &sk0[c32 * D];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const bf16x8_t kf = *(const bf16x8_t*)(k0 + kb * 32 * D + (2 * k + half ^ k_swizzle) * 8);
        S[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[k], k == 0 ? f32x16_t{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0} : S[kb], 0, 0, 0);
      }
    }
  };
  // Every key of a step by every row of the wavefront: keys up to seen_to, from seen_from on or among the first ones.
  const int seen_to = __builtin_amdgcn_readfirstlane(lo < s.keys ? lo : s.keys - 1);
  const int seen_from = __builtin_amdgcn_readfirstlane(a.window > 0 && hi >= a.window ? hi - a.window + 1 : 0);
  auto all_seen = [&](int step) {
    const int key0 = blocks.block(step) * kTileKeys, last = key0 + kTileKeys - 1;
    return last <= seen_to && (key0 >= seen_from || last < a.sinks);
  };
  auto largest = [&](const f32x16_t (&S)[2]) {
    float m = fmaxf(S[0][0], S[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) m = max3(m, S[0][i], S[1][i]);
    return m;
  };
  const RowSight sight(a, pos, s.keys);
  auto mask = [&](f32x16_t (&S)[2], int step) __attribute__((always_inline)) {    // what a row does not see: -infinity; a lane's largest logit
    const int key0 = blocks.block(step) * kTileKeys + 4 * half;
    const bool firsts = a.window > 0 && blocks.block(step) * kTileKeys < a.sinks;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int i = 0; i < 16; ++i) S[kb][i] = sight.sees(key0 + kb * 32 + i / 4 * 8 + i % 4) | (firsts & (key0 + kb * 32 + i / 4 * 8 + i % 4 < sight.first)) ? S[kb][i] : -__builtin_huge_valf();
    }
    return largest(S);
  };
  // the running maximum, moved where a logit (m: a lane's largest one) lies far above it
  auto raise = [&](float m) {
    if (__any(m > top + kSlack)) {
      const float n = fmaxf(top, halves_max(m)), f = __builtin_amdgcn_exp2f(top - n);
      top = n;
      sum *= f;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= f;
    }
  };
  const int v_row = 4 * half + lane % 16 / 4, v_swizzle = value_swizzle<D>(v_row);       // (of rows 8 and 16 further on too)
  // a lane's places: chunk 2 k + half of key c32, and the four features from 32 i on of its first key (the swizzle is an exclusive or too)
  const int k_at = c32 * D + (half ^ k_swizzle) * 8, v_at = v_row * D + (lane / 16 % 2 * 2 + lane % 4 / 2 ^ v_swizzle) * 8 + lane % 4 % 2 * 4;

  TileRaw<D> raw;
  // (ka, va: of this step;  kb, vb: of the next one)
  auto advance = [&](f32x16_t (&S)[2], f32x16_t (&next)[2], bf16_t* ka, bf16_t* kb, bf16_t* va, bf16_t* vb, int i) __attribute__((always_inline)) {
    constexpr int NA = 2 * KS, NB = 4 * DT;        // products of either kind
    constexpr int AHEAD = 4;                       // operands on their way out of LDS
    // Weights: logit, exponential and sum three places apart, so that none waits for the one before; `place` p takes logit p + 3, exponential p and sum
    // p - 3.  The first places beside the first kind of product (three operands of the second kind are then there), the others beside the second.
    constexpr int PLACES = 35, PA = 28;
    // Direct loads go one by one between the products: all at once they hold up the reads of LDS.
    const __amdgpu_buffer_rsrc_t next_k = rows_at(Kb, a.k_sn, i + 2), next_v = rows_at(Vb, a.v_sn, i + 1);
    const int hidden_k = hidden_rows(i + 2), hidden_v = hidden_rows(i + 1);
    if constexpr (SRC == kDense) load_v(raw, vb, i + 1);
    bf16x8_t kf[AHEAD], vf[AHEAD], P[4];
    float x[32], w[32];
    auto read_k = [&](int g) { kf[g % AHEAD] = *(const bf16x8_t*)(kb + g / KS * 32 * D + (k_at ^ g % KS * 16)); };
    auto read_v = [&](int g) {
      const bf16_t* v = va + 16 * (g / DT) * D + (v_at ^ g % DT * 32);
      const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t)v));
      const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t)(v + 8 * D)));
      vf[g % AHEAD] = __builtin_bit_cast(bf16x8_t, uint4{x.x, x.y, y.x, y.y});
    };
    auto place = [&](int p) {
      if (p + 3 < 32) x[p + 3] = fmaf(S[(p + 3) / 16][(p + 3) % 16], a.scale_log2e, -top);
      if (p < 32) w[p] = __builtin_amdgcn_exp2f(x[p]);
      const int e = p - 3;
      if (e >= 0) sum += w[e];
      if (e >= 0 && e % 8 == 7)
        P[e / 8] = __builtin_bit_cast(bf16x8_t, uint4{pack_bf16(w[e - 7], w[e - 6]), pack_bf16(w[e - 5], w[e - 4]), pack_bf16(w[e - 3], w[e - 2]), pack_bf16(w[e - 1], w[e])});
    };
#pragma unroll
    for (int e = 0; e < 3; ++e) x[e] = fmaf(S[0][e], a.scale_log2e, -top);
#pragma unroll
    for (int g = 0; g < AHEAD; ++g) read_k(g);
#pragma unroll
    for (int g = 0; g < NA; ++g) {
      __builtin_amdgcn_sched_barrier(0);
      next[g / KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[g % AHEAD], qf[g % KS], g % KS == 0 ? f32x16_t{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0} : next[g / KS], 0, 0, 0);
      if (g + AHEAD < NA) read_k(g + AHEAD);
      else if constexpr (SRC == kDenseDirect) read_v(g + AHEAD - NA);
      if constexpr (SRC == kDenseDirect) {
        if (g % 2 == 1 && g / 2 < NL) direct(next_k, hidden_k, ka, k_off, k_bytes, g / 2);
        else if (g % 2 == 1) direct(next_v, hidden_v, vb, v_off, v_bytes, g / 2 - NL);
      }
#pragma unroll
      for (int p = g * PA / NA; p < (g + 1) * PA / NA; ++p) place(p);
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (SRC != kDenseDirect) {
      store(raw, vb, false);
      load_k(raw, ka, i + 2);
#pragma unroll
      for (int g = 0; g < AHEAD; ++g) read_v(g);
    }
    float m[2] = {next[0][0], next[0][1]};
#pragma unroll
    for (int g = 0; g < NB; ++g) {
      __builtin_amdgcn_sched_barrier(0);
      o[g % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[g % AHEAD], P[g / DT], o[g % DT], 0, 0, 0);
      if (g + AHEAD < NB) read_v(g + AHEAD);
#pragma unroll
      for (int p = PA + g * 16 / NB; p < PA + (g + 1) * 16 / NB && p < PLACES; ++p) place(p);
      if (g >= NB / 2) {
#pragma unroll
        for (int e = (g - NB / 2) * 32 / NB; e < (g + 1 - NB / 2) * 32 / NB; ++e) m[e % 2] = max3(m[e % 2], next[e / 8][e % 8 * 2], next[e / 8][e % 8 * 2 + 1]);
      }
    }
    products_settle();
    if (i + 1 < end) raise((all_seen(i + 1) ? fmaxf(m[0], m[1]) : mask(next, i + 1)) * a.scale_log2e);
    store(raw, ka, true);
    arrived();
  };
  f32x16_t S0[2], S1[2];
  if (begin < end) {
    load_k(raw, sk0, begin);
    store(raw, sk0, true);
    load_v(raw, sv0, begin);
    store(raw, sv0, false);
    load_k(raw, sk1, begin + 1);
    store(raw, sk1, true);
  }
  {                                                // (behind the keys, which more has to wait for)
    const bf16_t* q = a.Q + (int64_t)b * a.q_sb + (int64_t)(h * a.group + g) * a.q_sh + (int64_t)t * a.q_sn + 8 * half;
#pragma unroll
    for (int k = 0; k < KS; ++k) __builtin_memcpy(&qf[k], q + 16 * k, 16);
  }
  arrived();
  if (begin < end) {
    logits(S0);
    products_settle();
    raise((all_seen(begin) ? largest(S0) : mask(S0, begin)) * a.scale_log2e);
  }
  __syncthreads();                                 // (the first keys are read before their buffer is filled again)
  for (int i = begin; i < end; i += 2) {
    advance(S0, S1, sk0, sk1, sv0, sv1, i);
    if (i + 1 < end) advance(S1, S0, sk1, sk0, sv1, sv0, i + 1);
  }

  sum += __shfl_xor(sum, 32);
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  const int first_row = row0 + 32 * wv;
  rows_out<D>(o, inv, (uint8_t*)(wv < 2 ? sk0 : sk1) + wv % 2 * 64 * D, [&](int row, int piece) -> void* {
    const int r = first_row + row, t = a.by_group.of(r);
    return r < rows ? a.O + (int64_t)b * a.o_sb + (int64_t)(h * a.group + r - t * a.group) * a.o_sh + (int64_t)t * a.o_sn + 8 * piece : nullptr;
  });
}

}  // namespace

void launch_dense_rows(const AttendArgs& a, int d_head, hipStream_t s) {
  const dim3 grid((unsigned)(a.B * a.H_kv * a.row_tiles)), threads(kTileThreads);
  // (straight into LDS: no registers, and no waiting for them.  16384 tokens 920 us, through registers 1110; two prompts of 675 tokens 19.6, 23.6.  Rows at odd
  // elements, which have to go through registers: 1158 and 25.8)
  const bool direct = (((uintptr_t)a.K | (uintptr_t)a.V) & 15) == 0 && ((a.k_sb | a.k_sh | a.k_sn | a.v_sb | a.v_sh | a.v_sn) & 7) == 0 &&
                      a.k_sn < (1 << 23) && a.v_sn < (1 << 23);
  if (d_head == 128) {
    if (direct) hipLaunchKernelGGL((tile_rows_kernel<128, kDenseDirect>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((tile_rows_kernel<128, kDense>), grid, threads, 0, s, a);
  } else {
    if (direct) hipLaunchKernelGGL((tile_rows_kernel<64, kDenseDirect>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((tile_rows_kernel<64, kDense>), grid, threads, 0, s, a);
  }
}

}  // namespace ficoco

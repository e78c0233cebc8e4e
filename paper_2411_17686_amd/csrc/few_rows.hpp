// Attention over pages of 8 bits for few rows: the work of one workgroup (16 rows, some of the keys), wherever its rows come from.
#pragma once
#include "attend.hpp"

namespace ficoco {

constexpr int kFewWaves = 4, kFewRows = 16;         // rows of a workgroup
constexpr int kFewKeys = 32;                 // keys of a step

// One step's keys, and values, of a lane as they come out of memory.
template <int D> struct FewKeys { uint4 x[2][D / 64]; };
template <int D> struct FewValues { uint32_t x[2][4][D / 64]; };

// Four dwords of four keys, each four features, as four dwords of four features, each four keys.
__device__ __forceinline__ void transpose4(const uint32_t (&a)[4], uint32_t (&t)[4]) {
  const uint32_t x = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), y = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u);
  const uint32_t z = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u), w = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
  t[0] = __builtin_amdgcn_perm(z, x, 0x05040100u);
  t[1] = __builtin_amdgcn_perm(z, x, 0x07060302u);
  t[2] = __builtin_amdgcn_perm(w, y, 0x05040100u);
  t[3] = __builtin_amdgcn_perm(w, y, 0x07060302u);
}

__device__ __forceinline__ float quarters_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float quarters_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// o = sum_j softmax_j(scale q . k_j) v_j for 16 rows, in one pass with a running maximum and sum.  Every wavefront takes steps of
// 32 keys of its own, straight from memory into registers, the next step's loads in flight while one is computed:
//   S^T[key][row] = K Q^T      operand A a lane's 32 bytes of key lane % 16 (the features of a lane are not in order: Q has them alike)
//   O^T[feature][row] += V^T P^T   contraction over 32 keys in the order in which a lane holds its logits, so that the weights
//                                  stay where they are; operand A eight keys of one feature, out of a byte transposition
// 8 bits become bfloat16 (exactly, the block's scale with them) in front of the products.  A row's maximum is the reference of its
// exponentials as long as no logit lies more than 8 (units of log2) above it: a weight then stays below 2^8.  Weights are rounded to bfloat16 for the second
// product (half a step, 2^-9 to 2^-8 of each; their sum is of the unrounded ones): single precision has a sixteenth of its rate, and two parts of bfloat16 would
// double it.  Against 64 bits results are off by 0.0021 of their size, the plain form by 0.0017, which is the rounding of the results.
//
// Bound by memory: 2 d_head bytes a token and head.  4 sequences of 40000 .. 65536 tokens, 32 heads on 8: 80 us, 5.7 TB/s, a plain read's rate; with the join 86 .. 89;
// 32 of 300 .. 4096: 37 us with the join, 4.1 TB/s (the longest sequences end last); one of 243: 6 us, a launch and three trips to memory.  24 sequences,
// 28 heads of 64 on 4, behind a window of 1 .. 32 tokens 5.2 us, of 2048 9.4, 4096 13.3, 8192 21.3: such a start, then 6.3 TB/s.
//
// tid: the thread.  A lane's row (lane % 16) has its queries at q and sees `sight`; `rows` of the 16 rows count.  Keys of head h are those of blocks begin .. end - 1 and of the table's `row`;
// lo, hi: the rows' first and last position, keys: how many keys each of them has at least.  put(r, feature, x, top, sum): eight features of
// row r, relative to the row's maximum, and its sum.  lds: where the wavefronts' parts meet: at(w, row, feature), eight features from a multiple of eight on next to each other, and top, sum
// [kFewWaves * kFewRows].
template <int D, typename Lds, typename Steps, typename Put>
__device__ __forceinline__ void few_rows(const AttendArgs& a, int tid, Lds& lds, int h, const bf16_t* q, const RowSight& sight, int rows, int lo, int hi, int keys,
                                         const int32_t* row, const Steps& blocks, int begin, int end, Put put) {
  constexpr int L = D / 64;                  // 16-byte loads of a key
  constexpr int M = D / 16;                  // blocks of 16 features; features of a lane's value load
  const int lane = tid % kWave, wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int c16 = lane % 16, q4 = lane / 16;
  // queries: features 64 l + 16 q4 + 8 u .. + 8
  bf16x8_t qf[L][2];
#pragma unroll
  for (int l = 0; l < L; ++l) {
#pragma unroll
    for (int u = 0; u < 2; ++u) __builtin_memcpy(&qf[l][u], q + 64 * l + 16 * q4 + 8 * u, 16);
  }
  f32x4_t o[M];
#pragma unroll
  for (int m = 0; m < M; ++m) o[m] = f32x4_t{0, 0, 0, 0};
  float top = kNoLogit, sum = 0.0f;

  // Pages and exponents of 32 steps (64 half steps of 16 keys, one a lane): the page or -1, and both bytes.  A half of which no row sees a key counts as one
  // without a page: nobody need have written its exponents, and a byte of 255 would make NaN of the zeros that its values become.
  struct Meta { int page, exps; };
  auto meta_of = [&](int chunk) {
    Meta m{-1, 0};
    const int i = begin + wv + (chunk * 32 + lane / 2) * kFewWaves;
    if (i < end) {
      const int key = blocks.block(i) * kFewKeys + 16 * (lane & 1);
      const bool some = key < blocks.end && (key + 16 > blocks.near_key || key < blocks.first_keys);       // (then key lies inside the row: see sight_of)
      int p = some ? row[key >> a.page_shift] : -1;
      p = p < a.n_pages ? p : -1;
      if (p >= 0) m.exps = a.k_exp[(int64_t)p * a.H_kv + h] | a.v_exp[(int64_t)p * a.H_kv + h] << 8;
      m.page = p;
    }
    return m;
  };
  const int steps = begin + wv < end ? (end - begin - wv + kFewWaves - 1) / kFewWaves : 0;
  Meta now = meta_of(0), next = steps > 32 ? meta_of(1) : Meta{-1, 0};
  const int page_bytes = D << a.page_shift;
  auto block_at = [&](int step, const Meta& m, int u) {           // bytes to half step u's first key
    const int key = blocks.block(begin + wv + step * kFewWaves) * kFewKeys + 16 * u, p = __builtin_amdgcn_readlane(m.page, (step & 31) * 2 + u);
    return ((int64_t)(p < 0 ? 0 : p) * a.H_kv + h) * page_bytes + (key & ((1 << a.page_shift) - 1)) * D;
  };
  auto load_keys = [&](FewKeys<D>& raw, int step, const Meta& m) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint8_t* k = a.k + block_at(step, m, u);
#pragma unroll
      for (int l = 0; l < L; ++l) raw.x[u][l] = *(const uint4*)(k + (c16 * D + 16 * q4) + 64 * l);
    }
  };
  auto load_values = [&](FewValues<D>& raw, int step, const Meta& m) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint8_t* v = a.v + block_at(step, m, u);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (L == 2) {
          const uint2 x = *(const uint2*)(v + (4 * q4 * D + c16 * M) + i * D);
          raw.x[u][i][0] = x.x;
          raw.x[u][i][1] = x.y;
        } else {
          raw.x[u][i][0] = *(const uint32_t*)(v + (4 * q4 * D + c16 * M) + i * D);
        }
      }
    }
  };
  auto compute = [&](const FewKeys<D>& k_raw, FewValues<D>& values, int step, const Meta& m) {
    const int key0 = blocks.block(begin + wv + step * kFewWaves) * kFewKeys;
    float ks[2], vs[2];
    bool there = true, have[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int e = __builtin_amdgcn_readlane(m.exps, (step & 31) * 2 + u);
      have[u] = __builtin_amdgcn_readlane(m.page, (step & 31) * 2 + u) >= 0;
      there &= have[u];
      ks[u] = exp_scale(e & 255);
      vs[u] = exp_scale(e >> 8);
    }
    f32x4_t S[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int l = 0; l < L; ++l) {
        const uint32_t w[4] = {k_raw.x[u][l].x, k_raw.x[u][l].y, k_raw.x[u][l].z, k_raw.x[u][l].w};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint2 x = widen_e4m3(w[2 * half], ks[u]), y = widen_e4m3(w[2 * half + 1], ks[u]);
          S[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, uint4{x.x, x.y, y.x, y.y}), qf[l][half], l + half == 0 ? f32x4_t{0, 0, 0, 0} : S[u], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);                  // (here and below: or the compiler runs ahead, and out of registers)
    }
    products_settle();
    const int last = key0 + kFewKeys - 1;
    const bool all_seen = there && last < keys && last <= lo && (a.window <= 0 || (int64_t)key0 > (int64_t)hi - a.window || last < a.sinks);
#pragma unroll
    for (int i = 0; i < 8; ++i) S[i / 4][i % 4] *= a.scale_log2e;
    if (!all_seen) {                                      // (uniform)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = key0 + 16 * u + 4 * q4 + i;
          const bool seen = have[u] & (sight.sees(key) | (key < sight.first));
          S[u][i] = seen ? S[u][i] : -__builtin_huge_valf();
          // what no row sees may hold anything, and 0 * NaN is NaN
          const bool some = have[u] & (key < blocks.end) & ((key >= blocks.near_key) | (key < blocks.first_keys));
#pragma unroll
          for (int l = 0; l < L; ++l) values.x[u][i][l] = some ? values.x[u][i][l] : 0u;
        }
      }
    }
    const float t = fmaxf(max3(S[0][0], S[0][1], S[0][2]), max3(S[0][3], max3(S[1][0], S[1][1], S[1][2]), S[1][3]));
    if (__any(t > top + kSlack)) {
      const float m = fmaxf(top, quarters_max(t)), f = __builtin_amdgcn_exp2f(top - m);
      top = m;
      sum *= f;
#pragma unroll
      for (int i = 0; i < M; ++i) o[i] *= f;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(S[i / 4][i % 4] - top);
      sum += p[i];
    }
    const bf16x8_t P = __builtin_bit_cast(bf16x8_t, uint4{pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])});
#pragma unroll
    for (int w = 0; w < M / 4; ++w) {                     // four features of the lane at a time
      uint32_t t[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t x[4] = {values.x[u][0][w], values.x[u][1][w], values.x[u][2][w], values.x[u][3][w]};
        transpose4(x, t[u]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint2 x = widen_e4m3(t[0][i], vs[0]), y = widen_e4m3(t[1][i], vs[1]);
        o[4 * w + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, uint4{x.x, x.y, y.x, y.y}), P, o[4 * w + i], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    products_settle();
  };

  // A step's values and the next step's keys are on their way while its logits are formed, the next step's keys beyond that.
  FewKeys<D> k0, k1;
  FewValues<D> values;
  if (steps > 0) load_keys(k0, 0, now);
  for (int i = 0; i < steps; i += 2) {
    // (a chunk is 32 steps: an even step and the next one are of the same chunk)
    load_values(values, i, now);
    if (i + 1 < steps) load_keys(k1, i + 1, now);
    compute(k0, values, i, now);
    if (i + 1 >= steps) break;
    load_values(values, i + 1, now);
    const bool turn = ((i + 2) & 31) == 0;
    if (i + 2 < steps) load_keys(k0, i + 2, turn ? next : now);
    compute(k1, values, i + 1, now);
    if (turn) {
      now = next;
      if (i + 34 < steps) next = meta_of((i + 34) / 32);
    }
  }

  // the wavefronts' parts
  const float total_here = quarters_sum(sum);
  if (q4 == 0) {
    lds.top[wv * kFewRows + c16] = top;
    lds.sum[wv * kFewRows + c16] = total_here;
  }
#pragma unroll
  for (int m = 0; m < M; ++m) {
#pragma unroll
    for (int i = 0; i < 4; ++i) *lds.at(wv, c16, (4 * q4 + i) * M + m) = o[m][i];
  }
  __syncthreads();
  for (int j = tid; j < kFewRows * D / 8; j += kFewWaves * kWave) {
    const int r = j / (D / 8), d = j % (D / 8) * 8;
    if (r >= rows) continue;
    float m = lds.top[r];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) m = fmaxf(m, lds.top[w * kFewRows + r]);
    float total = 0.0f, x[8] = {};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(lds.top[w * kFewRows + r] - m);
      total += f * lds.sum[w * kFewRows + r];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] += f * lds.at(w, r, d)[i];
    }
    put(r, d, x, m, total);
  }
}

// Eight features of a row, divided by its sum, as bfloat16.
__device__ __forceinline__ void put_row(bf16_t* o, const float (&x)[8], float total) {
  const float inv = total > 0.0f ? 1.0f / total : 0.0f;
  const uint4 w = {pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv), pack_bf16(x[4] * inv, x[5] * inv), pack_bf16(x[6] * inv, x[7] * inv)};
  __builtin_memcpy(o, &w, 16);
}

}  // namespace ficoco

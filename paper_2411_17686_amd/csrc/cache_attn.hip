// Attention over pages of 8 bits for few rows: single tokens of a decoder, the few of a draft and short questions, all query
// heads of a key / value head together.
#include <algorithm>

#include "attend.hpp"

namespace ficoco {
namespace {

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

// o = sum_j softmax_j(scale q . k_j) v_j for 16 rows a workgroup, in one pass with a running maximum and sum.  Every wavefront takes steps of
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
template <int D>
__global__ __launch_bounds__(kFewWaves * kWave, 2) void few_rows_kernel(AttendArgs a) {
  constexpr int L = D / 64;                  // 16-byte loads of a key
  constexpr int M = D / 16;                  // blocks of 16 features; features of a lane's value load
  __shared__ float so[kFewWaves][kFewRows][D + 4];
  __shared__ float sm[kFewWaves][kFewRows], ss[kFewWaves][kFewRows];
  const int lane = threadIdx.x % kWave, wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c16 = lane % 16, q4 = lane / 16;
  const int at = a.by_splits.of(blockIdx.x), split = blockIdx.x - at * a.splits, tile = a.by_all.of(at), bh = at - tile * a.B * a.H_kv;
  const int b = a.by_heads.of(bh), h = bh - b * a.H_kv, row0 = tile * kFewRows;
  int slot;
  const Sight s = sight_of<true>(a, b, slot);
  const int all_rows = s.queries * a.group, rows = all_rows - row0 < kFewRows ? all_rows - row0 : kFewRows;      // (of this workgroup)
  if (s.queries <= 0 || rows <= 0) return;
  const int lo = s.first + a.by_group.of(row0), hi = s.first + a.by_group.of(row0 + rows - 1);
  const Blocks<kFewKeys> blocks(a, s, lo, hi);
  int per = a.by_splits.of(blocks.count + a.splits - 1);
  per = (per + kFewWaves - 1) / kFewWaves * kFewWaves;
  const int begin = split * per, end = begin + per < blocks.count ? begin + per : blocks.count;

  // queries: row c16, features 64 l + 16 q4 + 8 u .. + 8
  bf16x8_t qf[L][2];
  const int my_r = row0 + (c16 < rows ? c16 : rows - 1);
  const int my_t = a.by_group.of(my_r);
  const RowSight sight(a, s.first + my_t, s.keys);
  {
    const bf16_t* q = a.Q + (int64_t)b * a.q_sb + (int64_t)(h * a.group + my_r - my_t * a.group) * a.q_sh + (int64_t)my_t * a.q_sn;
#pragma unroll
    for (int l = 0; l < L; ++l) {
#pragma unroll
      for (int u = 0; u < 2; ++u) __builtin_memcpy(&qf[l][u], q + 64 * l + 16 * q4 + 8 * u, 16);
    }
  }
  f32x4_t o[M];
#pragma unroll
  for (int m = 0; m < M; ++m) o[m] = f32x4_t{0, 0, 0, 0};
  float top = kNoLogit, sum = 0.0f;

  // Pages and exponents of 32 steps (64 half steps of 16 keys, one a lane): the page or -1, and both bytes.  A half of which no row sees a key counts as one
  // without a page: nobody need have written its exponents, and a byte of 255 would make NaN of the zeros that its values become.
  struct Meta { int page, exps; };
  const int32_t* row = a.table + (int64_t)slot * a.max_pages;
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
  auto compute = [&](const FewKeys<D>& keys, FewValues<D>& values, int step, const Meta& m) {
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
        const uint32_t w[4] = {keys.x[u][l].x, keys.x[u][l].y, keys.x[u][l].z, keys.x[u][l].w};
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
    const bool all_seen = there && last < s.keys && last <= lo && (a.window <= 0 || (int64_t)key0 > (int64_t)hi - a.window || last < a.sinks);
    S[0] *= a.scale_log2e;
    S[1] *= a.scale_log2e;
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
    sm[wv][c16] = top;
    ss[wv][c16] = total_here;
  }
#pragma unroll
  for (int m = 0; m < M; ++m) {
#pragma unroll
    for (int i = 0; i < 4; ++i) so[wv][c16][(4 * q4 + i) * M + m] = o[m][i];
  }
  __syncthreads();
  for (int j = threadIdx.x; j < kFewRows * D / 8; j += kFewWaves * kWave) {
    const int r = j / (D / 8), d = j % (D / 8) * 8;
    if (r >= rows) continue;
    float m = sm[0][r];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) m = fmaxf(m, sm[w][r]);
    float total = 0.0f, x[8] = {};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm[w][r] - m);
      total += f * ss[w][r];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] += f * so[w][r][d + i];
    }
    if (a.splits > 1) {
      const int64_t at = ((int64_t)bh * a.splits + split) * a.part_rows + row0 + r;
      if (d == 0) a.part_ms[at] = float2{m, total};
      __builtin_memcpy(a.part_o + at * D + d, x, 32);
    } else {
      const float inv = total > 0.0f ? 1.0f / total : 0.0f;
      const uint4 w = {pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv), pack_bf16(x[4] * inv, x[5] * inv),
                       pack_bf16(x[6] * inv, x[7] * inv)};
      const int t = a.by_group.of(row0 + r);
      __builtin_memcpy(a.O + (int64_t)b * a.o_sb + (int64_t)(h * a.group + row0 + r - t * a.group) * a.o_sh + (int64_t)t * a.o_sn + d, &w, 16);
    }
  }
}

// Rows whose keys were cut: the parts, relative to their largest maximum, eight at a time (all of their loads in flight).  D / 4 lanes a row and group of
// parts; the groups' sums meet in LDS.  Bound by memory and its latency: 16384 rows of 4 parts, 34 MB, 8 us; 128 rows of 16 parts 4 us.
template <int D, int GROUPS>
__global__ __launch_bounds__(kFewWaves * kWave) void join_rows_kernel(AttendArgs a) {
  constexpr int L = D / 4, AT_ONCE = 8;
  __shared__ f32x4_t sums[GROUPS > 1 ? kFewWaves * kWave : 1];
  __shared__ float2 tops[GROUPS > 1 ? kFewWaves * kWave / L : 1];
  const int rows = a.n_q * a.group, piece = threadIdx.x % L, group = threadIdx.x / L % GROUPS;
  const int64_t at = (int64_t)blockIdx.x * (kFewWaves * kWave / (L * GROUPS)) + threadIdx.x / (L * GROUPS);
  const bool there = at < (int64_t)rows * a.B * a.H_kv;
  const int bh = there ? (int)(at / rows) : 0, r = there ? (int)(at - (int64_t)bh * rows) : 0, b = a.by_heads.of(bh), h = bh - b * a.H_kv;
  const int t = a.by_group.of(r);
  const bool wanted = there && !(a.q_len && t >= a.q_len[b]);
  const int64_t part = (int64_t)bh * a.splits * a.part_rows + r;
  float m = kNoLogit, total = 0.0f;
  f32x4_t x = {0, 0, 0, 0};
  for (int i = group * AT_ONCE; wanted && i < a.splits; i += GROUPS * AT_ONCE) {
    float2 ms[AT_ONCE];
    f32x4_t v[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      ms[k] = float2{kNoLogit, 0.0f};
      v[k] = f32x4_t{0, 0, 0, 0};
      if (i + k < a.splits) {
        const int64_t p = part + (int64_t)(i + k) * a.part_rows;
        ms[k] = a.part_ms[p];
        v[k] = *(const f32x4_t*)(a.part_o + p * D + 4 * piece);
      }
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) top = fmaxf(top, ms[k].x);
    const float f = __builtin_amdgcn_exp2f(m - top);
    total *= f;
    x *= f;
    m = top;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const float w = __builtin_amdgcn_exp2f(ms[k].x - m);
      total += w * ms[k].y;
      x += v[k] * w;
    }
  }
  if constexpr (GROUPS > 1) {
    sums[threadIdx.x] = x;
    if (piece == 0) tops[threadIdx.x / L] = float2{m, total};
    __syncthreads();
    if (group > 0) return;
    const int first = threadIdx.x / L;
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) m = fmaxf(m, tops[first + g].x);
    const float f = __builtin_amdgcn_exp2f(tops[first].x - m);
    total *= f;
    x *= f;
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) {
      const float w = __builtin_amdgcn_exp2f(tops[first + g].x - m);
      total += w * tops[first + g].y;
      x += sums[threadIdx.x + g * L] * w;
    }
  }
  if (!wanted) return;
  const float inv = total > 0.0f ? 1.0f / total : 0.0f;
  const uint2 w = {pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
  __builtin_memcpy(a.O + (int64_t)b * a.o_sb + (int64_t)(h * a.group + r - t * a.group) * a.o_sh + (int64_t)t * a.o_sn + 4 * piece, &w, 8);
}

template <int D, int GROUPS>
void launch_join(const AttendArgs& a, hipStream_t s) {
  constexpr int per = kFewWaves * kWave / (D / 4 * GROUPS);
  const dim3 grid((unsigned)(((int64_t)a.B * a.H_kv * a.n_q * a.group + per - 1) / per));
  hipLaunchKernelGGL((join_rows_kernel<D, GROUPS>), grid, dim3(kFewWaves * kWave), 0, s, a);
}

}  // namespace

AttendPlan attend_plan(const ficoco_attention& a, int heads, int64_t max_keys, bool paged) {
  AttendPlan pl{};
  const int64_t rows = (int64_t)a.n_q * (a.H / heads), bh = (int64_t)a.B * heads;
  // Workgroups of 16 rows that stream the keys, or of 128 that have them in LDS.  One of 16: 4 rows of 243 tokens 6 us, the other way 11; of 40000 .. 65536 86 and 155.
  // Up to four of them, as long as there are few enough to have every key read and converted that often: 64 heads of 2400 tokens, 32 rows 17 and 25, 64 rows
  // 23 and 27.  1000 .. 2000 tokens, heads of 128 (of 64), this way and the other:
  //   heads   32 rows                       48 rows                       64 rows
  //   128     21 and 32 us (16 and 23)      27 and 32 (20 and 23)         27 and 33 (20 and 24)
  //   256     27 and 46 (20 and 34)         45 and 48 (24 and 34)         54 and 49 (29 and 35): the other way
  //   344     46 and 66 (23 and 48)         65 and 67 (33 and 49): 1032, the other way    77 and 68 (40 and 49): the other way
  //   512     66 and 71 (32 and 50)         93 and 72 (48 and 51): the other way          120 and 73 (61 and 52): the other way
  //   1024    151 and 137 (64 and 93): the other way for all
  // The line is drawn for heads of 128 and a few thousand tokens.  Beyond it heads of 64 take up to 1.6 times what they could (344 heads behind 300 .. 600, 48 rows:
  // 13 and 21 us), and short of it long sequences up to 1.3 times: behind 6000 .. 9000, 128 heads of 128, 48 rows 107 and 86 us, 256 heads 211 and 163; 512 heads, 32 rows 347 and 294.
  const int64_t tiles = (rows + kFewRows - 1) / kFewRows;
  pl.few = paged && (tiles <= 1 || (tiles <= 4 && bh * tiles <= (tiles <= 3 ? 1024 : 512)));
  pl.rows = pl.few ? kFewRows : kTileRows;
  pl.row_tiles = (int)std::max<int64_t>(1, (rows + pl.rows - 1) / pl.rows);
  pl.splits = 1;
  if (paged && bh > 0) {
    int64_t seen = max_keys;
    if (a.window > 0) seen = std::min(seen, (int64_t)a.window + a.sinks + a.n_q);
    // Keys are cut where there are too few workgroups: at most two a compute unit (what is resident at once; rounded up instead, the last few run alone: 20 questions of
    // 325 tokens, 4 heads, 61 us and 44; 40 single tokens behind 2000 .. 3000, 8 heads, 52 and 48), 256 keys each at least.  4 sequences of
    // 40000 .. 65536 tokens, 8 heads: 256 workgroups 93 us, 512 86, 1024 88; 32 of 300 .. 4096: 45, 37, 36; 8 questions of 64 tokens behind 1251 .. 2400:
    // 1024 52 us, 512 39.  One sequence of 1000 tokens: at least 128 keys 8.6 us, 256 9.1, 512 10.8; two of 4000: 11.3, 10.8, 12.2.
    const int64_t want = 512 / (bh * pl.row_tiles);
    pl.splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, seen / 256), 256));
  }
  const size_t parts = pl.splits > 1 ? (size_t)bh * pl.splits * pl.row_tiles * pl.rows : 0;
  pl.part_ms = 0;
  pl.part_o = (parts * sizeof(float2) + 255) / 256 * 256;
  pl.total = std::max<size_t>(256, pl.part_o + (parts * a.d_head * sizeof(float) + 255) / 256 * 256);
  return pl;
}

void launch_few_rows(const AttendArgs& a, int d_head, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.B * a.H_kv * a.row_tiles * a.splits)), threads(kFewWaves * kWave);
  if (d_head == 128) hipLaunchKernelGGL(few_rows_kernel<128>, grid, threads, 0, s, a);
  else hipLaunchKernelGGL(few_rows_kernel<64>, grid, threads, 0, s, a);
}

void launch_join_rows(const AttendArgs& a, int d_head, hipStream_t s) {
  // More than one batch of parts: by eight groups at once.  With the whole call, one sequence of 65536 tokens 32 us, by one group 39; 84 rows behind 30078 tokens
  // 19 and 29; 4 sequences of 40000 .. 65536 86 and 87.
  const bool many = a.splits > 8;
  if (d_head == 128) many ? launch_join<128, 8>(a, s) : launch_join<128, 1>(a, s);
  else many ? launch_join<64, 8>(a, s) : launch_join<64, 1>(a, s);
}

}  // namespace ficoco

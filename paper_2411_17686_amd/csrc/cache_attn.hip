// Attention over pages of 8 bits for few rows: single tokens of a decoder, the few of a draft and short questions, all query
// heads of a key / value head together.
#include <algorithm>

#include "few_rows.hpp"

namespace ficoco {
namespace {

template <int D>
struct FewLds {
  float o[kFewWaves][kFewRows][D + 4], top[kFewWaves * kFewRows], sum[kFewWaves * kFewRows];
  __device__ __forceinline__ float* at(int w, int row, int feature) { return &o[w][row][feature]; }
};

template <int D>
__global__ __launch_bounds__(kFewWaves * kWave, 2) void few_rows_kernel(AttendArgs a) {
  __shared__ FewLds<D> lds;
  const int at = a.by_splits.of(blockIdx.x), split = blockIdx.x - at * a.splits, tile = a.by_all.of(at), bh = at - tile * a.B * a.H_kv;
  const int b = a.by_heads.of(bh), h = bh - b * a.H_kv, row0 = tile * kFewRows;
  int slot;
  const Sight s = sight_of<true>(a, b, slot);
  const int all_rows = s.queries * a.group, rows = all_rows - row0 < kFewRows ? all_rows - row0 : kFewRows;      // (of this workgroup)
  if (s.queries <= 0 || rows <= 0) return;
  const int lo = s.first + a.by_group.of(row0), hi = s.first + a.by_group.of(row0 + rows - 1);
  const Blocks<kFewKeys> blocks(a, s.keys, lo, hi);
  int per = a.by_splits.of(blocks.count + a.splits - 1);
  per = (per + kFewWaves - 1) / kFewWaves * kFewWaves;
  const int begin = split * per, end = begin + per < blocks.count ? begin + per : blocks.count;
  const int c16 = threadIdx.x % kFewRows, my_r = row0 + (c16 < rows ? c16 : rows - 1), my_t = a.by_group.of(my_r);
  const bf16_t* q = a.Q + (int64_t)b * a.q_sb + (int64_t)(h * a.group + my_r - my_t * a.group) * a.q_sh + (int64_t)my_t * a.q_sn;
  few_rows<D>(a, threadIdx.x, lds, h, q, RowSight(a, s.first + my_t, s.keys), rows, lo, hi, s.keys, a.table + (int64_t)slot * a.max_pages, blocks, begin, end,
              [&](int r, int d, const float (&x)[8], float m, float total) {
    if (a.splits > 1) {
      const int64_t at = ((int64_t)bh * a.splits + split) * a.part_rows + row0 + r;
      if (d == 0) a.part_ms[at] = float2{m, total};
      __builtin_memcpy(a.part_o + at * D + d, x, 32);
    } else {
      const int t = a.by_group.of(row0 + r);
      put_row(a.O + (int64_t)b * a.o_sb + (int64_t)(h * a.group + row0 + r - t * a.group) * a.o_sh + (int64_t)t * a.o_sn + d, x, total);
    }
  });
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

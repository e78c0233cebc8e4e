// Attention of a batch whose sequences share pages, by the plan of share.hip: the common keys once for all rows of a group, each sequence's own keys for itself, and
// a second launch that joins the parts.
#include <algorithm>

#include "few_rows.hpp"
#include "page_rows.hpp"
#include "share.hpp"

namespace ficoco {
namespace {

// Row r of an item's owner: the sequence, the query and the head of the group that it is of, where it stands and whether it counts.
struct OwnerRow { int b, t, g, pos; bool live; };
__device__ __forceinline__ OwnerRow owner_row(const ShareArgs& s, const ShareOwner& it, int r) {
  OwnerRow x{it.owner, 0, 0, it.lo, true};
  int queries = 0x7fffffff;
  if (it.owner < -1) {
    const int m = s.by_rows.of(r);
    const ShareMember member = ((const ShareMember*)(s.plan + s.members))[-2 - it.owner + m];
    r -= m * (int)s.by_rows.d;
    x.b = member.b;
    x.pos = member.first;
    queries = member.queries;
  }
  x.t = s.a.by_group.of(r);
  x.g = r - x.t * s.a.group;
  x.pos += x.t;
  x.live = x.t < queries;
  return x;
}
__device__ __forceinline__ const bf16_t* query_at(const AttendArgs& a, const OwnerRow& x, int h) {
  return a.Q + (int64_t)x.b * a.q_sb + (int64_t)(h * a.group + x.g) * a.q_sh + (int64_t)x.t * a.q_sn;
}
__device__ __forceinline__ bf16_t* result_at(const AttendArgs& a, const OwnerRow& x, int h) {
  return a.O + (int64_t)x.b * a.o_sb + (int64_t)(h * a.group + x.g) * a.o_sh + (int64_t)x.t * a.o_sn;
}
__device__ __forceinline__ RowSight sight_of_row(const AttendArgs& a, const OwnerRow& x, int keys) {
  RowSight sight(a, x.pos, keys);
  if (!x.live) {
    sight.lo = 0x7fffffff;
    sight.first = 0;
    sight.span = 0;
  }
  return sight;
}

// Blocks of 64 keys as steps of 32.
struct HalfBlocks : Blocks<kTileKeys> {
  __device__ __forceinline__ explicit HalfBlocks(const Blocks<kTileKeys>& b) : Blocks<kTileKeys>(b) {}
  __device__ __forceinline__ int block(int i) const { return 2 * Blocks<kTileKeys>::block(i >> 1) + (i & 1); }
};

// The LDS of few_rows() inside that of page_rows(): 16 rows of a wavefront fill one of its arrays, each row turned by eight features a row, so that the rows of one feature
// lie on different banks.
template <int D>
struct FewInPages {
  float *top, *sum;
  __device__ __forceinline__ float* at(int w, int row, int feature) const {
    float* o = (float*)(w < 2 ? w == 0 ? PageLds<D>::template array<0>() : PageLds<D>::template array<1>() : w == 2 ? PageLds<D>::template array<2>() : PageLds<D>::template array<3>());
    return o + row * D + ((feature + 8 * row) & (D - 1));
  }
};

// The work of one item: 16 rows straight from memory (few_rows()) or 128 (page_rows()).
template <int D, bool FEW>
__device__ __forceinline__ void share_tile(const ShareArgs& s, const ShareItem& it, int tid, int h) {
  constexpr int TILE = FEW ? kFewRows : kTileRows;
  const AttendArgs& a = s.a;
  const ShareOwner& o = it.o;
  const int row0 = it.tile * TILE, rows = o.rows - row0 < TILE ? o.rows - row0 : TILE;
  auto pos_of = [&](int r) { return o.lo + a.by_group.of(r < o.rows ? r : o.rows - 1); };
  // (pieces of a tile have to be pieces of the same blocks as those of the others: of all that the owner sees)
  const bool narrow = o.owner >= 0 && !o.cut;
  const int lo = narrow ? pos_of(row0) : o.lo, hi = narrow ? pos_of(row0 + rows - 1) : o.hi;
  const Blocks<kTileKeys> blocks(a, o.keys, lo, hi, o.from);
  const int i0 = it.i0, i1 = it.i1 < blocks.count ? it.i1 : blocks.count;
  const int32_t* table = a.table + (int64_t)o.slot * a.max_pages;
  const int64_t part = (int64_t)it.part * a.H_kv + (int64_t)h * o.part_rows;
  const bool parts = it.part >= 0;
  if constexpr (FEW) {
    float* ms = (float*)PageLds<D>::meta();
    FewInPages<D> lds{ms, ms + kFewWaves * kFewRows};
    const int c16 = tid % kFewRows;
    const OwnerRow mine = owner_row(s, o, row0 + (c16 < rows ? c16 : rows - 1));
    few_rows<D>(a, tid, lds, h, query_at(a, mine, h), sight_of_row(a, mine, o.keys), rows, lo, hi, o.keys, table, HalfBlocks(blocks), 2 * i0, 2 * i1,
                [&](int r, int d, const float (&x)[8], float m, float total) {
      if (parts) {
        if (d == 0) a.part_ms[part + r] = float2{m, total};
        __builtin_memcpy(a.part_o + (part + r) * D + d, x, 32);
      } else {
        put_row(result_at(a, owner_row(s, o, row0 + r), h) + d, x, total);
      }
    });
  } else {
    const int first = 32 * __builtin_amdgcn_readfirstlane(tid / kWave), mine_at = first + tid % 32;
    auto row_of = [&] {
      const OwnerRow mine = owner_row(s, o, row0 + (mine_at < rows ? mine_at : rows - 1));
      return TileRow{query_at(a, mine, h), sight_of_row(a, mine, o.keys)};
    };
    page_rows<D>(a, tid, h, row_of, narrow ? pos_of(row0 + first) : lo, narrow ? pos_of(row0 + first + 31) : hi, o.keys, table, blocks, i0, i1, parts,
                 mine_at < rows ? a.part_ms + part + mine_at : nullptr,
                 [&](int row, int piece) -> void* { return first + row < rows ? a.part_o + (part + first + row) * D + 4 * piece : nullptr; },
                 [&](int row, int piece) -> void* { return first + row < rows ? result_at(a, owner_row(s, o, row0 + first + row), h) + 8 * piece : nullptr; });
  }
}

// Bound by what few_rows() and page_rows() are bound by, common keys counted once for a group.  Heads of 128:
//   8 answers behind 675 tokens, 32 heads          8.8 .. 10.3 us (9 MB) a launch, three trips to memory and the blocks of a workgroup
//   64 answers behind 16384, 32 heads on 8          39 us    (17.4 GFLOP of products for the common keys, 13 MB of own keys) tiles of 128 rows, two a compute unit: 11 blocks 24 to 32 us, 3 blocks 12 to 17, so
//                                                            7 us to begin and end and 1.65 a block; then the own keys of the last sequences
//   16 questions of 48 behind 9000, 32 heads on 8  143 .. 154 us (113 GFLOP, 0.74 to 0.79 PFLOP/s) vector instructions beside the products, as page_rows(): 54 blocks 95 to 136 us
// and 48 sequences, 5 prompts of up to 24000, 28 heads of 64 on 4 31 us (82 MB, 2.6 TB/s).  (36 to 48 scalars go over lanes of a vector register, since both kinds of tile are in one kernel; none over memory.)  Either kind of tile is in one launch, so that the one fills the places that the other leaves: a launch for each took 108 us instead of 102 for the last of these calls, 226 instead of 212 for the one before.
template <int D>
__global__ __launch_bounds__(kTileThreads, 2) void share_rows_kernel(ShareArgs s) {
  static_assert(kTileThreads == kFewWaves * kWave && kFewKeys * 2 == kTileKeys, "either kind of tile");
  const int wg = s.a.by_heads.of(blockIdx.x), h = blockIdx.x - wg * s.a.H_kv;
  const ShareItem* items = (const ShareItem*)(s.plan + s.items_at);
  int next = wg < s.pieces ? wg : wg + s.pieces;
  const uint64_t mark = ((const ShareHead*)s.plan)->mark;
  const int owner = items[next].o.owner;                             // (on its way with the mark)
  if (mark != s.mark || owner == -1) return;                         // (another mark: a plan for something else, of which nothing means anything)
  do {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));                                    // (or what follows from it is kept over the loop, in more registers than there are)
    const ShareItem it = items[next];
    if (it.o.few) share_tile<D, true>(s, it, tid, h);
    else share_tile<D, false>(s, it, tid, h);
    next = it.next;
    __syncthreads();                                                 // LDS is free again
  } while (next >= 0);
}

// The parts of row `r` of an owner: the first, and how many, one after the other `step` rows apart.
struct PartsOf { int64_t first, step; int count; };
__device__ __forceinline__ PartsOf parts_of(const ShareParts& p, int r, int h, int heads, int unit) {
  const int tile = p.tile == 16 ? r / 16 : r / kTileRows;
  int count = p.pieces > 0 ? 1 : 0;
  if (p.cut) {                                             // (quotients of whole numbers below 2^53: exact)
    const double at = p.at + (double)tile * p.stride, per = (double)unit;
    count = (int)((at + (p.blocks - 1)) / per) - (int)(at / per) + 1;
  }
  const int64_t step = (int64_t)p.rows * heads;
  return PartsOf{((int64_t)p.part + (int64_t)tile * p.pieces * p.rows) * heads + (int64_t)h * p.rows + (r - tile * p.tile), step, count};
}

// Rows that have parts: those of their own keys and of their group's, relative to their largest maximum, eight at a time; D / 4 lanes a row and group of parts, the
// groups' sums meet in LDS (as join_rows_kernel).
//
// Bound by memory and latency: 64 sequences, 32 heads of 128 8 us, 16 questions of 48 queries 14 us (the parts once, 3.6 and 4.5 TB/s); 8 sequences 4 us, a launch and three trips.
template <int D, int GROUPS>
__global__ __launch_bounds__(kFewWaves * kWave) void share_join_kernel(ShareArgs s) {
  constexpr int L = D / 4, AT_ONCE = 8;
  __shared__ f32x4_t sums[GROUPS > 1 ? kFewWaves * kWave : 1];
  __shared__ float2 tops[GROUPS > 1 ? kFewWaves * kWave / L : 1];
  const AttendArgs& a = s.a;
  if (((const ShareHead*)s.plan)->mark != s.mark) return;
  const int R = (int)s.by_rows.d, piece = threadIdx.x % L, group = threadIdx.x / L % GROUPS;
  const int64_t at = (int64_t)blockIdx.x * (kFewWaves * kWave / (L * GROUPS)) + threadIdx.x / (L * GROUPS);
  const bool there = at < (int64_t)R * a.B * a.H_kv;
  const int bh = there ? s.by_rows.of((int)at) : 0, r = there ? (int)at - bh * R : 0, b = a.by_heads.of(bh), h = bh - b * a.H_kv;
  const int t = a.by_group.of(r);
  const ShareEntry& e = ((const ShareEntry*)(s.plan + s.entries))[b];
  const bool wanted = there && !e.direct && t < e.queries;
  const int unit = ((const ShareHead*)s.plan)->unit;
  const PartsOf own = parts_of(e.own, r, h, a.H_kv, unit), common = parts_of(e.group, e.row0 + r, h, a.H_kv, unit);
  const int parts = own.count + common.count;
  float m = kNoLogit, total = 0.0f;
  f32x4_t x = {0, 0, 0, 0};
  for (int i = group * AT_ONCE; wanted && i < parts; i += GROUPS * AT_ONCE) {
    float2 ms[AT_ONCE];
    f32x4_t v[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      ms[k] = float2{kNoLogit, 0.0f};
      v[k] = f32x4_t{0, 0, 0, 0};
      const int j = i + k;
      if (j < parts) {
        const int64_t p = j < own.count ? own.first + j * own.step : common.first + (j - own.count) * common.step;
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
void launch_join(const ShareArgs& s, hipStream_t stream) {
  constexpr int per = kFewWaves * kWave / (D / 4 * GROUPS);
  const dim3 grid((unsigned)(((int64_t)s.a.B * s.a.H_kv * s.by_rows.d + per - 1) / per));
  hipLaunchKernelGGL((share_join_kernel<D, GROUPS>), grid, dim3(kFewWaves * kWave), 0, stream, s);
}

template <int D>
void launch_rows(const ShareArgs& s, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)(s.items - s.pieces) * s.a.H_kv));
  hipLaunchKernelGGL(share_rows_kernel<D>, grid, dim3(kTileThreads), 0, stream, s);
  // Groups of lanes a row: as many as take the parts of a tile at once, if all rows were of one group, and as fill the chip.  Rows and join, 16 rows of 60000 tokens by 8 groups 18.4 us, by 4 22.0, by 1 44; 64 of them
  // 32.1, 32.9 and 39.1; 960 of 9000 by 8 28.4, by 4 27.8, by 2 27.6; 2048 of 16384 52.6, 50.7 and 50.6, by 1 51.4; 6400 of 3000 67.0, 62.0, 59.1 and 57.4.
  const int64_t rows = (int64_t)s.a.B * s.by_rows.d, tiles = std::max<int64_t>(1, rows / kTileRows), threads = rows * s.a.H_kv * (D / 4);
  int groups = 1;
  while (groups < 8 && s.pieces / tiles > 8 * groups && 2 * groups * threads <= 1 << 17) groups *= 2;
  switch (groups) {
    case 8: launch_join<D, 8>(s, stream); break;
    case 4: launch_join<D, 4>(s, stream); break;
    case 2: launch_join<D, 2>(s, stream); break;
    default: launch_join<D, 1>(s, stream); break;
  }
}

}  // namespace

void launch_share_rows(const ShareArgs& s, int d_head, hipStream_t stream) {
  if (d_head == 128) launch_rows<128>(s, stream); else launch_rows<64>(s, stream);
}

}  // namespace ficoco

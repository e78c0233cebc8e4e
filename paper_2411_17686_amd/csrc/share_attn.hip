// Attention of a batch whose sequences share pages, by the plan of share.hip: the common keys once for all rows of a group, each sequence's own keys for itself, and
// a second launch that joins the parts.
#include <algorithm>

#include "few_rows.hpp"
#include "page_rows.hpp"
#include "share.hpp"

namespace ficoco {
namespace {

// What one workgroup does: its item, or nothing.
__device__ __forceinline__ bool item_of(const ShareArgs& s, bool few, ShareItem& it, int& h) {
  const int i = s.a.by_heads.of(blockIdx.x);
  h = blockIdx.x - i * s.a.H_kv;
  if (((const ShareHead*)s.plan)->mark != s.mark) return false;      // (a plan for something else: nothing of it means anything)
  it = ((const ShareItem*)(s.plan + s.items_at))[i];
  return it.owner != -1 && (it.few != 0) == few;
}
// Row r of an item's owner: the sequence, the query and the head of the group that it is of, where it stands and whether it counts.
struct OwnerRow { int b, t, g, pos; bool live; };
__device__ __forceinline__ OwnerRow owner_row(const ShareArgs& s, const ShareItem& it, int r) {
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

template <int D>
__global__ __launch_bounds__(kFewWaves * kWave, 2) void share_few_kernel(ShareArgs s) {
  __shared__ FewLds<D> lds;
  ShareItem it;
  int h;
  if (!item_of(s, true, it, h)) return;
  const AttendArgs& a = s.a;
  const bool own = it.owner >= 0;
  const int row0 = it.tile * kFewRows, rows = it.rows - row0 < kFewRows ? it.rows - row0 : kFewRows;
  const int lo = own ? it.lo + a.by_group.of(row0) : it.lo, hi = own ? it.lo + a.by_group.of(row0 + rows - 1) : it.hi;
  const Blocks<kFewKeys> blocks(a, it.keys, lo, hi, it.from);
  int per = (blocks.count + it.pieces - 1) / it.pieces;
  per = (per + kFewWaves - 1) / kFewWaves * kFewWaves;
  const int begin = it.piece * per, end = begin + per < blocks.count ? begin + per : blocks.count;
  const int c16 = threadIdx.x % kFewRows;
  const OwnerRow mine = owner_row(s, it, row0 + (c16 < rows ? c16 : rows - 1));
  few_rows<D>(a, lds, h, query_at(a, mine, h), sight_of_row(a, mine, it.keys), rows, lo, hi, it.keys, a.table + (int64_t)it.slot * a.max_pages, blocks, begin, end,
              [&](int r, int d, const float (&x)[8], float m, float total) {
    if (it.part >= 0) {
      const int64_t at = (int64_t)it.part * a.H_kv + (int64_t)h * it.part_rows + r;
      if (d == 0) a.part_ms[at] = float2{m, total};
      __builtin_memcpy(a.part_o + at * D + d, x, 32);
    } else {
      put_row(result_at(a, owner_row(s, it, row0 + r), h) + d, x, total);
    }
  });
}

template <int D>
__global__ __launch_bounds__(kTileThreads, 2) void share_tile_kernel(ShareArgs s) {
  ShareItem it;
  int h;
  if (!item_of(s, false, it, h)) return;
  const AttendArgs& a = s.a;
  const bool own = it.owner >= 0;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), c32 = threadIdx.x % 32;
  const int row0 = it.tile * kTileRows, first_row = row0 + 32 * wv, rows = it.rows;
  auto pos_of = [&](int r) { return it.lo + a.by_group.of(r < rows ? r : rows - 1); };
  const Blocks<kTileKeys> blocks(a, it.keys, own ? pos_of(row0) : it.lo, own ? pos_of(row0 + kTileRows - 1) : it.hi, it.from);
  const int per = (blocks.count + it.pieces - 1) / it.pieces;
  const int begin = it.piece * per, end = begin + per < blocks.count ? begin + per : blocks.count;
  const int r = first_row + c32;
  const OwnerRow mine = owner_row(s, it, r < rows ? r : rows - 1);
  const int64_t at = (int64_t)it.part * a.H_kv + (int64_t)h * it.part_rows + 32 * wv;
  page_rows<D>(a, h, query_at(a, mine, h), sight_of_row(a, mine, it.keys), own ? pos_of(first_row) : it.lo, own ? pos_of(first_row + 31) : it.hi, it.keys,
               a.table + (int64_t)it.slot * a.max_pages, blocks, begin, end, it.part >= 0, r < rows ? a.part_ms + at + c32 : nullptr,
               [&](int row, int piece) -> void* { return first_row + row < rows ? a.part_o + (at + row) * D + 4 * piece : nullptr; },
               [&](int row, int piece) -> void* { return first_row + row < rows ? result_at(a, owner_row(s, it, first_row + row), h) + 8 * piece : nullptr; });
}

// Rows that have parts: those of their own keys and of their group's, relative to their largest maximum, eight at a time; D / 4 lanes a row and group of parts, the
// groups' sums meet in LDS (as join_rows_kernel).
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
  const ShareEntry e = ((const ShareEntry*)(s.plan + s.entries))[b];
  const bool wanted = there && !e.direct && t < e.queries;
  const int own_tile = e.own_tile == 16 ? r / 16 : r / kTileRows, shared_row = e.row0 + r, group_tile = e.group_tile == 16 ? shared_row / 16 : shared_row / kTileRows;
  const int64_t own0 = ((int64_t)e.own_part + (int64_t)own_tile * e.own_pieces * e.own_rows) * a.H_kv + (int64_t)h * e.own_rows + (r - own_tile * e.own_tile);
  const int64_t group0 = ((int64_t)e.group_part + (int64_t)group_tile * e.group_pieces * e.group_rows) * a.H_kv + (int64_t)h * e.group_rows + (shared_row - group_tile * e.group_tile);
  const int parts = e.own_pieces + e.group_pieces;
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
        const int64_t p = j < e.own_pieces ? own0 + (int64_t)j * e.own_rows * a.H_kv : group0 + (int64_t)(j - e.own_pieces) * e.group_rows * a.H_kv;
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
  const dim3 grid((unsigned)((int64_t)s.items * s.a.H_kv));
  hipLaunchKernelGGL(share_tile_kernel<D>, grid, dim3(kTileThreads), 0, stream, s);
  hipLaunchKernelGGL(share_few_kernel<D>, grid, dim3(kFewWaves * kWave), 0, stream, s);
  if (s.pieces > 8) launch_join<D, 8>(s, stream); else launch_join<D, 1>(s, stream);
}

}  // namespace

void launch_share_rows(const ShareArgs& s, int d_head, hipStream_t stream) {
  if (d_head == 128) launch_rows<128>(s, stream); else launch_rows<64>(s, stream);
}

}  // namespace ficoco

// The plan of a batch whose sequences share pages: which keys a group has in common, and how all keys are cut over workgroups.
#include <algorithm>

#include "share.hpp"

namespace ficoco {
namespace {

// Blocks of a workgroup: 4 at least (8 answers behind 675 tokens, plan and four layers: 61 us, by 2 59 to 65, by 8 71 to 73; 64 behind 16384 99 to 101 by either).  Workgroups that all heads share: two a compute unit
// (64 answers behind 16384 tokens, plan and two layers: 101 us, by 384 108, by 768 113, by 1024 125; 16 questions behind 9000 153, by 384 169).
constexpr int kLeastBlocks = 4;
constexpr int kMostPieces = 512;
// Tiles of a group have 16 rows where 3 (tiles of 16) - 8 (tiles of 128), times its blocks, times the heads, is below this: three of the former take about as long for a block as one of the latter,
// which take 4 us more to begin and end.  64 rows of 8 heads of 128: behind 512 common tokens 10.9 us and 15.2, 2048 13.6 and 16.7, 8192 20.9 and 21.6, 16384 28.0 and 28.4; of 32 heads
// behind 2048 40.1 and 39.0, 8192 57.8 and 52.5; 32 rows 19.7 and 26 behind 16384; 112 rows of 4 heads of 64 behind 4096 11.7 and 13.9.
constexpr long long kFewWork = 2100;

// Sums over the threads before this one, and over all, of which the first `waves` wavefronts have any.  Whole numbers below 2^53.
struct Sums { double blocks; int cut, whole, parts, members; };
__device__ __forceinline__ Sums add(const Sums& x, const Sums& y) { return Sums{x.blocks + y.blocks, x.cut + y.cut, x.whole + y.whole, x.parts + y.parts, x.members + y.members}; }
template <int CTRL>
__device__ __forceinline__ double plus_shifted(double x) {
  return x + __hiloint2double(dpp_move_or_zero<CTRL>(__double2hiint(x)), dpp_move_or_zero<CTRL>(__double2loint(x)));
}
__device__ __forceinline__ double scan_inclusive(double v) {      // (as wave_scan_inclusive())
  v = plus_shifted<0x118>(plus_shifted<0x114>(plus_shifted<0x112>(plus_shifted<0x111>(v))));
  const double r0 = lane_value(v, 15), r1 = lane_value(v, 31), r2 = lane_value(v, 47);
  const int row = (int)(threadIdx.x % kWave) / 16;
  return v + (row >= 1 ? r0 : 0.0) + (row >= 2 ? r1 : 0.0) + (row >= 3 ? r2 : 0.0);
}
__device__ __forceinline__ Sums sums_before(const Sums& mine, Sums* scratch, int waves, Sums& all) {
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Sums x{0, 0, 0, 0, 0};
  if (wv < waves) x = Sums{scan_inclusive(mine.blocks), wave_scan_inclusive(mine.cut), wave_scan_inclusive(mine.whole), wave_scan_inclusive(mine.parts), wave_scan_inclusive(mine.members)};
  if (threadIdx.x % kWave == kWave - 1) scratch[wv] = x;
  __syncthreads();
  Sums before{0, 0, 0, 0, 0};
  all = before;
#pragma unroll 2
  for (int w = 0; w < waves; ++w) {
    if (w < wv) before = add(before, scratch[w]);
    all = add(all, scratch[w]);
  }
  before = add(before, x);
  return Sums{before.blocks - mine.blocks, before.cut - mine.cut, before.whole - mine.whole, before.parts - mine.parts, before.members - mine.members};
}

// Sums over all threads.
struct Six { double x, y, z, w; int u, v; };
__device__ __forceinline__ Six sum_of(Six p, Six* scratch, int waves) {
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (wv < waves) {
    auto plus = [](auto a, auto b) { return a + b; };
    p = Six{wave_reduce(p.x, plus), wave_reduce(p.y, plus), wave_reduce(p.z, plus), wave_reduce(p.w, plus), wave_reduce(p.u, plus), wave_reduce(p.v, plus)};
    if (threadIdx.x % kWave == 0) scratch[wv] = p;
  }
  __syncthreads();
  p = scratch[0];
#pragma unroll 2
  for (int w = 1; w < waves; ++w) p = Six{p.x + scratch[w].x, p.y + scratch[w].y, p.z + scratch[w].z, p.w + scratch[w].w, p.u + scratch[w].u, p.v + scratch[w].v};
  return p;
}

// What workgroups take, in sixteenths of a microsecond of one of two places of a compute unit (measured with heads of 128; of 64 as much for a sequence's own 16 rows, half of it for the others): a block of 64 keys for 16 rows
// of a sequence 13, of a group 18, for 128 rows 34; to begin and end 72, or 144.  From these the time of a call: what all workgroups take over all places, or the longest of them and the beginnings of those that have to wait for a place, and the join, which reads and writes
// the parts at 3 TB/s and takes 1.5 us to begin.  It decides whether the common keys of the groups are worth it, against this attention without them: 64 sequences, 32 heads on 8 of 128, behind 512 common tokens 15.6 us without,
// 17.7 with them; behind 1024 20.6 and 16.4 (where the rule still does without), 4096 53.2 and 22.8; 8 behind 512 10.1 and 10.4, 4096 16.6 and 13.2; 16 questions of 48 tokens behind 512 37.8 and 41.2, 9000 162 and 138.
// (ficoco_cache_attention, which needs no plan, launches what has work and joins only what is cut, in the same order: 12.3, 18.0, 52.5; 8.8, 14.2; 35.9, 159.  The rule does not know of it.)
struct Costs {
  int own, common, start;
  __device__ __forceinline__ Costs(const ShareArgs& s, bool few) : own(few ? 13 : 34), common(few ? 18 : 34), start(few ? 72 : 144) {
    if (s.d_head == 64) {
      common /= 2;
      own = few ? own : common;
    }
  }
  __device__ __forceinline__ float time(const ShareArgs& s, double work, double blocks, int tiles, int part_rows) const {
    const float each = (float)work / (float)s.pieces, unit = fmaxf((float)kLeastBlocks, (float)blocks / (float)s.pieces), longest = (float)start + (float)own * unit + 72.0f * (ceilf((float)tiles / (float)s.pieces) - 1.0f);
    const float parts = fminf((float)s.pieces, (float)blocks / (float)kLeastBlocks) * (float)part_rows + (float)s.a.B * (float)(s.a.n_q * s.a.group);
    return fmaxf(each, longest) + 24.0f + parts * (float)s.a.H_kv * (float)(4 * s.d_head + 8) * (16.0f / 3e6f);
  }
};

// The whole part of x / y, whole numbers, 0 <= x < 2^53: the quotient of the doubles lies on the same side of every whole number as the exact one (a division of 64-bit integers takes ten times
// as long).  It has to fit in an int.
__device__ __forceinline__ int quotient(double x, int y) { return (int)(x / (double)y); }

// The last of n ascending numbers that is not above x.
template <typename T>
__device__ __forceinline__ int last_below(const T* at, int n, T x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (at[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// One workgroup, a thread a sequence.  Every number is the same in every run: groups are in the order of their first members, members in that of the call.
//
// Bound by its chain: members of groups, rows of the table (read once, 16 bytes a lane, the bytes do not count), three sums over all threads, the items.  8 answers behind 675 tokens, pages of 64, 8.6 us;
// 64 behind 16384 13; 48 in 5 groups behind 24000 at most, pages of 32, 13.5; once for all layers of a step.
template <int NT>
__global__ __launch_bounds__(NT) void share_plan_kernel(ShareArgs s) {
  __shared__ __align__(16) int group[NT];
  __shared__ int slots[NT];
  __shared__ int common[NT], lows[NT], highs[NT];          // of the group whose first member is b
  __shared__ double at_blocks[2 * NT];                     // of owner i (group 2 b, sequence 2 b + 1): blocks, and tiles, that are cut before it
  __shared__ int at_cut[2 * NT];
  __shared__ Sums scratch[NT / kWave];
  __shared__ Six sixes[2][NT / kWave];
  const AttendArgs& a = s.a;
  const int b = threadIdx.x, R = a.n_q * a.group, waves = (a.B + kWave - 1) / kWave;
  ShareEntry* entries = (ShareEntry*)(s.plan + s.entries);
  ShareMember* members = (ShareMember*)(s.plan + s.members);
  ShareOwner* owners = (ShareOwner*)(s.plan + s.owners);
  ShareItem* items = (ShareItem*)(s.plan + s.items_at);
  Sight sight{0, 0, 0};
  int slot = 0, g = -1;
  if (b < a.B) {
    const int named = a.seq ? a.seq[b] : b;
    if (s.group) g = s.group[b];
    sight = sight_of<true>(a, b, slot);
    sight.queries = sight.queries > 0 ? sight.queries : 0;
    if (sight.queries == 0 || named < 0 || named >= a.n_seqs || g < 0 || g >= a.B) g = -1;
  }
  group[b] = g;
  slots[b] = slot;
  common[b] = 0x7fffffff;
  lows[b] = 0x7fffffff;
  highs[b] = -0x7fffffff - 1;
  __syncthreads();
  // members before this one, all of them, and the first
  int rank = 0, count = 0, leader = b;
  if (g >= 0) {
    constexpr int STEP = 16;
    for (int i = (a.B - 1) / STEP * STEP; i >= 0; i -= STEP) {      // (behind the last one: -1)
      int x[STEP];
#pragma unroll
      for (int k = 0; k < STEP; k += 4) *(int4*)&x[k] = *(const int4*)&group[i + k];
#pragma unroll
      for (int k = STEP - 1; k >= 0; --k) {
        const bool same = x[k] == g;
        count += same;
        rank += same && i + k < b;
        leader = same ? i + k : leader;
      }
    }
    atomicMin(&common[leader], sight.keys >> a.page_shift);
    atomicMin(&lows[leader], sight.first);
    atomicMax(&highs[leader], sight.first + sight.queries - 1);
  }
  __syncthreads();
  group[b] = g >= 0 ? leader : -1;
  __syncthreads();
  // the pages that all members of a group hold: a wavefront a member, some at a time, against the first one's
  const int lane = threadIdx.x % kWave, wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  constexpr int WAVES = NT / kWave, AT_ONCE = 4;
  for (int e0 = wv; e0 < a.B; e0 += AT_ONCE * WAVES) {
    int first[AT_ONCE], till[AT_ONCE], most = 0;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const int e = e0 + k * WAVES;
      first[k] = e < a.B ? group[e] : -1;
      if (first[k] == e || (first[k] >= 0 && slots[first[k]] == slots[e])) first[k] = -1;
      till[k] = first[k] >= 0 ? common[first[k]] : 0;      // (what others have found meanwhile may be less, and then decides)
      most = till[k] > most ? till[k] : most;
    }
    for (int i0 = 0; i0 < most; i0 += 8 * kWave) {         // eight pages a lane
      int x[AT_ONCE][8], y[AT_ONCE][8], differ[AT_ONCE];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        const int32_t* p = a.table + (first[k] >= 0 ? (int64_t)slots[first[k]] * a.max_pages : 0);
        const int32_t* q = a.table + (first[k] >= 0 ? (int64_t)slots[e0 + k * WAVES] * a.max_pages : 0);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int i = i0 + 4 * (j * kWave + lane);
          if (i < till[k] && i + 4 <= a.max_pages) {       // (what lies behind `till` in them does not count)
            __builtin_memcpy(&x[k][4 * j], p + i, 16);
            __builtin_memcpy(&y[k][4 * j], q + i, 16);
          } else if (i < till[k]) {
#pragma unroll
            for (int m = 0; m < 4; ++m) {
              x[k][4 * j + m] = i + m < till[k] ? p[i + m] : 0;
              y[k][4 * j + m] = i + m < till[k] ? q[i + m] : 0;
            }
          }
        }
      }
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        differ[k] = 0x7fffffff;
#pragma unroll
        for (int j = 7; j >= 0; --j) {
          const int i = i0 + 4 * (j / 4 * kWave + lane) + j % 4;
          differ[k] = i < till[k] && x[k][j] != y[k][j] ? i : differ[k];
        }
      }
      most = 0;
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        if (__any(differ[k] != 0x7fffffff)) {
          const int at = wave_reduce(differ[k], [](int u, int v) { return u < v ? u : v; });
          if (lane == 0) atomicMin(&common[first[k]], at);
          till[k] = 0;
        }
        most = till[k] > most ? till[k] : most;
      }
    }
  }
  __syncthreads();
  const int held = g >= 0 && count > 1 ? (int)(((int64_t)common[leader] << a.page_shift) & ~(int64_t)(kShareAlign - 1)) : 0;
  const int low = g >= 0 ? lows[leader] : 0, high = g >= 0 ? highs[leader] : 0;
  ShareOwner own{}, all{};
  own.owner = b; own.slot = all.slot = slot;
  own.keys = sight.keys;
  own.lo = sight.first; own.hi = sight.first + sight.queries - 1;
  own.rows = sight.queries * a.group; own.few = s.own_tile == 16;
  own.tiles = s.own_tile == 16 ? (own.rows + 15) / 16 : (own.rows + kTileRows - 1) / kTileRows;
  own.part_rows = R < s.own_tile ? R : s.own_tile;
  // Tiles of 16 or of 128 rows (kFewWork).
  const int group_rows = count * R, small = (group_rows + 15) / 16, large = (group_rows + kTileRows - 1) / kTileRows;      // (the host has seen to 32 bits)
  const int common_blocks = held > 0 ? Blocks<kTileKeys>(a, held, low, high).count : 0, more = 3 * small - 8 * large;
  const int group_tile = more <= 0 || (long long)more * common_blocks * a.H_kv < kFewWork ? 16 : kTileRows;
  if (held > 0 && leader == b) {
    all.lo = low; all.hi = high;
    all.rows = group_rows; all.few = group_tile == 16;
    all.tiles = all.few ? small : large;
    all.blocks = common_blocks;
  }
  all.part_rows = group_rows < group_tile ? group_rows : group_tile;
  // Whether the common keys are worth workgroups of their own.
  const int blocks_alone = own.tiles ? Blocks<kTileKeys>(a, own.keys, own.lo, own.hi).count : 0;
  const int blocks_beside = own.tiles ? Blocks<kTileKeys>(a, own.keys, own.lo, own.hi, held).count : 0;
  const Costs cost(s, own.few), group_cost(s, all.few);
  const double t = own.tiles, tg = all.tiles;
  auto takes = [](int each, int blocks, int start) { return (double)each * (double)blocks + (double)start; };
  const Six work = sum_of(Six{t * takes(cost.own, blocks_alone, cost.start), t * takes(cost.own, blocks_beside, cost.start) + tg * takes(group_cost.common, all.blocks, group_cost.start),
                              t * (double)blocks_alone, t * (double)blocks_beside + tg * (double)all.blocks, own.tiles, own.tiles + all.tiles}, sixes[0], waves);
  const bool tiles = __syncthreads_or(tg > 0 && !all.few), some = __syncthreads_or(tg > 0);
  const float alone = cost.time(s, work.x, work.z, work.u, own.part_rows), together = Costs(s, !tiles).time(s, work.y, work.w, work.v, tiles ? kTileRows : 16);
  const bool worth = some && (s.always || together < alone);
  const int from = worth ? held : 0;
  const bool shared = from > 0, leads = shared && leader == b;
  own.from = from;
  own.blocks = shared ? blocks_beside : blocks_alone;
  if (leads) all.keys = from;
  else all.tiles = all.blocks = 0;
  const double each = ((worth ? work.w : work.z) + (double)(s.pieces - 1)) / (double)s.pieces;
  int unit = (int)fmin(fmax(each, (double)kLeastBlocks), (double)0x3fffffff);
  // Whether every tile can begin with a workgroup of its own, if these take a little more each: a workgroup that begins a second tile takes as long as 5 blocks, or an eighth of them, more.
  const int larger = unit + (unit / 8 > 5 ? unit / 8 : 5);
  auto whole_pieces = [](const ShareOwner& o, int u) { return o.blocks > u ? (double)o.tiles * (double)((o.blocks + u - 1) / u) : 0.0; };
  const Six need = sum_of(Six{whole_pieces(all, unit) + whole_pieces(own, unit), whole_pieces(all, larger) + whole_pieces(own, larger), 0, 0, 0, 0}, sixes[1], waves);
  const bool apart = need.x <= (double)s.pieces || need.y <= (double)s.pieces;
  if (need.x > (double)s.pieces && apart) unit = larger;
  auto cut_up = [&](ShareOwner& o) {
    o.cut = o.blocks > unit;
    o.part_pieces = o.cut ? o.blocks / unit + 2 : 1;
    o.stride = apart ? (o.blocks + unit - 1) / unit * unit : o.blocks;
  };
  cut_up(own);
  cut_up(all);
  const bool direct = !shared && !own.cut;
  const double blocks_all = all.cut ? (double)all.stride * (double)all.tiles : 0.0, blocks_own = own.cut ? (double)own.stride * (double)own.tiles : 0.0;
  const int parts_all = all.tiles * all.part_pieces * all.part_rows, parts_own = direct ? 0 : own.tiles * own.part_pieces * own.part_rows;
  Sums sum;
  const Sums before = sums_before(Sums{blocks_all + blocks_own, (all.cut ? all.tiles : 0) + (own.cut ? own.tiles : 0), (all.cut ? 0 : all.tiles) + (own.cut ? 0 : own.tiles), parts_all + parts_own,
                                           leads ? count : 0}, scratch, waves, sum);
  all.owner = -2 - before.members;
  all.part = before.parts;
  own.part = direct ? -1 : before.parts + parts_all;
  at_blocks[2 * b] = before.blocks;
  at_blocks[2 * b + 1] = before.blocks + blocks_all;
  at_cut[2 * b] = before.cut;
  at_cut[2 * b + 1] = before.cut + (all.cut ? all.tiles : 0);
  if (b < a.B) {
    owners[2 * b] = all;
    owners[2 * b + 1] = own;
    int at = 2 * s.pieces + before.whole;
    auto whole = [&](const ShareOwner& o) {
      for (int t = 0; !o.cut && t < o.tiles; ++t, ++at) items[at] = ShareItem{o, t, 0, 0x3fffffff, o.part < 0 ? -1 : o.part + t * o.part_rows, -1, {0, 0, 0}};
    };
    whole(all);
    whole(own);
  }
  __syncthreads();
  if (b < a.B) {
    ShareEntry e{};
    e.queries = sight.queries;
    e.direct = direct;
    e.own = ShareParts{at_blocks[2 * b + 1], own.blocks, own.part, own.part_rows, own.tiles ? own.part_pieces : 0, s.own_tile, own.cut, own.stride, 0};
    if (shared) {
      const ShareOwner o = owners[2 * leader];
      e.group = ShareParts{at_blocks[2 * leader], o.blocks, o.part, o.part_rows, o.part_pieces, group_tile, o.cut, o.stride, 0};
      e.row0 = rank * R;
      members[-2 - o.owner + rank] = ShareMember{b, sight.first, sight.queries, 0};
    }
    entries[b] = e;
  }
  // workgroups of the owners that are cut
  for (int w = b; w < s.pieces; w += NT) {
    const double at = (double)w * (double)unit;
    if (at >= sum.blocks) {
      items[w].o.owner = -1;
      continue;
    }
    const int i = last_below(at_blocks, 2 * a.B, at);
    const ShareOwner o = owners[i];
    const double in = at - at_blocks[i];
    const int tile = quotient(in, o.stride), i0 = (int)(in - (double)tile * (double)o.stride), i1 = i0 + unit < o.blocks ? i0 + unit : o.blocks;
    const int piece = w - quotient(at_blocks[i] + (double)tile * (double)o.stride, unit), after = at_cut[i] + tile + 1;
    items[w] = ShareItem{o, tile, i0, i1, o.part + (tile * o.part_pieces + piece) * o.part_rows, !apart && i1 - i0 < unit && after < sum.cut ? s.pieces + after : -1, {0, 0, 0}};
  }
  for (int c = b; !apart && c < sum.cut; c += NT) {
    const int i = last_below(at_cut, 2 * a.B, c);
    const ShareOwner o = owners[i];
    const double begins = at_blocks[i] + (double)(c - at_cut[i]) * (double)o.blocks;
    const int tile = c - at_cut[i], behind = (int)(begins - (double)quotient(begins, unit) * (double)unit);      // (a tile has more than `unit` blocks)
    if (behind != 0) items[s.pieces + c] = ShareItem{o, tile, 0, unit - behind, o.part + tile * o.part_pieces * o.part_rows, -1, {0, 0, 0}};
  }
  for (int i = 2 * s.pieces + sum.whole + b; i < s.items; i += NT) items[i].o.owner = -1;
  if (b == 0) {
    ShareHead* head = (ShareHead*)s.plan;
    head->mark = s.mark;
    head->unit = unit;
  }
}

}  // namespace

SharePlan share_plan(const ficoco_cache& c, const ficoco_attention& a) {
  SharePlan pl{};
  const int64_t heads = c.heads, R = (int64_t)a.n_q * (a.H / heads), B = a.B;
  // own rows as in attend_plan()
  const int64_t few_tiles = (R + 15) / 16;
  pl.own_tile = few_tiles <= 1 || (few_tiles <= 4 && B * heads * few_tiles <= (few_tiles <= 3 ? 1024 : 512)) ? 16 : kTileRows;
  pl.own_tiles = (int)((R + pl.own_tile - 1) / pl.own_tile);
  const int64_t room = (int64_t)c.max_pages * c.page_size, longest = a.max_len > 0 ? std::min<int64_t>(room, a.max_len) : room;
  pl.pieces = (int)std::max<int64_t>(1, std::min<int64_t>(std::max<int64_t>(1, kMostPieces / heads), B * std::max(1, pl.own_tiles) * ((longest + 255) / 256)));
  // A group has two members at least, and a last tile that is not full.
  const int64_t most_groups = B / 2, own_items = B * pl.own_tiles, group_items = B * R / 16 + most_groups;
  pl.items = (int)std::min<int64_t>(0x3fffffff, 2 * pl.pieces + own_items + group_items);
  // Rows of parts: tiles of own rows, of groups in tiles of 16, or of 128 where they have more than 32 rows; of tiles that are cut (there are less than pl.pieces, of more blocks than a
  // workgroup's), two parts more than whole workgroups.
  const int64_t own_rows = own_items * std::min<int64_t>(R, pl.own_tile), group_rows = B * R + 16 * most_groups + B * R / 32 * 128;
  const int64_t parts = (own_rows + group_rows + 3 * (int64_t)pl.pieces * kTileRows) * heads;
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  pl.entries = 256;
  pl.members = pl.entries + up((size_t)B * sizeof(ShareEntry));
  pl.owners = pl.members + up((size_t)B * sizeof(ShareMember));
  pl.items_at = pl.owners + up((size_t)B * 2 * sizeof(ShareOwner));
  pl.bytes = pl.items_at + up((size_t)pl.items * sizeof(ShareItem));
  pl.part_ms = 0;
  pl.part_o = up((size_t)parts * sizeof(float2));
  pl.ws_bytes = std::max<size_t>(256, pl.part_o + up((size_t)parts * a.d_head * sizeof(float)));
  return pl;
}

void launch_share(const ShareArgs& s, hipStream_t stream) {
  // Few wavefronts wait less for each other, many compare more members at once: 64 members behind 256 pages 13 us by 1024 threads, 15 by 512, 19 by 256; 48 behind up to 750 13.5, 16 and 19; 8 behind 10
  // 8.6 by 256, 10.6 by 512; 16 behind 140 13.6 and 15.
  if (s.a.B <= 16) hipLaunchKernelGGL(share_plan_kernel<256>, dim3(1), dim3(256), 0, stream, s);
  else hipLaunchKernelGGL(share_plan_kernel<kMaxCall>, dim3(1), dim3(kMaxCall), 0, stream, s);
}

}  // namespace ficoco

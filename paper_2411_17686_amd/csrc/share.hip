// The plan of a batch whose sequences share pages: which keys a group has in common, and how all keys are cut over workgroups.
#include <algorithm>

#include "share.hpp"

namespace ficoco {
namespace {

constexpr int kShareLeast = 2 * kShareAlign;     // common keys below which a group's members attend for themselves
constexpr int kLeastBlocks = 4;                  // blocks of a workgroup
constexpr int kMostPieces = 512;                 // workgroups for a head: two a compute unit (see attend_plan())
constexpr int kFewGroup = 64;                    // rows of a group up to which its tiles have 16

// Sums over the threads before this one, and over all.
struct Sums { long long blocks; int cut, whole, parts, members; };
__device__ __forceinline__ Sums add(const Sums& x, const Sums& y) { return Sums{x.blocks + y.blocks, x.cut + y.cut, x.whole + y.whole, x.parts + y.parts, x.members + y.members}; }
template <int NT>
__device__ __forceinline__ Sums sums_before(const Sums& mine, Sums* scratch, Sums& all) {
  const int lane = threadIdx.x % kWave, wv = threadIdx.x / kWave;
  Sums x = mine;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const Sums y{__shfl_up(x.blocks, d), __shfl_up(x.cut, d), __shfl_up(x.whole, d), __shfl_up(x.parts, d), __shfl_up(x.members, d)};
    if (lane >= d) x = add(x, y);
  }
  if (lane == kWave - 1) scratch[wv] = x;
  __syncthreads();
  Sums before{0, 0, 0, 0, 0};
  all = before;
  for (int w = 0; w < NT / kWave; ++w) {
    if (w < wv) before = add(before, scratch[w]);
    all = add(all, scratch[w]);
  }
  before = add(before, x);
  return Sums{before.blocks - mine.blocks, before.cut - mine.cut, before.whole - mine.whole, before.parts - mine.parts, before.members - mine.members};
}

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
template <int NT>
__global__ __launch_bounds__(NT) void share_plan_kernel(ShareArgs s) {
  __shared__ __align__(16) int group[NT];
  __shared__ int slots[NT];
  __shared__ int common[NT], lows[NT], highs[NT];          // of the group whose first member is b
  __shared__ long long at_blocks[2 * NT];                  // of owner i (group 2 b, sequence 2 b + 1): blocks, and tiles, that are cut before it
  __shared__ int at_cut[2 * NT];
  __shared__ Sums scratch[NT / kWave];
  __shared__ unsigned long long totals[NT / kWave], needs[2][NT / kWave];
  const AttendArgs& a = s.a;
  const int b = threadIdx.x, R = a.n_q * a.group;
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
    for (int i = (a.B - 1) / 4 * 4; i >= 0; i -= 4) {      // (behind the last one: -1)
      const int4 x = *(const int4*)&group[i];
      const int y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int k = 3; k >= 0; --k) {
        const bool same = y[k] == g;
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
  // the pages that all members of a group hold: a wavefront a member, four at a time, against the first one's
  const int lane = threadIdx.x % kWave, wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  constexpr int WAVES = NT / kWave;
  for (int e0 = wv; e0 < a.B; e0 += 4 * WAVES) {
    int first[4], till[4], most = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int e = e0 + k * WAVES;
      first[k] = e < a.B ? group[e] : -1;
      if (first[k] == e || (first[k] >= 0 && slots[first[k]] == slots[e])) first[k] = -1;
      till[k] = first[k] >= 0 ? common[first[k]] : 0;      // (what others have found meanwhile may be less, and then decides)
      most = till[k] > most ? till[k] : most;
    }
    for (int i0 = 0; i0 < most; i0 += 8 * kWave) {         // eight pages a lane
      int x[4][8], y[4][8], differ[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int32_t* p = a.table + (first[k] >= 0 ? (int64_t)slots[first[k]] * a.max_pages : 0);
        const int32_t* q = a.table + (first[k] >= 0 ? (int64_t)slots[e0 + k * WAVES] * a.max_pages : 0);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int i = i0 + 4 * (j * kWave + lane);
          if (i + 4 <= till[k]) {
            __builtin_memcpy(&x[k][4 * j], p + i, 16);
            __builtin_memcpy(&y[k][4 * j], q + i, 16);
          } else {
#pragma unroll
            for (int m = 0; m < 4; ++m) {
              x[k][4 * j + m] = i + m < till[k] ? p[i + m] : 0;
              y[k][4 * j + m] = i + m < till[k] ? q[i + m] : 0;
            }
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        differ[k] = 0x7fffffff;
#pragma unroll
        for (int j = 7; j >= 0; --j) differ[k] = x[k][j] != y[k][j] ? i0 + 4 * (j / 4 * kWave + lane) + j % 4 : differ[k];
      }
      most = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
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
  const int from = g >= 0 && count > 1 ? (int)(((int64_t)common[leader] << a.page_shift) & ~(int64_t)(kShareAlign - 1)) : 0;
  const bool shared = from >= kShareLeast, leads = shared && leader == b;
  ShareOwner own{}, all{};
  own.owner = b; own.slot = all.slot = slot;
  own.from = shared ? from : 0; own.keys = sight.keys;
  own.lo = sight.first; own.hi = sight.first + sight.queries - 1;
  own.rows = sight.queries * a.group; own.few = s.own_tile == 16;
  own.tiles = s.own_tile == 16 ? (own.rows + 15) / 16 : (own.rows + kTileRows - 1) / kTileRows;
  own.blocks = own.tiles ? Blocks<kTileKeys>(a, own.keys, own.lo, own.hi, own.from).count : 0;
  own.part_rows = R < s.own_tile ? R : s.own_tile;
  const int group_rows = count * R, group_tile = group_rows <= kFewGroup ? 16 : kTileRows;       // (the host has seen to 32 bits)
  all.part_rows = group_rows < group_tile ? group_rows : group_tile;
  if (leads) {
    all.keys = from;
    all.lo = lows[b]; all.hi = highs[b];
    all.rows = group_rows; all.few = group_tile == 16;
    all.tiles = all.few ? (group_rows + 15) / 16 : (group_rows + kTileRows - 1) / kTileRows;
    all.blocks = Blocks<kTileKeys>(a, from, all.lo, all.hi).count;
  }
  unsigned long long total = (unsigned long long)own.blocks * own.tiles + (unsigned long long)all.blocks * all.tiles;
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) total += __shfl_xor(total, d);
  if (lane == 0) totals[wv] = total;
  __syncthreads();
  total = 0;
  for (int w = 0; w < WAVES; ++w) total += totals[w];
  const unsigned long long each = (total + s.pieces - 1) / s.pieces;
  int unit = (int)(each > kLeastBlocks ? each < 0x3fffffff ? each : 0x3fffffff : kLeastBlocks);
  // Whether every tile can begin with a workgroup of its own, if these take a little more each: a workgroup that begins a second tile takes as long as 5 blocks, or an eighth of them, more.
  const int larger = unit + (unit / 8 > 5 ? unit / 8 : 5);
  auto whole_pieces = [](const ShareOwner& o, int u) { return o.blocks > u ? (unsigned long long)o.tiles * ((o.blocks + u - 1) / u) : 0ull; };
  unsigned long long need = whole_pieces(all, unit) + whole_pieces(own, unit), need_larger = whole_pieces(all, larger) + whole_pieces(own, larger);
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) {
    need += __shfl_xor(need, d);
    need_larger += __shfl_xor(need_larger, d);
  }
  if (lane == 0) {
    needs[0][wv] = need;
    needs[1][wv] = need_larger;
  }
  __syncthreads();
  need = need_larger = 0;
  for (int w = 0; w < WAVES; ++w) {
    need += needs[0][w];
    need_larger += needs[1][w];
  }
  const bool apart = need <= (unsigned)s.pieces || need_larger <= (unsigned)s.pieces;
  if (need > (unsigned)s.pieces && apart) unit = larger;
  auto cut_up = [&](ShareOwner& o) {
    o.cut = o.blocks > unit;
    o.part_pieces = o.cut ? o.blocks / unit + 2 : 1;
    o.stride = apart ? (o.blocks + unit - 1) / unit * unit : o.blocks;
  };
  cut_up(own);
  cut_up(all);
  const bool direct = !shared && !own.cut;
  const long long blocks_all = all.cut ? (long long)all.stride * all.tiles : 0, blocks_own = own.cut ? (long long)own.stride * own.tiles : 0;
  const int parts_all = all.tiles * all.part_pieces * all.part_rows, parts_own = direct ? 0 : own.tiles * own.part_pieces * own.part_rows;
  Sums sum;
  const Sums before = sums_before<NT>(Sums{blocks_all + blocks_own, (all.cut ? all.tiles : 0) + (own.cut ? own.tiles : 0), (all.cut ? 0 : all.tiles) + (own.cut ? 0 : own.tiles), parts_all + parts_own,
                                           leads ? count : 0}, scratch, sum);
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
    e.own = ShareParts{(double)at_blocks[2 * b + 1], own.blocks, own.part, own.part_rows, own.tiles ? own.part_pieces : 0, s.own_tile, own.cut, own.stride, 0};
    if (shared) {
      const ShareOwner o = owners[2 * leader];
      e.group = ShareParts{(double)at_blocks[2 * leader], o.blocks, o.part, o.part_rows, o.part_pieces, group_tile, o.cut, o.stride, 0};
      e.row0 = rank * R;
      members[-2 - o.owner + rank] = ShareMember{b, sight.first, sight.queries, sight.keys};
    }
    entries[b] = e;
  }
  // workgroups of the owners that are cut
  for (int w = b; w < s.pieces; w += NT) {
    const long long at = (long long)w * unit;
    if (at >= sum.blocks) {
      items[w].o.owner = -1;
      continue;
    }
    const int i = last_below(at_blocks, 2 * a.B, at);
    const ShareOwner o = owners[i];
    const long long in = at - at_blocks[i];
    const int tile = (int)(in / o.stride), i0 = (int)(in - (long long)tile * o.stride), i1 = i0 + unit < o.blocks ? i0 + unit : o.blocks;
    const int piece = w - (int)((at_blocks[i] + (long long)tile * o.stride) / unit), after = at_cut[i] + tile + 1;
    items[w] = ShareItem{o, tile, i0, i1, o.part + (tile * o.part_pieces + piece) * o.part_rows, !apart && i1 - i0 < unit && after < sum.cut ? s.pieces + after : -1, {0, 0, 0}};
  }
  for (int c = b; !apart && c < sum.cut; c += NT) {
    const int i = last_below(at_cut, 2 * a.B, c);
    const ShareOwner o = owners[i];
    const int tile = c - at_cut[i], behind = (int)((at_blocks[i] + (long long)tile * o.blocks) % unit);      // (a tile has more than `unit` blocks)
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
  // Rows of parts: tiles of own rows, of groups in tiles of 16 (64 rows at most) or of 128 (more than 64 rows); of tiles that are cut (there are less than pl.pieces, of more blocks than a
  // workgroup's), two parts more than whole workgroups.
  const int64_t own_rows = own_items * std::min<int64_t>(R, pl.own_tile), group_rows = B * R + 16 * most_groups + B * R / kFewGroup * 128;
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
  // As many wavefronts as compare four members each at once, at least; fewer wait less for each other.
  if (s.a.B <= 16) hipLaunchKernelGGL(share_plan_kernel<256>, dim3(1), dim3(256), 0, stream, s);
  else hipLaunchKernelGGL(share_plan_kernel<kMaxCall>, dim3(1), dim3(kMaxCall), 0, stream, s);
}

}  // namespace ficoco

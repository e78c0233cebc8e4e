// The plan of a batch whose sequences share pages: which keys a group has in common, and how all keys are cut over workgroups.
#include <algorithm>

#include "share.hpp"

namespace ficoco {
namespace {

constexpr int kPlanThreads = kMaxCall;
constexpr int kShareLeast = 2 * kShareAlign;     // common keys below which a group's members attend for themselves
constexpr int kLeastBlocks = 4;                  // blocks of 64 keys of a piece
constexpr int kMostPieces = 256;
constexpr int kFewGroup = 64;                    // rows of a group up to which its tiles have 16

// One workgroup, a thread a sequence.  Every number is the same in every run: groups are in the order of their first members, members in that of the call.
__global__ __launch_bounds__(kPlanThreads) void share_plan_kernel(ShareArgs s) {
  __shared__ int group[kMaxCall], keys[kMaxCall], slots[kMaxCall];
  __shared__ int common[kMaxCall], lows[kMaxCall], highs[kMaxCall];      // of the group whose first member is b
  __shared__ int scratch[kPlanThreads / kWave];
  __shared__ unsigned long long total;
  const AttendArgs& a = s.a;
  const int b = threadIdx.x, P = 1 << a.page_shift, R = a.n_q * a.group;
  ShareEntry* entries = (ShareEntry*)(s.plan + s.entries);
  ShareMember* members = (ShareMember*)(s.plan + s.members);
  ShareItem* items = (ShareItem*)(s.plan + s.items_at);
  Sight sight{0, 0, 0};
  int slot = 0, g = -1;
  if (b < a.B) {
    sight = sight_of<true>(a, b, slot);
    sight.queries = sight.queries > 0 ? sight.queries : 0;
    const int named = a.seq ? a.seq[b] : b;
    if (s.group && sight.queries > 0 && named >= 0 && named < a.n_seqs) g = s.group[b];
    if (g < 0 || g >= a.B) g = -1;
  }
  group[b] = g;
  keys[b] = sight.keys;
  slots[b] = slot;
  if (b == 0) total = 0;
  __syncthreads();
  // members before this one, all of them, and the first
  int rank = 0, count = 0, leader = b;
  if (g >= 0) {
    for (int i = a.B - 1; i >= 0; --i) {
      const bool same = group[i] == g;
      count += same;
      rank += same && i < b;
      leader = same ? i : leader;
    }
  }
  common[b] = 0x7fffffff;
  lows[b] = 0x7fffffff;
  highs[b] = -0x7fffffff - 1;
  __syncthreads();
  if (g >= 0) {
    atomicMin(&common[leader], sight.keys >> a.page_shift);
    atomicMin(&lows[leader], sight.first);
    atomicMax(&highs[leader], sight.first + sight.queries - 1);
    group[b] = leader;                                     // (nobody looks for equal numbers any more; -1 elsewhere)
  }
  __syncthreads();
  // the pages that all members of a group hold: a wavefront a member, against the first one's
  const int lane = threadIdx.x % kWave, wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  for (int e = wv; e < a.B; e += kPlanThreads / kWave) {
    const int first = group[e];
    if (first < 0 || first == e || slots[first] == slots[e]) continue;
    const int32_t *x = a.table + (int64_t)slots[first] * a.max_pages, *y = a.table + (int64_t)slots[e] * a.max_pages;
    for (int i0 = 0; i0 < common[first]; i0 += 4 * kWave) {
      const int till = common[first];
      int differ = 0x7fffffff;
#pragma unroll
      for (int k = 3; k >= 0; --k) {
        const int i = i0 + k * kWave + lane;
        if (i < till && x[i] != y[i]) differ = i;
      }
      const uint64_t any = __ballot(differ != 0x7fffffff);
      if (any) {
        differ = wave_reduce(differ, [](int u, int v) { return u < v ? u : v; });
        if (lane == 0) atomicMin(&common[first], differ);
        break;
      }
    }
  }
  __syncthreads();
  const int from = g >= 0 && count > 1 ? (int)(((int64_t)common[leader] << a.page_shift) & ~(int64_t)(kShareAlign - 1)) : 0;
  const bool shared = from >= kShareLeast, leads = shared && leader == b;
  // owners: a sequence with its own keys, and, with its first member, a group with the common ones
  const Blocks<kTileKeys> own(a, sight.keys, sight.first, sight.first + sight.queries - 1, shared ? from : 0);
  const int own_tiles = sight.queries > 0 ? (sight.queries * a.group + s.own_tile - 1) / s.own_tile : 0;
  int group_blocks = 0, group_tiles = 0;
  const int group_rows = count * R;                        // (the host has seen to 32 bits)
  const int group_tile = group_rows <= kFewGroup ? 16 : kTileRows;
  if (leads) {
    group_blocks = Blocks<kTileKeys>(a, from, lows[b], highs[b]).count;
    group_tiles = (group_rows + group_tile - 1) / group_tile;
  }
  atomicAdd(&total, (unsigned long long)own.count * own_tiles + (unsigned long long)group_blocks * group_tiles);
  __syncthreads();
  const unsigned long long all = (total + s.pieces - 1) / s.pieces;
  const int unit = (int)(all > kLeastBlocks ? all < 0x3fffffff ? all : 0x3fffffff : kLeastBlocks);
  auto pieces_of = [&](int blocks) {
    const int n = (blocks + unit - 1) / unit;
    return n < 1 ? 1 : n < kMostPieces ? n : kMostPieces;
  };
  const int own_pieces = own_tiles ? pieces_of(own.count) : 0, group_pieces = leads ? pieces_of(group_blocks) : 0;
  const int own_part_rows = R < s.own_tile ? R : s.own_tile, group_part_rows = group_rows < group_tile ? group_rows : group_tile;
  const bool direct = !shared && own_pieces <= 1;
  // items: the groups', then the sequences'; rows of parts in the same order
  int n_group, n_own, p_group, p_own;
  const int my_group = group_tiles * group_pieces, my_own = own_tiles * own_pieces;
  const int at_group = block_scan_inclusive(my_group, scratch, &n_group) - my_group;
  const int at_own = block_scan_inclusive(my_own, scratch, &n_own) - my_own + n_group;
  const int rows_group = my_group * group_part_rows, rows_own = direct ? 0 : my_own * own_part_rows;
  const int part_group = block_scan_inclusive(rows_group, scratch, &p_group) - rows_group;
  const int part_own = block_scan_inclusive(rows_own, scratch, &p_own) - rows_own + p_group;
  int n_members;
  const int members_at = block_scan_inclusive(leads ? count : 0, scratch, &n_members) - (leads ? count : 0);
  // (common, lows and highs of a first member have served)
  const int low = g >= 0 ? lows[leader] : 0, high = g >= 0 ? highs[leader] : 0;
  __syncthreads();
  if (leads) {
    common[b] = members_at;
    lows[b] = part_group;
    highs[b] = group_pieces;
  }
  __syncthreads();
  if (b < a.B) {
    ShareEntry e{};
    e.queries = sight.queries;
    e.direct = direct;
    e.own_part = part_own; e.own_pieces = own_pieces; e.own_rows = own_part_rows; e.own_tile = s.own_tile;
    if (shared) {
      e.group_part = lows[leader]; e.group_pieces = highs[leader]; e.group_rows = group_part_rows; e.group_tile = group_tile;
      e.row0 = rank * R;
      members[common[leader] + rank] = ShareMember{b, sight.first, sight.queries, sight.keys};
    }
    entries[b] = e;
  }
  auto put = [&](int at, int i, ShareItem x, int part) {   // item i of an owner
    x.tile = i / x.pieces;
    x.piece = i - x.tile * x.pieces;
    x.part = part < 0 ? -1 : part + i * x.part_rows;
    items[at + i] = x;
  };
  if (my_own > 0) {
    const ShareItem x{b, 0, 0, own_pieces, slot, shared ? from : 0, sight.keys, sight.first, sight.first + sight.queries - 1, sight.queries * a.group, s.own_tile == 16, 0, own_part_rows, {0, 0, 0}};
    for (int i = 0; i < my_own; ++i) put(at_own, i, x, direct ? -1 : part_own);
  }
  if (leads) {
    const ShareItem x{-2 - members_at, 0, 0, group_pieces, slot, 0, from, low, high, group_rows, group_tile == 16, 0, group_part_rows, {0, 0, 0}};
    for (int i = 0; i < my_group; ++i) put(at_group, i, x, part_group);
  }
  for (int i = n_group + n_own + b; i < s.items; i += kPlanThreads) items[i].owner = -1;
  if (b == 0) {
    ShareHead* head = (ShareHead*)s.plan;
    head->mark = s.mark;
    head->items = n_group + n_own;
  }
}

}  // namespace

SharePlan share_plan(const ficoco_cache& c, const ficoco_attention& a) {
  SharePlan pl{};
  const int64_t heads = c.heads, group = a.H / heads, R = a.n_q * group, B = a.B;
  // own rows as in attend_plan()
  const int64_t few_tiles = (R + 15) / 16;
  pl.own_tile = few_tiles <= 1 || (few_tiles <= 4 && B * heads * few_tiles <= (few_tiles <= 3 ? 1024 : 512)) ? 16 : kTileRows;
  pl.own_tiles = (int)((R + pl.own_tile - 1) / pl.own_tile);
  // Two workgroups a compute unit (see attend_plan()).
  pl.pieces = (int)std::max<int64_t>(1, 512 / heads);
  const int64_t room = (int64_t)c.max_pages * c.page_size, longest = a.max_len > 0 ? std::min<int64_t>(room, a.max_len) : room;
  pl.pieces = (int)std::max<int64_t>(1, std::min<int64_t>(pl.pieces, B * std::max(1, pl.own_tiles) * ((longest + 255) / 256)));
  // Pieces beyond one a tile are as many as pl.pieces at most; a group has two members at least, and a last tile that is not full.
  const int64_t most_groups = B / 2, own_items = B * pl.own_tiles, group_items = B * R / 16 + most_groups;
  pl.items = (int)std::min<int64_t>(0x7fffffff, pl.pieces + own_items + group_items);
  // Rows of parts: tiles of own rows, of groups in tiles of 16 (64 rows at most) or of 128 (more than 64 rows), and the pieces beyond one a tile.
  const int64_t own_rows = own_items * std::min<int64_t>(R, pl.own_tile), group_rows = B * R + 16 * most_groups + B * R / kFewGroup * 128;
  const int64_t parts = (own_rows + group_rows + (int64_t)pl.pieces * kTileRows) * heads;
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  pl.entries = 256;
  pl.members = pl.entries + up((size_t)B * sizeof(ShareEntry));
  pl.items_at = pl.members + up((size_t)B * sizeof(ShareMember));
  pl.bytes = pl.items_at + up((size_t)pl.items * sizeof(ShareItem));
  pl.part_ms = 0;
  pl.part_o = up((size_t)parts * sizeof(float2));
  pl.ws_bytes = std::max<size_t>(256, pl.part_o + up((size_t)parts * a.d_head * sizeof(float)));
  return pl;
}

void launch_share(const ShareArgs& s, hipStream_t stream) {
  hipLaunchKernelGGL(share_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, s);
}

}  // namespace ficoco

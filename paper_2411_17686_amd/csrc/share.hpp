// Attention of a batch whose sequences share pages: what the plan (share.hip), the attention (share_attn.hip) and the host share.
#pragma once
#include "attend.hpp"

namespace ficoco {

constexpr int kShareAlign = 64;              // common keys are counted in whole steps of either kind of workgroup

// One workgroup's rows and keys, for each key / value head: tile `tile` of an owner's rows (a sequence's own ones, or all of a group's), piece `piece` of `pieces` of the owner's keys from `from` on.
struct ShareItem {
  int owner;                                 // the sequence, or -2 - the group's first member record; -1: nothing to do
  int tile, piece, pieces;
  int slot;                                  // whose row of the table
  int from, keys;
  int lo, hi;                                // positions of the owner's rows
  int rows;                                  // of the owner
  int few;                                   // 16 rows, else 128
  int part;                                  // first of its rows of parts (times the key / value heads); -1: straight into the result
  int part_rows;                             // rows of parts of a tile
  int pad[3];
};
// A sequence: where the parts of its rows are, its own and its group's.
struct ShareEntry {
  int queries, direct;
  int own_part, own_pieces, own_rows, own_tile;          // first row of parts, pieces, rows of parts of a tile, rows of a tile
  int group_part, group_pieces, group_rows, group_tile;  // pieces 0: no group
  int row0;                                  // its first row among the group's
  int pad[5];
};
struct ShareMember { int b, first, queries, keys; };
struct ShareHead { uint64_t mark; int items, pad[13]; };

struct SharePlan {
  int own_tile, own_tiles, pieces, items;    // rows of a tile of own rows; tiles of a sequence; pieces that the keys are cut into, about; most items
  size_t entries, members, items_at, bytes;  // offsets and size of the plan
  size_t part_ms, part_o, ws_bytes;          // of the workspace
};
SharePlan share_plan(const ficoco_cache& c, const ficoco_attention& a);

struct ShareArgs {
  AttendArgs a;
  uint64_t mark;                             // of the shapes that the plan was made for
  char* plan;
  const int32_t* group;
  Divisor by_rows;                           // n_q * group
  int own_tile, own_tiles, pieces, items;
  size_t entries, members, items_at;
};
void launch_share(const ShareArgs& s, hipStream_t stream);
void launch_share_rows(const ShareArgs& s, int d_head, hipStream_t stream);

}  // namespace ficoco

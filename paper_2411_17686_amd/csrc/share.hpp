// Attention of a batch whose sequences share pages: what the plan (share.hip), the attention (share_attn.hip) and the host share.
#pragma once
#include "attend.hpp"

namespace ficoco {

// Common keys are counted in whole blocks of 64, the steps of a tile of 128 rows; a tile of 16 takes two steps of 32.
constexpr int kShareAlign = kTileKeys;

// An owner of rows: a sequence with its own keys, or a group with the common ones.  Its rows are cut into tiles, each of which sees all of its keys.
struct ShareOwner {
  int owner;                                 // the sequence, or -2 - the group's first member record
  int slot;                                  // whose row of the table
  int from, keys;                            // keys [from, keys)
  int lo, hi;                                // positions of the rows
  int rows, few;                             // rows; tiles of 16 of them, else of 128
  int blocks, tiles;                         // of 64 keys; of rows
  int part, part_rows, part_pieces;          // first row of parts (-1: straight into the result), rows of a tile's part, parts of a tile that there is room for
  int cut;                                   // whether its blocks are cut over workgroups (else one workgroup a tile)
  int stride;                                // blocks from the beginning of a tile to that of the next, among all that are cut
  int pad;
};
// What a workgroup does, for one key / value head: blocks [i0, i1) of one tile, then item `next`, if that is not -1.
struct ShareItem {
  ShareOwner o;                              // owner -1: nothing to do
  int tile, i0, i1, part, next, pad[3];      // part: its first row of parts
};
// A sequence: where the parts of its rows are, its own and its group's.
struct ShareParts {
  double at;                                 // where the owner's blocks begin among all that are cut
  int blocks, part, rows, pieces, tile, cut; // of the owner: part_rows, part_pieces (0: no such owner); tile: rows of one
  int stride, pad;
};
struct ShareEntry {
  ShareParts own, group;
  int queries, direct, row0, pad;            // row0: its first row among the group's
};
struct ShareMember { int b, first, queries, pad; };
struct ShareHead { uint64_t mark; int unit, pad[13]; };        // unit: blocks of a workgroup

// The blocks of all tiles of the owners that are cut, one tile after the other, go to workgroups `unit` at a time: as many as are resident at once.  They have equally many blocks, not equally much to do: a block of
// a tile of 128 rows takes twice as long as one of 16 (22 blocks of the former 27 to 28 us, of the latter 13 to 18, in one launch of 30).  A workgroup that comes to the
// end of a tile goes on with the next one, or, where there are workgroups enough for that, every tile begins with one of its own.  (As workgroups of their own such beginnings wait, while others have ended, for a place on the shader engine whose turn it is: 8 sequences of 16484 tokens 48 us
// so.)  Items: [0, pieces) where these workgroups begin, [pieces, 2 pieces) beginnings of tiles that they come to, [2 pieces, items) tiles that are not cut.
struct SharePlan {
  int own_tile, own_tiles, pieces, items;    // rows of a tile of own rows; tiles of a sequence
  size_t entries, members, owners, items_at, bytes;      // offsets and size of the plan
  size_t part_ms, part_o, ws_bytes;          // of the workspace
};
SharePlan share_plan(const ficoco_cache& c, const ficoco_attention& a);

struct ShareArgs {
  AttendArgs a;
  uint64_t mark;                             // of the shapes that the plan was made for
  char* plan;
  const int32_t* group;
  Divisor by_rows;                           // n_q * group
  int own_tile, pieces, items, d_head, always;
  size_t entries, members, owners, items_at;
};
void launch_share(const ShareArgs& s, hipStream_t stream);
void launch_share_rows(const ShareArgs& s, int d_head, hipStream_t stream);

}  // namespace ficoco

// Attention over pages of 8 bits for many rows: the tokens of a question, or a piece of a prompt.
#include "page_rows.hpp"

namespace ficoco {
namespace {

template <int D>
__global__ __launch_bounds__(kTileThreads, 2) void page_rows_kernel(AttendArgs a) {
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), c32 = threadIdx.x % 32;
  // (the last rows of all heads first: see tile_rows_kernel; five prompts of up to 2400 tokens in pages, five heads of 64: 56.2 us in the other order, 48.5)
  const int rest = a.by_all.of(blockIdx.x), bh = blockIdx.x - rest * a.B * a.H_kv, b = a.by_heads.of(bh), h = bh - b * a.H_kv;
  const int back = a.by_splits.of(rest), split = rest - back * a.splits, tile = a.row_tiles - 1 - back;
  int slot;
  const Sight s = sight_of<true>(a, b, slot);
  const int rows = s.queries * a.group, row0 = tile * kTileRows;
  if (s.queries <= 0 || row0 >= rows) return;
  auto pos_of = [&](int r) { return s.first + a.by_group.of(r < rows ? r : rows - 1); };
  const Blocks<kTileKeys> blocks(a, s.keys, pos_of(row0), pos_of(row0 + kTileRows - 1));
  const int per = a.by_splits.of(blocks.count + a.splits - 1);
  const int begin = split * per, end = begin + per < blocks.count ? begin + per : blocks.count;

  const int first_row = row0 + 32 * wv, r = first_row + c32, my_r = r < rows ? r : rows - 1;
  const int t = a.by_group.of(my_r), g = my_r - t * a.group;
  const bf16_t* q = a.Q + (int64_t)b * a.q_sb + (int64_t)(h * a.group + g) * a.q_sh + (int64_t)t * a.q_sn;
  const int64_t at = ((int64_t)bh * a.splits + split) * a.part_rows + first_row;
  page_rows<D>(a, threadIdx.x, h, [&] { return TileRow{q, RowSight(a, s.first + t, s.keys)}; }, pos_of(first_row), pos_of(first_row + 31), s.keys, a.table + (int64_t)slot * a.max_pages, blocks, begin, end,
               a.splits > 1, r < rows ? a.part_ms + at + c32 : nullptr,
               [&](int row, int piece) -> void* { return first_row + row < rows ? a.part_o + (at + row) * D + 4 * piece : nullptr; },
               [&](int row, int piece) -> void* {
                 const int r = first_row + row, t = a.by_group.of(r);
                 return r < rows ? a.O + (int64_t)b * a.o_sb + (int64_t)(h * a.group + r - t * a.group) * a.o_sh + (int64_t)t * a.o_sn + 8 * piece : nullptr;
               });
}

}  // namespace

void launch_page_rows(const AttendArgs& a, int d_head, hipStream_t s) {
  const dim3 grid((unsigned)(a.B * a.H_kv * a.row_tiles * a.splits)), threads(kTileThreads);
  if (d_head == 128) hipLaunchKernelGGL(page_rows_kernel<128>, grid, threads, 0, s, a);
  else hipLaunchKernelGGL(page_rows_kernel<64>, grid, threads, 0, s, a);
}

}  // namespace ficoco

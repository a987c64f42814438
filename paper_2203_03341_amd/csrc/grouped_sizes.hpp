// What the grouped products' host code and kernels count, in plain C++, so that it can be tested at any size without a GPU.
#pragma once
#include <cstdint>

namespace ecgemm {

constexpr int kGroupedTile = 128;

// Tiles along `extent` rows or columns.  64 bits: an extent next to 2^31 is allowed, and rounding it up passes 32.
constexpr int64_t grouped_tiles(int64_t extent) { return (extent + kGroupedTile - 1) / kGroupedTile; }

// A launch has fewer than 2^32 threads along x.
constexpr bool launchable(int64_t blocks, int threads) { return blocks <= (((int64_t)1 << 32) - 1) / threads; }

// ---- the kernels of narrow_kernel.hpp: what a block takes, and whether a launch holds a call
constexpr int kNarrowWaves = 8, kNarrowThreads = 64 * kNarrowWaves;
constexpr int64_t kNarrowTallBlocks = 256;
// Blocks of 16 rows the operand that is read once is taken in: four where its rows are contiguous, else two where that leaves
// enough blocks and there are enough columns for it to matter (4096 deep times 32 columns, 8192 rows 49.6 us / 33.8 with 32 rows
// a block, 4096 rows 25.5 / 33.5).
constexpr int narrow_fr(bool depth, int64_t groups, int64_t rows, int64_t columns) {
  return !depth ? 4 : columns > 16 && groups * ((rows + 31) / 32) >= kNarrowTallBlocks ? 2 : 1;
}
constexpr int64_t narrow_row_blocks(int fr, int64_t rows) { return (rows + 16 * fr - 1) / (16 * fr); }
// `more`: rows of blocks beside the groups' own
constexpr bool narrow_fits(bool depth, int64_t groups, int64_t rows, int64_t columns, int more) {
  return launchable((groups + more) * narrow_row_blocks(narrow_fr(depth, groups, rows, columns), rows), kNarrowThreads);
}

constexpr int kShallowThreads = 256, kShallowRows = 256, kShallowColumns = 64;
constexpr int64_t shallow_row_blocks(int64_t M) { return (M + kShallowRows - 1) / kShallowRows; }
constexpr int64_t shallow_column_blocks(int64_t N) { return (N + kShallowColumns - 1) / kShallowColumns; }
// (M x N is held below 2^30 tiles)
constexpr bool shallow_fits(int64_t groups, int64_t M, int64_t N) {
  return launchable(groups * (shallow_row_blocks(M) * shallow_column_blocks(N)), kShallowThreads);
}

constexpr int kAdapterUpThreads = 256, kAdapterUpRows = 256, kAdapterUpColumns = 64, kAdapterUpColumnsShort = 8;
constexpr int64_t adapter_up_row_blocks(int64_t M) { return (M + kAdapterUpRows - 1) / kAdapterUpRows; }
constexpr int64_t adapter_up_blocks(int64_t M, int64_t N, int64_t columns) { return adapter_up_row_blocks(M) * ((N + columns - 1) / columns); }

}  // namespace ecgemm

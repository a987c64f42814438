// What the grouped products' host code and kernels count, in plain C++, so that it can be tested at any size without a GPU.
#pragma once
#include <cstdint>

namespace ecgemm {

constexpr int kGroupedTile = 128;

// Tiles along `extent` rows or columns.  64 bits: an extent next to 2^31 is allowed, and rounding it up passes 32.
constexpr int64_t grouped_tiles(int64_t extent) { return (extent + kGroupedTile - 1) / kGroupedTile; }

}  // namespace ecgemm

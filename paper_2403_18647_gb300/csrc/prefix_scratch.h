// The size of the prefix attention's scratch (plain C++, for the host and the device).
#pragma once

#include <stddef.h>

namespace sdsat {

constexpr int PX_ROWS = 64;   // rows of a tile

// Rows of partial results, each hd values, a reference and four sums: two for each row and head (of the
// shared pages, of the others) and a tile for each CTA.
constexpr size_t px_scratch_rows(size_t row_heads, int ctas) {
  return (2 * row_heads + (size_t)PX_ROWS * ctas + 31) / 32 * 32;
}
constexpr size_t px_scratch_floats(size_t row_heads, int hd, int ctas) { return px_scratch_rows(row_heads, ctas) * (5 + hd); }

// ... floats for every call of b q H hd <= row_dims values: as rows of 64 dimensions, or half as many of 128
constexpr size_t prefix_attention_scratch(size_t row_dims, int ctas) {
  const size_t a = px_scratch_floats(row_dims / 64, 64, ctas), z = px_scratch_floats(row_dims / 128, 128, ctas);
  return a > z ? a : z;
}

}  // namespace sdsat

// The rows between two offsets that only the device knows, whatever they hold.  Plain C++ (nothing from HIP), so that it can be looked at on
// the CPU.
#pragma once

#include <cstdint>

namespace moe {

// of rows 0 .. rows - 1
constexpr int32_t row_within(int32_t at, int32_t rows) {
  const int32_t below = at < rows ? at : rows;
  return below < 0 ? 0 : below;
}
struct RowRange {
  int32_t first, count;
};
// The end is brought behind the first row ahead of the difference, which then cannot pass 32 bits.  An end ahead of the first row: none.
constexpr RowRange row_range(int32_t from, int32_t to, int32_t rows) {
  const int32_t first = row_within(from, rows), below = to < rows ? to : rows;
  return {first, (below > first ? below : first) - first};
}

}  // namespace moe

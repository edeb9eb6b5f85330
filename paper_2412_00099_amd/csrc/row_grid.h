// The grid of a launch whose workgroups take rows in turn.  Plain C++ (nothing from HIP), so that it can be looked at on the CPU.
//
// HIP takes fewer than 2^32 threads along a dimension of a grid, which 2^26 rows of some wavefronts each pass: more workgroups than
// fit into x go on in y.
#pragma once

#include <cstdint>

namespace moe {

constexpr int64_t kRowGridX = 1 << 21;  // of up to 1024 threads
struct RowGrid {
  uint32_t x, y;
};
inline RowGrid row_grid(int64_t groups) {
  const int64_t x = groups < kRowGridX ? groups : kRowGridX;
  return {(uint32_t)x, (uint32_t)((groups + x - 1) / x)};
}

}  // namespace moe

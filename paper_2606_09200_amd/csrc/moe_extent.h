// Where the expert layer's descriptors of 16 rows of a matrix lie: arithmetic that the host can check.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace occ {

// `bytes` from byte `at` on of an expert's codes or values, or of its scales.
struct MoeExtent {
  size_t at;
  uint32_t bytes;
};

// Rows row0 .. row0 + 15, as far as the matrix has them, of `pitch` bytes each.
constexpr MoeExtent moe_rows_extent(uint32_t pitch, int row0, int rows) {
  return MoeExtent{(size_t)row0 * pitch, (uint32_t)(rows - row0 < 16 ? rows - row0 : 16) * pitch};
}

// Their scale tile.  row0 = rows, where a task's blocks are more than the matrix has, may lie past the last one.
constexpr MoeExtent moe_scales_extent(uint32_t pitch, int row0, int rows) {
  return MoeExtent{(size_t)(row0 >> 4) * pitch, row0 < rows ? pitch : 0u};
}

// First row of block `block` of a task whose rows start at row0; `rows` where none are left.
constexpr int moe_block_row(int row0, int block, int rows) {
  return row0 + block * 16 < rows ? row0 + block * 16 : rows;
}

}  // namespace occ

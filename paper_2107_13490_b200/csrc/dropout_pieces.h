// The launches of a dropout call.  A launch numbers the chunks of its rows (16 bytes, or a pair of elements) in 31
// bits, so larger tensors go in pieces of whole rows, and a row that is too long for one launch goes alone, in pieces
// of its columns.
#pragma once

#include <algorithm>
#include <cstdint>

namespace adapt {

struct DropoutPieces {
  int64_t rows, cols;
  int64_t unit;                 // elements of a chunk
  int64_t per_row;              // chunks of a row (the most that any alignment needs)
  int64_t row_step, col_step;   // rows and columns of a piece (col_step a multiple of unit where it cuts a row)

  DropoutPieces(int64_t rows, int64_t cols, int64_t unit) : rows(rows), cols(cols), unit(unit) {
    constexpr int64_t kMost = 1ll << 30;   // chunks of a launch
    col_step = std::min<int64_t>(cols, (kMost - 2) / 8 * unit);
    per_row = (col_step + unit - 1) / unit + 1;
    row_step = col_step < cols ? 1 : std::max<int64_t>(1, kMost / per_row);
  }
  // f(first row, first column, rows, columns) of every piece, until one returns other than 0.
  template <typename F>
  int each(F f) const {
    for (int64_t row = 0; row < rows; row += row_step)
      for (int64_t col = 0; col < cols; col += col_step)
        if (const int rc = f(row, col, std::min(row_step, rows - row), std::min(col_step, cols - col))) return rc;
    return 0;
  }
};

}  // namespace adapt

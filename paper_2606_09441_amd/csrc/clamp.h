// Clamps of what kernels read from a caller's tables: any value leads inside the
// caller's buffers.  No difference is taken before both its terms are in range.
// (constexpr: for the host and the device)
#pragma once

#include <stdint.h>

namespace sift {

// x inside 0 .. most.
constexpr int32_t within(int32_t x, int32_t most) { return x < 0 ? 0 : x > most ? most : x; }

// New tokens of a sequence: row pointers row0 (inside 0 .. rows already) and end, of
// `rows` rows, at most max_rows.
constexpr int32_t rows_between(int32_t row0, int32_t end, int32_t rows, int32_t max_rows) {
  return within(within(end, rows) - row0, max_rows);
}

// Keys of 16 rows of a page from its row `in` (a page's) on; page_len: how many the
// page is said to hold; left: of the sequence.
constexpr int32_t keys_of_page(int32_t page_len, int32_t in, int32_t left) {
  const int32_t held = (page_len > 0 ? page_len : 0) - in;
  return within(held < left ? held : left, 16);
}

}  // namespace sift

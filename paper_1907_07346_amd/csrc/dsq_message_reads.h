// Where the products' kernels read in a row of a 4-bit message: offsets from the row's first byte, in plain arithmetic that a program
// on the host can go through for every width.  A row is blocks of 4 + block / 2 bytes (a scale, then a word for every eight
// columns), of which the last may be shorter; a matrix's last row has nothing behind it.
#pragma once

#include <stdint.h>

namespace dsq {

constexpr uint32_t block_pitch(uint32_t block_log2) { return 4 + (1u << block_log2) / 2; }

// One token: 16 bytes of codes for the 32 columns from col, a multiple of 32, and their scale.  The last lane with columns may have fewer than four
// words: it reads the four that end with the row instead, of which the first `missing` are none of its.  A lane behind the last column
// reads the row's first four words, and counts for nothing.  Needs a row of four words: cols > 24.
constexpr uint32_t missing_words(uint64_t col, uint64_t cols) { return col < cols && col + 24 >= cols ? 4 - (uint32_t)((cols - col + 7) / 8) : 0u; }
struct LaneRead {
    uint64_t scale, codes;
};
constexpr LaneRead lane_read(uint64_t col, uint64_t cols, uint32_t block_log2) {
    const uint64_t from = col < cols ? col : 0, scale = (from >> block_log2) * block_pitch(block_log2);
    return {scale, scale + 4 + (from & ((1u << block_log2) - 1)) / 2 - 4 * missing_words(col, cols)};
}

}  // namespace dsq

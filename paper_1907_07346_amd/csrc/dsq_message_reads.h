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

// Few tokens: a stage is 256 columns that start at one.  Blocks of at most as many lie there whole, scales among the codes, in nine pieces of 16 bytes or
// fewer; of longer blocks eight pieces of codes are read.
constexpr uint32_t kStageColumns = 256, kRowPieces = 9;
constexpr bool scales_apart(uint32_t block_log2) { return (1u << block_log2) > kStageColumns; }
constexpr uint32_t stage_pieces(uint32_t block_log2) { return scales_apart(block_log2) ? kRowPieces - 1 : kRowPieces; }
constexpr uint32_t stage_scale(uint32_t col, uint32_t block_log2) { return (col >> block_log2) * block_pitch(block_log2); }
constexpr uint32_t stage_codes(uint32_t col, uint32_t block_log2) {
    return stage_scale(col, block_log2) + (scales_apart(block_log2) ? 4 + (col & ((1u << block_log2) - 1)) / 2 : 0);
}
// With blocks of 128 and 256 a stage fills two words and one of its last piece.  In the matrix's last rows that piece is read where it ends with its row at
// the latest, `back` words too early: 2 (block 128) or 3 (256) where the row ends with the stage, 1 where one word more follows with its scale (256).
// What the stage has of it is then moved to its front.  (Of all other pieces nothing lies behind the row.)
constexpr uint32_t words_back(uint32_t at, uint32_t pieces, uint32_t row_bytes) { return at + 16 * pieces > row_bytes ? (at + 16 * pieces - row_bytes) / 4 : 0; }
constexpr uint32_t piece_read(uint32_t piece, uint32_t row_bytes) { return piece + 16 <= row_bytes ? piece : row_bytes - 16; }
struct Front {
    uint32_t x, y;
};
constexpr Front moved_to_front(uint32_t back, uint32_t y, uint32_t z, uint32_t w) { return {back == 1 ? y : back == 2 ? z : w, back == 1 ? z : w}; }

}  // namespace dsq

// Goes through the products' reads of a message (paper_1907_07346_amd/csrc/dsq_message_reads.h) on the host: every read inside the row it
// belongs to, and the words that come out the ones that are meant.  Built and run by tests/test_message_reads.py.
#include <cstdio>
#include <cstring>
#include <vector>

#include "dsq_message_reads.h"

namespace {

int failures = 0;
void fail(const char* what, uint64_t cols, uint32_t block, uint64_t at) {
    if (++failures <= 20) std::printf("FAILED %s: cols %llu, block %u, at %llu\n", what, (unsigned long long)cols, block, (unsigned long long)at);
}

uint64_t row_bytes(uint64_t cols, uint32_t block) {
    const uint64_t tail = cols % block;
    return cols / block * (4 + block / 2) + (tail ? 4 + 4 * ((tail + 7) / 8) : 0);
}
uint64_t word_of(uint64_t col, uint32_t block) { return col / block * (4 + block / 2) + 4 + 4 * (col % block / 8); }

// One token: all lanes of all slices, for a slice of `lanes` lanes.
void one_token(uint64_t cols, uint32_t block_log2, uint64_t lanes) {
    const uint32_t block = 1u << block_log2;
    const uint64_t end = row_bytes(cols, block);
    for (uint64_t slice = 0; slice < cols; slice += 32 * lanes)
        for (uint64_t lane = 0; lane < lanes; ++lane) {
            const uint64_t col = slice + 32 * lane;
            const dsq::LaneRead read = dsq::lane_read(col, cols, block_log2);
            if (read.scale + 4 > end || read.codes + 16 > end) fail("a lane reads behind the row", cols, block, col);
            if (col >= cols) continue;
            if (read.scale != col / block * (4 + block / 2)) fail("scale", cols, block, col);
            const uint32_t missing = dsq::missing_words(col, cols);
            for (uint32_t w = 0; w < 4; ++w) {                    // word w of the lane is number (w + missing) % 4 of those that are read
                if (col + 8 * w >= cols) continue;
                const uint32_t place = (w + missing) % 4;
                if (read.codes + 4 * place != word_of(col + 8 * w, block)) fail("word", cols, block, col);
            }
        }
}

// Few tokens: all whole stages of one of the matrix's last rows, or (inner) of another, whose last piece may end in the next row.
void few_tokens(uint64_t cols, uint32_t block_log2, bool inner) {
    const uint32_t block = 1u << block_log2, end = (uint32_t)row_bytes(cols, block), pieces = dsq::stage_pieces(block_log2);
    const uint32_t readable = inner ? 2 * end : end;
    for (uint32_t col = 0; col + dsq::kStageColumns <= cols; col += dsq::kStageColumns) {
        const uint32_t at = dsq::stage_codes(col, block_log2), scale = dsq::stage_scale(col, block_log2);
        if (scale != col / block * (4 + block / 2) || scale + 4 > end) fail("a stage's scale", cols, block, col);
        const uint32_t back = inner ? 0 : dsq::words_back(at, pieces, end);
        uint32_t words[4 * dsq::kRowPieces];                      // the bytes' offsets in the row that the stage's words came from
        for (uint32_t p = 0; p < pieces; ++p) {
            const uint32_t from = inner ? at + 16 * p : dsq::piece_read(at + 16 * p, end);
            if (from + 16 > readable) fail("a piece behind the row", cols, block, col);
            for (uint32_t w = 0; w < 4; ++w) words[4 * p + w] = from + 4 * w;
            if (back && p == dsq::kRowPieces - 1) {
                const dsq::Front f = dsq::moved_to_front(back, words[4 * p + 1], words[4 * p + 2], words[4 * p + 3]);
                words[4 * p] = f.x;
                words[4 * p + 1] = f.y;
            }
        }
        // where the kernel looks: scales and codes of blocks of at most 256 columns one behind the other, of longer ones codes alone
        for (uint32_t c = col; c < col + dsq::kStageColumns; c += 8) {
            const uint32_t in = c - col, word = dsq::scales_apart(block_log2) ? in / 8 : in / block * (1 + block / 8) + 1 + in % block / 8;
            if (words[word] != word_of(c, block)) fail("a stage's word", cols, block, c);
            if (!dsq::scales_apart(block_log2) && words[in / block * (1 + block / 8)] != c / block * (4 + block / 2)) fail("a block's scale", cols, block, c);
        }
    }
}

}  // namespace

int main() {
    for (uint32_t block_log2 = 6; block_log2 <= 11; ++block_log2) {
        for (uint64_t lanes : {4, 16, 32, 64, 128, 256, 512}) {
            for (uint64_t cols = 25; cols < 2200; ++cols) one_token(cols, block_log2, lanes);
            for (uint64_t slices = 1; slices <= 3; ++slices)      // around the ends of slices
                for (int off = -70; off <= 70; ++off) one_token(512 * 32 * slices + off, block_log2, lanes);
        }
        for (uint64_t cols = 256; cols < 5000; ++cols) {
            few_tokens(cols, block_log2, false);
            few_tokens(cols, block_log2, true);
        }
    }
    if (!failures) std::printf("message reads ok\n");
    return failures ? 1 : 0;
}

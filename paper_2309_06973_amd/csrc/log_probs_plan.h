// Log probabilities: how a call's rows are shared out, its workspace and the checks of its sizes.  Plain C++: the host
// and the tests share it.
#pragma once

#include <algorithm>

#include "q8_plan.h"

namespace shifter {

constexpr uint32_t LOGP_MAX_TOP = 32;              // alternatives of a row
constexpr uint32_t LOGP_MAX_PARTS = 64;            // parts of a row: a wavefront joins them
constexpr uint64_t LOGP_PART = 8192;               // columns of a part: 256 threads, four pieces of eight
constexpr uint64_t LOGP_SHARED_ROWS = 512;         // only fewer rows than these are shared by blocks
// The front of a workspace of a call whose blocks join their sums: counters, zero before a call and after it.
constexpr uint64_t LEARN_TICKETS = 4 * LOGP_SHARED_ROWS;
constexpr uint64_t LOGP_MAX_BLOCKS = 1u << 21;     // a launch holds less than 2^32 threads; blocks take further rows in turn

// What a logit is multiplied with before differences are taken.  From 2^-64 on, logits whose difference is beyond fp32 (2^128 and more) are 2^64 and
// more apart with the scale: minus infinity gives the same, no probability.  Below, the difference counts, and in 2^-64 it stays within 2^65;
// what falls below fp32's steps there is less than 2^-148 with the scale.
inline float log_probs_unit(float scale) { return scale < 0x1p-64f ? 0x1p-64f : 1.0f; }

struct LogProbsPlan {
    uint32_t threads;      // of a row's part: 16 or 64, several rows a block; 256, a block
    uint32_t parts;        // blocks that share a row; the last of them joins their sums
    uint32_t part_cols;    // columns of a part, a multiple of 8
    uint64_t bytes;        // of the workspace, 0: none needed
};

inline uint64_t logp_entry(uint32_t top) { return 16u + 8u * (uint64_t)top; }      // what a part leaves: its sums, its alternatives

// Rows up to 256 columns have 16 threads each, up to 1024 a wavefront (more alternatives than groups of 16 give a bound for: a wavefront too),
// longer ones 256 threads.  us in fp32, 16 threads / 64: 10000 x 200 with five alternatives 9.1 / 18.7, 65536 x 100 13.9 / 45.0,
// 10000 x 256 5.7 / 8.9 (10000 x 200 with 16 threads, without alternatives and with five: fp32 5.1 8.9, bf16 5.2 12.2, fp16 5.0 11.8, which have more equal
// logits to be told apart by their columns); 64 / 256: 4096 x 1000 6.4 / 12.8, with five 10.4 / 27.1.  And where there are too few
// rows to fill the chip, several such blocks, each of which fetches its 8192 columns at once.  us of bf16 with 20 alternatives, by blocks a
// row: 1 x 50001 1: 13.9, 6 (two fetches each): 14.8, 8: 13.4, 24: 14.9; 1 x 131072 1: 23.0, 8: 14.5, 16: 14.4, 32: 15.4;
// 128 x 131072 1: 29.3, 4: 21.6, 8: 21.7; 300 x 131072 1: 38.0, 2: 33.9, 4: 35.3; 8 x 10000 1: 11.3, 2: 14.4.  512 threads a block are
// faster where one block has a long row (300 x 131072 32.4), and slower elsewhere (128 x 131072 23.0, 1000 x 2000 25.4 for 14.2).
inline LogProbsPlan log_probs_plan(uint64_t rows, uint64_t cols, uint32_t top) {
    LogProbsPlan p{};
    p.parts = 1;
    p.part_cols = (uint32_t)((cols + 7u) & ~7ull);
    if (cols <= 256 && top <= 8) p.threads = 16;
    else if (cols <= 1024) p.threads = 64;
    else p.threads = 256;
    if (cols > 2 * LOGP_PART && rows < LOGP_SHARED_ROWS) {
        uint64_t parts = (LOGP_SHARED_ROWS + rows - 1u) / (rows ? rows : 1u);
        parts = std::min<uint64_t>({parts, (cols + LOGP_PART - 1u) / LOGP_PART, LOGP_MAX_PARTS});
        const uint64_t each = ((cols + parts - 1u) / parts + 7u) & ~7ull;
        p.part_cols = (uint32_t)each;
        p.parts = (uint32_t)((cols + each - 1u) / each);
    }
    if (p.parts > 1) p.bytes = LEARN_TICKETS + rows * p.parts * logp_entry(top);
    return p;
}

}  // namespace shifter

// Low-rank adapters: how a call is shared out, its workspace and the checks of its sizes.  Plain C++: the host and the
// tests share it.
#pragma once

#include "log_probs_plan.h"

namespace shifter {

constexpr uint32_t ADAPT_MAX_RANK = 128;
constexpr uint64_t ADAPT_MAX_ROWS = 1ull << 25;    // tiles of 16 rows, up to four blocks of 256 threads each: less than 2^32 threads
// From so many adapters on (up to those that fit the block's LDS) more than a few rows are put in order first, whatever order they have.  us of
// 8192 rows, 4096 x 4096 with rank 16, in order / as they come: 4 adapters of random rows 77 / 101, of runs 70 / 59; 8: 79 / 160, 73 / 62;
// 16: 81 / 260, 79 / 63.
constexpr uint64_t ADAPT_SORT_FROM = 8, ADAPT_SORT_MOST = 4094;
// Up to so many adapters the gradient's sums over rows are cut into parts as if one adapter had all the rows; beyond, as if all had as many.
// us of a training step of 4096 x 2048 x 2048 with rank 32, as one / as all: 3 adapters 87 / 94, 8 98 / 121, 16 110 / 109, 32 134 / 106.  That goes by
// the adapters that are loaded, not by where the rows are: 64 of which one has all rows take 181 (105 where all have as many, 79 with one loaded).
constexpr uint64_t ADAPT_FEW_ADAPTERS = 8;
constexpr uint32_t ADAPT_STEP = 64;                // columns of a step of the products over long rows
// Up to ADAPT_FEW_ROWS rows each adapter of a tile has blocks of its own; beyond, tiles are taken with all of theirs, or in the order of the
// adapters.  us of 4096 x 4096 with rank 16, apart / together: 256 rows of 32 adapters as they come 33.7 / 20.2, 1024 of them 83 / 19.3;
// 256 rows in six runs 10.2 / 11.8, 1024 16.7 / 13.7.
// From ADAPT_TWO_TILES rows on a block has two tiles of the product over long rows (1024 rows in three runs, one tile / two: 13.9 / 17.4,
// 2048 20.1 / 19.4, 4096 34.3 / 31.5).
constexpr uint64_t ADAPT_FEW_ROWS = 128, ADAPT_TWO_TILES = 2048;
// With more rows, their product with B holds so many parts in registers.  us, one part / two, 4096 x 4096 with rank 16 and six adapters, 8 bits: 129
// rows 12.1 / 9.9, 512 13.1 / 10.8, 1024 15.3 / 12.9, 2048 23.6 / 19.0, 4096 31.5 / 28.9, 8192 46.3 / 44.7; a training step of 2048 x 2048, rank 32: 1024
// rows 47.3 / 43.3, 4096 of one adapter 81.2 / 78.5, of three 83.1 / 86.4.
constexpr uint32_t ADAPT_MANY_ROWS_PARTS = 2;
constexpr uint32_t ADAPT_UP_BLOCKS = 2048;         // of the product with B, as far as there are columns (1024 and 4096: within 4 %)
constexpr uint64_t ADAPT_ONE_BYTES = 144u << 10;
constexpr uint32_t ADAPT_SLAB = 128;               // columns of a block of the gradient's sums over rows

inline uint64_t adapt_pad(uint64_t rank) { return (rank + 15u) & ~15ull; }

// Tiles of 16 rows that a block works on together: they share what it reads of an adapter.  (Two tiles of 64 ranks do not fit the registers.)
inline uint32_t adapt_tiles(uint64_t m, uint32_t rank) { return adapt_pad(rank) > 32 || m < ADAPT_TWO_TILES ? 1u : 2u; }

// Blocks that share a tile of few rows, one for each adapter that its rows may have.
inline uint32_t adapt_jobs(uint64_t m, uint64_t adapters) {
    return m > ADAPT_FEW_ROWS ? 1u : (uint32_t)std::max<uint64_t>(1u, std::min<uint64_t>({16u, m, adapters}));
}

// The same for the product over long rows, of any number of rows.
inline uint32_t adapt_down_jobs(uint64_t m, uint64_t adapters) {
    return m <= ADAPT_FEW_ROWS ? adapt_jobs(m, adapters) : adapters >= 2 ? 2u : 1u;
}

// Whether one launch does for both products: each of its blocks reads a tile's rows and their adapter's A, which is less than a second launch
// costs up to ADAPT_ONE_BYTES of rows that start on 16 bytes.  us of two launches / one, bf16, square: one row, rank 16, 1024 columns 10.1 / 6.7,
// 2048 9.6 / 7.2, 4096 (139 KB) 9.8 / 8.8, 8192 with rank 8 (147 KB) 10.7 / 10.0; eight rows, 2048 9.6 / 7.2, 4096 (197 KB) 9.7 / 9.6; sixteen rows, 2048
// 9.6 / 8.4, 4096 (262 KB) 9.8 / 11.1; fp32, one row, 2048 (139 KB) 9.6 / 8.7, eight (197 KB) 10.3 / 10.0.  48 rows of 32 adapters, 2048 10.0 / 8.4; 128
// 12.2 / 9.7.  Rows of 3541 in fp16, which start anywhere: 48 of 32 adapters with rank 4 13.3 / 19.9.  It needs no workspace.
inline bool adapt_one(uint64_t m, uint64_t k, uint64_t ld_x, uint32_t rank, uint64_t adapters, uint64_t size) {
    return m <= ADAPT_FEW_ROWS && rank <= 32 && adapters >= 1 && k % 8u == 0 && ld_x % 8u == 0 &&
           (rank + std::min<uint64_t>(m, 16u)) * k * size <= ADAPT_ONE_BYTES;
}
// Its blocks that share the columns of a tile's rows and adapter.  More than 256 blocks take a compute unit's turn each (128 rows of 32 adapters,
// 4096 x 1024: 256 9.9 us, 512 13.8, 1024 21.0).
inline uint32_t adapt_one_blocks(uint64_t m, uint64_t n, uint64_t adapters) {
    const uint64_t shared = (m + 15u) / 16u * adapt_jobs(m, adapters), groups = (n + 255u) / 256u;
    return (uint32_t)std::max<uint64_t>(1u, std::min<uint64_t>(groups, 256u / shared));
}

// Whether the rows are put in order of their adapters first: one more launch, of 6 to 11 us, where tiles of rows as they come could have many.
inline bool adapt_sorted(uint64_t m, uint64_t adapters) { return m > ADAPT_FEW_ROWS && adapters >= ADAPT_SORT_FROM && adapters <= ADAPT_SORT_MOST; }

// Blocks that share the k columns of a tile's rows; each leaves its sums.
inline uint32_t adapt_parts(uint64_t m, uint64_t k, uint32_t rank) {
    const uint64_t rows = 16u * adapt_tiles(m, rank), blocks = (m + rows - 1u) / rows, steps = (k + ADAPT_STEP - 1u) / ADAPT_STEP;
    uint64_t parts = blocks ? 512u / blocks : 1u;
    if (parts > steps / 4u) parts = steps / 4u;    // each of a block's four wavefronts has a step
    const uint64_t most = m > ADAPT_FEW_ROWS ? ADAPT_MANY_ROWS_PARTS : 32u;
    return parts < 1 ? 1u : parts > most ? (uint32_t)most : (uint32_t)parts;
}

struct AdaptersPlan {
    uint32_t parts;
    uint64_t order;                    // rows in the order of their adapters, behind the sums
    uint64_t bytes;
};
inline AdaptersPlan adapters_plan(uint64_t m, uint64_t k, uint32_t rank, uint64_t adapters) {
    AdaptersPlan p{};
    p.parts = adapt_parts(m, k, rank);
    p.order = p.parts * m * adapt_pad(rank) * 4u;
    p.bytes = p.order + (adapt_sorted(m, adapters) ? 4u * m : 0u);
    return p;
}

// The gradient's workspace: offsets of its pieces.
struct AdaptersGradPlan {
    uint32_t parts_x, parts_g;         // of x A' and of g B
    uint32_t parts_rows, rows_each;    // blocks that share an adapter's rows, if it has them all; rows of one
    uint64_t down, up;                 // [m][pad]: x A' where it is not given, and g B
    uint64_t sums;                     // [parts][m][pad]
    uint64_t a, b;                     // the adapters, turned: [adapters][k][rank], [adapters][rank][n]
    uint64_t rows, first;              // rows sorted by their adapter; each adapter's first, and the number of all
    uint64_t partial;                  // [parts_rows + adapters][k + n][rank]: see adapters_grad_kernel
    uint64_t bytes;
};
inline AdaptersGradPlan adapters_grad_plan(uint64_t m, uint64_t n, uint64_t k, uint32_t rank, uint64_t adapters, uint64_t size) {
    AdaptersGradPlan p{};
    const uint64_t pad = adapt_pad(rank);
    p.parts_x = adapt_parts(m, k, rank);
    p.parts_g = adapt_parts(m, n, rank);
    // Few adapters may have any share of the rows: as many parts as would do for one that has all.
    const uint64_t slabs = ((k + ADAPT_SLAB - 1u) / ADAPT_SLAB + (n + ADAPT_SLAB - 1u) / ADAPT_SLAB) * (adapters > ADAPT_FEW_ADAPTERS ? adapters : 1u);
    uint64_t parts = slabs ? 512u / slabs : 1u;
    parts = std::max<uint64_t>(1u, std::min<uint64_t>({parts, m / 64u, 16u}));
    p.rows_each = (uint32_t)((((m + parts - 1u) / parts) + 15u) & ~15ull);
    p.parts_rows = m ? (uint32_t)((m + p.rows_each - 1u) / p.rows_each) : 1u;
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t was = at;
        at += (bytes + 255u) & ~255ull;
        return was;
    };
    p.down = take(m * pad * 4u);
    p.up = take(m * pad * 4u);
    p.sums = take((p.parts_x > p.parts_g ? p.parts_x : p.parts_g) * m * pad * 4u);
    p.a = take(adapters * k * rank * size);
    p.b = take(adapters * n * rank * size);
    p.rows = take(4u * m);
    p.first = take(4u * (adapters + 2u));
    p.partial = take(p.parts_rows > 1 ? (p.parts_rows + adapters) * (k + n) * rank * 4u : 0u);
    p.bytes = at;
    return p;
}

// What is wrong with the sizes, or nullptr; *capacity: they are more than a call holds.
inline const char* adapters_bad_sizes(uint64_t m, uint64_t n, uint64_t k, uint64_t rank, uint64_t adapters, bool* capacity) {
    *capacity = false;
    if (rank < 1 || rank > ADAPT_MAX_RANK) return "a rank that is not 1 to 128";
    if (n > Q8_MAX_ROWS || k > Q8_MAX_ROWS || adapters > (1u << 24)) return "more than 2^31 - 1 columns or 2^24 adapters";
    *capacity = true;
    if (m > ADAPT_MAX_ROWS) return "more than 2^25 rows";
    // the gradient's blocks of 64 columns of all adapters, 256 threads each
    if (adapters * (1u + (k + 63u) / 64u + (n + 63u) / 64u) + 1u >= 1ull << 24) return "more columns of all adapters than a launch holds";
    *capacity = false;
    return nullptr;
}

}  // namespace shifter

// 8-bit matrices: the layout, the checks of a call's arguments and the gradient's workspace.  Plain C++: the
// host and the test that holds the checks to the interface share it.
//
// A matrix of rows x cols is held as int8 codes, a row at a stride that is a multiple of 16
// bytes from a base on 16 bytes, and one fp32 scale a row: the value is code * scale.  What a
// row holds behind its last column is never relied on.
#pragma once

#include <stdint.h>

#include <cmath>

namespace shifter {

constexpr uint32_t Q8_ALIGN = 16;                  // bytes: a row's start, and the granule of its stride
constexpr uint64_t Q8_MAX_STRIDE = 1u << 22;       // bytes between rows: 256 rows stay inside 32-bit offsets
constexpr uint64_t Q8_MAX_ROWS = 0x7fffffffull;    // rows, or columns, of one call
constexpr uint64_t Q8_MAX_LD = 1ull << 32;         // elements between rows of a matrix of elements
constexpr uint64_t Q8_MAX_K = 131071;              // products whose sum 32 bits hold: 131071 * 128 * 128 < 2^31

constexpr uint64_t q8_pad(uint64_t cols) { return (cols + Q8_ALIGN - 1u) & ~(uint64_t)(Q8_ALIGN - 1u); }

inline bool q8_off(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1u)) != 0; }

// What is wrong with a matrix of elements of `size` bytes, or nullptr.
inline const char* q8_bad_rows(const void* p, uintptr_t size, uint64_t rows, uint64_t cols, uint64_t ld) {
    if (rows > Q8_MAX_ROWS || cols > Q8_MAX_ROWS) return "more than 2^31 - 1 rows or columns";
    if (rows == 0 || cols == 0) return nullptr;
    if (!p) return "NULL pointer argument";
    if (q8_off(p, size)) return "a pointer is not aligned to its elements";
    if (rows > 1 && ld < cols) return "a stride is smaller than a row";
    if (ld > Q8_MAX_LD) return "a stride is larger than 2^32 elements";
    return nullptr;
}

// The same for an 8-bit matrix.
inline const char* q8_bad_codes(const void* q, const void* scale, uint64_t rows, uint64_t cols, uint64_t ld) {
    if (rows > Q8_MAX_ROWS || cols > Q8_MAX_ROWS) return "more than 2^31 - 1 rows or columns";
    if (rows == 0) return nullptr;
    if (!scale || (!q && cols)) return "NULL pointer argument";
    if (q8_off(q, Q8_ALIGN) || ld % Q8_ALIGN) return "8-bit rows must start on 16 bytes (pointer and stride)";
    if (q8_off(scale, 4)) return "a pointer is not aligned to its elements";
    if (ld < q8_pad(cols)) return "the stride of 8-bit rows is smaller than a row rounded up to 16";
    if (ld > Q8_MAX_STRIDE) return "the stride of 8-bit rows is larger than 2^22";
    return nullptr;
}

// The product's kernels.  Tiles of rows x columns, a block each; Q8_FEW and Q8_GROUPS: no tiles, both factors are read straight
// into registers by blocks of 16 columns and all of a few rows, or groups of them.
enum Q8Kernel { Q8_FEW, Q8_GROUPS, Q8_TILE_64x64, Q8_TILE_64x128, Q8_TILE_128x128, Q8_TILE_128x256, Q8_TILE_256x256, Q8_KERNELS };
struct Q8TileCost {
    uint32_t rows, cols;
    // us: a launch and a tile's ends; then a stage of 128 bytes: a tile alone on the chip, one on each compute unit, and, where
    // two share a unit, a tile's part of it (0: they do not, and rounds are whole numbers)
    double start, alone, one, shared;
};
// Measured on 256 compute units, us of the kernel by tile:
//    m x n x k             64x64   64x128  128x128  128x256  256x256
//    128 x 4096 x 4096     10.5     12.0     16.1     24.8     39.5
//    512 x 4096 x 4096     15.7     14.7     18.1     25.2     40.4
//    1024 x 4096 x 4096    30.1     24.1     21.5     26.2     41.3
//    2048 x 4096 x 4096    55.2     44.3     39.8     33.8     42.5
//    4096 x 4096 x 4096     106     85.4     77.7     65.0     57.4
//    777 x 1873 x 977       6.8      6.1      7.6     10.8     17.4
//    2048 x 2048 x 2048    16.9     13.4     12.8     16.2     24.8
//    4096 x 1024 x 8192    53.0     43.7     37.7     45.5     73.4
//    16384 x 100 x 2048     9.4      9.1     11.4     16.8     26.4
// The costs below say these within 17 %; the kernel of the least cost is taken, the fastest one in all these rows but 777 x 1873 x 977
// (64x64 for 64x128).
constexpr int Q8_TILES_N = 5;
constexpr Q8TileCost Q8_TILES[Q8_TILES_N] = {{64, 64, 3.2, 0.21, 0.235, 0.20},
                                             {64, 128, 3.2, 0.265, 0.36, 0.325},
                                             {128, 128, 4.0, 0.37, 0.56, 0.0},
                                             {128, 256, 5.0, 0.60, 0.88, 0.0},
                                             {256, 256, 7.0, 0.99, 1.58, 0.0}};
constexpr double Q8_UNITS = 256.0;      // compute units

// Blocks a compute unit of m x n sums, each made by `parts` of them.
inline double q8_rounds(const Q8TileCost& c, uint64_t m, uint64_t n, uint64_t parts) {
    return (double)((m + c.rows - 1u) / c.rows) * (double)((n + c.cols - 1u) / c.cols) * (double)parts / Q8_UNITS;
}

// us of these sums, over k bytes.
inline double q8_tile_us(const Q8TileCost& c, uint64_t m, uint64_t n, uint64_t k, uint64_t parts = 1) {
    const double rounds = q8_rounds(c, m, n, parts), stages = (double)(((k + 127u) / 128u + parts - 1u) / parts);
    if (rounds <= 1.0) return c.start + stages * (c.alone + (c.one - c.alone) * rounds);
    if (c.shared > 0.0) return c.start + stages * (c.shared * rounds > c.one ? c.shared * rounds : c.one);
    return c.start + stages * c.one * std::ceil(rounds);
}

// Up to 16 rows the reading of the weights is all there is, and the kernel without LDS does it best: 1 x 4096 x 4096 5.4 us
// against 9.8 with tiles, 1 x 256 x 8192 6.4 / 16.3, 1 x 8192 x 8192 13.5 / 16.6.  Its blocks read all of A: up to 48 rows it still
// wins where the weights are few (17 x 1000 x 1000 4.0 / 4.7, 32 x 4096 x 4096 8.3 / 10.0, 48 x 3541 x 3277 7.5 / 9.4; but
// 32 x 8192 x 8192 24.1 / 16.8, 64 x 4096 x 4096 12.2 / 10.1).
constexpr uint64_t Q8_FEW_ROWS = 16, Q8_FEW_ROWS_MOST = 48, Q8_FEW_WEIGHTS = 1ull << 24;

// Few results go the same way whatever their rows, in groups of 16 F rows, F as small as leaves a block a compute unit, or 3.  us,
// with F = 1, 2 and 3 / 64 x 64 tiles: 100 x 500 x 8000 7.2 9.4 11.7 / 16.4 (224 blocks with F = 1), 128 x 256 x 4096 5.5 7.4 9.2 / 9.7,
// 64 x 1024 x 1024 3.1 3.6 4.1 / 4.7, 500 x 300 x 2000 5.4 6.0 4.4 / 6.5 (209 blocks with F = 3), 2000 x 64 x 4000 7.0 5.9 7.2 / 9.5 (252
// with F = 2); beyond a block a unit, 512 x 512 x 4096 16.2 13.7 17.4 / 9.7.
inline uint64_t q8_group_blocks(uint64_t m, uint64_t n, uint64_t f) { return (n + 15u) / 16u * ((m + 16u * f - 1u) / (16u * f)); }
inline uint32_t q8_group(uint64_t m, uint64_t n) {
    for (uint32_t f = 1; f < 3; ++f)
        if (m <= 16u * f || q8_group_blocks(m, n, f) <= (uint64_t)Q8_UNITS) return f;
    return 3;
}

// A launch holds less than 2^32 threads along an axis.  Results whose tiles do not fit that: the smallest tiles have 64 x 64
// results, the largest blocks 512 threads; blocks of 16 columns for few rows up to 1024.
constexpr uint64_t Q8_LAUNCH = 1ull << 32;
inline bool q8_tiles_fit(uint64_t rows, uint64_t cols) { return (rows + 63u) / 64u * ((cols + 63u) / 64u) * 512u < Q8_LAUNCH; }
inline const char* q8_too_many(uint64_t m, uint64_t n) {
    return !q8_tiles_fit(m, n) || (m <= Q8_FEW_ROWS_MOST && (n + 15u) / 16u * 1024u >= Q8_LAUNCH) ? "a result of more tiles than a launch holds"
                                                                                                   : nullptr;
}

inline Q8Kernel q8_kernel_for(uint64_t m, uint64_t n, uint64_t k) {
    if (m <= Q8_FEW_ROWS || (m <= Q8_FEW_ROWS_MOST && n * k <= Q8_FEW_WEIGHTS)) return Q8_FEW;
    if (q8_group_blocks(m, n, 3) <= (uint64_t)Q8_UNITS) return Q8_GROUPS;
    int best = 0;
    for (int i = 1; i < Q8_TILES_N; ++i)
        if (q8_tile_us(Q8_TILES[i], m, n, k) < q8_tile_us(Q8_TILES[best], m, n, k)) best = i;
    return (Q8Kernel)(Q8_TILE_64x64 + best);
}

// The gradient's workspace: the largest |g s| of every column by slices of rows and of all rows, then the columns'
// three planes of digits, then the codes, both with the rows of a call side by side.
constexpr uint32_t Q8_SLICES = 128, Q8_SLICE_ROWS = 32;      // most slices; a slice's rows are a multiple of the other
// Up to so many rows a block holds its columns whole in registers and makes their digits from there, in one launch that
// reads g once; beyond, the rows are read in slices for the columns' largest first.  us a call, one launch / two: 966 x 232 x 320
// 15.2 / 19.2, 1000 x 4096 x 4096 70.7 / 75.9; equal at 2048 rows; 4096 x 64 x 1024 30.8 / 26.2, 4096 x 4096 x 1024 74.5 / 82.3.
constexpr uint32_t Q8_WHOLE_ROWS = 2048;
// The gradient's kernels, tiles of (columns of g) x (columns of the checkpoint), the costs as above.  DEEP: three stages in LDS
// for two, so that one block fills a compute unit: taken where there is a unit for every block.  Measured, us of the tiles' kernel:
//    m x n x k             64x64  deep  64x128  deep  64x256  128x256
//    16384 x 4096 x 4096     912  1066     703   797     689      638
//    2048 x 2048 x 2048     32.9  41.7    27.5  30.2    26.5     37.1
//    2048 x 1873 x 977      18.8  25.1    18.2  17.2    23.0     37.3
//    512 x 4096 x 1024      14.2  21.7    11.4  13.7    12.2     18.1
//    3000 x 1500 x 700      20.6  28.9    22.0  18.6    28.0     47.4
//    8192 x 1000 x 300      40.9  31.9    47.0  38.9    61.0      106
//    16384 x 512 x 512      76.0  57.2    83.9  72.0     113      198
//    256 x 2048 x 512        5.8   6.0     6.1   6.2     8.3     13.0
// (on random digits).  The costs below say these within 11 % from 3000 rows on; fewer rows cost more than they say, up to 27 %, and
// with three stages up to 47 % (512 x 4096 x 1024).  3000 x 1500 x 700 takes 64x64, 11 % slower than the fastest, 256 x 2048 x 512
// 64x64 deep, 3 %; the first four rows take the fastest, the other two are split as below.
// Q8_GRAD_SMALL and _WIDE: no digits and no workspace, sums in 64-bit floating point, in one launch.
enum Q8GradientKernel { Q8_GRAD_WIDE = -2, Q8_GRAD_SMALL = -1, Q8_GRAD_64x64, Q8_GRAD_64x64_DEEP, Q8_GRAD_64x128, Q8_GRAD_64x128_DEEP,
                        Q8_GRAD_64x256, Q8_GRAD_128x256, Q8_GRAD_KERNELS };
constexpr double Q8_ALONE = -1.0;       // in the place of `shared`: only where every block has a unit
constexpr Q8TileCost Q8_GRAD_TILES[] = {{64, 64, 3.5, 0.57, 0.62, 0.43},
                                        {64, 64, 3.5, 0.41, 0.50, Q8_ALONE},
                                        {64, 128, 4.3, 0.60, 0.86, 0.72},
                                        {64, 128, 4.3, 0.52, 0.74, Q8_ALONE},
                                        {64, 256, 5.0, 0.85, 1.32, 0.0},
                                        {128, 256, 7.0, 1.50, 2.29, 0.0}};
// Where tiles are few the rows are split among `parts` blocks a tile; their sums, fp32, are joined by a launch of its own,
// which costs that and the traffic.  us of both by parts, with the tiles that are taken:
//    m x n x k                       1     2     4     8    16    32
//    8192 x 1000 x 300   64x64     41.5  28.8  25.3  29.8  34.9  44.6   (4 taken; 64x128 deep would take 21.6)
//    16384 x 512 x 512   64x128 d. 72.2  42.5  27.4  26.9  34.4  49.8   (8 taken)
//    20000 x 60 x 50     64x64 d.  67.4  40.5  25.5  19.0  17.3  20.2   (32 taken)
//    4100 x 260 x 520    64x64     18.8  17.5  14.3  14.6  15.7  20.9   (8 taken)
constexpr uint64_t Q8_PARTS = 32;
// Little work, and few rows of whatever size, go to one launch.  us, that / digits and tiles: 64 x 512 x 512 3.3 / 9.3, 300 x 300 x 300
// 4.4 / 9.5, 500 x 250 x 333 5.8 / 12, 1000 x 100 x 200 7.1 / 14, 2000 x 250 x 260 16 / 21, 128 x 1024 x 1024
// 9.6 / 9.6, 64 x 1400 x 1400 11.8 / 11.6, 256 x 1024 x 1024 14.5 / 11.5; 16 x 4096 x 4096 24.8 / 27.8 (1 x 4096 x 4096 15.5).
constexpr uint64_t Q8_SMALL_ROWS = 2048, Q8_SMALL_RESULTS = 1ull << 20, Q8_SMALL_WORK = 1ull << 27, Q8_WIDE_ROWS = 16;
constexpr bool q8_small(uint64_t m, uint64_t n, uint64_t k) {
    return m <= Q8_SMALL_ROWS && n * k <= Q8_SMALL_RESULTS && m * n * k <= Q8_SMALL_WORK;
}
constexpr double q8_join_us(uint64_t parts, uint64_t n, uint64_t k) {
    return parts > 1 ? 3.5 + 2.0e-6 * (double)parts * (double)n * (double)k : 0.0;
}
struct Q8GradientPlan {
    Q8GradientKernel kernel;
    uint32_t parts, part_rows;                // blocks a tile, and the rows (a multiple of 128) that each has
    uint64_t ld;                              // bytes of a transposed row: the call's rows, rounded up to 128
    uint32_t slices, slice_rows;              // 0 slices: up to Q8_WHOLE_ROWS rows
    uint64_t tops, slice_tops, digits, codes, sums, bytes;      // offsets, and the whole
};
// The rows of the transposed operands, and the slices that more than Q8_WHOLE_ROWS of them are read in.
constexpr uint64_t q8_gradient_ld(uint64_t m) { return (m + 127u) & ~(uint64_t)127u; }
inline uint32_t q8_slice_rows(uint64_t m) {
    const uint64_t per = (m + Q8_SLICES * Q8_SLICE_ROWS - 1u) / (Q8_SLICES * Q8_SLICE_ROWS);
    return (uint32_t)(Q8_SLICE_ROWS * (per ? per : 1u));
}
// The grids that make the operands.  Threads of a block that holds columns whole; blocks of `threads` that turn the checkpoint, 128
// rows and columns by each 256 of them; blocks of the slices' columns; of the digits, whose blocks each read the slices: as many
// times 128 rows a block as leave 2048 blocks.
constexpr uint32_t q8_columns_threads(uint64_t ld) { return ld <= 512 ? 256u : ld <= 1024 ? 512u : 1024u; }
constexpr uint64_t q8_columns_blocks(uint64_t n) { return (n + 15u) / 16u; }
constexpr uint64_t q8_turn_blocks(uint64_t k, uint64_t ld, uint32_t threads) {
    return ((k + 127u) / 128u * (ld / 128u) + threads / 256u - 1u) / (threads / 256u);
}
constexpr uint64_t q8_tops_blocks(uint64_t n, uint64_t slices) { return (n + 511u) / 512u * slices; }
inline uint32_t q8_digits_deep(uint64_t n, uint64_t ld) {
    const uint64_t deep = (n + 63u) / 64u * (ld / 128u) / 2048u;
    return deep < 1u ? 1u : deep > 8u ? 8u : (uint32_t)deep;
}
inline uint64_t q8_digits_blocks(uint64_t n, uint64_t ld) {
    const uint64_t deep = q8_digits_deep(n, ld);
    return (n + 63u) / 64u * ((ld / 128u + deep - 1u) / deep);
}

// The same for the gradient: its tiles, or the blocks of few rows, and what makes the tiles' operands.  m, n and k are less than 2^31.
inline const char* q8_gradient_too_many(uint64_t m, uint64_t n, uint64_t k) {
    bool fits = true;
    if (q8_small(m, n, k)) {
    } else if (m <= Q8_WIDE_ROWS) {
        fits = (n + 15u) / 16u * ((k + 255u) / 256u) * 256u < Q8_LAUNCH;
    } else {
        const uint64_t ld = q8_gradient_ld(m), threads = q8_columns_threads(ld), rows = q8_slice_rows(m);
        fits = q8_tiles_fit(n, k);
        if (m <= Q8_WHOLE_ROWS) fits = fits && (q8_columns_blocks(n) + q8_turn_blocks(k, ld, (uint32_t)threads)) * threads < Q8_LAUNCH;
        else
            fits = fits && (q8_tops_blocks(n, (m + rows - 1u) / rows) + q8_turn_blocks(k, ld, 256)) * 256u < Q8_LAUNCH &&
                   q8_digits_blocks(n, ld) * 256u < Q8_LAUNCH;
    }
    return fits ? nullptr : "a gradient of more tiles than a launch holds";
}

inline Q8GradientPlan q8_gradient_plan(uint64_t m, uint64_t n, uint64_t k) {
    Q8GradientPlan p;
    p.ld = q8_gradient_ld(m);
    p.slice_rows = q8_slice_rows(m);
    p.slices = m <= Q8_WHOLE_ROWS ? 0u : (uint32_t)((m + p.slice_rows - 1u) / p.slice_rows);
    p.tops = 0;
    p.slice_tops = 4u * n;
    p.digits = (p.slice_tops + 4u * n * p.slices + 255u) & ~(uint64_t)255u;
    p.codes = p.digits + 3u * n * p.ld;
    p.sums = p.codes + k * p.ld;
    p.parts = 1;
    p.part_rows = (uint32_t)p.ld;
    if (q8_small(m, n, k) || m <= Q8_WIDE_ROWS) {
        p.kernel = q8_small(m, n, k) ? Q8_GRAD_SMALL : Q8_GRAD_WIDE;
        p.bytes = 0;
        return p;
    }
    p.kernel = Q8_GRAD_64x64;
    uint64_t parts = 1;
    double least = 0.0;
    for (int i = 0; i < Q8_GRAD_KERNELS; ++i)
        for (uint64_t x = 1; x <= Q8_PARTS && (x == 1 || 2u * 128u * x <= p.ld); x *= 2) {
            if (Q8_GRAD_TILES[i].shared == Q8_ALONE && q8_rounds(Q8_GRAD_TILES[i], n, k, x) > 1.0) continue;
            const double us = q8_tile_us(Q8_GRAD_TILES[i], n, k, m, x) + q8_join_us(x, n, k);
            if ((i == 0 && x == 1) || us < least) { least = us; p.kernel = (Q8GradientKernel)i; parts = x; }
        }
    p.part_rows = (uint32_t)((p.ld / 128u + parts - 1u) / parts * 128u);
    p.parts = (uint32_t)((p.ld + p.part_rows - 1u) / p.part_rows);
    p.bytes = p.sums + (p.parts > 1 ? 4u * (uint64_t)p.parts * n * k : 0u);
    return p;
}

}  // namespace shifter

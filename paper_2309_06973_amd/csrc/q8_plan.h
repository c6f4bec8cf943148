// 8-bit matrices: the layout, the checks of a call's arguments and the gradient's workspace.  Plain C++: the
// host and the test that holds the checks to the interface share it.
//
// A matrix of rows x cols is held as int8 codes, a row at a stride that is a multiple of 16
// bytes from a base on 16 bytes, and one fp32 scale a row: the value is code * scale.  What a
// row holds behind its last column is never relied on.
#pragma once

#include <stdint.h>

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

// The gradient's workspace: the largest |g s| of every column by slices of rows, then the columns' three
// planes of digits, then the codes, both with the rows of a call side by side.
constexpr uint32_t Q8_SLICES = 64;
struct Q8GradientPlan {
    uint64_t ld;                              // bytes of a transposed row: the call's rows, rounded up to 128
    uint32_t slices, slice_rows;
    uint64_t tops, digits, codes, bytes;      // offsets, and the whole
};
inline Q8GradientPlan q8_gradient_plan(uint64_t m, uint64_t n, uint64_t k) {
    Q8GradientPlan p;
    p.ld = (m + 127u) & ~(uint64_t)127u;
    const uint64_t tiles = p.ld / 128u;                       // slices are whole tiles of 128 rows
    const uint64_t per = (tiles + Q8_SLICES - 1u) / Q8_SLICES;
    p.slice_rows = (uint32_t)(128u * (per ? per : 1u));
    p.slices = (uint32_t)((m + p.slice_rows - 1u) / p.slice_rows);
    p.tops = 0;
    p.digits = (4u * n * p.slices + 255u) & ~(uint64_t)255u;
    p.codes = p.digits + 3u * n * p.ld;
    p.bytes = p.codes + k * p.ld;
    return p;
}

}  // namespace shifter

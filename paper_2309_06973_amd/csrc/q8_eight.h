// Eight neighbouring elements of a row at a time: what the 8-bit operators read rows of fp32, bf16 and fp16 with.
#pragma once

#include "q8.h"

namespace shifter {

// Eight neighbouring elements as they lie in memory, at any element's address.
template <typename T>
struct Eight {
    static constexpr uint32_t WORDS = 2 * sizeof(T);
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const T* p) {
        typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
        const vec* q = reinterpret_cast<const vec*>(p);
#pragma unroll
        for (uint32_t x = 0; x < WORDS / 4u; ++x) {
            const vec v = q[x];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) w[4u * x + i] = v[i];
        }
    }
    __device__ __forceinline__ void store(T* p) const {
        typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
        vec* q = reinterpret_cast<vec*>(p);
#pragma unroll
        for (uint32_t x = 0; x < WORDS / 4u; ++x) q[x] = vec{w[4u * x], w[4u * x + 1u], w[4u * x + 2u], w[4u * x + 3u]};
    }
    __device__ __forceinline__ void store_through(T* p) const {          // not kept in the caches
        typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
        vec* q = reinterpret_cast<vec*>(p);
#pragma unroll
        for (uint32_t x = 0; x < WORDS / 4u; ++x) __builtin_nontemporal_store(vec{w[4u * x], w[4u * x + 1u], w[4u * x + 2u], w[4u * x + 3u]}, q + x);
    }
    // the elements from the n-th on, zeros behind them: n < 8
    __device__ __forceinline__ void drop(uint32_t n) {
        const uint32_t bits = n * 8u * sizeof(T), words = bits / 32u, rest = bits % 32u;
#pragma unroll
        for (uint32_t d = WORDS / 2u; d > 0; d >>= 1)
#pragma unroll
            for (uint32_t i = 0; i < WORDS; ++i)
                if (words & d) w[i] = i + d < WORDS ? w[i + d] : 0u;
        if (sizeof(T) == 2 && rest) {
#pragma unroll
            for (uint32_t i = 0; i < WORDS; ++i) w[i] = w[i] >> 16 | (i + 1u < WORDS ? w[i + 1u] << 16 : 0u);
        }
    }
    __device__ __forceinline__ void floats(float (&f)[8]) const {
        typedef T vec __attribute__((ext_vector_type(8)));
        vec v;
        __builtin_memcpy(&v, w, sizeof(v));
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
    }
    __device__ __forceinline__ void from(const float (&f)[8]) {
        typedef T vec __attribute__((ext_vector_type(8)));
        vec v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (T)f[i];
        __builtin_memcpy(w, &v, sizeof(v));
    }
};

// The elements from column c on of a row of `cols`, zeros behind its end.  A row's last elements are fetched
// with the ones before them and moved into place, so that no load stands in a branch and all of a row's are under way
// together; only rows of less than eight elements are read one by one.
template <typename T>
__device__ __forceinline__ void fetch8(const T* row, uint32_t c, uint32_t cols, Eight<T>& e) {
    if (cols >= 8u) {
        e.load(row + min(c, cols - 8u));
    } else {
        float f[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) f[i] = c + i < cols ? (float)row[c + i] : 0.0f;
        e.from(f);
    }
}
template <typename T>
__device__ __forceinline__ void place8(uint32_t c, uint32_t cols, Eight<T>& e) {
    if (c + 8u > cols && cols >= 8u) {
        if (c < cols) e.drop(c + 8u - cols);
        else {
#pragma unroll
            for (uint32_t i = 0; i < Eight<T>::WORDS; ++i) e.w[i] = 0u;
        }
    }
}

}  // namespace shifter

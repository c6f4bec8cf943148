// Products of 8-bit matrices on the integer matrix units.
//
// The product   c = sa sb (A B') + bias    of two 8-bit matrices, and the weight gradient
// dW = (g s)' Q from an 8-bit checkpoint Q.  Both are sums over the bytes of two rows that
// lie side by side in memory, exact in 32-bit integers, so no result depends on how the work
// is split; they share one tiled loop.
//
// The gradient's other factor is p = g s in fp32.  Per column it is brought to 24-bit whole
// numbers v (the column's largest |p| becomes 8355711 = 127 (2^16 + 2^8 + 1)), and those to three
// balanced digits, v = d2 2^16 + d1 2^8 + d0, digits from -128 to 127.  Three integer products
// with the same Q give the sum to fp32 accuracy at 1.5 times the cost of one bf16 product (the
// matrix units take 8-bit integers twice as fast), where fp32 products run at a sixteenth.
#include <algorithm>

#include "dev_common.h"
#include "q8.h"

namespace shifter {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

constexpr uint32_t STEP = 128;     // bytes of a row per stage
constexpr uint32_t UNIT = 16;      // bytes a lane moves

// 16 bytes a lane from global memory to LDS: lane l's go to base + 16 l, base the same in all lanes.
__device__ __forceinline__ void to_lds(const int8_t* from, int8_t* base) {
    typedef __attribute__((address_space(1))) const void gptr;
    typedef __attribute__((address_space(3))) void lptr;
    __builtin_amdgcn_global_load_lds((gptr*)from, (lptr*)base, 16, 0, 0);
}

// The tiled loop: WA x WB wavefronts, each with FA x FB tiles of 32 x 32 (FA for each of P planes of A).
// A stage holds STEP bytes of every row of the block's tile, the 16-byte units of a row permuted by its
// number so that the 8 lanes that LDS serves at once read 8 different units.
template <uint32_t P, uint32_t WA, uint32_t WB, uint32_t FA, uint32_t FB>
struct Tile {
    static constexpr uint32_t THREADS = 64 * WA * WB;
    static constexpr uint32_t RA = 32 * WA * FA, RB = 32 * WB * FB;      // rows of A (per plane) and of B
    static constexpr uint32_t ROWS = P * RA + RB;
    static constexpr uint32_t BYTES = ROWS * STEP;
    static constexpr uint32_t PER = ROWS * (STEP / UNIT) / THREADS;      // units a thread moves per stage
    static constexpr uint32_t PASS = THREADS / (STEP / UNIT);            // rows per pass of all threads
    static_assert(ROWS * (STEP / UNIT) % THREADS == 0 && RA % PASS == 0 && RB % PASS == 0, "whole passes");
    v16i acc[P][FA][FB];

    // a, b: first rows of the block; rows_a, rows_b: how many of them there are (1 at least); k: bytes of a row
    __device__ __forceinline__ void run(const int8_t* a, uint64_t ld_a, uint64_t plane, uint32_t rows_a,
                                        const int8_t* b, uint64_t ld_b, uint32_t rows_b, uint32_t k, int8_t* lds) {
#pragma unroll
        for (uint32_t p = 0; p < P; ++p)
#pragma unroll
            for (uint32_t i = 0; i < FA; ++i)
#pragma unroll
                for (uint32_t j = 0; j < FB; ++j)
#pragma unroll
                    for (uint32_t e = 0; e < 16; ++e) acc[p][i][j][e] = 0;
        if (k == 0) return;
        const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = uniform_u32(tid >> 6);
        const uint32_t wa = wave % WA, wb = wave / WA;
        const uint32_t row_in_pass = tid / (STEP / UNIT);
        const uint32_t unit = ((tid % (STEP / UNIT)) ^ (row_in_pass & 7u)) * UNIT;    // PASS is a multiple of 8
        const uint32_t pad = (k + UNIT - 1u) & ~(UNIT - 1u);
        const uint32_t stages = (k + STEP - 1u) / STEP;
        uint32_t off[PER];
#pragma unroll
        for (uint32_t j = 0; j < PER; ++j) {
            const uint32_t r = j * PASS + row_in_pass;
            // rows and units behind the matrix' end: its last ones again, their sums are not used
            off[j] = j * PASS < P * RA ? min(r % RA, rows_a - 1u) * (uint32_t)ld_a
                                       : min(r - P * RA, rows_b - 1u) * (uint32_t)ld_b;
        }
        auto fetch = [&](uint32_t s, int8_t* to) {
            const uint32_t at = s * STEP;
            const uint32_t u = at + min(unit, pad - UNIT - at);
#pragma unroll
            for (uint32_t j = 0; j < PER; ++j) {
                const int8_t* base = j * PASS < P * RA ? a + (uint64_t)(j * PASS / RA) * plane : b;
                to_lds(base + (uint64_t)(off[j] + u), to + (j * THREADS + wave * 64u) * UNIT);
            }
        };
        const uint32_t half = lane >> 5;
        const uint32_t turn = (half ^ (lane & 7u)) * UNIT;
        const int8_t* lane_a = lds + (wa * FA * 32u + (lane & 31u)) * STEP;
        const int8_t* lane_b = lds + (P * RA + wb * FB * 32u + (lane & 31u)) * STEP;
        fetch(0, lds);
        for (uint32_t s = 0; s < stages; ++s) {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // this wavefront's part has come, its reads are done
            __builtin_amdgcn_s_barrier();          // the stage is there, and the other half is free
            asm volatile("" ::: "memory");
            if (s + 1u < stages) fetch(s + 1u, lds + ((s + 1u) & 1u) * BYTES);
            const uint32_t buf = (s & 1u) * BYTES;
            const uint32_t left = k - s * STEP;
#pragma unroll
            for (uint32_t x = 0; x < STEP / 32u; ++x) {
                const uint32_t at = buf + (turn ^ (x * 32u));
                v4i fa[P][FA], fb[FB];
#pragma unroll
                for (uint32_t j = 0; j < FB; ++j) fb[j] = *reinterpret_cast<const v4i*>(lane_b + at + j * 32u * STEP);
#pragma unroll
                for (uint32_t p = 0; p < P; ++p)
#pragma unroll
                    for (uint32_t i = 0; i < FA; ++i)
                        fa[p][i] = *reinterpret_cast<const v4i*>(lane_a + at + (p * RA + i * 32u) * STEP);
                if (left < STEP) {                 // bytes behind the row's end count as zero in A
                    const int32_t n = (int32_t)left - (int32_t)(x * 32u + half * UNIT);
#pragma unroll
                    for (int32_t e = 0; e < 4; ++e) {
                        const int32_t m = min(max(n - 4 * e, 0), 4);
                        const int32_t keep = m == 4 ? -1 : (1 << (8 * m)) - 1;
#pragma unroll
                        for (uint32_t p = 0; p < P; ++p)
#pragma unroll
                            for (uint32_t i = 0; i < FA; ++i) fa[p][i][e] &= keep;
                    }
                }
#pragma unroll
                for (uint32_t p = 0; p < P; ++p)
#pragma unroll
                    for (uint32_t i = 0; i < FA; ++i)
#pragma unroll
                        for (uint32_t j = 0; j < FB; ++j)
                            acc[p][i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[p][i], fb[j], acc[p][i][j], 0, 0, 0);
            }
        }
    }

    // Row (of A) and column (of B) of the block's tile that element e of acc[.][i][j] belongs to.
    __device__ __forceinline__ static uint32_t row(uint32_t i, uint32_t e) {
        const uint32_t lane = threadIdx.x & 63u, wa = uniform_u32(threadIdx.x >> 6) % WA;
        return (wa * FA + i) * 32u + 8u * (e / 4u) + 4u * (lane >> 5) + (e & 3u);
    }
    __device__ __forceinline__ static uint32_t col(uint32_t j) {
        const uint32_t lane = threadIdx.x & 63u, wb = uniform_u32(threadIdx.x >> 6) / WA;
        return (wb * FB + j) * 32u + (lane & 31u);
    }
};

template <typename T, uint32_t WA, uint32_t WB, uint32_t FA, uint32_t FB>
__global__ __launch_bounds__(64 * WA * WB) void q8_product_kernel(Q8ProductArgs g) {
    using Tl = Tile<1, WA, WB, FA, FB>;
    extern __shared__ __align__(16) int8_t lds[];
    const uint32_t tiles_m = (g.m + Tl::RA - 1u) / Tl::RA;
    const uint32_t m0 = (blockIdx.x % tiles_m) * Tl::RA, n0 = (blockIdx.x / tiles_m) * Tl::RB;
    Tl t;
    t.run(g.a + (uint64_t)m0 * g.ld_a, g.ld_a, 0, g.m - m0, g.b + (uint64_t)n0 * g.ld_b, g.ld_b, g.n - n0, g.k, lds);
    T* c = static_cast<T*>(g.c);
#pragma unroll
    for (uint32_t j = 0; j < FB; ++j) {
        const uint32_t n = n0 + Tl::col(j);
        if (n >= g.n) continue;
        const float sb = g.sb[n], bias = g.bias ? g.bias[n] : 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < FA; ++i)
#pragma unroll
            for (uint32_t e = 0; e < 16; ++e) {
                const uint32_t m = m0 + Tl::row(i, e);
                if (m >= g.m) continue;
                // the token's scale first: the product of both could leave the range that their values stay in
                float v = fmaf((float)t.acc[0][i][j][e] * g.sa[m], sb, bias);
                if (g.relu) v = v < 0.0f ? 0.0f : v;
                c[(uint64_t)m * g.ld_c + n] = (T)v;
            }
    }
}

template <typename T>
static void launch_product_of(shifter_ctx* ctx, const Q8ProductArgs& g) {
    constexpr uint32_t WA = 2, WB = 2, FA = 1, FB = 1;
    using Tl = Tile<1, WA, WB, FA, FB>;
    const uint64_t tiles = (uint64_t)((g.m + Tl::RA - 1u) / Tl::RA) * ((g.n + Tl::RB - 1u) / Tl::RB);
    q8_product_kernel<T, WA, WB, FA, FB><<<(uint32_t)tiles, Tl::THREADS, 2 * Tl::BYTES, ctx->stream>>>(g);
}

void launch_q8_product(shifter_ctx* ctx, int dtype, const Q8ProductArgs& g) {
    ProfileScope ps(ctx, K_Q8_PRODUCT);
    if (dtype == SHIFTER_F32) launch_product_of<float>(ctx, g);
    else if (dtype == SHIFTER_BF16) launch_product_of<__bf16>(ctx, g);
    else launch_product_of<_Float16>(ctx, g);
}

// ---- the weight gradient --------------------------------------------------------------

constexpr float DIGITS_TOP = 8355711.0f;     // 127 * (2^16 + 2^8 + 1): the largest v whose digits stay in a byte

// A column whose largest |p| is c is worked on times up: a small one's factor would overflow, its unit would
// fall below the normal numbers.
__device__ __forceinline__ float digits_up(float c) { return c < 0x1p-90f ? 0x1p90f : 1.0f; }
__device__ __forceinline__ float digits_down(float c) { return c < 0x1p-90f ? 0x1p-90f : 1.0f; }

// p = fl(g s) as 32 bits of magnitude: the order of |p|, with infinity and NaN on top.
template <typename T>
__device__ __forceinline__ float scaled(const T* g, float s) { return __fmul_rn((float)*g, s); }

// Largest |p| of every column over a slice of rows.  One column a thread.
template <typename T>
__global__ __launch_bounds__(BLOCK) void q8_tops_kernel(Q8GradientArgs a, uint32_t slice_rows, uint32_t* __restrict__ tops) {
    const uint32_t n = blockIdx.x * BLOCK + threadIdx.x, r0 = blockIdx.y * slice_rows;
    if (n >= a.n) return;
    const T* g = static_cast<const T*>(a.g) + (uint64_t)r0 * a.ld_g + n;
    const uint32_t rows = min(slice_rows, a.m - r0);
    uint32_t top = 0;
    for (uint32_t r = 0; r < rows; ++r) top = max(top, key_of(scaled(g + (uint64_t)r * a.ld_g, a.s[r0 + r])));
    tops[(uint64_t)blockIdx.y * a.n + n] = top;
}

// The digits of 64 columns and 128 rows, the rows of a column side by side.
template <typename T>
__global__ __launch_bounds__(BLOCK) void q8_digits_kernel(Q8GradientArgs a, Q8GradientPlan pl) {
    __shared__ float s_factor[64];
    __shared__ float s_up[64];
    __shared__ int8_t s_d[3][64][128 + 4];
    uint32_t* tops = reinterpret_cast<uint32_t*>(a.work + pl.tops);
    const uint32_t n0 = blockIdx.x * 64u, m0 = blockIdx.y * 128u;
    if (threadIdx.x < 64u) {
        const uint32_t n = n0 + threadIdx.x;
        uint32_t top = 0;
        if (n < a.n)
            for (uint32_t s = 0; s < pl.slices; ++s) top = max(top, tops[(uint64_t)s * a.n + n]);
        const float c = __uint_as_float(top);
        const float up = digits_up(c);
        s_up[threadIdx.x] = up;
        s_factor[threadIdx.x] = top == 0u || top >= 0x7f800000u ? 0.0f : DIGITS_TOP / (c * up);
    }
    __syncthreads();
    const uint32_t col = threadIdx.x & 63u, n = n0 + col;
    const float f = s_factor[col], up = s_up[col];
    for (uint32_t r = threadIdx.x / 64u; r < 128u; r += BLOCK / 64u) {
        const uint32_t m = m0 + r;
        int32_t v = 0;
        if (m < a.m && n < a.n && f != 0.0f) {
            const float p = scaled(static_cast<const T*>(a.g) + (uint64_t)m * a.ld_g + n, a.s[m]);
            v = (int32_t)fminf(fmaxf(rintf(p * up * f), -DIGITS_TOP), DIGITS_TOP);
        }
        const int32_t d0 = (int8_t)v, w = (v - d0) >> 8, d1 = (int8_t)w;
        s_d[0][col][r] = (int8_t)d0;
        s_d[1][col][r] = (int8_t)d1;
        s_d[2][col][r] = (int8_t)((w - d1) >> 8);
    }
    __syncthreads();
    int8_t* out = reinterpret_cast<int8_t*>(a.work + pl.digits);
    for (uint32_t i = threadIdx.x; i < 3u * 64u * 32u; i += BLOCK) {
        const uint32_t word = i & 31u, c = (i >> 5) & 63u, p = i >> 11;
        if (n0 + c < a.n)
            *reinterpret_cast<uint32_t*>(out + ((uint64_t)p * a.n + n0 + c) * pl.ld + m0 + 4u * word) =
                *reinterpret_cast<const uint32_t*>(&s_d[p][c][4u * word]);
    }
}

// 64 columns and 128 rows of the checkpoint, turned.
__global__ __launch_bounds__(BLOCK) void q8_turn_kernel(Q8GradientArgs a, Q8GradientPlan pl) {
    __shared__ int8_t s_q[64][128 + 4];
    const uint32_t k0 = blockIdx.x * 64u, m0 = blockIdx.y * 128u;
    const uint32_t col = threadIdx.x & 63u;
    for (uint32_t r = threadIdx.x / 64u; r < 128u; r += BLOCK / 64u) {
        const uint32_t m = m0 + r, k = k0 + col;
        s_q[col][r] = m < a.m && k < a.k ? a.q[(uint64_t)m * a.ld_q + k] : (int8_t)0;
    }
    __syncthreads();
    int8_t* out = reinterpret_cast<int8_t*>(a.work + pl.codes);
    for (uint32_t i = threadIdx.x; i < 64u * 32u; i += BLOCK) {
        const uint32_t word = i & 31u, c = i >> 5;
        if (k0 + c < a.k)
            *reinterpret_cast<uint32_t*>(out + (uint64_t)(k0 + c) * pl.ld + m0 + 4u * word) =
                *reinterpret_cast<const uint32_t*>(&s_q[c][4u * word]);
    }
}

template <uint32_t WA, uint32_t WB, uint32_t FA, uint32_t FB>
__global__ __launch_bounds__(64 * WA * WB) void q8_gradient_kernel(Q8GradientArgs g, Q8GradientPlan pl) {
    using Tl = Tile<3, WA, WB, FA, FB>;
    extern __shared__ __align__(16) int8_t lds[];
    const uint32_t tiles_n = (g.n + Tl::RA - 1u) / Tl::RA;
    const uint32_t n0 = (blockIdx.x % tiles_n) * Tl::RA, k0 = (blockIdx.x / tiles_n) * Tl::RB;
    const int8_t* digits = reinterpret_cast<const int8_t*>(g.work + pl.digits);
    const int8_t* codes = reinterpret_cast<const int8_t*>(g.work + pl.codes);
    const uint32_t* tops = reinterpret_cast<const uint32_t*>(g.work + pl.tops);
    Tl t;
    t.run(digits + (uint64_t)n0 * pl.ld, pl.ld, (uint64_t)g.n * pl.ld, g.n - n0, codes + (uint64_t)k0 * pl.ld, pl.ld,
          g.k - k0, (uint32_t)pl.ld, lds);
#pragma unroll
    for (uint32_t i = 0; i < FA; ++i)
#pragma unroll
        for (uint32_t e = 0; e < 16; ++e) {
            const uint32_t n = n0 + Tl::row(i, e);
            if (n >= g.n) continue;
            uint32_t top = 0;
            for (uint32_t s = 0; s < pl.slices; ++s) top = max(top, tops[(uint64_t)s * g.n + n]);
            const float c = __uint_as_float(top), unit = c * digits_up(c) / DIGITS_TOP, down = digits_down(c);
            const bool bad = top >= 0x7f800000u;
#pragma unroll
            for (uint32_t j = 0; j < FB; ++j) {
                const uint32_t k = k0 + Tl::col(j);
                if (k >= g.k) continue;
                const bool keep = !g.mask || g.mask[(uint64_t)n * g.ld_mask + k];
                float v = fmaf((float)t.acc[2][i][j][e], 65536.0f, fmaf((float)t.acc[1][i][j][e], 256.0f, (float)t.acc[0][i][j][e]));
                v = bad ? __uint_as_float(0x7fc00000u) : v * unit * down;
                float* out = g.dw + (uint64_t)n * g.ld_dw + k;
                if (g.accumulate) { if (keep) *out += v; }
                else *out = keep ? v : 0.0f;
            }
        }
}

template <typename T>
static void launch_digits(shifter_ctx* ctx, const Q8GradientArgs& g, const Q8GradientPlan& pl) {
    if (pl.slices == 0) return;
    q8_tops_kernel<T><<<dim3((g.n + BLOCK - 1u) / BLOCK, pl.slices), BLOCK, 0, ctx->stream>>>(
        g, pl.slice_rows, reinterpret_cast<uint32_t*>(g.work + pl.tops));
    q8_digits_kernel<T><<<dim3((g.n + 63u) / 64u, (uint32_t)(pl.ld / 128u)), BLOCK, 0, ctx->stream>>>(g, pl);
    q8_turn_kernel<<<dim3((g.k + 63u) / 64u, (uint32_t)(pl.ld / 128u)), BLOCK, 0, ctx->stream>>>(g, pl);
}

void launch_q8_gradient(shifter_ctx* ctx, int dtype, const Q8GradientArgs& g) {
    const Q8GradientPlan pl = q8_gradient_plan(g.m, g.n, g.k);
    {
        ProfileScope ps(ctx, K_Q8_DIGITS);
        if (dtype == SHIFTER_F32) launch_digits<float>(ctx, g, pl);
        else if (dtype == SHIFTER_BF16) launch_digits<__bf16>(ctx, g, pl);
        else launch_digits<_Float16>(ctx, g, pl);
    }
    ProfileScope ps(ctx, K_Q8_GRADIENT);
    constexpr uint32_t WA = 2, WB = 2, FA = 1, FB = 1;
    using Tl = Tile<3, WA, WB, FA, FB>;
    const uint64_t tiles = (uint64_t)((g.n + Tl::RA - 1u) / Tl::RA) * ((g.k + Tl::RB - 1u) / Tl::RB);
    q8_gradient_kernel<WA, WB, FA, FB><<<(uint32_t)tiles, Tl::THREADS, 2 * Tl::BYTES, ctx->stream>>>(g, pl);
}

}  // namespace shifter

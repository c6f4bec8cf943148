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
#include <type_traits>

#include "dev_common.h"
#include "q8.h"

namespace shifter {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

constexpr uint32_t UNIT = 16;      // bytes a lane moves

// 16 bytes a lane from global memory to LDS: lane l's go to base + 16 l, base the same in all lanes.
__device__ __forceinline__ void to_lds(const int8_t* from, int8_t* base) {
    typedef __attribute__((address_space(1))) const void gptr;
    typedef __attribute__((address_space(3))) void lptr;
    __builtin_amdgcn_global_load_lds((gptr*)from, (lptr*)base, 16, 0, 0);
}

// Waits until at most N of this wavefront's moves are under way, and until its LDS reads are done.
template <uint32_t N>
__device__ __forceinline__ void wait_moves() {
    static_assert(N < 64, "six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15u) | (N >> 4) << 14 | 7u << 4);      // a builtin: the compiler knows what is done
    asm volatile("" ::: "memory");
}

// The tiled loop: WA x WB wavefronts, each with FA x FB tiles of 32 x 32 (FA for each of P planes of A).
// A stage holds STEP bytes of every row of the block's tile, the 16-byte units of a row permuted by its
// number so that 16 lanes of a read meet 64 different banks.  NS stages are in LDS or on their
// way to it.  A stage is worked off in steps of 32 bytes, whose operands are read one step
// ahead: the first ones of the next stage before the last step of this one, behind the stage's only barrier.
template <uint32_t P, uint32_t WA, uint32_t WB, uint32_t FA, uint32_t FB, uint32_t NS, uint32_t STEP>
struct Tile {
    static constexpr uint32_t UNITS = STEP / UNIT, STEPS = STEP / 32;
    static constexpr uint32_t COLS = 32 * FB;                            // columns of a wavefront
    static constexpr uint32_t THREADS = 64 * WA * WB;
    static constexpr uint32_t RA = 32 * WA * FA, RB = 32 * WB * FB;      // rows of A (per plane) and of B
    static constexpr uint32_t ROWS = P * RA + RB;
    static constexpr uint32_t BYTES = ROWS * STEP;
    static constexpr uint32_t LDS = NS * BYTES;
    static constexpr uint32_t PER = ROWS * UNITS / THREADS;              // units a thread moves per stage
    static constexpr uint32_t PASS = THREADS / UNITS;                    // rows per pass of all threads
    // a row's turn: rows that share the 256 bytes of all banks have the same one
    __device__ __forceinline__ static uint32_t turn_of(uint32_t row) { return row / (256u / STEP) & (UNITS - 1u); }
    static_assert(STEPS % 2 == 0 && PASS % 16 == 0 && ROWS * UNITS % THREADS == 0 && RA % PASS == 0 && RB % PASS == 0, "whole passes");
    v16i acc[P][FA][FB];

    struct Operands { v4i a[P][FA], b[FB]; };

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
        const uint32_t row_in_pass = tid / UNITS;
        const uint32_t unit = ((tid % UNITS) ^ turn_of(row_in_pass)) * UNIT;    // PASS is a multiple of 16
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
        auto fetch = [&](uint32_t s, uint32_t buf) {
            const uint32_t at = s * STEP;
            const uint32_t u = at + min(unit, pad - UNIT - at);
#pragma unroll
            for (uint32_t j = 0; j < PER; ++j) {
                const int8_t* base = j * PASS < P * RA ? a + (uint64_t)(j * PASS / RA) * plane : b;
                to_lds(base + (uint64_t)(off[j] + u), lds + buf + (j * THREADS + wave * 64u) * UNIT);
            }
        };
        const uint32_t half = lane >> 5;
        const uint32_t turn = (half ^ turn_of(lane & 31u)) * UNIT;
        const int8_t* lane_a = lds + (wa * FA * 32u + (lane & 31u)) * STEP;
        const int8_t* lane_b = lds + (P * RA + wb * FB * 32u + (lane & 31u)) * STEP;
        auto read = [&](Operands& o, uint32_t buf, uint32_t x) {
            const uint32_t at = buf + (turn ^ (x * 32u));
#pragma unroll
            for (uint32_t j = 0; j < FB; ++j) o.b[j] = *reinterpret_cast<const v4i*>(lane_b + at + j * 32u * STEP);
#pragma unroll
            for (uint32_t p = 0; p < P; ++p)
#pragma unroll
                for (uint32_t i = 0; i < FA; ++i)
                    o.a[p][i] = *reinterpret_cast<const v4i*>(lane_a + at + (p * RA + i * 32u) * STEP);
        };
        auto multiply = [&](const Operands& o) {
#pragma unroll
            for (uint32_t p = 0; p < P; ++p)
#pragma unroll
                for (uint32_t i = 0; i < FA; ++i)
#pragma unroll
                    for (uint32_t j = 0; j < FB; ++j)
                        acc[p][i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(o.a[p][i], o.b[j], acc[p][i][j], 0, 0, 0);
        };

#pragma unroll
        for (uint32_t s = 0; s < NS; ++s)
            if (s < stages) fetch(s, s * BYTES);
        Operands o[2];
        if (stages >= NS) wait_moves<(NS - 1u) * PER>(); else wait_moves<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        uint32_t buf = 0, s = 0;
        read(o[0], 0, 0);
        auto stage = [&](auto more) {              // more: there is a stage to be fetched
            const uint32_t next = buf + BYTES == LDS ? 0u : buf + BYTES;
#pragma unroll
            for (uint32_t x = 0; x < STEPS; ++x) {
                if (x + 1u < STEPS) {
                    read(o[(x + 1) & 1], buf, x + 1);
                } else {
                    // the next stage's parts have come and this one's reads are done, in this wavefront and, behind
                    // the barrier, in all: the buffer is free
                    wait_moves<more.value ? (NS - 2u) * PER : 0u>();
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    read(o[0], next, 0);
                    if (more.value) fetch(s + NS, buf);
                }
                multiply(o[x & 1]);
                // one LDS read, then its share of the products, in turn
                constexpr int READS = P * FA + FB, PRODUCTS = P * FA * FB;
#pragma unroll
                for (int z = 0; z < READS; ++z) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x8, PRODUCTS / READS, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x8, PRODUCTS % READS, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            buf = next;
        };
        for (; s + NS < stages; ++s) stage(std::true_type{});
        for (; s + 1u < stages; ++s) stage(std::false_type{});
        const uint32_t left = k - (stages - 1u) * STEP;      // bytes of the last stage, 1 at least
#pragma unroll
        for (uint32_t x = 0; x < STEPS; ++x) {
            if (x * 32u >= left) break;
            if (x + 1u < STEPS) read(o[(x + 1) & 1], buf, x + 1);
            if (left < x * 32u + 32u) {                      // bytes behind the row's end count as zero in A
                const int32_t n = (int32_t)left - (int32_t)(x * 32u + half * UNIT);
#pragma unroll
                for (int32_t e = 0; e < 4; ++e) {
                    const int32_t m = min(max(n - 4 * e, 0), 4);
                    const int32_t keep = m == 4 ? -1 : (1 << (8 * m)) - 1;
#pragma unroll
                    for (uint32_t p = 0; p < P; ++p)
#pragma unroll
                        for (uint32_t i = 0; i < FA; ++i) o[x & 1].a[p][i][e] &= keep;
                }
            }
            multiply(o[x & 1]);
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

// The tile of a block, of `tiles_a` x `tiles_b`: blocks go to the 8 chiplets in turn, and each of those takes a
// run of tiles in bands of GROUP along a, so that the 32 tiles it works on share rows of both factors in its L2.
template <uint32_t GROUP>
__device__ __forceinline__ void tile_of_block(uint32_t tiles_a, uint32_t tiles_b, uint32_t* ta, uint32_t* tb) {
    const uint32_t all = tiles_a * tiles_b, xcd = blockIdx.x % 8u, nth = blockIdx.x / 8u;
    const uint32_t each = all / 8u, more = all % 8u;
    const uint32_t t = xcd * each + min(xcd, more) + nth;
    const uint32_t band = t / (GROUP * tiles_b), in = t - band * GROUP * tiles_b;
    const uint32_t high = min(GROUP, tiles_a - band * GROUP);
    *tb = in / high;
    *ta = band * GROUP + in - *tb * high;
}

// Writes a wavefront's 32 rows x COLS values of LDS (rows `pitch` bytes apart) to c: 16 bytes a lane, rows and
// columns behind the matrix' end left out.
template <typename T, uint32_t COLS>
__device__ __forceinline__ void store_rows(const int8_t* from, uint32_t pitch, T* c, uint64_t ld, uint32_t rows, uint32_t cols) {
    constexpr uint32_t E = 16 / sizeof(T), LANES = COLS / E;             // elements of a lane, lanes of a row
    typedef T vec __attribute__((ext_vector_type(E)));
    typedef T loose __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    const uint32_t lane = threadIdx.x & 63u, n = lane % LANES * E;
#pragma unroll
    for (uint32_t r = lane / LANES; r < 32u; r += 64u / LANES) {
        const vec v = *reinterpret_cast<const vec*>(from + r * pitch + n * sizeof(T));
        if (r >= rows) continue;
        T* to = c + (uint64_t)r * ld + n;
        if (n + E <= cols) {
            *reinterpret_cast<loose*>(to) = v;
        } else {
#pragma unroll
            for (uint32_t i = 0; i < E; ++i)
                if (n + i < cols) to[i] = v[i];
        }
    }
}

template <typename T, uint32_t WA, uint32_t WB, uint32_t FA, uint32_t FB, uint32_t NS, uint32_t STEP, uint32_t GROUP>
__global__ __launch_bounds__(64 * WA * WB) void q8_product_kernel(Q8ProductArgs g) {
    using Tl = Tile<1, WA, WB, FA, FB, NS, STEP>;
    constexpr uint32_t PITCH = Tl::COLS * sizeof(T) + 16u;               // of the results' rows, in bytes
    constexpr uint32_t OUT = WA * WB * 32u * PITCH;
    constexpr uint32_t BEHIND = OUT + 4u * Tl::RA;                       // the tokens' scales lie behind them
    __shared__ __align__(16) int8_t lds[Tl::LDS > BEHIND ? Tl::LDS : BEHIND];
    static_assert(Tl::THREADS >= Tl::RA, "a scale a thread");
    uint32_t ta, tb;
    tile_of_block<GROUP>((g.m + Tl::RA - 1u) / Tl::RA, (g.n + Tl::RB - 1u) / Tl::RB, &ta, &tb);
    const uint32_t m0 = ta * Tl::RA, n0 = tb * Tl::RB;
    const float mine = g.sa[min(m0 + threadIdx.x % Tl::RA, g.m - 1u)];
    float sb[FB], bias[FB];
#pragma unroll
    for (uint32_t j = 0; j < FB; ++j) {
        const uint32_t n = min(n0 + Tl::col(j), g.n - 1u);
        sb[j] = g.sb[n];
        bias[j] = g.bias ? g.bias[n] : 0.0f;
    }
    Tl t;
    t.run(g.a + (uint64_t)m0 * g.ld_a, g.ld_a, 0, g.m - m0, g.b + (uint64_t)n0 * g.ld_b, g.ld_b, g.n - n0, g.k, lds);
    // results go through LDS, each wavefront by itself, so that rows are written in long pieces
    __syncthreads();
    float* s_a = reinterpret_cast<float*>(lds + OUT);
    if (threadIdx.x < Tl::RA) s_a[threadIdx.x] = mine;
    __syncthreads();
    const uint32_t lane = threadIdx.x & 63u;
    int8_t* out = lds + uniform_u32(threadIdx.x >> 6) * 32u * PITCH;
    T* c = static_cast<T*>(g.c);
#pragma unroll
    for (uint32_t i = 0; i < FA; ++i) {
        const uint32_t first = Tl::row(i, 0) - 4u * (lane >> 5), m = m0 + first, n = n0 + Tl::col(0) - (lane & 31u);
#pragma unroll
        for (uint32_t e4 = 0; e4 < 4; ++e4) {
            const float4 sa = *reinterpret_cast<const float4*>(&s_a[Tl::row(i, 4 * e4)]);
            const float s[4] = {sa.x, sa.y, sa.z, sa.w};
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e)
#pragma unroll
                for (uint32_t j = 0; j < FB; ++j) {
                    // the token's scale first: the product of both could leave the range that their values stay in
                    float v = fmaf((float)t.acc[0][i][j][4 * e4 + e] * s[e], sb[j], bias[j]);
                    if (g.relu) v = v < 0.0f ? 0.0f : v;
                    *reinterpret_cast<T*>(out + (8u * e4 + 4u * (lane >> 5) + e) * PITCH + (j * 32u + (lane & 31u)) * sizeof(T)) = (T)v;
                }
        }
        __builtin_amdgcn_wave_barrier();       // a wavefront's LDS accesses are done in order
        if (m < g.m && n < g.n)
            store_rows<T, Tl::COLS>(out, PITCH, c + (uint64_t)m * g.ld_c + n, g.ld_c, g.m - m, g.n - n);
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename T, uint32_t WA, uint32_t WB, uint32_t FA, uint32_t FB, uint32_t NS, uint32_t STEP, uint32_t GROUP>
static void launch_product_as(shifter_ctx* ctx, const Q8ProductArgs& g) {
    using Tl = Tile<1, WA, WB, FA, FB, NS, STEP>;
    const uint64_t tiles = (uint64_t)((g.m + Tl::RA - 1u) / Tl::RA) * ((g.n + Tl::RB - 1u) / Tl::RB);
    q8_product_kernel<T, WA, WB, FA, FB, NS, STEP, GROUP><<<(uint32_t)tiles, Tl::THREADS, 0, ctx->stream>>>(g);
}

// Few tokens: the weights are read once, straight into registers, and that read is the time.  A block has 16
// columns of the result and all of the up to 16 F tokens; its WAVES wavefronts take pieces of 128 bytes of the
// rows in turn and join their sums in LDS.  (Weights are the first factor of the 16 x 16 x 64 products: a
// lane then holds four neighbouring columns of one token.)
template <typename T, uint32_t F, uint32_t WAVES>
__global__ __launch_bounds__(64 * WAVES) void q8_product_few_kernel(Q8ProductArgs g) {
    constexpr uint32_t PIECE = 128, DEPTH = 4;                           // bytes; pieces under way
    __shared__ v4i s_sum[WAVES][F][64];
    const uint32_t lane = threadIdx.x & 63u, wave = uniform_u32(threadIdx.x >> 6);
    const uint32_t n0 = blockIdx.x * 16u, at = lane / 16u * UNIT;
    const int8_t* b = g.b + (uint64_t)min(n0 + (lane & 15u), g.n - 1u) * g.ld_b;
    const int8_t* a[F];
#pragma unroll
    for (uint32_t f = 0; f < F; ++f) a[f] = g.a + (uint64_t)min(16u * f + (lane & 15u), g.m - 1u) * g.ld_a;
    v4i acc[F];
#pragma unroll
    for (uint32_t f = 0; f < F; ++f) acc[f] = v4i{0, 0, 0, 0};
    const uint32_t whole = g.k / PIECE;
    uint32_t p = wave;
    for (; p + (DEPTH - 1u) * WAVES < whole; p += DEPTH * WAVES) {
        v4i vb[DEPTH][2], va[DEPTH][F][2];
#pragma unroll
        for (uint32_t d = 0; d < DEPTH; ++d)
#pragma unroll
            for (uint32_t x = 0; x < 2; ++x) {
                const uint32_t k = (p + d * WAVES) * PIECE + x * 64u + at;
                vb[d][x] = *reinterpret_cast<const v4i*>(b + k);
#pragma unroll
                for (uint32_t f = 0; f < F; ++f) va[d][f][x] = *reinterpret_cast<const v4i*>(a[f] + k);
            }
#pragma unroll
        for (uint32_t d = 0; d < DEPTH; ++d)
#pragma unroll
            for (uint32_t x = 0; x < 2; ++x)
#pragma unroll
                for (uint32_t f = 0; f < F; ++f)
                    acc[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb[d][x], va[d][f][x], acc[f], 0, 0, 0);
    }
    for (; p * PIECE < g.k; p += WAVES) {
#pragma unroll
        for (uint32_t x = 0; x < 2; ++x) {
            const uint32_t k = p * PIECE + x * 64u + at;
            const uint32_t from = min(k, (g.k - 1u) & ~(UNIT - 1u));     // behind the row's end: its last unit again
            const v4i vb = *reinterpret_cast<const v4i*>(b + from);
#pragma unroll
            for (uint32_t f = 0; f < F; ++f) {
                v4i va = *reinterpret_cast<const v4i*>(a[f] + from);
#pragma unroll
                for (int32_t e = 0; e < 4; ++e) {                        // bytes behind it count as zero
                    const int32_t n = min(max((int32_t)g.k - (int32_t)k - 4 * e, 0), 4);
                    va[e] &= n == 4 ? -1 : (1 << (8 * n)) - 1;
                }
                acc[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb, va, acc[f], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (uint32_t f = 0; f < F; ++f) s_sum[wave][f][lane] = acc[f];
    __syncthreads();
    static_assert(WAVES >= F, "a wavefront for 16 tokens' sums");
    if (wave >= F) return;
    const uint32_t m = wave * 16u + (lane & 15u), n = n0 + lane / 16u * 4u;
    v4i sum = s_sum[0][wave][lane];
#pragma unroll
    for (uint32_t w = 1; w < WAVES; ++w) sum += s_sum[w][wave][lane];
    if (m >= g.m) return;
    const float sa = g.sa[m];
    T* c = static_cast<T*>(g.c) + (uint64_t)m * g.ld_c + n;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
        if (n + e >= g.n) break;
        float v = fmaf((float)sum[e] * sa, g.sb[n + e], g.bias ? g.bias[n + e] : 0.0f);
        if (g.relu) v = v < 0.0f ? 0.0f : v;
        c[e] = (T)v;
    }
}

template <typename T, uint32_t F, uint32_t WAVES>
static void launch_product_few(shifter_ctx* ctx, const Q8ProductArgs& g) {
    q8_product_few_kernel<T, F, WAVES><<<(g.n + 15u) / 16u, 64 * WAVES, 0, ctx->stream>>>(g);
}

template <typename T>
static void launch_product_of(shifter_ctx* ctx, const Q8ProductArgs& g) {
    switch (q8_kernel_for(g.m, g.n, g.k)) {
        case Q8_FEW:
            if (g.m <= 16) launch_product_few<T, 1, 8>(ctx, g);
            else if (g.m <= 32) launch_product_few<T, 2, 16>(ctx, g);
            else launch_product_few<T, 3, 16>(ctx, g);
            break;
        case Q8_TILE_64x64: launch_product_as<T, 2, 2, 1, 1, 4, 128, 16>(ctx, g); break;
        case Q8_TILE_64x128: launch_product_as<T, 2, 2, 1, 2, 3, 128, 8>(ctx, g); break;
        case Q8_TILE_128x256: launch_product_as<T, 2, 4, 2, 2, 2, 128, 8>(ctx, g); break;
        default: launch_product_as<T, 2, 4, 4, 2, 2, 128, 4>(ctx, g); break;
    }
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

template <uint32_t WA, uint32_t WB, uint32_t FA, uint32_t FB, uint32_t NS>
__global__ __launch_bounds__(64 * WA * WB) void q8_gradient_kernel(Q8GradientArgs g, Q8GradientPlan pl) {
    using Tl = Tile<3, WA, WB, FA, FB, NS, 128>;
    __shared__ __align__(16) int8_t lds[Tl::LDS];
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
    constexpr uint32_t WA = 2, WB = 2, FA = 1, FB = 1, NS = 2;
    using Tl = Tile<3, WA, WB, FA, FB, NS, 128>;
    const uint64_t tiles = (uint64_t)((g.n + Tl::RA - 1u) / Tl::RA) * ((g.k + Tl::RB - 1u) / Tl::RB);
    q8_gradient_kernel<WA, WB, FA, FB, NS><<<(uint32_t)tiles, Tl::THREADS, 0, ctx->stream>>>(g, pl);
}

}  // namespace shifter

// Products of 8-bit matrices on the integer matrix units.
//
// The product   c = sa sb (A B') + bias    of two 8-bit matrices, and the weight gradient
// dW = (g s)' Q from an 8-bit checkpoint Q.  Both are sums over the bytes of two rows that
// lie side by side in memory, exact in 32-bit integers, so a product's result does not depend on how the
// work is split (a gradient's rows split into parts round once a part); they share one tiled loop.
//
// The gradient's other factor is p = g s in fp32.  Per column it is brought to 24-bit whole
// numbers v (the column's largest |p| becomes 8355711 = 127 (2^16 + 2^8 + 1)), and those to three
// balanced digits, v = d2 2^16 + d1 2^8 + d0, digits from -128 to 127.  Three integer products
// with the same Q give the sum of v q exactly at 1.5 times the cost of one bf16 product (the
// matrix units take 8-bit integers twice as fast), where fp32 products run at a sixteenth.  What that
// rounds to fewer bits is p, once: a p that is 2^j below its column's largest keeps 24 - j of its bits, so
// the column's largest bounds the error of all its sums.  Norm-wise, 4096 rows behind a ReLU: 5e-7 with rows whose
// sizes spread by e^1, 1.7e-6 by e^2 (fp32 products 3e-7); with one row 10^4 above the others 3e-4 in the entries where that
// row has nothing, with 10^6 4e-2.  Such rows are for a call of their own (SHIFTER_Q8_ACCUMULATE), whose columns have their own
// largest.  Where there is little work, 64-bit products in one launch, without that rounding, are faster than the two
// launches that digits need.
#include <algorithm>
#include <type_traits>

#include "dev_common.h"
#include "q8_eight.h"

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

// c[m][n] = (sum over k of A[m][k] B[n][k]) sa[m] sb[n] + bias[n]: the sum exact, then two roundings in fp32 and the one to
// c's type.  8192 x 8192 x 8192 to bf16 takes 425 us on the same operands again and again and 445 on new ones (434 to 555 under a
// profiler), 2.5 to 2.6 POP/s, against 2.42 of the library's bare integer product: the matrix units are busy in 71 % of the
// cycles, and there are 1.66 GHz of those under this load where the chip has up to 2.4; LDS reads conflict in 1 % of their
// cycles.  A band of GROUP tiles keeps memory out of the way: 0.8 GB are read, 1.8 TB/s.  Eight wavefronts of 128 x 64 each
// for 256 x 256: four of 128 x 128 would read a fifth less LDS but spill (505 us or more).
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

// Few tokens, or few results: the weights are read once (by each group of tokens), straight into registers, and that read is the
// time.  A block has 16 columns of the result and 16 F tokens; its WAVES wavefronts take pieces of 128 bytes of the
// rows in turn and join their sums in LDS.  (Weights are the first factor of the 16 x 16 x 64 products: a
// lane then holds four neighbouring columns of one token.)  1 x 4096 x 4096 takes 5.3 us, 6.3 with the weights in no cache, of
// which 3.4 are their 16.8 MB at a large copy's rate, 5.0 TB/s; 1 x 8192 x 8192 14.6 us, 4.6 TB/s; 48 x 3277 x 3541 7.6 and 9.6 us.
// Four pieces of each wavefront are under way: 16 KB to 64 KB a block.
template <typename T, uint32_t F, uint32_t WAVES>
__global__ __launch_bounds__(64 * WAVES) void q8_product_few_kernel(Q8ProductArgs g) {
    constexpr uint32_t PIECE = 128, DEPTH = 4;                           // bytes; pieces under way
    __shared__ v4i s_sum[WAVES][F][64];
    const uint32_t lane = threadIdx.x & 63u, wave = uniform_u32(threadIdx.x >> 6);
    const uint32_t n0 = blockIdx.x * 16u, m0 = blockIdx.y * 16u * F, at = lane / 16u * UNIT;
    const int8_t* b = g.b + (uint64_t)min(n0 + (lane & 15u), g.n - 1u) * g.ld_b;
    const int8_t* a[F];
#pragma unroll
    for (uint32_t f = 0; f < F; ++f) a[f] = g.a + (uint64_t)min(m0 + 16u * f + (lane & 15u), g.m - 1u) * g.ld_a;
    v4i acc[F];
#pragma unroll
    for (uint32_t f = 0; f < F; ++f) acc[f] = v4i{0, 0, 0, 0};
    // what the sums are finished with is on its way while they are made
    const uint32_t m = m0 + wave * 16u + (lane & 15u), n = n0 + lane / 16u * 4u;
    float sa = 0.0f, sb[4], bias[4];
    if (wave < F) {
        sa = g.sa[min(m, g.m - 1u)];
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
            sb[e] = g.sb[min(n + e, g.n - 1u)];
            bias[e] = g.bias ? g.bias[min(n + e, g.n - 1u)] : 0.0f;
        }
    }
    const uint32_t whole = g.k / PIECE, pieces = (g.k + PIECE - 1u) / PIECE;
    uint32_t p = wave;
    // D pieces, `ends`: the row may end in or before them
    auto round = [&](auto depth, auto ends) {
        constexpr uint32_t D = depth.value;
        v4i vb[D][2], va[D][F][2];
#pragma unroll
        for (uint32_t d = 0; d < D; ++d)
#pragma unroll
            for (uint32_t x = 0; x < 2; ++x) {
                uint32_t k = (p + d * WAVES) * PIECE + x * 64u + at;
                if (ends.value) k = min(k, (g.k - 1u) & ~(UNIT - 1u));   // behind the row's end: its last unit again
                vb[d][x] = *reinterpret_cast<const v4i*>(b + k);
#pragma unroll
                for (uint32_t f = 0; f < F; ++f) va[d][f][x] = *reinterpret_cast<const v4i*>(a[f] + k);
            }
#pragma unroll
        for (uint32_t d = 0; d < D; ++d)
#pragma unroll
            for (uint32_t x = 0; x < 2; ++x) {
                if (ends.value) {                                        // bytes behind it count as zero
                    const int32_t left = (int32_t)g.k - (int32_t)((p + d * WAVES) * PIECE + x * 64u + at);
#pragma unroll
                    for (int32_t e = 0; e < 4; ++e) {
                        const int32_t c = min(max(left - 4 * e, 0), 4), keep = c == 4 ? -1 : (1 << (8 * c)) - 1;
                        vb[d][x][e] &= keep;
                    }
                }
#pragma unroll
                for (uint32_t f = 0; f < F; ++f)
                    acc[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vb[d][x], va[d][f][x], acc[f], 0, 0, 0);
            }
        p += D * WAVES;
    };
    while (p + (DEPTH - 1u) * WAVES < whole) round(std::integral_constant<uint32_t, DEPTH>{}, std::false_type{});
    while (p < pieces) {
        if (p + 2u * WAVES < pieces) round(std::integral_constant<uint32_t, DEPTH>{}, std::true_type{});
        else if (p + WAVES < pieces) round(std::integral_constant<uint32_t, 2>{}, std::true_type{});
        else round(std::integral_constant<uint32_t, 1>{}, std::true_type{});
    }
#pragma unroll
    for (uint32_t f = 0; f < F; ++f) s_sum[wave][f][lane] = acc[f];
    __syncthreads();
    static_assert(WAVES >= F, "a wavefront for 16 tokens' sums");
    if (wave >= F) return;
    v4i sum = s_sum[0][wave][lane];
#pragma unroll
    for (uint32_t w = 1; w < WAVES; ++w) sum += s_sum[w][wave][lane];
    if (m >= g.m) return;
    T* c = static_cast<T*>(g.c) + (uint64_t)m * g.ld_c + n;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
        if (n + e >= g.n) break;
        float v = fmaf((float)sum[e] * sa, sb[e], bias[e]);
        if (g.relu) v = v < 0.0f ? 0.0f : v;
        c[e] = (T)v;
    }
}

template <typename T, uint32_t F, uint32_t WAVES>
static void launch_product_few(shifter_ctx* ctx, const Q8ProductArgs& g) {
    q8_product_few_kernel<T, F, WAVES><<<dim3((g.n + 15u) / 16u, (g.m + 16u * F - 1u) / (16u * F)), 64 * WAVES, 0, ctx->stream>>>(g);
}

template <typename T>
static void launch_product_of(shifter_ctx* ctx, const Q8ProductArgs& g) {
    switch (q8_kernel_for(g.m, g.n, g.k)) {
        case Q8_FEW:
        case Q8_GROUPS: {
            const uint32_t f = q8_group(g.m, g.n);
            // long rows and a block a compute unit: more wavefronts (1 x 4096 x 14336 14.1 -> 13.6 us, 8 x 1024 x 16384 15.6 -> 14.5;
            // but 1 x 8192 x 4200 9.0 -> 10.0, 16 x 8192 x 8192 20.1 -> 20.5)
            if (f == 1 && g.k >= 8192 && q8_group_blocks(g.m, g.n, 1) <= 256u) launch_product_few<T, 1, 16>(ctx, g);
            else if (f == 1) launch_product_few<T, 1, 8>(ctx, g);
            else if (f == 2) launch_product_few<T, 2, 16>(ctx, g);
            else launch_product_few<T, 3, 16>(ctx, g);
            break;
        }
        case Q8_TILE_64x64: launch_product_as<T, 2, 2, 1, 1, 4, 128, 16>(ctx, g); break;
        case Q8_TILE_64x128: launch_product_as<T, 2, 4, 1, 1, 3, 128, 8>(ctx, g); break;
        case Q8_TILE_128x128: launch_product_as<T, 2, 4, 2, 1, 3, 128, 8>(ctx, g); break;
        case Q8_TILE_128x256: launch_product_as<T, 2, 4, 2, 2, 3, 128, 8>(ctx, g); break;
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

// Four words of four bytes, turned: byte i of word j becomes byte j of word i.
__device__ __forceinline__ void turn_bytes(uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
    const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
    const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
    a = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
    b = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
    c = __builtin_amdgcn_perm(cd1, ab1, 0x05040100u);
    d = __builtin_amdgcn_perm(cd1, ab1, 0x07060302u);
}

constexpr uint32_t TURN_ROWS = 128, TURN_PITCH = TURN_ROWS / 4 + 1;      // words of a turned row in LDS

// `rows` turned rows of 128 bytes from LDS to memory, 16 bytes a thread of 256.
__device__ __forceinline__ void store_turned(uint32_t tid, const uint32_t* s, uint32_t rows, int8_t* to, uint64_t ld) {
    for (uint32_t i = tid; i < rows * 8u; i += BLOCK) {
        const uint32_t* w = s + (i / 8u) * TURN_PITCH + (i & 7u) * 4u;
        *reinterpret_cast<uint4*>(to + (uint64_t)(i / 8u) * ld + (i & 7u) * 16u) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// 128 columns and 128 rows of the checkpoint, turned, by each 256 threads of a block: a thread has 16 columns of
// four rows.  lds: 128 rows of TURN_PITCH words for each.
template <uint32_t THREADS>
__device__ __forceinline__ void turn_codes(const Q8GradientArgs& a, const Q8GradientPlan& pl, uint32_t block, uint32_t* lds) {
    const uint32_t across = (a.k + 127u) / 128u, tid = threadIdx.x % BLOCK, group = threadIdx.x / BLOCK;
    const uint32_t tile = block * (THREADS / BLOCK) + group;
    const bool there = tile < across * (uint32_t)(pl.ld / TURN_ROWS);
    const uint32_t k0 = tile % across * 128u, m0 = tile / across * TURN_ROWS;
    const uint32_t kg = tid & 7u, rg = tid >> 3, k = k0 + kg * 16u;
    lds += group * (128u * TURN_PITCH);
    uint32_t w[4][4];                                                    // [row][word of its columns]
#pragma unroll
    for (uint32_t r = 0; r < 4; ++r) {
        const uint32_t m = m0 + rg * 4u + r;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (there && m < a.m && k < a.k) v = *reinterpret_cast<const uint4*>(a.q + (uint64_t)m * a.ld_q + k);
        w[r][0] = v.x; w[r][1] = v.y; w[r][2] = v.z; w[r][3] = v.w;
    }
#pragma unroll
    for (uint32_t x = 0; x < 4; ++x) {
        turn_bytes(w[0][x], w[1][x], w[2][x], w[3][x]);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) lds[(kg * 16u + x * 4u + i) * TURN_PITCH + rg] = w[i][x];
    }
    __syncthreads();
    if (there)
        store_turned(tid, lds, min(128u, a.k - k0), reinterpret_cast<int8_t*>(a.work + pl.codes) + (uint64_t)k0 * pl.ld + m0, pl.ld);
}

// What a column's digits are made with, from its largest |p|.  No factor: zeros, or a column that is not finite.
struct ColumnScale {
    float up, factor;
    ColumnScale() = default;
    __device__ __forceinline__ explicit ColumnScale(uint32_t top) {
        const float c = __uint_as_float(top);
        up = digits_up(c);
        // a little less than the quotient, so that the largest p stays at DIGITS_TOP with both roundings
        factor = top == 0u || top >= 0x7f800000u ? 0.0f : DIGITS_TOP / (c * up) * (1.0f - 0x1p-22f);
    }
    // 0x808080 + the whole number of p: with 128 added to each, the balanced digits are the number's bytes
    __device__ __forceinline__ uint32_t operator()(float p) const {
        // a column that is not finite has factor 0; its NaN become some number, in their own column alone
        return (uint32_t)((int32_t)rintf(__fmul_rn(__fmul_rn(p, up), factor)) + 0x808080);
    }
    // what a whole number of 1 stands for, without `up`; NaN for a column that is not finite
    __device__ __forceinline__ static float unit(uint32_t top) {
        return top >= 0x7f800000u ? __uint_as_float(0x7fc00000u)
                                  : __uint_as_float(top) * digits_up(__uint_as_float(top)) / DIGITS_TOP * (1.0f + 0x1p-22f);
    }
};

// Four of its numbers as the digits' three words, the first number's in the lowest bytes.
__device__ __forceinline__ void digit_words(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t& d0, uint32_t& d1, uint32_t& d2) {
    const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x05010400u), cd = __builtin_amdgcn_perm(d, c, 0x05010400u);
    d0 = __builtin_amdgcn_perm(cd, ab, 0x05040100u) ^ 0x80808080u;
    d1 = __builtin_amdgcn_perm(cd, ab, 0x07060302u) ^ 0x80808080u;
    const uint32_t hi = __builtin_amdgcn_perm(b, a, 0x0c0c0602u), lo = __builtin_amdgcn_perm(d, c, 0x06020c0cu);
    d2 = (hi | lo) ^ 0x80808080u;
}

// Digits of 16 columns and all rows by a block that holds them in registers, eight columns of four rows a thread: g is
// read once, and what a thread has of a column leaves as four bytes.  Neighbouring blocks, which share lines of g, are
// on one chiplet.  Behind the blocks for digits come those that turn the checkpoint.  300 x 1100 with 1000 columns of checkpoint
// takes 5 us, little more than a launch; 2048 x 1873 (bf16, odd stride) and 977 12 to 14 us for 23 MB, 1.8 TB/s: 118 blocks for
// digits and 32 for the checkpoint leave units idle; 2048 x 4096 and 4096 13.5 us for 58 MB, 4.3 TB/s.
template <typename T, uint32_t THREADS>
__global__ __launch_bounds__(THREADS) void q8_columns_kernel(Q8GradientArgs a, Q8GradientPlan pl, uint32_t blocks) {
    constexpr uint32_t COLS = 16, DEEP = 4;                              // a block's columns, a thread's rows
    static_assert(THREADS / 2 * DEEP <= Q8_WHOLE_ROWS, "all rows");
    __shared__ uint32_t lds[THREADS / BLOCK * 128 * TURN_PITCH];
    if (blockIdx.x >= blocks) return turn_codes<THREADS>(a, pl, blockIdx.x - blocks, lds);
    const uint32_t xcd = blockIdx.x % 8u, block = xcd * (blocks / 8u) + min(xcd, blocks % 8u) + blockIdx.x / 8u;
    const uint32_t cg = threadIdx.x % 2u, m0 = threadIdx.x / 2u * DEEP, n = block * COLS + cg * 8u;
    Eight<T> e[DEEP];
    float s[DEEP];
#pragma unroll
    for (uint32_t r = 0; r < DEEP; ++r) {
        const uint32_t m = min(m0 + r, a.m - 1u);                        // behind the last one: it again
        fetch8(static_cast<const T*>(a.g) + (uint64_t)m * a.ld_g, n, a.n, e[r]);
        s[r] = a.s[m];
    }
    if (threadIdx.x < COLS) lds[threadIdx.x] = 0;
    __syncthreads();
    uint32_t top[8] = {};
#pragma unroll
    for (uint32_t r = 0; r < DEEP; ++r) {
        float f[8];
        place8(n, a.n, e[r]);
        e[r].floats(f);
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) top[i] = max(top[i], key_of(__fmul_rn(f[i], s[r])));
    }
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {                                   // lanes of the same columns: every other one
        top[i] = max(top[i], (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top[i], 0x4E, 0xf, 0xf, true));
        top[i] = max(top[i], (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top[i], 0x124, 0xf, 0xf, true));
        top[i] = max(top[i], (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top[i], 0x128, 0xf, 0xf, true));
        if ((threadIdx.x & 15u) < 2u) atomicMax(&lds[cg * 8u + i], top[i]);
    }
    __syncthreads();
    float* s_scale = reinterpret_cast<float*>(lds + COLS);               // factor and up of every column
    if (threadIdx.x < COLS) {
        const ColumnScale scale(lds[threadIdx.x]);
        s_scale[2u * threadIdx.x] = scale.factor;
        s_scale[2u * threadIdx.x + 1u] = scale.up;
        if (block * COLS + threadIdx.x < a.n) reinterpret_cast<uint32_t*>(a.work + pl.tops)[block * COLS + threadIdx.x] = lds[threadIdx.x];
    }
    __syncthreads();
    if (m0 >= (uint32_t)pl.ld) return;
    int8_t* out = reinterpret_cast<int8_t*>(a.work + pl.digits) + m0;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        if (n + i >= a.n) break;
        ColumnScale scale;
        scale.factor = s_scale[2u * (cg * 8u + i)];
        scale.up = s_scale[2u * (cg * 8u + i) + 1u];
        uint32_t u[DEEP];
#pragma unroll
        for (uint32_t r = 0; r < DEEP; ++r) {
            float f[8];
            e[r].floats(f);
            u[r] = scale(m0 + r < a.m ? __fmul_rn(f[i], s[r]) : 0.0f);       // rows behind the last one count as zero
        }
        uint32_t d[3];
        digit_words(u[0], u[1], u[2], u[3], d[0], d[1], d[2]);
#pragma unroll
        for (uint32_t p = 0; p < 3; ++p)
            *reinterpret_cast<uint32_t*>(out + ((uint64_t)p * a.n + n + i) * pl.ld) = d[p];
    }
}

// Largest |p| of eight columns over the rows from r0 on, every `step`-th.  As magnitudes' bits: infinity and NaN are on top.
template <typename T>
__device__ __forceinline__ void column_tops(const Q8GradientArgs& a, uint32_t n, uint32_t r0, uint32_t r1, uint32_t step, uint32_t (&top)[8]) {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) top[i] = 0;
    if (n >= a.n) return;
    const T* g = static_cast<const T*>(a.g);
    for (uint32_t r = r0; r < r1; r += 8u * step) {                      // eight rows under way
        Eight<T> e[8];
        float s[8];
#pragma unroll
        for (uint32_t x = 0; x < 8; ++x) {
            const uint32_t at = min(r + x * step, r1 - 1u);              // behind the last one: it again
            fetch8(g + (uint64_t)at * a.ld_g, n, a.n, e[x]);
            s[x] = a.s[at];
        }
#pragma unroll
        for (uint32_t x = 0; x < 8; ++x) {
            float f[8];
            place8(n, a.n, e[x]);
            e[x].floats(f);
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) top[i] = max(top[i], key_of(__fmul_rn(f[i], s[x])));
        }
    }
}

// The columns' largest over one slice of rows, 512 columns a block and eight a thread; behind those blocks, the
// ones that turn the checkpoint.  16384 x 4096 bf16 and as much checkpoint take 52 to 58 us: 271 MB, 5 TB/s.
template <typename T>
__global__ __launch_bounds__(BLOCK) void q8_tops_kernel(Q8GradientArgs a, Q8GradientPlan pl, uint32_t blocks) {
    __shared__ uint32_t lds[128 * TURN_PITCH];
    if (blockIdx.x >= blocks) return turn_codes<BLOCK>(a, pl, blockIdx.x - blocks, lds);
    const uint32_t across = blocks / pl.slices, slice = blockIdx.x / across, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t n = blockIdx.x % across * 512u + lane * 8u, r0 = slice * pl.slice_rows;
    uint32_t top[8];
    column_tops<T>(a, n, r0 + wave, min(r0 + pl.slice_rows, a.m), BLOCK / 64u, top);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) lds[(wave * 8u + i) * 64u + lane] = top[i];
    __syncthreads();
    if (wave != 0) return;
    uint32_t* to = reinterpret_cast<uint32_t*>(a.work + pl.slice_tops) + (uint64_t)slice * a.n;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        for (uint32_t w = 1; w < BLOCK / 64u; ++w) top[i] = max(top[i], lds[(w * 8u + i) * 64u + lane]);
        if (n + i < a.n) to[n + i] = top[i];
    }
}

// The digits of 64 columns and `deep` times 128 rows, the rows of a column side by side: a thread has eight columns
// of four rows at a time, and the next ones on their way while it works.  g is read again here because a column's unit is not
// known before its last row: 16384 x 4096 bf16 takes 68 to 73 us, 341 MB, 4.8 TB/s.
template <typename T>
__global__ __launch_bounds__(BLOCK) void q8_digits_kernel(Q8GradientArgs a, Q8GradientPlan pl, uint32_t deep) {
    __shared__ uint32_t lds[3 * 64 * TURN_PITCH];
    __shared__ uint32_t s_top[64];
    const uint32_t across = (a.n + 63u) / 64u, n0 = blockIdx.x % across * 64u;
    const uint32_t first = blockIdx.x / across * deep * TURN_ROWS, last = min(first + deep * TURN_ROWS, (uint32_t)pl.ld);
    const uint32_t cg = threadIdx.x & 7u, rg = threadIdx.x >> 3, n = n0 + cg * 8u;
    Eight<T> e[4];
    float s[4];
    auto fetch = [&](uint32_t m0) {
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) {
            const uint32_t m = min(m0 + rg * 4u + r, a.m - 1u);              // behind the last one: it again
            fetch8(static_cast<const T*>(a.g) + (uint64_t)m * a.ld_g, n, a.n, e[r]);
            s[r] = a.s[m];
        }
    };
    fetch(first);
    if (threadIdx.x < 64u) s_top[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t* tops = reinterpret_cast<const uint32_t*>(a.work + pl.slice_tops);
    const uint32_t col = threadIdx.x & 63u;
    if (n0 + col < a.n) {
        uint32_t top = 0;
#pragma unroll 8
        for (uint32_t x = threadIdx.x / 64u; x < pl.slices; x += BLOCK / 64u) top = max(top, tops[(uint64_t)x * a.n + n0 + col]);
        atomicMax(&s_top[col], top);
    }
    __syncthreads();
    if (first == 0 && threadIdx.x < 64u && n0 + threadIdx.x < a.n)
        reinterpret_cast<uint32_t*>(a.work + pl.tops)[n0 + threadIdx.x] = s_top[threadIdx.x];
    int8_t* out = reinterpret_cast<int8_t*>(a.work + pl.digits);
    const ColumnScale scale[8] = {ColumnScale(s_top[cg * 8u]), ColumnScale(s_top[cg * 8u + 1u]), ColumnScale(s_top[cg * 8u + 2u]),
                                  ColumnScale(s_top[cg * 8u + 3u]), ColumnScale(s_top[cg * 8u + 4u]), ColumnScale(s_top[cg * 8u + 5u]),
                                  ColumnScale(s_top[cg * 8u + 6u]), ColumnScale(s_top[cg * 8u + 7u])};
    for (uint32_t m0 = first; m0 < last; m0 += TURN_ROWS) {
        uint32_t u[4][8];
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) {
            const bool there = m0 + rg * 4u + r < a.m;                       // rows behind the last one count as zero
            float f[8];
            place8(n, a.n, e[r]);
            e[r].floats(f);
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) u[r][i] = scale[i](there ? __fmul_rn(f[i], s[r]) : 0.0f);
        }
        if (m0 + TURN_ROWS < last) fetch(m0 + TURN_ROWS);
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            uint32_t d[3];
            digit_words(u[0][i], u[1][i], u[2][i], u[3][i], d[0], d[1], d[2]);
#pragma unroll
            for (uint32_t p = 0; p < 3; ++p) lds[(p * 64u + cg * 8u + i) * TURN_PITCH + rg] = d[p];
        }
        __syncthreads();
#pragma unroll
        for (uint32_t p = 0; p < 3; ++p)
            store_turned(threadIdx.x, lds + p * 64u * TURN_PITCH, min(64u, a.n - n0), out + ((uint64_t)p * a.n + n0) * pl.ld + m0, pl.ld);
        __syncthreads();
    }
}

// A wavefront's 32 rows x COLS values of LDS to dw, under the mask, or added to it.
template <uint32_t COLS>
__device__ __forceinline__ void store_gradient(const int8_t* from, uint32_t pitch, const Q8GradientArgs& g, uint32_t n0, uint32_t k0) {
    constexpr uint32_t LANES = COLS / 4;
    typedef float vec __attribute__((ext_vector_type(4)));
    typedef float loose __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t lane = threadIdx.x & 63u, k = k0 + lane % LANES * 4u;
    if (k >= g.k) return;
    const bool whole = k + 4u <= g.k;
#pragma unroll 4
    for (uint32_t r = lane / LANES; r < 32u; r += 64u / LANES) {
        vec v = *reinterpret_cast<const vec*>(from + r * pitch + (k - k0) * 4u);
        const uint32_t n = n0 + r;
        if (n >= g.n) continue;
        float* to = g.dw + (uint64_t)n * g.ld_dw + k;
        const uint8_t* mask = g.mask + (uint64_t)n * g.ld_mask + k;
        if (whole) {
            uint32_t keep = 0xffffffffu;
            if (g.mask) keep = *reinterpret_cast<const u32_a1*>(mask);
            vec old = {0.0f, 0.0f, 0.0f, 0.0f};
            if (g.accumulate) old = *reinterpret_cast<const loose*>(to);
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) v[i] = keep >> (8u * i) & 255u ? (g.accumulate ? old[i] + v[i] : v[i]) : old[i];
            *reinterpret_cast<loose*>(to) = v;
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                if (k + i >= g.k) break;
                const float old = g.accumulate ? to[i] : 0.0f;
                to[i] = !g.mask || mask[i] ? (g.accumulate ? old + v[i] : v[i]) : old;
            }
        }
    }
}

// dW[n][k] = unit[n] (2^16 D2 + 2^8 D1 + D0), Dp the exact sum of digit plane p of column n times column k of the codes.  One
// tile of Q serves the three planes, whose sums all stay in registers: 128 x 256 of them fill eight wavefronts' 192
// accumulators.  16384 x 4096 x 4096 takes 640 to 690 us, 2.5 POP/s over the three products: the matrix units are busy in 69 % of
// the cycles, at 1.73 GHz as in the product, and LDS reads do not conflict.  2048 x 1873 x 977 takes 20 to 22 us on tiles of 64 x 128,
// one on a compute unit, the matrix units busy in 36 % of its cycles and the LDS in 27 %: eight wavefronts, of which one reads while
// another multiplies, take 17.2 us on random digits where four of 64 x 64 take 18.8; the rest is a launch, the digits' and the mask's way from memory.
template <uint32_t WA, uint32_t WB, uint32_t FA, uint32_t FB, uint32_t NS, uint32_t STEP, uint32_t GROUP>
__global__ __launch_bounds__(64 * WA * WB) void q8_gradient_kernel(Q8GradientArgs g, Q8GradientPlan pl) {

    using Tl = Tile<3, WA, WB, FA, FB, NS, STEP>;
    constexpr uint32_t PITCH = Tl::COLS * 4u + 16u, OUT = WA * WB * 32u * PITCH, BEHIND = OUT + 8u * Tl::RA;
    __shared__ __align__(16) int8_t lds[Tl::LDS > BEHIND ? Tl::LDS : BEHIND];
    static_assert(Tl::THREADS >= Tl::RA, "a column's unit a thread");
    uint32_t ta, tb;
    tile_of_block<GROUP>((g.n + Tl::RA - 1u) / Tl::RA, (g.k + Tl::RB - 1u) / Tl::RB, &ta, &tb);
    const uint32_t n0 = ta * Tl::RA, k0 = tb * Tl::RB;
    const int8_t* digits = reinterpret_cast<const int8_t*>(g.work + pl.digits);
    const int8_t* codes = reinterpret_cast<const int8_t*>(g.work + pl.codes);
    const float top = reinterpret_cast<const float*>(g.work + pl.tops)[min(n0 + threadIdx.x % Tl::RA, g.n - 1u)];
    Tl t;
    const uint32_t m0 = blockIdx.y * pl.part_rows;
    t.run(digits + (uint64_t)n0 * pl.ld + m0, pl.ld, (uint64_t)g.n * pl.ld, g.n - n0, codes + (uint64_t)k0 * pl.ld + m0, pl.ld,
          g.k - k0, min(pl.part_rows, (uint32_t)pl.ld - m0), lds);
    if (pl.parts > 1) {                        // one part of the rows: its sums go to the workspace as they are
        g.dw = reinterpret_cast<float*>(g.work + pl.sums) + (uint64_t)blockIdx.y * g.n * g.k;
        g.ld_dw = g.k;
        g.mask = nullptr;
        g.accumulate = 0;
    }
    __syncthreads();
    float* s_unit = reinterpret_cast<float*>(lds + OUT);
    float* s_down = s_unit + Tl::RA;
    if (threadIdx.x < Tl::RA) {
        s_unit[threadIdx.x] = ColumnScale::unit(key_of(top));
        s_down[threadIdx.x] = digits_down(top);
    }
    __syncthreads();
    const uint32_t lane = threadIdx.x & 63u;
    int8_t* out = lds + uniform_u32(threadIdx.x >> 6) * 32u * PITCH;
#pragma unroll
    for (uint32_t i = 0; i < FA; ++i) {
#pragma unroll
        for (uint32_t e = 0; e < 16; ++e) {
            const uint32_t row = Tl::row(i, e);
            const float unit = s_unit[row], down = s_down[row];
#pragma unroll
            for (uint32_t j = 0; j < FB; ++j) {
                const float v = fmaf((float)t.acc[2][i][j][e], 65536.0f, fmaf((float)t.acc[1][i][j][e], 256.0f, (float)t.acc[0][i][j][e]));
                *reinterpret_cast<float*>(out + (8u * (e / 4u) + 4u * (lane >> 5) + (e & 3u)) * PITCH + (j * 32u + (lane & 31u)) * 4u) = v * unit * down;
            }
        }
        __builtin_amdgcn_wave_barrier();       // a wavefront's LDS accesses are done in order
        store_gradient<Tl::COLS>(out, PITCH, g, n0 + Tl::row(i, 0) - 4u * (lane >> 5), k0 + Tl::col(0) - (lane & 31u));
        __builtin_amdgcn_wave_barrier();
    }
}

typedef double v4d __attribute__((ext_vector_type(4)));

// Little work: one launch, no digits and no workspace, 64-bit products on the matrix units (as fast as the vector units', but
// an operand serves 16 of them), in which a p times a code is exact.  A block has 16 FA columns of g and 16 FB of the
// checkpoint; its WAVES wavefronts take 16 rows in turn, read straight into registers, the next ones on their way while these
// are multiplied, and join their sums in LDS.  64 x 512 x 512 takes 3.3 us, little more than a launch; 300 x 300 x 300 4.4,
// 512 x 512 x 512 9.5,
// where the matrix units' rate and the conversions bound it: as fast with 32 rows a turn.
template <typename T, uint32_t FA, uint32_t FB, uint32_t WAVES>
__global__ __launch_bounds__(64 * WAVES) void q8_gradient_small_kernel(Q8GradientArgs a) {
    constexpr uint32_t ROWS = 16, STEPS = ROWS / 4;                      // of a turn; four rows a step
    typedef uint8_t codes __attribute__((ext_vector_type(FB), aligned(FB)));
    __shared__ double s_sum[WAVES][FA * 4][FB][64];
    const uint32_t across = (a.k + 16u * FB - 1u) / (16u * FB), n0 = blockIdx.x / across * (16u * FA), k0 = blockIdx.x % across * (16u * FB);
    const uint32_t lane = threadIdx.x & 63u, wave = uniform_u32(threadIdx.x >> 6), col = lane & 15u, row = lane / 16u;
    const uint32_t k = k0 + col * FB, pad = (a.k + Q8_ALIGN - 1u) & ~(Q8_ALIGN - 1u);
    const int8_t* q = a.q + min(k, pad - FB);                            // columns behind the last one: in the row's padding
    const T* g[FA];
#pragma unroll
    for (uint32_t i = 0; i < FA; ++i) g[i] = static_cast<const T*>(a.g) + min(n0 + 16u * i + col, a.n - 1u);
    T e[STEPS][FA];
    codes c[STEPS];
    float s[STEPS];
    auto fetch = [&](uint32_t from) {
#pragma unroll
        for (uint32_t x = 0; x < STEPS; ++x) {
            const uint64_t m = min(from + 4u * x + row, a.m - 1u);       // behind the last one: it again
#pragma unroll
            for (uint32_t i = 0; i < FA; ++i) e[x][i] = g[i][m * a.ld_g];
            c[x] = *reinterpret_cast<const codes*>(q + m * a.ld_q);
            s[x] = a.s[m];
        }
    };
    v4d acc[FA][FB];
#pragma unroll
    for (uint32_t i = 0; i < FA; ++i)
#pragma unroll
        for (uint32_t j = 0; j < FB; ++j) acc[i][j] = v4d{0.0, 0.0, 0.0, 0.0};
    uint32_t from = wave * ROWS;
    if (from < a.m) fetch(from);
    while (from < a.m) {
        double p[STEPS][FA], b[STEPS][FB];
#pragma unroll
        for (uint32_t x = 0; x < STEPS; ++x) {
            const bool there = from + 4u * x + row < a.m;                // rows behind the last one count as zero
#pragma unroll
            for (uint32_t i = 0; i < FA; ++i) p[x][i] = there ? (double)__fmul_rn((float)e[x][i], s[x]) : 0.0;
#pragma unroll
            for (uint32_t j = 0; j < FB; ++j) b[x][j] = (double)(int8_t)c[x][j];
        }
        from += WAVES * ROWS;
        if (from < a.m) fetch(from);
#pragma unroll
        for (uint32_t x = 0; x < STEPS; ++x)
#pragma unroll
            for (uint32_t i = 0; i < FA; ++i)
#pragma unroll
                for (uint32_t j = 0; j < FB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f64_16x16x4f64(p[x][i], b[x][j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (uint32_t i = 0; i < FA; ++i)
#pragma unroll
        for (uint32_t j = 0; j < FB; ++j)
#pragma unroll
            for (uint32_t x = 0; x < 4; ++x) s_sum[wave][i * 4u + x][j][lane] = acc[i][j][x];
    __syncthreads();
    // row 4 x + lane / 16 of 16 is in the x-th number of a lane
#pragma unroll
    for (uint32_t u = 0; u < FA * 4u; u += WAVES) {
        const uint32_t at = u + wave;
        if (at >= FA * 4u) break;
        double sum[FB];
#pragma unroll
        for (uint32_t j = 0; j < FB; ++j) {
            sum[j] = s_sum[0][at][j][lane];
#pragma unroll
            for (uint32_t w = 1; w < WAVES; ++w) sum[j] += s_sum[w][at][j][lane];
        }
        const uint32_t n = n0 + at / 4u * 16u + at % 4u * 4u + row;
        if (n >= a.n || k >= a.k) continue;
        float* to = a.dw + (uint64_t)n * a.ld_dw + k;
        const uint8_t* mask = a.mask + (uint64_t)n * a.ld_mask + k;
        float v[FB];
#pragma unroll
        for (uint32_t j = 0; j < FB; ++j) {
            // a column with a p that is not finite: NaN in the whole row, as where digits are made
            v[j] = isfinite(sum[j]) ? (float)sum[j] : __uint_as_float(0x7fc00000u);
            if (k + j >= a.k) continue;
            const float old = a.accumulate ? to[j] : 0.0f;
            v[j] = !a.mask || mask[j] ? (a.accumulate ? old + v[j] : v[j]) : old;
        }
        if (k + FB <= a.k) {
            typedef float loose __attribute__((ext_vector_type(FB), aligned(4)));
            loose w;
#pragma unroll
            for (uint32_t j = 0; j < FB; ++j) w[j] = v[j];
            *reinterpret_cast<loose*>(to) = w;
        } else {
#pragma unroll
            for (uint32_t j = 0; j < FB; ++j)
                if (k + j < a.k) to[j] = v[j];
        }
    }
}

// Up to 16 rows and a large dW, whose writing is the time: a block has 16 columns of g, their p in LDS, and 256 of the
// checkpoint; a thread 4 x 4 of the sums, 64-bit on the vector units.  1 x 4096 x 4096 15.5 us, the 67 MB of dW at 4.3 TB/s
// (25 with the kernel above and a wavefront a block).
template <typename T>
__global__ __launch_bounds__(BLOCK) void q8_gradient_wide_kernel(Q8GradientArgs a) {
    constexpr uint32_t I = 4, COLS = 4 * I, DEEP = Q8_WIDE_ROWS;
    __shared__ double s_p[DEEP][COLS];
    const uint32_t across = (a.k + 255u) / 256u, n0 = blockIdx.x / across * COLS, k0 = blockIdx.x % across * 256u;
    const uint32_t lane = threadIdx.x & 63u, wave = uniform_u32(threadIdx.x >> 6), k = k0 + lane * 4u;
    const bool there = k < a.k;                                          // the codes behind the last column are in the row's padding
    uint32_t q[DEEP];
#pragma unroll
    for (uint32_t r = 0; r < DEEP; ++r)
        q[r] = there && a.m ? *reinterpret_cast<const uint32_t*>(a.q + (uint64_t)min(r, a.m - 1u) * a.ld_q + k) : 0u;
    static_assert(DEEP * COLS == BLOCK, "a p a thread");
    const uint32_t m = threadIdx.x / COLS, c = threadIdx.x % COLS;
    float mine = 0.0f;                                                   // rows behind the last one count as zero
    if (m < a.m) mine = __fmul_rn((float)static_cast<const T*>(a.g)[(uint64_t)m * a.ld_g + min(n0 + c, a.n - 1u)], a.s[m]);
    s_p[m][c] = (double)mine;
    __syncthreads();
    double acc[I][4] = {};
#pragma unroll
    for (uint32_t r = 0; r < DEEP; ++r) {
        if (r % 4u == 0 && r >= a.m) break;
        double p[I];
#pragma unroll
        for (uint32_t i = 0; i < I; ++i) p[i] = s_p[r][wave * I + i];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const double c = (double)(int8_t)(q[r] >> (8u * j));
#pragma unroll
            for (uint32_t i = 0; i < I; ++i) acc[i][j] = fma(p[i], c, acc[i][j]);
        }
    }
    if (!there) return;
#pragma unroll
    for (uint32_t i = 0; i < I; ++i) {
        const uint32_t n = n0 + wave * I + i;
        if (n >= a.n) break;
        float* to = a.dw + (uint64_t)n * a.ld_dw + k;
        const uint8_t* mask = a.mask + (uint64_t)n * a.ld_mask + k;
        typedef float loose __attribute__((ext_vector_type(4), aligned(4)));
        float v[4];
        uint32_t keep = 0xffffffffu;
        const bool whole = k + 4u <= a.k;
        if (a.mask) {
            keep = 0;
            if (whole) keep = *reinterpret_cast<const u32_a1*>(mask);
            else
                for (uint32_t j = 0; k + j < a.k; ++j) keep |= (uint32_t)mask[j] << (8u * j);
        }
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            // a column with a p that is not finite: NaN in the whole row, as where digits are made
            v[j] = isfinite(acc[i][j]) ? (float)acc[i][j] : __uint_as_float(0x7fc00000u);
            const float old = a.accumulate && k + j < a.k ? to[j] : 0.0f;
            v[j] = keep >> (8u * j) & 255u ? (a.accumulate ? old + v[j] : v[j]) : old;
        }
        if (whole) *reinterpret_cast<loose*>(to) = loose{v[0], v[1], v[2], v[3]};
        else
            for (uint32_t j = 0; k + j < a.k; ++j) to[j] = v[j];
    }
}

template <typename T, uint32_t FA, uint32_t FB, uint32_t WAVES>
static void launch_gradient_small_as(shifter_ctx* ctx, const Q8GradientArgs& g) {
    const uint64_t blocks = (uint64_t)((g.n + 16u * FA - 1u) / (16u * FA)) * ((g.k + 16u * FB - 1u) / (16u * FB));
    q8_gradient_small_kernel<T, FA, FB, WAVES><<<(uint32_t)blocks, 64 * WAVES, 0, ctx->stream>>>(g);
}
template <typename T>
static void launch_gradient_small(shifter_ctx* ctx, const Q8GradientArgs& g, Q8GradientKernel kernel) {
    ProfileScope ps(ctx, K_Q8_GRADIENT);
    if (kernel == Q8_GRAD_WIDE) {
        const uint64_t blocks = (uint64_t)((g.n + 15u) / 16u) * ((g.k + 255u) / 256u);
        q8_gradient_wide_kernel<T><<<(uint32_t)blocks, BLOCK, 0, ctx->stream>>>(g);
    } else if ((uint64_t)((g.n + 15u) / 16u) * ((g.k + 15u) / 16u) <= 256u) {
        // a narrowest block a compute unit, up to four narrow ones, then wider ones: us with 16 x 16, 16 x 32 and 32 x 32 results,
        // 1000 x 100 x 200 7.1 8.9 19, 2000 x 250 x 260 20 16 35, 64 x 512 x 512 3.6 3.4 3.7, 300 x 300 x 300 5.0 4.5 7.5,
        // 64 x 1024 x 1024 9.1 7.1 6.5, 128 x 1024 x 1024 13 11 9.2
        launch_gradient_small_as<T, 1, 1, 8>(ctx, g);
    } else if ((uint64_t)((g.n + 15u) / 16u) * ((g.k + 31u) / 32u) <= 1024u) {
        launch_gradient_small_as<T, 1, 2, 8>(ctx, g);
    } else {
        launch_gradient_small_as<T, 2, 2, 4>(ctx, g);
    }
}

template <typename T, uint32_t THREADS>
static void launch_columns(shifter_ctx* ctx, const Q8GradientArgs& g, const Q8GradientPlan& pl) {
    const uint32_t blocks = (uint32_t)q8_columns_blocks(g.n);
    q8_columns_kernel<T, THREADS><<<blocks + (uint32_t)q8_turn_blocks(g.k, pl.ld, THREADS), THREADS, 0, ctx->stream>>>(g, pl, blocks);
}

template <typename T>
static void launch_digits(shifter_ctx* ctx, const Q8GradientArgs& g, const Q8GradientPlan& pl) {
    if (g.m <= Q8_WHOLE_ROWS) {
        const uint32_t threads = q8_columns_threads(pl.ld);
        if (threads == 256) return launch_columns<T, 256>(ctx, g, pl);
        if (threads == 512) return launch_columns<T, 512>(ctx, g, pl);
        return launch_columns<T, 1024>(ctx, g, pl);
    }
    const uint32_t tops = (uint32_t)q8_tops_blocks(g.n, pl.slices);
    q8_tops_kernel<T><<<tops + (uint32_t)q8_turn_blocks(g.k, pl.ld, BLOCK), BLOCK, 0, ctx->stream>>>(g, pl, tops);
    q8_digits_kernel<T><<<(uint32_t)q8_digits_blocks(g.n, pl.ld), BLOCK, 0, ctx->stream>>>(g, pl, q8_digits_deep(g.n, pl.ld));
}

// The parts' sums joined, in 64 bits so that only the parts' own roundings count; under the mask, or added to dw.
// One pass over parts x n x k fp32 that are mostly still in cache: q8_join_us, 3.5 us and 2 us per million of them.
__global__ __launch_bounds__(BLOCK) void q8_join_kernel(Q8GradientArgs g, Q8GradientPlan pl) {
    const float* sums = reinterpret_cast<const float*>(g.work + pl.sums);
    const uint64_t all = (uint64_t)g.n * g.k;
    for (uint64_t i = ((uint64_t)blockIdx.x * BLOCK + threadIdx.x) * 4u; i < all; i += (uint64_t)gridDim.x * BLOCK * 4u) {
        double v[4] = {0.0, 0.0, 0.0, 0.0};
        const uint32_t there = (uint32_t)min(all - i, (uint64_t)4u);
#pragma unroll 4
        for (uint32_t p = 0; p < pl.parts; ++p) {
            const float* from = sums + p * all + i;
            if (there == 4u) {
                const uint4 f = load_u4<false>(from);
                v[0] += __uint_as_float(f.x); v[1] += __uint_as_float(f.y); v[2] += __uint_as_float(f.z); v[3] += __uint_as_float(f.w);
            } else {
                for (uint32_t e = 0; e < there; ++e) v[e] += from[e];
            }
        }
        const uint64_t row = i / g.k;
        uint32_t k = (uint32_t)(i - row * g.k);
        float* to = g.dw + row * g.ld_dw;
        const uint8_t* mask = g.mask + row * g.ld_mask;
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
            if (e >= there) break;
            if (k == g.k) { k = 0; to += g.ld_dw; mask += g.ld_mask; }
            const float old = g.accumulate ? to[k] : 0.0f;
            to[k] = !g.mask || mask[k] ? (g.accumulate ? old + (float)v[e] : (float)v[e]) : old;
            ++k;
        }
    }
}

template <uint32_t WA, uint32_t WB, uint32_t FA, uint32_t FB, uint32_t NS, uint32_t STEP, uint32_t GROUP>
static void launch_gradient_as(shifter_ctx* ctx, const Q8GradientArgs& g, const Q8GradientPlan& pl) {
    using Tl = Tile<3, WA, WB, FA, FB, NS, STEP>;
    const uint64_t tiles = (uint64_t)((g.n + Tl::RA - 1u) / Tl::RA) * ((g.k + Tl::RB - 1u) / Tl::RB);
    q8_gradient_kernel<WA, WB, FA, FB, NS, STEP, GROUP><<<dim3((uint32_t)tiles, pl.parts), Tl::THREADS, 0, ctx->stream>>>(g, pl);
    if (pl.parts > 1)
        q8_join_kernel<<<(uint32_t)std::min<uint64_t>(((uint64_t)g.n * g.k + 4u * BLOCK - 1u) / (4u * BLOCK), 4096u), BLOCK, 0, ctx->stream>>>(g, pl);
}

void launch_q8_gradient(shifter_ctx* ctx, int dtype, const Q8GradientArgs& g) {
    const Q8GradientPlan pl = q8_gradient_plan(g.m, g.n, g.k);
    if (pl.kernel < 0) {
        if (dtype == SHIFTER_F32) launch_gradient_small<float>(ctx, g, pl.kernel);
        else if (dtype == SHIFTER_BF16) launch_gradient_small<__bf16>(ctx, g, pl.kernel);
        else launch_gradient_small<_Float16>(ctx, g, pl.kernel);
        return;
    }
    {
        ProfileScope ps(ctx, K_Q8_DIGITS);
        if (dtype == SHIFTER_F32) launch_digits<float>(ctx, g, pl);
        else if (dtype == SHIFTER_BF16) launch_digits<__bf16>(ctx, g, pl);
        else launch_digits<_Float16>(ctx, g, pl);
    }
    ProfileScope ps(ctx, K_Q8_GRADIENT);
    switch (pl.kernel) {
        case Q8_GRAD_64x64: launch_gradient_as<2, 2, 1, 1, 2, 128, 8>(ctx, g, pl); break;
        case Q8_GRAD_64x64_DEEP: launch_gradient_as<2, 2, 1, 1, 3, 128, 8>(ctx, g, pl); break;
        case Q8_GRAD_64x128: launch_gradient_as<2, 4, 1, 1, 2, 128, 8>(ctx, g, pl); break;
        case Q8_GRAD_64x128_DEEP: launch_gradient_as<2, 4, 1, 1, 3, 128, 8>(ctx, g, pl); break;
        case Q8_GRAD_64x256: launch_gradient_as<2, 4, 1, 2, 2, 128, 8>(ctx, g, pl); break;
        default: launch_gradient_as<4, 2, 1, 4, 4, 64, 4>(ctx, g, pl); break;
    }
}

}  // namespace shifter

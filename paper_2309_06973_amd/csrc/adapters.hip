// Low-rank adapters beside a projection that rows of many requests share:
//
//   out_r = y_r + c_i (x_r A_i') B_i',   i = which[r]
//
// and their gradients.  The product over the long side, s_r = c_i x_r A_i', is the narrow one: rank numbers a row, held in 32 bits.
// It is multiplied with B_i in all of these bits, so that out is rounded once.
//
// Rows are taken in tiles of 16 as they come, whatever requests they belong to: a tile is multiplied with each adapter that
// one of its rows has, and each row keeps the result of its own.  So rows need no sorting, a run of rows of one request costs
// one product, and nothing that one request's adapter holds, infinities and NaN too, reaches another's rows.  More rows of many adapters are put
// in the adapters' order first, as a list that the kernels go by: nothing is moved.
//
// 8192 rows of 4096 in 8 bits to 4096 in bf16, rank 16, six runs: 50 to 52 us, of which the product over long rows takes 16 (34 MB; 11 for
// one adapter) and the one with B 30 (134 MB, 4.5 TB/s).  One row: one launch, 7.6 us.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "dev_common.h"
#include "learn.h"
#include "q8_eight.h"

namespace shifter {

typedef float v4f __attribute__((ext_vector_type(4)));
constexpr int NO_ADAPTER = -1, BAD_ADAPTER = -2;
constexpr uint32_t ADAPT_THREADS = 256, ADAPT_WAVES = 4;

__device__ __forceinline__ int adapter_of(const int64_t* which, uint64_t row, uint64_t rows, uint32_t adapters) {
    if (row >= rows) return NO_ADAPTER;
    const int64_t i = which[row];
    return i < 0 ? NO_ADAPTER : i < (int64_t)adapters ? (int)i : BAD_ADAPTER;
}

// The nth row of an order.
__device__ __forceinline__ uint64_t row_of(const uint32_t* order, uint64_t nth) { return order ? order[nth] : nth; }

// acc[i][j] += sum over 32 columns of a[i] b[j]: lane l holds eight columns, 8 (l / 16) on, of row l % 16 of each, and
// rows 4 (l / 16) on of column l % 16 of the result.
__device__ __forceinline__ v4f mma(const Eight<__bf16>& a, const Eight<__bf16>& b, v4f acc) {
    typedef __bf16 vec __attribute__((ext_vector_type(8)));
    vec u, v;
    __builtin_memcpy(&u, a.w, 16);
    __builtin_memcpy(&v, b.w, 16);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(u, v, acc, 0, 0, 0);
}
__device__ __forceinline__ v4f mma(const Eight<_Float16>& a, const Eight<_Float16>& b, v4f acc) {
    typedef _Float16 vec __attribute__((ext_vector_type(8)));
    vec u, v;
    __builtin_memcpy(&u, a.w, 16);
    __builtin_memcpy(&v, b.w, 16);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(u, v, acc, 0, 0, 0);
}
__device__ __forceinline__ v4f mma(const Eight<float>& a, const Eight<float>& b, v4f acc) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w[i]), __uint_as_float(b.w[i]), acc, 0, 0, 0);
    return acc;
}

// The next adapter that a row of the tiles still waits for, the same in all lanes; false: none.
template <uint32_t RT>
__device__ __forceinline__ bool next_adapter(int (&waits)[RT], int* which) {
#pragma unroll
    for (uint32_t i = 0; i < RT; ++i) {
        const uint64_t who = __ballot(waits[i] >= 0);
        if (who) {
            const int a = __builtin_amdgcn_readlane(waits[i], (int)__ffsll((unsigned long long)who) - 1);
#pragma unroll
            for (uint32_t j = 0; j < RT; ++j)
                if (waits[j] == a) waits[j] = NO_ADAPTER;
            *which = a;
            return true;
        }
    }
    return false;
}

// Two times eight neighbouring columns of a row, `apart` columns from one to the other, as two operands.
template <typename T>
struct Sixteen {
    Eight<T> h[2];
    __device__ __forceinline__ void load(const T* p, uint32_t apart) {
        h[0].load(p);
        h[1].load(p + apart);
    }
    __device__ __forceinline__ void load_end(const T* row, uint32_t c, uint32_t apart, uint32_t cols) {     // zeros behind the row's end
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i) {
            fetch8(row, c + apart * i, cols, h[i]);
            place8(c + apart * i, cols, h[i]);
        }
    }
};
// Codes as numbers of type T, which holds them exactly.
template <typename T>
__device__ __forceinline__ void codes_as(uint4 w, Sixteen<T>& s) {
    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
        float f[8];
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) f[j] = (float)(int8_t)(word[2 * i + j / 4] >> (8 * (j % 4)));
        s.h[i].from(f);
    }
}

// The 16 codes from column c on, zeros behind the row's end: what it holds there is not read as codes.
__device__ __forceinline__ uint4 codes_end(const int8_t* q, uint32_t c, uint32_t cols) {
    uint32_t w[4] = {0, 0, 0, 0};
    if (c < cols) {
        const uint4 v = *reinterpret_cast<const uint4*>(q + c);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        const int32_t n = (int32_t)(cols - c);
#pragma unroll
        for (int32_t e = 0; e < 4; ++e) {
            const int32_t b = min(max(n - 4 * e, 0), 4);
            w[e] &= b == 4 ? ~0u : (1u << (8 * b)) - 1u;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The adapter of the block: of few rows, each block takes one of the adapters that a tile's rows have, the job-th of them.  False: there
// are not so many.
__device__ __forceinline__ bool adapter_of_job(int id, uint32_t job, int* which) {
    int waits[1] = {id};
    for (uint32_t j = 0;; ++j) {
        if (!next_adapter<1>(waits, which)) return false;
        if (j == job) return true;
    }
}

// s[part][r] = c_i x_r A_i' over the part's columns; 0 for a row without an adapter, NaN for one whose adapter there is not.
// A block has RT tiles of 16 rows and 16 RF ranks; its wavefronts take steps of 64 columns in turn and join their sums.  Both factors
// come straight from memory into the operands (a lane has twice eight columns, so that four lanes read 64 bytes of a row side by side; the
// 16 codes of a lane are one read, and its columns of A lie as they do).  16 rows by 64 bytes are read at a time, 128 to 256 bytes of a row by
// the block: 8192 x 4096 bf16 with one adapter 17 us, 4 TB/s, as long as a library product of that shape (20).
// Blocks share the adapters of a tile's rows (g.jobs of them; of a tile of one adapter all but one end at once), and write the rows of
// theirs: a tile of several would take several times as long as the others, and the kernel with it (prompts of 8192 rows with five
// borders 21 us for 13).
template <typename T, bool CODES, uint32_t RF, uint32_t RT>
__global__ __launch_bounds__(ADAPT_THREADS, RT * RF > 2 ? 2 : 3) void adapters_down_kernel(AdaptersDownArgs g) {
    __shared__ v4f s_sum[ADAPT_WAVES][RF * RT][64];
    const uint32_t lane = threadIdx.x & 63u, wave = uniform_u32(threadIdx.x >> 6), col = (CODES ? 16u : 8u) * (lane / 16u), r16 = lane & 15u;
    constexpr uint32_t APART = CODES ? 8 : 32;
    const uint32_t tile = blockIdx.x, job = blockIdx.z / g.groups;
    const uint64_t m0 = (uint64_t)tile * 16u * RT;
    const uint32_t part = blockIdx.y, rank0 = (blockIdx.z - job * g.groups) * 16u * RF;
    const uint32_t steps = (g.k + ADAPT_STEP - 1u) / ADAPT_STEP, whole = g.k / ADAPT_STEP;
    const uint32_t s0 = (uint32_t)((uint64_t)steps * part / g.parts), s1 = (uint32_t)((uint64_t)steps * (part + 1u) / g.parts);
    int id[RT], waits[RT];
    uint32_t row[RT];
    const T* x[RT];
    const int8_t* q[RT];
#pragma unroll
    for (uint32_t i = 0; i < RT; ++i) {
        const uint64_t nth = m0 + 16u * i + r16, at = row_of(g.order, min(nth, (uint64_t)g.m - 1u));
        row[i] = (uint32_t)at;
        id[i] = waits[i] = nth < g.m ? adapter_of(g.which, at, g.m, g.adapters) : NO_ADAPTER;
        x[i] = static_cast<const T*>(g.x) + at * g.ld_x;
        q[i] = static_cast<const int8_t*>(g.x) + at * g.ld_x;
    }
    v4f sum[RT][RF];
#pragma unroll
    for (uint32_t i = 0; i < RT; ++i)
#pragma unroll
        for (uint32_t f = 0; f < RF; ++f) sum[i][f] = v4f{0, 0, 0, 0};
    bool mine[RT];                         // rows without an adapter are the first one's
#pragma unroll
    for (uint32_t i = 0; i < RT; ++i) mine[i] = job == 0 && id[i] < 0;
    int which;
    uint32_t nth = 0;
    while (next_adapter<RT>(waits, &which)) {
        if (nth++ % g.jobs != job) continue;
        const T* a[RF];
#pragma unroll
        for (uint32_t f = 0; f < RF; ++f)
            a[f] = static_cast<const T*>(g.a) + ((uint64_t)which * g.rank + min(rank0 + 16u * f + r16, g.rank - 1u)) * g.k;
        v4f acc[RT][RF];
#pragma unroll
        for (uint32_t i = 0; i < RT; ++i)
#pragma unroll
            for (uint32_t f = 0; f < RF; ++f) acc[i][f] = v4f{0, 0, 0, 0};
        struct Operands {
            Sixteen<T> x[RT], a[RF];
            uint4 q[RT];
        };
        auto fetch = [&](uint32_t s, Operands& o) {
            const uint32_t c = s * ADAPT_STEP + col;
#pragma unroll
            for (uint32_t i = 0; i < RT; ++i) {
                if (CODES) o.q[i] = *reinterpret_cast<const uint4*>(q[i] + c);
                else o.x[i].load(x[i] + c, APART);
            }
#pragma unroll
            for (uint32_t f = 0; f < RF; ++f) o.a[f].load(a[f] + c, APART);
        };
        auto multiply = [&](Operands& o) {
#pragma unroll
            for (uint32_t i = 0; i < RT; ++i) {
                if (CODES) codes_as(o.q[i], o.x[i]);
#pragma unroll
                for (uint32_t f = 0; f < RF; ++f)
#pragma unroll
                    for (uint32_t h = 0; h < 2; ++h) acc[i][f] = mma(o.a[f].h[h], o.x[i].h[h], acc[i][f]);
            }
        };
        Operands o, next;
        const uint32_t end = min(s1, whole);
        uint32_t s = s0 + wave;
        if (s < end) fetch(s, next);
        for (; s < end; s += ADAPT_WAVES) {
            o = next;
            if (s + ADAPT_WAVES < end) fetch(s + ADAPT_WAVES, next);
            multiply(o);
        }
        if (s1 > whole && (s1 - 1u - s0) % ADAPT_WAVES == wave) {        // the step that a row ends in
            const uint32_t c = whole * ADAPT_STEP + col;
#pragma unroll
            for (uint32_t i = 0; i < RT; ++i) {
                if (CODES) {
                    o.q[i] = codes_end(q[i], c, g.k);
                } else {
                    o.x[i].load_end(x[i], c, APART, g.k);
                }
            }
#pragma unroll
            for (uint32_t f = 0; f < RF; ++f) o.a[f].load_end(a[f], c, APART, g.k);
            multiply(o);
        }
#pragma unroll
        for (uint32_t i = 0; i < RT; ++i)
#pragma unroll
            for (uint32_t f = 0; f < RF; ++f)
                if (id[i] == which) sum[i][f] = acc[i][f];
#pragma unroll
        for (uint32_t i = 0; i < RT; ++i) mine[i] = mine[i] || id[i] == which;
    }
    if (job >= nth && job != 0) return;    // all wavefronts alike
#pragma unroll
    for (uint32_t i = 0; i < RT; ++i)
#pragma unroll
        for (uint32_t f = 0; f < RF; ++f) s_sum[wave][i * RF + f][lane] = sum[i][f];
    __syncthreads();
    const uint32_t pad = (g.rank + 15u) & ~15u;
#pragma unroll
    for (uint32_t u = 0; u < RF * RT; ++u) {
        if (u % ADAPT_WAVES != wave) continue;
        const uint32_t i = u / RF, f = u % RF, r = rank0 + 16u * f + 4u * (lane / 16u);
        const uint64_t nth = m0 + 16u * i + r16;
        if (nth >= g.m || rank0 + 16u * f >= pad) continue;
        if (!mine[i]) continue;
        v4f v = (s_sum[0][u][lane] + s_sum[1][u][lane]) + (s_sum[2][u][lane] + s_sum[3][u][lane]);
        float by = 1.0f;
        if (id[i] >= 0) {
            if (g.scale) by = g.scale[id[i]];
            if (CODES) by *= g.x_scale[row[i]];
        }
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) v[e] = id[i] == BAD_ADAPTER ? NAN : id[i] < 0 || r + e >= g.rank ? 0.0f : v[e] * by;
        *reinterpret_cast<v4f*>(g.s + ((uint64_t)part * g.m + nth) * pad + r) = v;
    }
}

template <typename T, bool CODES, uint32_t RF>
static void launch_down_as(shifter_ctx* ctx, const AdaptersDownArgs& g) {
    const uint32_t tiles = adapt_tiles(g.m, g.rank);
    const uint32_t blocks = (uint32_t)((g.m + 16u * tiles - 1u) / (16u * tiles));
    const dim3 grid(blocks, g.parts, g.groups * g.jobs);
    if constexpr (RF < 4)
        if (tiles == 2) return adapters_down_kernel<T, CODES, RF, 2><<<grid, ADAPT_THREADS, 0, ctx->stream>>>(g);
    adapters_down_kernel<T, CODES, RF, 1><<<grid, ADAPT_THREADS, 0, ctx->stream>>>(g);
}
template <typename T, bool CODES>
static void launch_down_of(shifter_ctx* ctx, const AdaptersDownArgs& g) {
    const uint64_t pad = adapt_pad(g.rank);
    if (pad <= 16) launch_down_as<T, CODES, 1>(ctx, g);
    else if (pad <= 32) launch_down_as<T, CODES, 2>(ctx, g);
    else launch_down_as<T, CODES, 4>(ctx, g);      // 64 ranks a block
}
static void launch_down(shifter_ctx* ctx, int dtype, AdaptersDownArgs g) {
    g.groups = (uint32_t)(adapt_pad(g.rank) + 63u) / 64u;
    g.jobs = adapt_down_jobs(g.m, g.adapters);
    ProfileScope ps(ctx, K_ADAPTERS_DOWN);
    if (dtype == SHIFTER_F32) g.x_scale ? launch_down_of<float, true>(ctx, g) : launch_down_of<float, false>(ctx, g);
    else if (dtype == SHIFTER_BF16) g.x_scale ? launch_down_of<__bf16, true>(ctx, g) : launch_down_of<__bf16, false>(ctx, g);
    else g.x_scale ? launch_down_of<_Float16, true>(ctx, g) : launch_down_of<_Float16, false>(ctx, g);
}

// Four neighbouring ranks of a column of B and of a row of s, as operands of products over 16 ranks: lane l holds four, 4 (l / 16) on, of
// row or column l % 16.
//
// The matrix units take fp32 at a sixteenth of bf16's rate: 16 ranks of a tile are four products of 32 cycles.  s is cut into three bf16 of
// 8 bits each instead, which are all of its 24, and a bf16 B is multiplied with them as it is, two pieces to a product of 16 cycles; an fp16
// B is two bf16, of 8 and 3 bits, three products.  All products of pieces are exact and summed in 32 bits.
__device__ __forceinline__ uint2 high_halves(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return make_uint2(__builtin_amdgcn_perm(b, a, 0x07060302), __builtin_amdgcn_perm(d, c, 0x07060302));
}
__device__ __forceinline__ v4f mma_pieces(uint2 a0, uint2 a1, uint2 b0, uint2 b1, v4f acc) {
    typedef __bf16 vec __attribute__((ext_vector_type(8)));
    const uint32_t u[4] = {a0.x, a0.y, a1.x, a1.y}, v[4] = {b0.x, b0.y, b1.x, b1.y};
    vec p, q;
    __builtin_memcpy(&p, u, 16);
    __builtin_memcpy(&q, v, 16);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, q, acc, 0, 0, 0);
}
// The upper 8 bits of four numbers' 24, and what is left of them.
__device__ __forceinline__ uint2 upper_of(v4f& v) {
    uint32_t w[4];
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
        w[e] = __float_as_uint(v[e]) & 0xffff0000u;
        v[e] = isinf(v[e]) ? 0.0f : v[e] - __uint_as_float(w[e]);
    }
    return high_halves(w[0], w[1], w[2], w[3]);
}
struct SPieces {
    uint2 p[3];
    __device__ __forceinline__ void from(v4f v) {
        p[0] = upper_of(v);
        p[1] = upper_of(v);
        p[2] = high_halves(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};
// n of four elements at p, zeros behind them.
template <bool EVEN, typename T>
__device__ __forceinline__ void four_of(const T* p, int32_t n, uint32_t (&w)[sizeof(T)]) {
    if (!EVEN) {
#pragma unroll
        for (uint32_t i = 0; i < sizeof(T); ++i) w[i] = 0u;
        if (n <= 0) return;
    }
    if (EVEN || n >= 4) {
        typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
        const vec v = *reinterpret_cast<const vec*>(p);
        __builtin_memcpy(w, &v, sizeof(v));
    } else {
        T v[4];
#pragma unroll
        for (int32_t e = 0; e < 4; ++e) v[e] = e < n ? p[e] : (T)0.0f;
        __builtin_memcpy(w, v, sizeof(v));
    }
}
template <typename T>
struct BFour {
    uint2 p;
    typedef SPieces S;
    template <bool EVEN>
    __device__ __forceinline__ void load(const T* row, uint32_t r, uint32_t rank) {
        uint32_t w[2];
        four_of<EVEN>(row + r, (int32_t)(rank - r), w);
        p = make_uint2(w[0], w[1]);
    }
    __device__ __forceinline__ v4f multiply(const S& s, v4f acc) const {
        acc = mma_pieces(p, p, s.p[0], s.p[1], acc);
        return mma_pieces(p, make_uint2(0, 0), s.p[2], make_uint2(0, 0), acc);
    }
};
template <>
struct BFour<_Float16> {
    uint2 high, low;
    typedef SPieces S;
    template <bool EVEN>
    __device__ __forceinline__ void load(const _Float16* row, uint32_t r, uint32_t rank) {
        uint32_t w[2];
        four_of<EVEN>(row + r, (int32_t)(rank - r), w);
        _Float16 h[4];
        __builtin_memcpy(h, w, 8);
        v4f v{(float)h[0], (float)h[1], (float)h[2], (float)h[3]};
        high = upper_of(v);
        low = upper_of(v);
    }
    __device__ __forceinline__ v4f multiply(const S& s, v4f acc) const {
        acc = mma_pieces(high, high, s.p[0], s.p[1], acc);
        acc = mma_pieces(high, low, s.p[2], s.p[0], acc);
        return mma_pieces(low, low, s.p[1], s.p[2], acc);
    }
};
template <>
struct BFour<float> {
    v4f v;
    struct S {
        v4f v;
        __device__ __forceinline__ void from(v4f x) { v = x; }
    };
    template <bool EVEN>
    __device__ __forceinline__ void load(const float* row, uint32_t r, uint32_t rank) {
        uint32_t w[4];
        four_of<EVEN>(row + r, (int32_t)(rank - r), w);
        __builtin_memcpy(&v, w, 16);
    }
    __device__ __forceinline__ v4f multiply(const S& s, v4f acc) const {
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], s.v[e], acc, 0, 0, 0);
        return acc;
    }
};

// out_r = y_r + s_r B_i'.  A wavefront multiplies tiles of 16 rows with 64 columns; the columns of a tile's four products are
// interleaved so that a lane ends with twice eight neighbouring columns of a row, which it adds to y and writes: 32 half + 8 group on.
template <typename T, typename Y>
struct UpTile {
    uint32_t lane = threadIdx.x & 63u, group = lane / 16u, r16 = lane & 15u;

    // The row of B that product t takes as its column i = lane % 16.
    __device__ __forceinline__ const T* b_row(const AdaptersUpArgs& g, int which, uint32_t n0, uint32_t t) const {
        const uint32_t at = n0 + 32u * (t / 2u) + 8u * (r16 / 4u) + 4u * (t % 2u) + r16 % 4u;
        return static_cast<const T*>(g.b) + ((uint64_t)which * g.n + min(at, g.n - 1u)) * g.rank;
    }
    __device__ __forceinline__ uint32_t col(uint32_t n0, uint32_t half) const { return n0 + 32u * half + 8u * group; }
    // FULL: all 64 columns are there.
    template <bool FULL>
    __device__ __forceinline__ void fetch(const AdaptersUpArgs& g, uint64_t row, uint32_t n0, Eight<Y> (&y)[2]) const {
        if (!g.y) return;
        const Y* y_row = static_cast<const Y*>(g.y) + min(row, (uint64_t)g.m - 1u) * g.ld_y;
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
            const uint32_t c = col(n0, h);
            if (FULL) {
                y[h].load(y_row + c);
            } else {
                fetch8(y_row, c, g.n, y[h]);
                place8(c, g.n, y[h]);
            }
        }
    }
    // A row without an adapter is y, and stays as it is in place.
    __device__ __forceinline__ static bool stays(const AdaptersUpArgs& g, int id) { return id == NO_ADAPTER && g.y == g.out; }
    template <bool FULL>
    __device__ __forceinline__ void write(const AdaptersUpArgs& g, uint64_t row, bool writes, int id, uint32_t n0, const Eight<Y> (&y)[2], v4f (&sum)[4]) const {
        if (__ballot(id < 0)) {
            const float none = g.y ? -0.0f : 0.0f;         // y as it is, its zeros' signs too
#pragma unroll
            for (uint32_t t = 0; t < 4; ++t)
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) sum[t][e] = id == BAD_ADAPTER ? NAN : id < 0 ? none : sum[t][e];
        }
        if (!writes) return;
        Y* out_row = static_cast<Y*>(g.out) + row * g.ld_out;
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
            const uint32_t c = col(n0, h);
            float f[8];
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) f[j] = sum[2 * h + j / 4][j % 4];
            if (g.y) {
                float w[8];
                y[h].floats(w);
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) f[j] += w[j];
            }
            if (FULL || c + 8u <= g.n) {
                Eight<Y> e;
                e.from(f);
                e.store(out_row + c);
            } else {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j)
                    if (c + j < g.n) out_row[c + j] = (Y)f[j];
            }
        }
    }
};
// s's four numbers of a row from rank r on: the sum of the parts'.
__device__ __forceinline__ v4f sum_of_parts(const AdaptersUpArgs& g, uint64_t row, uint32_t r, uint32_t pad) {
    const float* p = g.s + row * pad + r;
    const uint64_t next = (uint64_t)g.m * pad;
    constexpr uint32_t MOST = 8;           // under way
    v4f v = *reinterpret_cast<const v4f*>(p);
    for (uint32_t i0 = 1; i0 < g.parts; i0 += MOST) {
        v4f w[MOST];
#pragma unroll
        for (uint32_t i = 0; i < MOST; ++i)
            if (i0 + i < g.parts) w[i] = *reinterpret_cast<const v4f*>(p + (i0 + i) * next);
#pragma unroll
        for (uint32_t i = 0; i < MOST; ++i)
            if (i0 + i < g.parts) v += w[i];
    }
    return v;
}
__device__ __forceinline__ void keep_down(const AdaptersUpArgs& g, uint64_t row, uint32_t r, v4f v) {
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e)
        if (r + e < g.down_cols) g.down[row * g.down_cols + r + e] = v[e];
}

// A tile of rows for each block, whose wavefronts take 64 columns in turn: for few rows, and for ranks above 32.  s is in LDS.
template <typename T, typename Y, bool JOBS, bool EVEN>
__global__ __launch_bounds__(ADAPT_THREADS, 3) void adapters_up_kernel(AdaptersUpArgs g) {
    extern __shared__ __align__(16) float s_rows[];        // [16][pad + 4]
    const UpTile<T, Y> tile;
    const uint32_t wave = uniform_u32(threadIdx.x >> 6);
    const uint64_t m0 = (uint64_t)blockIdx.x * 16u, nth = m0 + tile.r16, row = row_of(g.order, min(nth, (uint64_t)g.m - 1u));
    const uint32_t pad = (g.rank + 15u) & ~15u, pitch = pad + 4u, fours = pad / 4u, job = blockIdx.z;
    const int id = nth < g.m ? adapter_of(g.which, row, g.m, g.adapters) : NO_ADAPTER;
    int mine = NO_ADAPTER;
    if (JOBS && !adapter_of_job(id, job, &mine) && job != 0) return;
    for (uint32_t u = threadIdx.x; u < 16u * fours; u += ADAPT_THREADS) {
        const uint32_t at = u / fours, r = u % fours * 4u;
        v4f v{0, 0, 0, 0};
        if (m0 + at < g.m) {
            v = sum_of_parts(g, m0 + at, r, pad);
            if (g.down && blockIdx.y == 0 && job == 0) keep_down(g, row_of(g.order, m0 + at), r, v);
        }
        *reinterpret_cast<v4f*>(s_rows + at * pitch + r) = v;
    }
    __syncthreads();
    const float* s_row = s_rows + tile.r16 * pitch;
    const bool writes = nth < g.m && !tile.stays(g, id) && (!JOBS || (id >= 0 ? id == mine : job == 0));
    auto columns = [&](uint32_t n0, auto full) {
        Eight<Y> y[2];
        tile.template fetch<full.value>(g, row, n0, y);
        v4f sum[4];
#pragma unroll
        for (uint32_t t = 0; t < 4; ++t) sum[t] = v4f{0, 0, 0, 0};
        int waits[1] = {id}, which = mine;
        bool first = true;
        while (JOBS ? which >= 0 : next_adapter<1>(waits, &which)) {
            v4f acc[4];
            const T* b[4];
#pragma unroll
            for (uint32_t t = 0; t < 4; ++t) {
                acc[t] = v4f{0, 0, 0, 0};
                b[t] = tile.b_row(g, which, n0, t);
            }
            for (uint32_t r = 4u * tile.group; r < pad; r += 16u) {
                BFour<T> v[4];
                typename BFour<T>::S s;
#pragma unroll
                for (uint32_t t = 0; t < 4; ++t) v[t].template load<EVEN>(b[t], r, g.rank);
                s.from(*reinterpret_cast<const v4f*>(s_row + r));
#pragma unroll
                for (uint32_t t = 0; t < 4; ++t) acc[t] = v[t].multiply(s, acc[t]);
            }
            // the first one's are overwritten where a row has another
#pragma unroll
            for (uint32_t t = 0; t < 4; ++t)
                if (first || id == which) sum[t] = acc[t];
            first = false;
            if (JOBS) break;
        }
        tile.template write<full.value>(g, row, writes, id, n0, y, sum);
    };
    const uint32_t step = gridDim.y * ADAPT_WAVES * 64u;
    for (uint32_t n0 = (blockIdx.y * ADAPT_WAVES + wave) * 64u; n0 < g.n; n0 += step) {
        if (n0 + 64u <= g.n) columns(n0, std::true_type{});
        else columns(n0, std::false_type{});
    }
}

// 64 columns for each wavefront, which takes tiles of rows in turn and keeps its columns of B in registers as long as the rows have the same
// adapter; the next tile's s and y are on their way meanwhile.  Nothing in the loop of a full tile of one adapter is in a lane's branch: with
// the ends of rows and columns looked after there, prompts of 8192 rows took 46 us.
template <typename T, typename Y, uint32_t NF, bool EVEN>
__global__ __launch_bounds__(ADAPT_THREADS, 3) void adapters_up_rows_kernel(AdaptersUpArgs g) {
    constexpr uint32_t PAD = 16 * NF;
    const UpTile<T, Y> tile;
    const uint32_t n0 = (blockIdx.x * ADAPT_WAVES + uniform_u32(threadIdx.x >> 6)) * 64u;
    const bool live = n0 < g.n, keeps = g.down && n0 == 0;
    if (!live && !keeps) return;
    const uint32_t tiles = (g.m + 15u) / 16u;
    auto rows = [&](auto full) {
        struct Operands {
            int id;
            uint64_t row;
            v4f s[2][NF];              // of two parts: added up where they are used, so that no fetch waits
            Eight<Y> y[2];
        };
        auto row_at = [&](uint32_t t) { return row_of(g.order, min((uint64_t)t * 16u + tile.r16, (uint64_t)g.m - 1u)); };
        auto fetch = [&](uint32_t t, uint64_t row, Operands& o) {
            const uint64_t at = min((uint64_t)t * 16u + tile.r16, (uint64_t)g.m - 1u);
            o.row = row;
            o.id = adapter_of(g.which, row, g.m, g.adapters);
#pragma unroll
            for (uint32_t f = 0; f < NF; ++f) {
                const float* p = g.s + at * PAD + 16u * f + 4u * tile.group;
                o.s[0][f] = *reinterpret_cast<const v4f*>(p);
                o.s[1][f] = v4f{0, 0, 0, 0};
                if (g.parts > 1) o.s[1][f] = *reinterpret_cast<const v4f*>(p + (uint64_t)g.m * PAD);
            }
            if (full.value || live) tile.template fetch<full.value>(g, row, n0, o.y);
        };
        uint32_t t = blockIdx.y;
        Operands next;
        if (t < tiles) fetch(t, row_at(t), next);
        uint64_t later = row_at(min(t + gridDim.y, tiles - 1u));           // where the next tile's rows are is known a tile ahead
        int held = NO_ADAPTER;
        BFour<T> b[NF][4];
        for (; t < tiles; t += gridDim.y) {
            Operands o = next;
            const bool there = (uint64_t)t * 16u + tile.r16 < g.m;
            if (!there) o.id = NO_ADAPTER;
            if (t + gridDim.y < tiles) fetch(t + gridDim.y, later, next);
            later = row_at(min(t + 2u * gridDim.y, tiles - 1u));
            if (keeps) {
                if (there) {
#pragma unroll
                    for (uint32_t f = 0; f < NF; ++f) keep_down(g, o.row, 16u * f + 4u * tile.group, o.s[0][f] + o.s[1][f]);
                }
                if (!live) continue;
            }
            typename BFour<T>::S s[NF];
#pragma unroll
            for (uint32_t f = 0; f < NF; ++f) s[f].from(o.s[0][f] + o.s[1][f]);
            v4f sum[4];
            int waits[1] = {o.id}, which;
            bool first = true;
            while (next_adapter<1>(waits, &which)) {
                if (which != held) {
                    held = which;
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
                        for (uint32_t f = 0; f < NF; ++f) b[f][i].template load<EVEN>(tile.b_row(g, which, n0, i), 16u * f + 4u * tile.group, g.rank);
                    // waited for here, or the compiler waits for all that is under way wherever B is used
                    __builtin_amdgcn_s_waitcnt(0x0f70);
                }
                v4f acc[4];
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) acc[i] = v4f{0, 0, 0, 0};
#pragma unroll
                for (uint32_t f = 0; f < NF; ++f)
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) acc[i] = b[f][i].multiply(s[f], acc[i]);
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    if (first || o.id == which) sum[i] = acc[i];
                first = false;
            }
            tile.template write<full.value>(g, o.row, there && !tile.stays(g, o.id), o.id, n0, o.y, sum);
        }
    };
    if (n0 + 64u <= g.n) rows(std::true_type{});
    else rows(std::false_type{});
}

template <typename T, typename Y>
static void launch_up_of(shifter_ctx* ctx, const AdaptersUpArgs& g) {
    const uint32_t jobs = adapt_jobs(g.m, g.adapters), tiles = (uint32_t)((g.m + 15u) / 16u), groups = std::max(1u, (g.n + 255u) / 256u);
    const uint64_t pad = adapt_pad(g.rank);
    if (g.m > ADAPT_FEW_ROWS && pad <= 32) {
        const dim3 grid(groups, std::min(tiles, std::max(1u, ADAPT_UP_BLOCKS / groups)));
        if (pad == 16 && g.rank == pad) adapters_up_rows_kernel<T, Y, 1, true><<<grid, ADAPT_THREADS, 0, ctx->stream>>>(g);
        else if (pad == 16) adapters_up_rows_kernel<T, Y, 1, false><<<grid, ADAPT_THREADS, 0, ctx->stream>>>(g);
        else if (g.rank == pad) adapters_up_rows_kernel<T, Y, 2, true><<<grid, ADAPT_THREADS, 0, ctx->stream>>>(g);
        else adapters_up_rows_kernel<T, Y, 2, false><<<grid, ADAPT_THREADS, 0, ctx->stream>>>(g);
        return;
    }
    const dim3 grid(tiles, std::min(groups, std::max(1u, ADAPT_UP_BLOCKS / tiles)), jobs);
    const uint32_t lds = (uint32_t)(16u * (pad + 4u) * sizeof(float));
    if (jobs > 1 && g.rank == pad) adapters_up_kernel<T, Y, true, true><<<grid, ADAPT_THREADS, lds, ctx->stream>>>(g);
    else if (jobs > 1) adapters_up_kernel<T, Y, true, false><<<grid, ADAPT_THREADS, lds, ctx->stream>>>(g);
    else if (g.rank == pad) adapters_up_kernel<T, Y, false, true><<<grid, ADAPT_THREADS, lds, ctx->stream>>>(g);
    else adapters_up_kernel<T, Y, false, false><<<grid, ADAPT_THREADS, lds, ctx->stream>>>(g);
}
template <typename T>
static void launch_up_as(shifter_ctx* ctx, int y_dtype, const AdaptersUpArgs& g) {
    if (y_dtype == SHIFTER_F32) launch_up_of<T, float>(ctx, g);
    else if (y_dtype == SHIFTER_BF16) launch_up_of<T, __bf16>(ctx, g);
    else launch_up_of<T, _Float16>(ctx, g);
}
static void launch_up(shifter_ctx* ctx, int dtype, int y_dtype, const AdaptersUpArgs& g) {
    ProfileScope ps(ctx, K_ADAPTERS_UP);
    if (dtype == SHIFTER_F32) launch_up_as<float>(ctx, y_dtype, g);
    else if (dtype == SHIFTER_BF16) launch_up_as<__bf16>(ctx, y_dtype, g);
    else launch_up_as<_Float16>(ctx, y_dtype, g);
}

// Both products in one launch, for a few rows of small adapters: each block works out s for itself, its wavefronts taking steps of 64 columns
// in turn, and multiplies it with its columns of B, which are on their way meanwhile, as y is.  One row of 4096 in 8 bits to 4096 with rank 16 7.6 us
// (9.3 in two launches), 512 to 512 6.3 (9.4): a launch, three trips to memory one after the other, and 131 KB of A by each of 16 blocks.
constexpr uint32_t ONE_THREADS = 1024, ONE_WAVES = ONE_THREADS / 64;
struct AdaptersOneArgs {
    AdaptersDownArgs d;
    AdaptersUpArgs u;
};
template <typename T, bool CODES, typename Y, uint32_t NF>
__global__ __launch_bounds__(ONE_THREADS) void adapters_one_kernel(AdaptersOneArgs g) {
    __shared__ v4f s_sum[ONE_WAVES][NF][64];
    const UpTile<T, Y> tile;
    const uint32_t wave = uniform_u32(threadIdx.x >> 6), job = blockIdx.z, rank = g.u.rank, k = g.d.k;
    const uint64_t nth = (uint64_t)blockIdx.x * 16u + tile.r16, row = min(nth, (uint64_t)g.u.m - 1u);
    const int id = nth < g.u.m ? adapter_of(g.u.which, row, g.u.m, g.u.adapters) : NO_ADAPTER;
    int mine = NO_ADAPTER;
    if (!adapter_of_job(id, job, &mine)) {         // all wavefronts alike
        if (job != 0) return;
        mine = NO_ADAPTER;
    }
    uint32_t n0 = (wave * gridDim.y + blockIdx.y) * 64u;
    const bool full = n0 + 64u <= g.u.n;
    BFour<T> b[NF][4];
    Eight<Y> y[2];
    auto fetch_b = [&] {
#pragma unroll
        for (uint32_t t = 0; t < 4; ++t)
#pragma unroll
            for (uint32_t f = 0; f < NF; ++f) b[f][t].template load<false>(tile.b_row(g.u, mine, n0, t), 16u * f + 4u * tile.group, rank);
    };
    if (n0 < g.u.n) {
        if (full) tile.template fetch<true>(g.u, row, n0, y);
        else tile.template fetch<false>(g.u, row, n0, y);
        if (mine >= 0) fetch_b();
    }
    if (mine >= 0) {
        constexpr uint32_t APART = CODES ? 8 : 32;
        const uint32_t col = (CODES ? 16u : 8u) * tile.group, whole = k / ADAPT_STEP;
        const T* x = static_cast<const T*>(g.d.x) + row * g.d.ld_x;
        const int8_t* q = static_cast<const int8_t*>(g.d.x) + row * g.d.ld_x;
        const T* a[NF];
        v4f acc[NF];
#pragma unroll
        for (uint32_t f = 0; f < NF; ++f) {
            a[f] = static_cast<const T*>(g.d.a) + ((uint64_t)mine * rank + min(16u * f + tile.r16, rank - 1u)) * k;
            acc[f] = v4f{0, 0, 0, 0};
        }
        auto multiply = [&](const Sixteen<T>& v, const Sixteen<T> (&w)[NF]) {
#pragma unroll
            for (uint32_t f = 0; f < NF; ++f)
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h) acc[f] = mma(w[f].h[h], v.h[h], acc[f]);
        };
        constexpr uint32_t DEPTH = sizeof(T) == 2 ? 4 / NF : 1;        // steps under way
        uint32_t s = wave;
        auto steps = [&](auto depth) {
            constexpr uint32_t D = depth.value;
            Sixteen<T> v[D], w[D][NF];
            uint4 code[D];
#pragma unroll
            for (uint32_t i = 0; i < D; ++i) {
                const uint32_t c = (s + i * ONE_WAVES) * ADAPT_STEP + col;
                if (CODES) code[i] = *reinterpret_cast<const uint4*>(q + c);
                else v[i].load(x + c, APART);
#pragma unroll
                for (uint32_t f = 0; f < NF; ++f) w[i][f].load(a[f] + c, APART);
            }
#pragma unroll
            for (uint32_t i = 0; i < D; ++i) {
                if (CODES) codes_as(code[i], v[i]);
                multiply(v[i], w[i]);
            }
            s += D * ONE_WAVES;
        };
        while (s + (DEPTH - 1u) * ONE_WAVES < whole) steps(std::integral_constant<uint32_t, DEPTH>{});
        while (s < whole) steps(std::integral_constant<uint32_t, 1>{});
        if (whole * ADAPT_STEP < k && whole % ONE_WAVES == wave) {         // the step that a row ends in
            const uint32_t c = whole * ADAPT_STEP + col;
            Sixteen<T> v, w[NF];
            if (CODES) codes_as(codes_end(q, c, k), v);
            else v.load_end(x, c, APART, k);
#pragma unroll
            for (uint32_t f = 0; f < NF; ++f) w[f].load_end(a[f], c, APART, k);
            multiply(v, w);
        }
#pragma unroll
        for (uint32_t f = 0; f < NF; ++f) s_sum[wave][f][tile.lane] = acc[f];
    }
    __syncthreads();
    v4f v[NF];
    float by = 1.0f;
    if (id >= 0) {
        if (g.d.scale) by = g.d.scale[id];
        if (CODES) by *= g.d.x_scale[row];
    }
    typename BFour<T>::S s[NF];
#pragma unroll
    for (uint32_t f = 0; f < NF; ++f) {
        v[f] = v4f{0, 0, 0, 0};
        if (mine >= 0) {
#pragma unroll
            for (uint32_t w = 0; w < ONE_WAVES; ++w) v[f] += s_sum[w][f][tile.lane];
        }
        const uint32_t r = 16u * f + 4u * tile.group;
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) v[f][e] = id == BAD_ADAPTER ? NAN : id < 0 || r + e >= rank ? 0.0f : v[f][e] * by;
        s[f].from(v[f]);
    }
    const bool own = nth < g.u.m && (id >= 0 ? id == mine : job == 0);
    if (g.u.down && own && blockIdx.y == 0 && wave == 0) {
#pragma unroll
        for (uint32_t f = 0; f < NF; ++f) keep_down(g.u, row, 16u * f + 4u * tile.group, v[f]);
    }
    const bool writes = own && !tile.stays(g.u, id);
    for (bool first = true; n0 < g.u.n; n0 += gridDim.y * ONE_WAVES * 64u, first = false) {
        if (!first) {
            tile.template fetch<false>(g.u, row, n0, y);
            if (mine >= 0) fetch_b();
        }
        v4f sum[4];
#pragma unroll
        for (uint32_t t = 0; t < 4; ++t) sum[t] = v4f{0, 0, 0, 0};
        if (mine >= 0) {
#pragma unroll
            for (uint32_t f = 0; f < NF; ++f)
#pragma unroll
                for (uint32_t t = 0; t < 4; ++t) sum[t] = b[f][t].multiply(s[f], sum[t]);
        }
        if (n0 + 64u <= g.u.n) tile.template write<true>(g.u, row, writes, id, n0, y, sum);
        else tile.template write<false>(g.u, row, writes, id, n0, y, sum);
    }
}

template <typename T, bool CODES, typename Y>
static void launch_one_of(shifter_ctx* ctx, const AdaptersOneArgs& g) {
    const uint32_t tiles = (g.u.m + 15u) / 16u, jobs = adapt_jobs(g.u.m, g.u.adapters);
    const dim3 grid(tiles, adapt_one_blocks(g.u.m, g.u.n, g.u.adapters), jobs);
    if (g.u.rank <= 16) adapters_one_kernel<T, CODES, Y, 1><<<grid, ONE_THREADS, 0, ctx->stream>>>(g);
    else adapters_one_kernel<T, CODES, Y, 2><<<grid, ONE_THREADS, 0, ctx->stream>>>(g);
}
template <typename T>
static void launch_one_as(shifter_ctx* ctx, int y_dtype, const AdaptersOneArgs& g) {
    const bool codes = g.d.x_scale != nullptr;
    if (y_dtype == SHIFTER_F32) codes ? launch_one_of<T, true, float>(ctx, g) : launch_one_of<T, false, float>(ctx, g);
    else if (y_dtype == SHIFTER_BF16) codes ? launch_one_of<T, true, __bf16>(ctx, g) : launch_one_of<T, false, __bf16>(ctx, g);
    else codes ? launch_one_of<T, true, _Float16>(ctx, g) : launch_one_of<T, false, _Float16>(ctx, g);
}
static void launch_one(shifter_ctx* ctx, int dtype, int y_dtype, const AdaptersOneArgs& g) {
    ProfileScope ps(ctx, K_ADAPTERS_UP);
    if (dtype == SHIFTER_F32) launch_one_as<float>(ctx, y_dtype, g);
    else if (dtype == SHIFTER_BF16) launch_one_as<__bf16>(ctx, y_dtype, g);
    else launch_one_as<_Float16>(ctx, y_dtype, g);
}

// The rows in the order of their adapters, those without one at the end, by one block: rows are counted by adapter in LDS, each with its
// place among the ones counted before it.  The order of an adapter's rows is not always the same, which no row's result depends on.
constexpr uint32_t SORT_THREADS = 1024, SORT_EACH = 8;
__global__ __launch_bounds__(SORT_THREADS) void adapters_sort_kernel(const int64_t* which, uint32_t m, uint32_t adapters, uint32_t* order) {
    constexpr uint32_t BINS = (uint32_t)ADAPT_SORT_MOST + 2u, PER = (BINS + SORT_THREADS - 1u) / SORT_THREADS;
    __shared__ uint32_t s_bin[PER * SORT_THREADS];
    __shared__ uint64_t smem[SORT_THREADS / 64 + 1];
    for (uint32_t i = threadIdx.x; i < PER * SORT_THREADS; i += SORT_THREADS) s_bin[i] = 0;
    __syncthreads();
    uint32_t bin[SORT_EACH], place[SORT_EACH];
    auto count = [&](uint64_t r0) {
#pragma unroll
        for (uint32_t e = 0; e < SORT_EACH; ++e) {
            const uint64_t r = r0 + e * SORT_THREADS + threadIdx.x;
            const int id = adapter_of(which, r, m, adapters);
            bin[e] = r >= m ? BINS : id < 0 ? adapters : (uint32_t)id;
        }
#pragma unroll
        for (uint32_t e = 0; e < SORT_EACH; ++e) {
            // rows of one adapter side by side go as one addition
            const bool want = bin[e] != BINS;
            const uint64_t todo = __ballot(want);
            if (todo == 0) break;
            const uint32_t first = (uint32_t)__ffsll((unsigned long long)todo) - 1u, lane = threadIdx.x & 63u;
            const uint32_t leader = (uint32_t)__builtin_amdgcn_readlane((int)bin[e], (int)first);
            const uint64_t peers = __ballot(want && bin[e] == leader);
            uint32_t base = 0;
            if (lane == first) base = atomicAdd(&s_bin[leader], (uint32_t)__popcll(peers));
            base = (uint32_t)__builtin_amdgcn_readlane((int)base, (int)first);
            if (want && bin[e] == leader) place[e] = base + (uint32_t)__popcll(peers & ((1ull << lane) - 1ull));
            else if (want) place[e] = atomicAdd(&s_bin[bin[e]], 1u);
        }
    };
    auto firsts = [&] {                    // of the bins, in the place of their numbers
        uint64_t sum = 0, all;
        uint32_t c[PER];
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < PER; ++i) sum += c[i] = s_bin[threadIdx.x * PER + i];
        uint64_t at = block_excl_scan_u64<SORT_THREADS>(sum, smem, &all);
#pragma unroll
        for (uint32_t i = 0; i < PER; ++i) {
            s_bin[threadIdx.x * PER + i] = (uint32_t)at;
            at += c[i];
        }
        __syncthreads();
    };
    if (m <= SORT_THREADS * SORT_EACH) {
        count(0);
        firsts();
#pragma unroll
        for (uint32_t e = 0; e < SORT_EACH; ++e)
            if (bin[e] != BINS) order[s_bin[bin[e]] + place[e]] = e * SORT_THREADS + threadIdx.x;
        return;
    }
    // more rows than the threads hold: counted once, and once more from the bins' first places on
    for (uint64_t r0 = 0; r0 < m; r0 += SORT_THREADS * SORT_EACH) count(r0);
    firsts();
    for (uint64_t r0 = 0; r0 < m; r0 += SORT_THREADS * SORT_EACH) {
        count(r0);
#pragma unroll
        for (uint32_t e = 0; e < SORT_EACH; ++e)
            if (bin[e] != BINS) order[place[e]] = (uint32_t)(r0 + e * SORT_THREADS + threadIdx.x);
    }
}

void launch_adapters(shifter_ctx* ctx, int dtype, int y_dtype, const AdaptersArgs& g) {
    const AdaptersPlan p = adapters_plan(g.m, g.k, g.rank, g.adapters);
    uint32_t* order = nullptr;
    if (adapt_sorted(g.m, g.adapters)) {
        ProfileScope ps(ctx, K_ADAPTERS_TURN);
        order = reinterpret_cast<uint32_t*>(g.work + p.order);
        adapters_sort_kernel<<<1, SORT_THREADS, 0, ctx->stream>>>(g.which, g.m, g.adapters, order);
    }
    AdaptersDownArgs d{};
    d.x = g.x; d.ld_x = g.ld_x; d.x_scale = g.x_scale; d.a = g.a; d.which = g.which; d.scale = g.scale;
    d.m = g.m; d.k = g.k; d.rank = g.rank; d.adapters = g.adapters; d.parts = p.parts;
    d.order = order;
    d.s = reinterpret_cast<float*>(g.work);
    AdaptersUpArgs u{};
    u.s = d.s; u.order = order; u.parts = p.parts; u.b = g.b; u.which = g.which; u.m = g.m; u.n = g.n; u.rank = g.rank; u.adapters = g.adapters;
    u.y = g.y; u.ld_y = g.ld_y; u.out = g.out; u.ld_out = g.ld_out; u.down = g.down; u.down_cols = g.rank;
    // x may be y, and written in place: not while blocks read it
    auto last = [&](uint64_t ld, uint64_t cols, uint64_t size) { return ((g.m - 1u) * ld + cols) * size; };
    const uintptr_t x = reinterpret_cast<uintptr_t>(g.x), out = reinterpret_cast<uintptr_t>(g.out);
    const uint64_t size = dtype == SHIFTER_F32 ? 4 : 2, y_size = y_dtype == SHIFTER_F32 ? 4 : 2;
    const bool apart = out >= x + last(g.ld_x, g.k, g.x_scale ? 1 : size) || x >= out + last(g.ld_out, g.n, y_size);
    if (apart && adapt_one(g.m, g.k, g.ld_x, g.rank, g.adapters, size)) return launch_one(ctx, dtype, y_dtype, AdaptersOneArgs{d, u});
    launch_down(ctx, dtype, d);
    launch_up(ctx, dtype, y_dtype, u);
}

// ---- gradients ----
//
//   up_r = c_i g_r B_i,   dx_r = up_r A_i,   dA_i = sum up_r' x_r,   dB_i = sum g_r' down_r   (down_r = c_i x_r A_i')
//
// up and dx are the products above with the adapters turned.  The sums over rows take fp32 products as well: both factors are rows as they
// lie, a lane's eight neighbouring columns are one operand of eight products.  A training step of 4096 x 2048 x 2048 with rank 32 and three
// adapters, forward and back, is seven launches, 88 us: the products over long rows 2 x 11, with A and B 2 x 16, turning 9, the sums over rows 24 and
// their join 4.

// Blocks up to `adapters`: the rows of an adapter in order, behind those of the ones before it; at the end those of none.  Each of them reads all of
// `which` twice (256 columns to 256 with rank 8: 4096 rows of 64 adapters 10 us, 16384 of 1000 43, 65536 of 4000 510 out of 670 for all of the
// gradient).  Further ones turn 64 columns of an
// adapter: A [rank][k] to [k][rank], or B [n][rank] to [rank][n].
template <typename T>
__global__ __launch_bounds__(ADAPT_THREADS) void adapters_turn_kernel(AdaptersTurnArgs g) {
    __shared__ T s_tile[ADAPT_MAX_RANK * 65];
    __shared__ uint32_t s_before[ADAPT_WAVES], s_mine[ADAPT_WAVES];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    uint64_t b = blockIdx.x;
    if (b <= g.adapters) {
        // the last bin: rows without an adapter, or with one that is not there
        auto bin_of = [&](uint64_t r) {
            const int id = adapter_of(g.which, r, g.m, g.adapters);
            return r >= g.m ? ~0u : id < 0 ? g.adapters : (uint32_t)id;
        };
        constexpr uint32_t EACH = 8;           // neighbouring rows of a thread
        uint32_t before = 0;                   // rows of bins before this one
        for (uint64_t r0 = 0; r0 < g.m; r0 += ADAPT_THREADS * EACH) {
            uint32_t bin[EACH];
#pragma unroll
            for (uint32_t e = 0; e < EACH; ++e) bin[e] = bin_of(r0 + e * ADAPT_THREADS + threadIdx.x);
#pragma unroll
            for (uint32_t e = 0; e < EACH; ++e) before += bin[e] < b;
        }
        for (uint32_t d = 1; d < 64; d <<= 1) before += __shfl_xor(before, d, 64);
        if (lane == 0) s_before[wave] = before;
        __syncthreads();
        uint32_t at = s_before[0] + s_before[1] + s_before[2] + s_before[3];
        if (threadIdx.x == 0) g.first[b] = at;
        for (uint64_t r0 = 0; r0 < g.m; r0 += ADAPT_THREADS * EACH) {
            const uint64_t r = r0 + threadIdx.x * EACH;
            uint32_t mine = 0, n = 0;
#pragma unroll
            for (uint32_t e = 0; e < EACH; ++e) mine |= (uint32_t)(bin_of(r + e) == b) << e;
            n = (uint32_t)__popc(mine);
            uint32_t upto = n;                 // this lane's and those before it
#pragma unroll
            for (uint32_t d = 1; d < 64; d <<= 1) {
                const uint32_t o = __shfl_up(upto, d, 64);
                if (lane >= d) upto += o;
            }
            __syncthreads();
            if (lane == 63) s_mine[wave] = upto;
            __syncthreads();
            uint32_t to = at + upto - n;
            for (uint32_t w = 0; w < wave; ++w) to += s_mine[w];
            for (; mine; mine &= mine - 1u) g.rows[to++] = (uint32_t)r + (uint32_t)__ffs(mine) - 1u;
            at += s_mine[0] + s_mine[1] + s_mine[2] + s_mine[3];
        }
        return;
    }
    b -= g.adapters + 1u;
    const uint32_t tiles_a = (g.k + 63u) / 64u, tiles_b = (g.n + 63u) / 64u;
    const bool of_a = b < (uint64_t)tiles_a * g.adapters;
    if (!of_a) b -= (uint64_t)tiles_a * g.adapters;
    const uint32_t tiles = of_a ? tiles_a : tiles_b, cols = of_a ? g.k : g.n;
    const uint64_t i = b / tiles;
    const uint32_t c0 = (uint32_t)(b % tiles) * 64u, width = min(64u, cols - c0), all = width * g.rank;
    if (of_a) {
        const T* from = static_cast<const T*>(g.a) + i * g.rank * cols;
        T* to = static_cast<T*>(g.a_turned) + (i * cols + c0) * g.rank;
        for (uint32_t u = threadIdx.x; u < 64u * g.rank; u += ADAPT_THREADS)
            if (u % 64u < width) s_tile[u / 64u * 65u + u % 64u] = from[(uint64_t)(u / 64u) * cols + c0 + u % 64u];
        __syncthreads();
        for (uint32_t u = threadIdx.x; u < all; u += ADAPT_THREADS) to[u] = s_tile[u % g.rank * 65u + u / g.rank];
    } else {
        const T* from = static_cast<const T*>(g.b) + (i * cols + c0) * g.rank;
        T* to = static_cast<T*>(g.b_turned) + i * g.rank * cols + c0;
        for (uint32_t u = threadIdx.x; u < all; u += ADAPT_THREADS) s_tile[u % g.rank * 65u + u / g.rank] = from[u];
        __syncthreads();
        for (uint32_t u = threadIdx.x; u < 64u * g.rank; u += ADAPT_THREADS)
            if (u % 64u < width) to[(uint64_t)(u / 64u) * cols + u % 64u] = s_tile[u / 64u * 65u + u % 64u];
    }
}

// An adapter's parts have places of their own among `parts + adapters`: the ones before it that its rows' first number gives, and one more for
// each adapter before it, whose last part may not be whole.
__device__ __forceinline__ uint64_t part_of(uint32_t first, uint32_t adapter, uint32_t rows_each) { return first / rows_each + adapter; }

// Sums over the rows of an adapter, rows_each of them from blockIdx.y rows_each on: 128 columns of dA_i = sum up' x or, further blocks, of
// dB_i = sum g' down, 16 ranks a block.  Wavefronts take 16 rows in turn and join their sums in LDS.
template <typename T, bool CODES>
__global__ __launch_bounds__(ADAPT_THREADS, 3) void adapters_grad_kernel(AdaptersSumArgs g) {
    constexpr uint32_t DEPTH = 4;              // four rows each
    __shared__ v4f s_sum[2][8][64];
    const uint32_t lane = threadIdx.x & 63u, wave = uniform_u32(threadIdx.x >> 6), group = lane / 16u, r16 = lane & 15u;
    const uint32_t slabs_a = (g.k + ADAPT_SLAB - 1u) / ADAPT_SLAB, slabs = slabs_a + (g.n + ADAPT_SLAB - 1u) / ADAPT_SLAB;
    const uint32_t adapter = blockIdx.x / slabs, nth_slab = blockIdx.x - adapter * slabs;
    const bool of_a = nth_slab < slabs_a;
    const uint32_t slab = of_a ? nth_slab : nth_slab - slabs_a, cols = of_a ? g.k : g.n;
    const uint32_t c = slab * ADAPT_SLAB + 8u * r16;
    const float* s = of_a ? g.up : g.down;
    const uint64_t ld_s = of_a ? g.ld_up : g.ld_down;
    const uint32_t from = g.first[adapter], count = g.first[adapter + 1] - from;
    const uint32_t q0 = min(blockIdx.y * g.rows_each, count), q1 = min(q0 + g.rows_each, count);
    if (g.parts > 1 && q0 == q1) return;       // all wavefronts alike
    const uint32_t* list = g.rows + from;
    const bool codes = CODES && of_a, full = slab * ADAPT_SLAB + ADAPT_SLAB <= cols;
    const uint8_t* rows_x = static_cast<const uint8_t*>(of_a ? g.x : g.g);
    const uint64_t pitch = (of_a ? g.ld_x : g.ld_g) * (codes ? 1u : sizeof(T));
    struct Operands {
        Eight<T> v[DEPTH];
        uint2 w[DEPTH];
        float p[DEPTH], by[DEPTH];
    };
    const uint32_t rank0 = blockIdx.z * 16u, rank_at = min(rank0 + r16, g.rank - 1u);
    v4f acc[8];
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) acc[j] = v4f{0, 0, 0, 0};
    auto rows_at = [&](uint32_t at, uint32_t (&row)[DEPTH]) {
#pragma unroll
        for (uint32_t d = 0; d < DEPTH; ++d) row[d] = list[min(at + 4u * d + group, q1 - 1u)];
    };
    auto fetch = [&](const uint32_t (&row)[DEPTH], Operands& o) {
#pragma unroll
        for (uint32_t d = 0; d < DEPTH; ++d) {
            const uint8_t* from_row = rows_x + row[d] * pitch;
            if (codes) {                   // they are there up to a multiple of 16
                o.w[d] = make_uint2(0u, 0u);
                if (full || c < cols) o.w[d] = *reinterpret_cast<const uint2*>(from_row + c);
                o.by[d] = g.x_scale[row[d]];
            } else if (full) {
                o.v[d].load(reinterpret_cast<const T*>(from_row) + c);
            } else {
                fetch8(reinterpret_cast<const T*>(from_row), c, cols, o.v[d]);
            }
            o.p[d] = s[row[d] * ld_s + rank_at];
        }
    };
    // the next rows are on their way while these are multiplied, and where the ones after them are is known
    constexpr uint32_t TURN = ADAPT_WAVES * 4u * DEPTH;
    uint32_t at = q0 + wave * 4u * DEPTH, row[DEPTH];
    Operands next;
    if (at < q1) {
        rows_at(at, row);
        fetch(row, next);
        rows_at(at + TURN, row);
    }
    for (; at < q1; at += TURN) {
        const Operands o = next;
        if (at + TURN < q1) {
            fetch(row, next);
            rows_at(at + 2u * TURN, row);
        }
#pragma unroll
        for (uint32_t d = 0; d < DEPTH; ++d) {
            float x[8];
            if (codes) {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) x[j] = (float)(int8_t)((j < 4 ? o.w[d].x : o.w[d].y) >> (8 * (j % 4)));
            } else {
                Eight<T> v = o.v[d];
                if (!full) place8(c, cols, v);
                v.floats(x);
            }
            float p = codes ? o.p[d] * o.by[d] : o.p[d];
            if (at + 4u * DEPTH > q1) {    // behind the last row: its numbers once more, which do not count
                const bool in = at + 4u * d + group < q1;
                p = in ? p : 0.0f;
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) x[j] = in ? x[j] : 0.0f;
            }
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(p, x[j], acc[j], 0, 0, 0);
        }
    }
    // wavefronts 2 and 3 to 0 and 1, then 1 to 0
#pragma unroll
    for (uint32_t half = 2; half > 0; half >>= 1) {
        __syncthreads();
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) s_sum[wave - half][j][lane] = acc[j];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) acc[j] += s_sum[wave][j][lane];
        }
    }
    if (wave != 0) return;
    // lane: ranks 4 group on, columns c on
    float* out = g.parts == 1 ? (of_a ? g.da : g.db) + (uint64_t)adapter * cols * g.rank
                              : g.partial + ((part_of(from, adapter, g.rows_each) + blockIdx.y) * (g.k + g.n) + (of_a ? 0 : g.k)) * g.rank;
    typedef float loose __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t r = rank0 + 4u * group;
    if (of_a) {
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
            if (r + e >= g.rank) continue;
            float* to = out + (uint64_t)(r + e) * cols + c;
            if (full) {
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h)
                    reinterpret_cast<loose*>(to)[h] = loose{acc[4 * h][e], acc[4 * h + 1][e], acc[4 * h + 2][e], acc[4 * h + 3][e]};
            } else {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j)
                    if (c + j < cols) to[j] = acc[j][e];
            }
        }
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
            if (c + j >= cols) continue;
            float* to = out + (uint64_t)(c + j) * g.rank + r;
            if (r + 4u <= g.rank) {
                *reinterpret_cast<loose*>(to) = loose{acc[j][0], acc[j][1], acc[j][2], acc[j][3]};
            } else {
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e)
                    if (r + e < g.rank) to[e] = acc[j][e];
            }
        }
    }
}

// The parts' sums of all adapters, in order; 0 for an adapter without rows.
__global__ __launch_bounds__(ADAPT_THREADS) void adapters_join_kernel(AdaptersSumArgs g) {
    const uint64_t of_a = (uint64_t)g.k * g.rank, each = of_a + (uint64_t)g.n * g.rank;
    const uint32_t adapter = blockIdx.y, from = g.first[adapter], count = g.first[adapter + 1] - from, parts = (count + g.rows_each - 1u) / g.rows_each;
    const float* p = g.partial + part_of(from, adapter, g.rows_each) * each;
    for (uint64_t u = (uint64_t)blockIdx.x * ADAPT_THREADS + threadIdx.x; u < each; u += (uint64_t)gridDim.x * ADAPT_THREADS) {
        float v = 0.0f, w[4];
        for (uint32_t i0 = 0; i0 < parts; i0 += 4) {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (i0 + i < parts) w[i] = p[(i0 + i) * each + u];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (i0 + i < parts) v += w[i];
        }
        if (u < of_a) g.da[adapter * of_a + u] = v;
        else g.db[adapter * (each - of_a) + u - of_a] = v;
    }
}

template <typename T, bool CODES>
static void launch_sums_as(shifter_ctx* ctx, const AdaptersSumArgs& g) {
    const dim3 grid(((g.k + ADAPT_SLAB - 1u) / ADAPT_SLAB + (g.n + ADAPT_SLAB - 1u) / ADAPT_SLAB) * g.adapters, g.parts, (uint32_t)adapt_pad(g.rank) / 16u);
    adapters_grad_kernel<T, CODES><<<grid, ADAPT_THREADS, 0, ctx->stream>>>(g);
}

template <typename T>
static void launch_gradients(shifter_ctx* ctx, int dtype, const AdaptersGradArgs& g) {
    const AdaptersGradPlan p = adapters_grad_plan(g.m, g.n, g.k, g.rank, g.adapters, sizeof(T));
    auto at = [&](uint64_t offset) { return g.work + offset; };
    const uint32_t pad = (uint32_t)adapt_pad(g.rank);
    AdaptersTurnArgs t{};
    t.which = g.which; t.a = g.a; t.b = g.b; t.m = g.m; t.n = g.n; t.k = g.k; t.rank = g.rank; t.adapters = g.adapters;
    t.a_turned = at(p.a); t.b_turned = at(p.b);
    t.rows = reinterpret_cast<uint32_t*>(at(p.rows)); t.first = reinterpret_cast<uint32_t*>(at(p.first));
    {
        ProfileScope ps(ctx, K_ADAPTERS_TURN);
        const uint64_t blocks = 1ull + g.adapters * (1ull + (g.k + 63u) / 64u + (g.n + 63u) / 64u);
        adapters_turn_kernel<T><<<(uint32_t)blocks, ADAPT_THREADS, 0, ctx->stream>>>(t);
    }
    AdaptersDownArgs d{};
    d.which = g.which; d.scale = g.scale; d.m = g.m; d.rank = g.rank; d.adapters = g.adapters;
    d.s = reinterpret_cast<float*>(at(p.sums));
    // rows are taken in the lists' order where they would be put in order without a gradient too: not with more than ADAPT_SORT_MOST adapters
    d.order = adapt_sorted(g.m, g.adapters) ? t.rows : nullptr;
    AdaptersUpArgs u{};
    u.s = d.s; u.order = d.order; u.which = g.which; u.m = g.m; u.rank = g.rank; u.adapters = g.adapters;
    const float* down = g.down;
    uint64_t ld_down = g.rank;
    if (!down && g.m) {                        // once more; its sums are joined by a pass that writes no columns
        d.x = g.x; d.ld_x = g.ld_x; d.x_scale = g.x_scale; d.a = g.a; d.k = g.k; d.parts = p.parts_x;
        launch_down(ctx, dtype, d);
        u.parts = p.parts_x; u.n = 0; u.b = g.b; u.down = reinterpret_cast<float*>(at(p.down)); u.down_cols = pad;
        launch_up(ctx, dtype, dtype, u);
        down = u.down;
        ld_down = pad;
    }
    d.x = g.g; d.ld_x = g.ld_g; d.x_scale = nullptr; d.a = at(p.b); d.k = g.n; d.parts = p.parts_g;
    if (g.m) launch_down(ctx, dtype, d);
    u.parts = p.parts_g; u.n = g.dx ? g.k : 0; u.b = at(p.a); u.out = g.dx; u.ld_out = g.ld_dx;
    u.down = reinterpret_cast<float*>(at(p.up)); u.down_cols = pad;
    if (g.m) launch_up(ctx, dtype, dtype, u);
    if (g.adapters == 0 || (g.n == 0 && g.k == 0)) return;
    AdaptersSumArgs s{};
    s.x = g.x; s.ld_x = g.ld_x; s.x_scale = g.x_scale; s.g = g.g; s.ld_g = g.ld_g;
    s.up = u.down; s.ld_up = pad; s.down = down; s.ld_down = ld_down;
    s.rows = t.rows; s.first = t.first; s.n = g.n; s.k = g.k; s.rank = g.rank; s.adapters = g.adapters; s.parts = p.parts_rows; s.rows_each = p.rows_each;
    s.da = g.da; s.db = g.db; s.partial = reinterpret_cast<float*>(at(p.partial));
    ProfileScope ps(ctx, K_ADAPTERS_GRAD);
    if (g.x_scale) launch_sums_as<T, true>(ctx, s);
    else launch_sums_as<T, false>(ctx, s);
    if (s.parts > 1) {
        const uint64_t each = (uint64_t)(g.k + g.n) * g.rank;
        const dim3 grid((uint32_t)std::min<uint64_t>((each + ADAPT_THREADS - 1u) / ADAPT_THREADS, 1024), g.adapters);
        adapters_join_kernel<<<grid, ADAPT_THREADS, 0, ctx->stream>>>(s);
    }
}

void launch_adapters_grad(shifter_ctx* ctx, int dtype, const AdaptersGradArgs& g) {
    if (dtype == SHIFTER_F32) launch_gradients<float>(ctx, dtype, g);
    else if (dtype == SHIFTER_BF16) launch_gradients<__bf16>(ctx, dtype, g);
    else launch_gradients<_Float16>(ctx, dtype, g);
}

}  // namespace shifter

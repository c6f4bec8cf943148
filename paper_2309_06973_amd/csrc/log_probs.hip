// Log probabilities of given targets, entropies and the likeliest alternatives of rows of logits, and their gradient.
//
//   z = scale x,  lse = log sum e^z,  log p = z - lse,  H = -sum p log p
//
// One read of x: a thread holds m = max x, s = sum 2^d and u = sum d 2^d with d = (x - m) scale log2 e of what it has seen,
// and scales s and u when m grows (u' = f (u + D s) for a step of D, f = 2^D).  Sums of two threads join in the same way.  Then
// lse = scale m + log s and H = log s - (u log 2) / s: no difference of large numbers, u <= 0.  m, s and u are in 32 bits, what is
// worked out of them in 64.  A logit of minus infinity has no probability and adds nothing, also where all d 2^d
// would be 0 times infinity; +infinity and NaN make s NaN, and with it whatever the row gives.
//
// Alternatives are the largest in the order of (logit, lower index), as one 64-bit number.  While a row is read each thread keeps
// the largest logit of its own and the eight columns that hold it.  The k-th largest of 64 groups of threads is a bound that
// k logits at least reach and hardly more than k do (24 of random ones for k = 20), and only the threads that do are looked at again, from the
// cache: their logits above the bound are ranked by counting.  That leaves one maximum a logit in the loop.
//
// Memory bounds long rows; see the figures at the kernels.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "dev_common.h"
#include "learn.h"
#include "q8_eight.h"

namespace shifter {

constexpr float LOG2E = 1.44269504088896341f;
constexpr double LN2 = 0.693147180559945309;
constexpr float LEAST = -3.402823466e38f;          // where m starts: a row of minus infinities has s = 0
constexpr float FAR = -1000.0f;                    // 2^FAR is 0 in 32 bits

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// d of two logits.  Both are taken in `unit`, 1 or less, as their difference may be beyond fp32 where the scale brings it back; a power of two, so that
// nothing is rounded but the difference and the product, and with 1 the difference is x - m to the bit.
struct Distance {
    float unit, c;                     // c: log2 e times the scale, of logits in that unit
    __device__ __forceinline__ float operator()(float x, float m) const { return fmaf(x, unit, -(m * unit)) * c; }
};

struct Sums {
    float m, s, u;
};

// The sums of both.  The same to the bit whichever comes first, so that all lanes that exchange theirs hold the same.
template <bool H>
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b, const Distance& c) {
    const bool first = a.m >= b.m;
    const float m = first ? a.m : b.m, less = first ? b.m : a.m, s = first ? b.s : a.s;
    const float d = c(less, m), f = exp2_of(d);
    Sums r;
    r.m = m;
    r.s = fmaf(f, s, first ? a.s : b.s);
    r.u = 0.0f;
    if constexpr (H) r.u = fmaf(f, fmaf(fmaxf(d, FAR), s, first ? b.u : a.u), first ? a.u : b.u);
    return r;
}

// Logits in order as whole numbers, both zeros alike, NaN last with minus infinity; with the column, lower ones first.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0x007fffffu;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t order) {
    return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order);
}
__device__ __forceinline__ uint64_t place_of(uint32_t order, uint32_t col) { return (uint64_t)order << 32 | (uint32_t)~col; }

// What a thread has seen of a row.
struct Best {
    float x = -INFINITY;
    uint32_t at = 0xffffffffu;         // first of the eight columns that hold it
};

// U pieces of 8 logits whose first columns are c0, c0 + step, ..., of a row that ends at `end`.
template <uint32_t U, bool H, bool TOP>
__device__ __forceinline__ void take(const float (&f)[8 * U], uint32_t c0, uint32_t step, uint32_t end, const Distance& c, Sums& a, Best& best) {
    float most = a.m;
#pragma unroll
    for (uint32_t p = 0; p < U; ++p) {
        const float top = fmaxf(fmaxf(fmaxf(f[8 * p], f[8 * p + 1]), fmaxf(f[8 * p + 2], f[8 * p + 3])),
                                fmaxf(fmaxf(f[8 * p + 4], f[8 * p + 5]), fmaxf(f[8 * p + 6], f[8 * p + 7])));
        most = fmaxf(most, top);
        if constexpr (TOP) {
            if ((top > best.x || best.at == 0xffffffffu) && c0 + p * step < end) {
                best.x = fmaxf(top, -INFINITY);
                best.at = c0 + p * step;
            }
        }
    }
    const float d = c(a.m, most), g = exp2_of(d);
    if constexpr (H) a.u = g * fmaf(fmaxf(d, FAR), a.s, a.u);
    a.s *= g;
    a.m = most;
#pragma unroll
    for (uint32_t i = 0; i < 8 * U; ++i) {
        const float t = c(f[i], most), e = exp2_of(t);
        a.s += e;
        if constexpr (H) a.u = fmaf(e, fmaxf(t, FAR), a.u);
    }
}

// The columns [c0, end) of a row by TPR threads, U pieces of 8 columns of each under way, the last of which stay in `e`.  Pieces behind
// the end and the one that holds it are fetched from inside the row, so that no load stands in a branch.
template <typename T, uint32_t TPR, uint32_t U, bool H, bool TOP>
__device__ __forceinline__ void scan(const T* row, uint32_t c0, uint32_t end, uint32_t t, const Distance& c, Sums& a, Best& best,
                                     Eight<T> (&e)[U]) {
    constexpr uint32_t STEP = 8 * TPR;
    auto batch = [&](uint32_t at, auto last) {
        float f[8 * U];
#pragma unroll
        for (uint32_t p = 0; p < U; ++p) {
            if constexpr (last.value) fetch8(row, at + p * STEP, end, e[p]);
            else e[p].load(row + at + p * STEP);
        }
#pragma unroll
        for (uint32_t p = 0; p < U; ++p) {
            float g[8];
            if constexpr (last.value) place8(at + p * STEP, end, e[p]);
            e[p].floats(g);
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) f[8 * p + i] = !last.value || at + p * STEP + i < end ? g[i] : -INFINITY;
        }
        take<U, H, TOP>(f, at, STEP, last.value ? end : 0xffffffffu, c, a, best);
    };
    uint32_t at = c0;
    for (; at + U * STEP <= end; at += U * STEP) batch(at + 8 * t, std::false_type{});
    if (at < end) batch(at + 8 * t, std::true_type{});
}

// The TPR threads of a row together.
template <uint32_t TPR>
__device__ __forceinline__ void meet() {
    if constexpr (TPR > 64) {
        __syncthreads();
    } else {                            // a wavefront's LDS accesses are done in order
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
}

// LDS of a row.  CAP: places that are ranked at once.
template <uint32_t TPR, bool TOP>
struct RowShared {
    static constexpr uint32_t WAVES = TPR > 64 ? TPR / 64 : 1, CAP = !TOP ? 1 : TPR == 16 ? 128 : TPR == 64 ? 512 : 1024;
    Sums sums[WAVES];
    uint64_t group[WAVES][TOP && TPR > 64 ? 64 : 1];
    uint64_t place[CAP + 8];
    uint64_t bound;
    uint32_t count, winners, last;
    uint16_t winner[TOP && TPR > 64 ? TPR : 1];
};

// The lane's value that DPP pattern CTRL pairs it with: neighbours by 1 and 2, mirrors of 8 and 16.
template <int CTRL>
__device__ __forceinline__ float beside(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL, bool H>
__device__ __forceinline__ void join_beside(Sums& a, const Distance& c) {
    a = join<H>(a, Sums{beside<CTRL>(a.m), beside<CTRL>(a.s), H ? beside<CTRL>(a.u) : 0.0f}, c);
}
// The sums of a wavefront's lanes, or of 16 of them, in all of these.
template <uint32_t LANES, bool H>
__device__ __forceinline__ Sums sum_lanes(Sums a, const Distance& c) {
    join_beside<0xB1, H>(a, c);
    join_beside<0x4E, H>(a, c);
    join_beside<0x141, H>(a, c);
    join_beside<0x140, H>(a, c);
    if constexpr (LANES == 64) {
        auto of = [&](int lane) {
            auto one = [&](float v) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); };
            return Sums{one(a.m), one(a.s), H ? one(a.u) : 0.0f};
        };
        a = join<H>(join<H>(of(0), of(16), c), join<H>(of(32), of(48), c), c);
    }
    return a;
}

template <uint32_t TPR, bool H, bool TOP>
__device__ __forceinline__ Sums sum_up(Sums a, uint32_t t, const Distance& c, RowShared<TPR, TOP>& sh) {
    a = sum_lanes<(TPR < 64 ? TPR : 64), H>(a, c);
    if constexpr (TPR > 64) {
        if ((t & 63u) == 0) sh.sums[t / 64] = a;
        meet<TPR>();
        a = sh.sums[0];
#pragma unroll
        for (uint32_t w = 1; w < TPR / 64; ++w) a = join<H>(a, sh.sums[w], c);
    }
    return a;
}

// The k-th largest of the numbers that the lanes of a wavefront (of a group of 16 of them) hold, or a lower one that no further
// lane reaches; 0 where fewer than k hold one.  Zero is none.  Bit by bit, the upper word first: mostly that is enough.
template <uint32_t LANES>
__device__ __forceinline__ uint64_t kth_of(uint64_t v, uint32_t k) {
    const uint32_t high = (uint32_t)(v >> 32), low = (uint32_t)v;
    uint32_t top = 0, rest = 0;
    if constexpr (LANES == 64) {
        if ((uint32_t)__popcll(__ballot(v != 0)) < k) return 0;
        for (uint32_t bit = 1u << 31; bit; bit >>= 1) {
            const uint32_t n = (uint32_t)__popcll(__ballot(high >= (top | bit)));
            if (n >= k) top |= bit;
            if (n == k) return (uint64_t)top << 32;
        }
        const uint64_t over = __ballot(high > top);
        for (uint32_t bit = 1u << 31; bit; bit >>= 1) {
            const uint32_t n = (uint32_t)__popcll(over | __ballot(high == top && low >= (rest | bit)));
            if (n >= k) rest |= bit;
            if (n == k) break;
        }
    } else {                            // a bound for each group, until all have theirs
        const uint64_t mine = ((1ull << LANES) - 1ull) << ((threadIdx.x & 63u) / LANES * LANES);
        bool done = (uint32_t)__popcll(__ballot(v != 0) & mine) < k;
        for (uint32_t bit = 1u << 31; bit && __ballot(!done); bit >>= 1) {
            const uint32_t n = (uint32_t)__popcll(__ballot(high >= (top | bit)) & mine);
            if (!done && n >= k) top |= bit;
            done = done || n == k;
        }
        if (__ballot(!done)) {
            const uint64_t over = __ballot(high > top) & mine;
            for (uint32_t bit = 1u << 31; bit && __ballot(!done); bit >>= 1) {
                const uint32_t n = (uint32_t)__popcll(over | (__ballot(high == top && low >= (rest | bit)) & mine));
                if (!done && n >= k) rest |= bit;
                done = done || n == k;
            }
        }
    }
    return (uint64_t)top << 32 | rest;
}

// Puts a place that reaches the bound on the list, if there is room.  Zero is none.
template <uint32_t TPR, bool TOP>
__device__ __forceinline__ void list(RowShared<TPR, TOP>& sh, uint64_t v, uint64_t bound) {
    if (v < bound || v == 0) return;
    const uint32_t n = atomicAdd(&sh.count, 1u);
    if (n < RowShared<TPR, TOP>::CAP) sh.place[n] = v;
}
// The same for the eight columns from `at` on of a row that ends at `end`.
template <typename T, uint32_t TPR, bool TOP>
__device__ __forceinline__ void list8(RowShared<TPR, TOP>& sh, const Eight<T>& e, uint32_t at, uint32_t end, uint64_t bound) {
    float f[8];
    e.floats(f);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
        if (at + i < end) list(sh, place_of(order_of(f[i]), at + i), bound);
}

// The k largest of the places that find(bound) lists, place(rank, v) for each.  Where more than the list holds reach the
// bound, the k-th of those that are on it is a higher one that at least k reach, and they are looked for again: the list's others are
// out each time.
template <uint32_t TPR, bool TOP, typename Find, typename Put>
__device__ __forceinline__ void rank(RowShared<TPR, TOP>& sh, uint32_t t, uint32_t k, uint64_t bound, Find find, Put put) {
    constexpr uint32_t CAP = RowShared<TPR, TOP>::CAP;
    for (;;) {
        if (t == 0) sh.count = 0;
        meet<TPR>();
        find(bound);
        meet<TPR>();
        const uint32_t n = sh.count, held = min(n, CAP);
        for (uint32_t i = t; i < held; i += TPR) {
            const uint64_t v = sh.place[i];
            uint32_t above = 0;
            for (uint32_t j = 0; j < held; j += 8) {
                uint64_t w[8];
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) w[e] = sh.place[j + e];
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) above += (uint32_t)(j + e < held) & (uint32_t)(w[e] > v);
            }
            if (n <= CAP) {
                if (above < k) put(above, v);
            } else if (above == k - 1) {
                sh.bound = v;
            }
        }
        meet<TPR>();
        if (n <= CAP) return;
        bound = sh.bound;
    }
}

// A row's results from its sums.
struct RowEnd {
    double most, log_s;                // scale m, log s
    __device__ __forceinline__ RowEnd(const Sums& a, float scale) : most((double)a.m * scale), log_s(log((double)a.s)) {}
    __device__ __forceinline__ float of(float x, float m, float scale) const {
        return (float)(((double)x - (double)m) * scale - log_s);
    }
};

// One launch: where blocks share a row, the last of them to end joins what all have left.  8192 x 32768 bf16 without alternatives or
// entropy 91 us by itself (537 MB, 5.9 TB/s), 112 behind a gradient whose results are still on their way to memory (4.8), 2048 x 50001 fp16 with entropy 51 (205 MB, 4.0 TB/s: eleven instructions a logit and an exponential),
// 128 x 131072 bf16 with entropy and 20 alternatives 20.4, without alternatives 10.1 (34 MB, 3.3 TB/s).  A single row of 50001 with 20
// takes 14.0, 6.2 without: a launch and one trip to memory, and with alternatives two rankings of some 24 places and the trip between
// blocks, each step of which waits for the one before.
template <typename T, uint32_t TPR, bool H, bool TOP>
__global__ __launch_bounds__(TPR < BLOCK ? BLOCK : TPR) void log_probs_kernel(LogProbsArgs g, LogProbsPlan plan) {
    constexpr uint32_t AT_ONCE = TPR < BLOCK ? BLOCK / TPR : 1u, U = TPR > 64 ? (sizeof(T) == 2 ? 4 : 2) : 2;
    __shared__ RowShared<TPR, TOP> shared[AT_ONCE];
    const uint32_t t = threadIdx.x % TPR;
    RowShared<TPR, TOP>& sh = shared[threadIdx.x / TPR];
    const Distance c{g.unit, g.by * LOG2E};
    const uint64_t all = (uint64_t)g.rows * plan.parts;
    for (uint64_t i = (uint64_t)blockIdx.x * AT_ONCE + threadIdx.x / TPR; i < all; i += (uint64_t)gridDim.x * AT_ONCE) {
        const uint64_t r = plan.parts == 1 ? i : i / plan.parts;
        const uint32_t part = (uint32_t)(i - r * plan.parts), c0 = part * plan.part_cols, end = min(c0 + plan.part_cols, g.cols);
        const T* row = static_cast<const T*>(g.x) + r * g.ld_x;
        int64_t target = -1;
        if (g.target && t == 0) target = g.target[r];
        Sums a{LEAST, 0.0f, 0.0f};
        Best best;
        Eight<T> e[U];
        scan<T, TPR, U, H, TOP>(row, c0, end, t, c, a, best, e);
        // the target's logit is on its way while the sums are joined
        float x_t = 0.0f;
        if (target >= 0 && target < (int64_t)g.cols) x_t = (float)row[target];
        a = sum_up<TPR, H, TOP>(a, t, c, sh);

        uint64_t bound = 0;
        // the part's own alternatives: as many as are asked for, or all that it has
        const uint32_t k = TOP ? min(g.top, end - c0) : 0u;
        auto find = [&](uint64_t least) {
            static_assert(TPR > 64 || U * 8 * TPR == 16 * TPR, "as many columns as the plan gives so many threads");
            const bool wins = best.at != 0xffffffffu && place_of(order_of(best.x), best.at) >= least;
            if constexpr (TPR <= 64) {             // a thread still holds all that it has seen
                if (!wins) return;
#pragma unroll
                for (uint32_t p = 0; p < U; ++p) list8(sh, e[p], c0 + 8 * (p * TPR + t), end, least);
            } else {                    // all pieces of the threads that do, by all threads
                if (t == 0) sh.winners = 0;
                meet<TPR>();
                if (wins) sh.winner[atomicAdd(&sh.winners, 1u)] = (uint16_t)t;
                meet<TPR>();
                const uint32_t pieces = (end - c0 + 8 * TPR - 1) / (8 * TPR), todo = pieces * sh.winners;
                for (uint32_t i = t; i < todo; i += TPR) {
                    const uint32_t w = i / pieces, at = c0 + 8 * ((i - w * pieces) * TPR + sh.winner[w]);
                    if (at < end) {
                        Eight<T> x;
                        fetch8(row, at, end, x);
                        place8(at, end, x);
                        list8(sh, x, at, end, least);
                    }
                }
            }
        };
        if constexpr (TOP) {
            // the last column that may hold a thread's largest: a place that its logits reach
            const uint64_t v = best.at == 0xffffffffu ? 0ull : place_of(order_of(best.x), min(best.at + 7u, end - 1u));
            if constexpr (TPR <= 64) {
                bound = kth_of<TPR>(v, k);
            } else {
                sh.group[t / 64][t & 63u] = v;
                meet<TPR>();
                if (t < 64) {
                    uint64_t most = v;
#pragma unroll
                    for (uint32_t w = 1; w < TPR / 64; ++w) most = max(most, sh.group[w][t]);
                    most = kth_of<64>(most, k);
                    if (t == 0) sh.bound = most;
                }
                meet<TPR>();
                bound = sh.bound;
            }
        }

        auto finish = [&](const Sums& s, const RowEnd& e) {
            if (t == 0) {
                g.norm[2 * r] = s.m;
                g.norm[2 * r + 1] = (float)e.log_s;
                g.lse[r] = (float)(e.most + e.log_s);
                if (g.logp) g.logp[r] = target < 0 ? 0.0f : target < (int64_t)g.cols ? e.of(x_t, s.m, g.scale) : NAN;
                if (H) g.entropy[r] = (float)(e.log_s - LN2 * (double)s.u / (double)s.s);
            }
        };
        auto put = [&](const Sums& s, const RowEnd& e, uint32_t n, uint64_t v) {
            const float x = logit_of((uint32_t)(v >> 32));
            g.top_logp[r * g.top + n] = e.of(x, s.m, g.scale);
            g.index[r * g.top + n] = (int64_t)(uint32_t)~(uint32_t)v;
        };
        if (plan.parts == 1) {
            const RowEnd e(a, g.scale);
            finish(a, e);
            if constexpr (TOP) rank(sh, t, k, bound, find, [&](uint32_t n, uint64_t v) { put(a, e, n, v); });
            else meet<TPR>();
            continue;
        }
        if constexpr (TPR > 64) {
            const uint32_t entry = 2 + g.top;          // words of 8 bytes
            unsigned long long* left = reinterpret_cast<unsigned long long*>(g.work + LEARN_TICKETS) + r * plan.parts * entry;
            unsigned long long* mine = left + (uint64_t)part * entry;
            auto leave = [](unsigned long long* p, uint64_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
            auto found = [](const unsigned long long* p) { return (uint64_t)__hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
            if (t == 0) {
                leave(mine, (uint64_t)__float_as_uint(a.s) << 32 | __float_as_uint(a.m));
                leave(mine + 1, __float_as_uint(a.u));
            }
            if constexpr (TOP) {
                for (uint32_t n = k + t; n < g.top; n += TPR) leave(mine + 2 + n, 0);
                rank(sh, t, k, bound, find, [&](uint32_t n, uint64_t v) { leave(mine + 2 + n, v); });
            }
            uint32_t* ticket = reinterpret_cast<uint32_t*>(g.work) + r;
            if (last_block(ticket, plan.parts, &sh.last)) {
                // the counter is as it was before the call, for the next one
                if (t == 0) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                const uint32_t lane = t & 63u;
                Sums b{LEAST, 0.0f, 0.0f};
                uint64_t first = 0;
                if (lane < plan.parts) {               // every wavefront by itself
                    const uint64_t ms = found(left + (uint64_t)lane * entry);
                    b.m = __uint_as_float((uint32_t)ms);
                    b.s = __uint_as_float((uint32_t)(ms >> 32));
                    b.u = __uint_as_float((uint32_t)found(left + (uint64_t)lane * entry + 1));
                }
                if constexpr (TOP) {                   // the best of each part, 33 or more, or all
                    const uint32_t each = min(g.top, 64u / plan.parts);
                    if (lane < plan.parts * each) first = found(left + (uint64_t)(lane / each) * entry + 2 + lane % each);
                }
                b = sum_lanes<64, H>(b, c);
                const RowEnd e(b, g.scale);
                finish(b, e);
                if constexpr (TOP) {
                    bound = kth_of<64>(first, g.top);
                    auto lists = [&](uint64_t least) {
                        for (uint32_t n = t; n < plan.parts * g.top; n += TPR)
                            list(sh, found(left + (uint64_t)(n / g.top) * entry + 2 + n % g.top), least);
                    };
                    rank(sh, t, g.top, bound, lists, [&](uint32_t n, uint64_t v) { put(b, e, n, v); });
                }
            }
            meet<TPR>();
        }
    }
}

template <typename T, uint32_t TPR>
static void launch_log_probs_as(shifter_ctx* ctx, const LogProbsArgs& g, const LogProbsPlan& p) {
    constexpr uint32_t AT_ONCE = TPR < BLOCK ? BLOCK / TPR : 1u, THREADS = TPR < BLOCK ? BLOCK : TPR;
    const uint64_t blocks = ((uint64_t)g.rows * p.parts + AT_ONCE - 1u) / AT_ONCE;
    const uint32_t grid = (uint32_t)std::min<uint64_t>(blocks, LOGP_MAX_BLOCKS);
    if (g.top && g.entropy) log_probs_kernel<T, TPR, true, true><<<grid, THREADS, 0, ctx->stream>>>(g, p);
    else if (g.top) log_probs_kernel<T, TPR, false, true><<<grid, THREADS, 0, ctx->stream>>>(g, p);
    else if (g.entropy) log_probs_kernel<T, TPR, true, false><<<grid, THREADS, 0, ctx->stream>>>(g, p);
    else log_probs_kernel<T, TPR, false, false><<<grid, THREADS, 0, ctx->stream>>>(g, p);
}

template <typename T>
static void launch_log_probs_of(shifter_ctx* ctx, const LogProbsArgs& g) {
    const LogProbsPlan p = log_probs_plan(g.rows, g.cols, g.top);
    if (p.threads == 16) launch_log_probs_as<T, 16>(ctx, g, p);
    else if (p.threads == 64) launch_log_probs_as<T, 64>(ctx, g, p);
    else launch_log_probs_as<T, 256>(ctx, g, p);
}

void launch_log_probs(shifter_ctx* ctx, int dtype, const LogProbsArgs& g) {
    if (g.rows == 0) return;
    ProfileScope ps(ctx, K_LOG_PROBS);
    if (dtype == SHIFTER_F32) launch_log_probs_of<float>(ctx, g);
    else if (dtype == SHIFTER_BF16) launch_log_probs_of<__bf16>(ctx, g);
    else launch_log_probs_of<_Float16>(ctx, g);
}

// The gradient, in one read of x: p = 2^((scale (x - m) - log s) log2 e) once more, x - m in the same unit, from the row's m and log s: lse, their sum,
// would have lost log s where all that is left of a row is the type's lowest value.  A row whose factors are all 0 is zeros,
// whatever it holds.  Memory bounds it: 8192 x 32768 bf16, a fifth of the rows left out, 144 to 155 us right behind the sums, with 430 MB read and 537
// written (183, with no row left out, where the logits are in no cache).  Threads a row as for the sums, where 16, 64 and 256 are within a tenth of each other but for
// rows of 200 (8192 x 200 10.5 us with 16, 14.4 with 256).
template <typename T, uint32_t TPR, bool H>
__global__ __launch_bounds__(BLOCK) void log_probs_grad_kernel(LogProbsGradArgs g, uint32_t parts, uint32_t part_cols) {
    constexpr uint32_t AT_ONCE = BLOCK / TPR, U = 2;
    const uint32_t t = threadIdx.x % TPR;
    const uint64_t all = (uint64_t)g.rows * parts;
    for (uint64_t i = (uint64_t)blockIdx.x * AT_ONCE + threadIdx.x / TPR; i < all; i += (uint64_t)gridDim.x * AT_ONCE) {
        // from the last row to the first: the last ones are in the last-level cache still, where the sums have just been made
        const uint64_t nth = parts == 1 ? i : i / parts, r = g.rows - 1u - nth;
        const uint32_t c0 = (uint32_t)(i - nth * parts) * part_cols, end = min(c0 + part_cols, g.cols);
        const T* row = static_cast<const T*>(g.x) + r * g.ld_x;
        T* out = static_cast<T*>(g.dx) + r * g.ld_dx;
        const int64_t target = g.target ? g.target[r] : -1;
        float one = g.g_logp && target >= 0 ? g.g_logp[r] : 0.0f;
        if (target >= (int64_t)g.cols) one = NAN;
        const float m = g.norm[2 * r] * g.unit, log_s = g.norm[2 * r + 1], of_lse = g.g_lse ? g.g_lse[r] : 0.0f;
        const float by = isinf(of_lse - one) ? 0.5f : 1.0f, scale = g.scale / by;      // factors that only their difference takes beyond fp32: halves of them
        one *= by;
        const float all_p = of_lse * by - one;
        float h = 0.0f, by_h = 0.0f;
        if constexpr (H) {
            h = g.entropy[r];
            by_h = -g.g_entropy[r] * by;
        }
        const bool none = all_p == 0.0f && one == 0.0f && by_h == 0.0f;
        auto value = [&](float x, uint32_t col) {
            const float d = fmaf(fmaf(x, g.unit, -m), g.by, -log_s), p = exp2_of(d * LOG2E);
            // p first and the scale last: no factor of a row comes to the end of fp32 before p makes it small, and where p is 0 this is 0
            float v = all_p * p;
            if constexpr (H) v = fmaf(by_h, p * (fmaxf(d, FAR) + h), v);
            return (col == (uint32_t)target && target >= 0 ? v + one : v) * scale;
        };
        auto piece = [&](uint32_t at, const Eight<T>& e) {
            float f[8];
            e.floats(f);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) f[j] = value(f[j], at + j);
            Eight<T> o;
            o.from(f);
            o.store_through(out + at);       // past the caches, which hold what is read next (8192 x 32768 with its sums 273 -> 258 us)
        };
        if (none) {
            const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            Eight<T> o;
            o.from(zero);
            for (uint32_t at = c0 + 8 * t; at < end; at += 8 * TPR) {
                if (at + 8 <= end) o.store(out + at);
                else for (uint32_t j = at; j < end; ++j) out[j] = (T)0.0f;
            }
            continue;
        }
        uint32_t at = c0;
        for (; at + U * 8 * TPR <= end; at += U * 8 * TPR) {
            Eight<T> e[U];
#pragma unroll
            for (uint32_t p = 0; p < U; ++p) e[p].load(row + at + 8 * (p * TPR + t));
#pragma unroll
            for (uint32_t p = 0; p < U; ++p) piece(at + 8 * (p * TPR + t), e[p]);
        }
        for (at += 8 * t; at < end; at += 8 * TPR) {
            if (at + 8 <= end) {
                Eight<T> e;
                e.load(row + at);
                piece(at, e);
            } else {
                for (uint32_t j = at; j < end; ++j) out[j] = (T)value((float)row[j], j);
            }
        }
    }
}

template <typename T, uint32_t TPR>
static void launch_log_probs_grad_as(shifter_ctx* ctx, const LogProbsGradArgs& g, uint32_t parts, uint32_t part_cols) {
    const uint64_t blocks = ((uint64_t)g.rows * parts + BLOCK / TPR - 1u) / (BLOCK / TPR);
    const uint32_t grid = (uint32_t)std::min<uint64_t>(blocks, LOGP_MAX_BLOCKS);
    if (g.g_entropy) log_probs_grad_kernel<T, TPR, true><<<grid, BLOCK, 0, ctx->stream>>>(g, parts, part_cols);
    else log_probs_grad_kernel<T, TPR, false><<<grid, BLOCK, 0, ctx->stream>>>(g, parts, part_cols);
}

template <typename T>
static void launch_log_probs_grad_of(shifter_ctx* ctx, const LogProbsGradArgs& g) {
    const uint32_t cols8 = (g.cols + 7u) & ~7u;
    if (g.cols <= 256) return launch_log_probs_grad_as<T, 16>(ctx, g, 1, cols8);
    if (g.cols <= 1024) return launch_log_probs_grad_as<T, 64>(ctx, g, 1, cols8);
    // parts of 8192 columns at least: blocks that end evenly where rows are long and few
    const uint32_t parts = std::max(1u, g.cols / 8192u), each = ((g.cols + parts - 1u) / parts + 7u) & ~7u;
    launch_log_probs_grad_as<T, 256>(ctx, g, (g.cols + each - 1u) / each, each);
}

void launch_log_probs_grad(shifter_ctx* ctx, int dtype, const LogProbsGradArgs& g) {
    if (g.rows == 0 || g.cols == 0) return;
    ProfileScope ps(ctx, K_LOG_PROBS_GRAD);
    if (dtype == SHIFTER_F32) launch_log_probs_grad_of<float>(ctx, g);
    else if (dtype == SHIFTER_BF16) launch_log_probs_grad_of<__bf16>(ctx, g);
    else launch_log_probs_grad_of<_Float16>(ctx, g);
}

}  // namespace shifter

// The norm of many tensors' elements, and their clipping: N = sqrt(sum g^2) over what the masks keep, then
// min(1, max / (N + 1e-6)) g.
//
// Two streaming passes, a launch each (for up to GRAD_LIST tensors).  Squares are summed in 64 bits: no square overflows or is lost, and a
// sum's error is far below the one rounding of the result, whatever the order.  The order is fixed all the same: each block
// leaves the sum of its chunks, and the last block of the launch adds those up.  The second pass takes the chunks from the
// last to the first, so that what the first pass left in the last-level cache (256 MB) is read from there.  268 M fp32 in 17 tensors
// to others: 212 + 424 us, 3.2 GB at 5.0 TB/s, a large copy's rate; 25.5 M fp32 in 161 with masks 43 + 42 us (127 and 229 MB, from memory,
// which holds other tensors' results in its cache still).  268 M bf16 in 17 tensors 345 us, fp16 381 (1.6 GB, 4.7 and 4.2 TB/s), with masks fp32 722, bf16 508,
// fp16 623: there vector instructions take 42 % of the compute units' cycles in bf16's clipping and 71 % in fp16's, 24 % in the norm.  512 blocks with long runs: with 2048 the search for a block's first tensor and its
// ends cost as much as its elements (161 tensors 90 us for 85).
#include <cmath>
#include <type_traits>

#include "dev_common.h"
#include "learn.h"
#include "q8_eight.h"

namespace shifter {

constexpr uint32_t GRAD_THREADS = 256;
static_assert(GRAD_CHUNK == 8 * GRAD_THREADS, "a piece of eight elements a thread");

enum GradPart { GRAD_IN, GRAD_OUT, GRAD_MASK };

// Neighbouring elements of one tensor.
struct GradRun {
    uint64_t in, out, mask, n;         // addresses of the first one; how many
    uint32_t dtype;
};

// f(run) for the block's share of the list: the chunks [chunks part / parts, chunks (part + 1) / parts), a run for each tensor.
template <typename F>
__device__ __forceinline__ void each_run(const GradList& l, uint32_t part, uint32_t parts, F f) {
    uint32_t at = (uint32_t)((uint64_t)l.chunks * part / parts);
    const uint32_t stop = (uint32_t)((uint64_t)l.chunks * (part + 1u) / parts);
    if (at == stop) return;
    for (uint32_t i = find_tensor(l.first, l.n, at); at < stop; ++i) {
        const uint32_t first = l.first[i], end = i + 1 < l.n ? l.first[i + 1] : l.chunks, last = l.last[i], to = min(end, stop);
        GradRun r;
        r.dtype = last >> 13;
        r.n = (uint64_t)(to - at) * GRAD_CHUNK - (to == end ? GRAD_CHUNK - 1u - (last & 8191u) : 0u);
        const uint64_t off = (uint64_t)(at - first) * GRAD_CHUNK, size = r.dtype == SHIFTER_F32 ? 4 : 2;
        auto address = [&](int part) { return (uint64_t)l.high[part][i] << 32 | l.low[part][i]; };
        r.in = address(GRAD_IN) + off * size;
        r.out = address(GRAD_OUT) + off * size;
        r.mask = address(GRAD_MASK);
        if (r.mask) r.mask += off;
        f(r);
        at = to;
    }
}

// An address of device memory as a pointer: that it is no other kind of memory is not to be found out by each access.
template <typename T>
__device__ __forceinline__ T* global(uint64_t address) {
    return (T*)(__attribute__((address_space(1))) T*)address;
}

// Eight of a mask's bytes, at any address.
__device__ __forceinline__ uint2 mask8(const uint8_t* p) {
    typedef uint32_t vec __attribute__((ext_vector_type(2), aligned(1)));
    const vec v = *reinterpret_cast<const vec*>(p);
    return make_uint2(v.x, v.y);
}
__device__ __forceinline__ bool kept(uint2 m, uint32_t i) { return ((i < 4 ? m.x : m.y) >> (8 * (i % 4)) & 255u) != 0; }

// Eight of a mask's bytes from `at` on of a run of n, zeros behind its end.
__device__ __forceinline__ uint2 mask_end(const uint8_t* p, uint64_t at, uint64_t n) {
    uint64_t w = 0;
    if (n >= 8) {
        if (at < n) {
            const uint64_t from = min(at, n - 8);
            const uint2 m = mask8(p + from);
            w = ((uint64_t)m.y << 32 | m.x) >> 8 * (at - from);
        }
    } else {
        for (uint32_t i = 0; i < 8; ++i)
            if (at + i < n) w |= (uint64_t)p[at + i] << 8 * i;
    }
    return make_uint2((uint32_t)w, (uint32_t)(w >> 32));
}

// f(first element, values, kept bytes) for the eights of a run, U of a thread's under way.  Behind the end are zeros.
template <typename T, bool MASK, uint32_t U, typename F>
__device__ __forceinline__ void each8(const GradRun& r, F f) {
    const T* in = global<const T>(r.in);
    const uint8_t* mask = global<const uint8_t>(r.mask);
    auto batch = [&](uint64_t at, auto last) {
        Eight<T> e[U];
        uint2 m[U];
        const uint32_t left = (uint32_t)min(r.n - (at - 8 * threadIdx.x), (uint64_t)U * GRAD_CHUNK);
        const T* from = in + (at - 8 * threadIdx.x);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint64_t a = at + u * GRAD_CHUNK;
            if constexpr (last.value) {
                if (r.n >= 8) e[u].load(in + min(a, r.n - 8));
                else fetch8(from, 8 * threadIdx.x + u * GRAD_CHUNK, left, e[u]);
                m[u] = MASK ? mask_end(mask, a, r.n) : make_uint2(~0u, ~0u);
            } else {
                e[u].load(in + a);
                m[u] = MASK ? mask8(mask + a) : make_uint2(~0u, ~0u);
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            float v[8];
            if constexpr (last.value) {
                // a run of eight and more: as a row of what is left, or of eight where less is
                const uint32_t c = 8 * threadIdx.x + u * GRAD_CHUNK;
                if (r.n >= 8 && c + 8u > left) {
                    if (c < left) e[u].drop(c + 8u - left);
                    else {
#pragma unroll
                        for (uint32_t i = 0; i < Eight<T>::WORDS; ++i) e[u].w[i] = 0u;
                    }
                }
            }
            e[u].floats(v);
            if (!last.value || at + u * GRAD_CHUNK < r.n) f(at + u * GRAD_CHUNK, v, m[u]);
        }
    };
    uint64_t at = 8 * threadIdx.x;
    for (uint64_t to = U * GRAD_CHUNK; to <= r.n; to += U * GRAD_CHUNK, at += U * GRAD_CHUNK) batch(at, std::false_type{});
    if (at - 8 * threadIdx.x < r.n) batch(at, std::true_type{});
}

template <typename T>
__device__ __forceinline__ void squares(const GradRun& r, double (&sum)[4]) {
    auto add = [&](uint64_t, const float (&v)[8], uint2 m) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const double x = kept(m, i) ? v[i] : 0.0f;
            sum[i % 4] = fma(x, x, sum[i % 4]);
        }
    };
    if (r.mask) each8<T, true, 4>(r, add);
    else each8<T, false, 4>(r, add);
}

template <uint32_t THREADS>
__device__ __forceinline__ double sum_of_block(double v, double* smem) {
#pragma unroll
    for (uint32_t d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if ((threadIdx.x & 63u) == 0) smem[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (uint32_t w = 0; w < THREADS / 64; ++w) v += smem[w];
    return v;
}

// sums: one a block of this launch, those of earlier launches before them; before: how many of those.  The last launch ends
// with the norm: in 64 bits at `norm64`, rounded at `norm`.
__global__ __launch_bounds__(GRAD_THREADS) void grad_norm_kernel(GradList l, double* sums, uint32_t before, uint32_t* ticket, double* norm64,
                                                                 float* norm) {
    __shared__ double smem[GRAD_THREADS / 64];
    __shared__ uint32_t s_last;
    double part[4] = {0.0, 0.0, 0.0, 0.0};
    each_run(l, blockIdx.x, gridDim.x, [&](const GradRun& r) {
        if (r.dtype == SHIFTER_F32) squares<float>(r, part);
        else if (r.dtype == SHIFTER_BF16) squares<__bf16>(r, part);
        else squares<_Float16>(r, part);
    });
    const double sum = sum_of_block<GRAD_THREADS>((part[0] + part[1]) + (part[2] + part[3]), smem);
    auto words = [](double* p) { return reinterpret_cast<unsigned long long*>(p); };
    if (threadIdx.x == 0) __hip_atomic_store(words(sums + before + blockIdx.x), (unsigned long long)__double_as_longlong(sum), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (!norm) return;
    if (!last_block(ticket, gridDim.x, &s_last)) return;
    double all = 0.0;
    for (uint32_t i = threadIdx.x; i < before + gridDim.x; i += GRAD_THREADS)
        all += __longlong_as_double((long long)__hip_atomic_load(words(sums + i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    all = sum_of_block<GRAD_THREADS>(all, smem);
    if (threadIdx.x == 0) {
        *norm64 = sqrt(all);
        *norm = (float)sqrt(all);
        *ticket = 0;                   // as it was, for the next call
    }
}

// min(1, max_norm / (norm + 1e-6)); NaN stays.
__device__ __forceinline__ double clip_factor(double norm, float max_norm) {
    const double by = (double)max_norm / (norm + 1e-6);
    return by >= 1.0 ? 1.0 : by;
}
// Up to eight elements: the product in 64 bits is right whatever the factor's size.
template <typename T>
__device__ __forceinline__ void write_scaled(T* out, uint64_t left, const float (&v)[8], uint2 m, double factor) {
    float r[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) r[i] = kept(m, i) ? (float)((double)v[i] * factor) : 0.0f;
    if (left >= 8) {
        Eight<T> e;
        e.from(r);
        e.store(out);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < left) out[i] = (T)r[i];
    }
}
template <typename T>
__device__ __forceinline__ void scale_run(const GradRun& r, double factor) {
    T* out = global<T>(r.out);
    auto write = [&](uint64_t at, const float (&v)[8], uint2 m) { write_scaled(out + at, r.n - at, v, m, factor); };
    if (r.mask) each8<T, true, 2>(r, write);
    else each8<T, false, 4>(r, write);
}

// Runs whose result is what they hold already are left: in place, without a mask, with a factor of 1.
__global__ __launch_bounds__(GRAD_THREADS) void grad_clip_kernel(GradList l, const double* norm64, float max_norm) {
    const double factor = clip_factor(*norm64, max_norm);
    each_run(l, gridDim.x - 1u - blockIdx.x, gridDim.x, [&](const GradRun& r) {
        if (factor == 1.0 && r.in == r.out && !r.mask) return;
        if (r.dtype == SHIFTER_F32) scale_run<float>(r, factor);
        else if (r.dtype == SHIFTER_BF16) scale_run<__bf16>(r, factor);
        else scale_run<_Float16>(r, factor);
    });
}

// Few elements by one block, which holds them in registers from the norm to the clipping: one launch, and one read.  The list's chunks
// are eights here.
constexpr uint32_t GRAD_SMALL_THREADS = 1024, GRAD_HELD = GRAD_SMALL / GRAD_SMALL_THREADS;
template <bool CLIP>
__global__ __launch_bounds__(GRAD_SMALL_THREADS) void grad_small_kernel(GradList l, float max_norm, float* norm) {
    __shared__ double smem[GRAD_SMALL_THREADS / 64];
    __shared__ uint32_t s_first[GRAD_LIST];
    for (uint32_t i = threadIdx.x; i < l.n; i += GRAD_SMALL_THREADS) s_first[i] = l.first[i];
    __syncthreads();
    float v[GRAD_HELD][8];
    uint2 m[GRAD_HELD];
    uint64_t out[GRAD_HELD];
    uint32_t n[GRAD_HELD], dtype[GRAD_HELD];
    double sum = 0.0;
#pragma unroll
    for (uint32_t h = 0; h < GRAD_HELD; ++h) {
        const uint32_t eight = threadIdx.x + h * GRAD_SMALL_THREADS;
        n[h] = 0;
        if (eight >= l.chunks) continue;
        uint32_t lo = 0, hi = l.n;             // the largest tensor whose first is not behind it
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (s_first[mid] <= eight) lo = mid; else hi = mid;
        }
        const uint32_t last = l.last[lo], end = lo + 1 < l.n ? s_first[lo + 1] : l.chunks, at = 8u * (eight - s_first[lo]);
        auto address = [&](int part) { return (uint64_t)l.high[part][lo] << 32 | l.low[part][lo]; };
        dtype[h] = last >> 13;
        n[h] = eight + 1 == end ? (last & 8191u) + 1u : 8u;
        const uint64_t in = address(GRAD_IN), mask = address(GRAD_MASK);
        out[h] = address(GRAD_OUT) + at * (dtype[h] == SHIFTER_F32 ? 4u : 2u);
        auto read = [&](auto* p) {
            p += at;
            if (n[h] == 8) {
                Eight<std::remove_const_t<std::remove_pointer_t<decltype(p)>>> e;
                e.load(p);
                e.floats(v[h]);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) v[h][i] = i < n[h] ? (float)p[i] : 0.0f;
            }
        };
        if (dtype[h] == SHIFTER_F32) read(global<const float>(in));
        else if (dtype[h] == SHIFTER_BF16) read(global<const __bf16>(in));
        else read(global<const _Float16>(in));
        m[h] = mask ? mask_end(global<const uint8_t>(mask) + at, 0, n[h]) : make_uint2(~0u, ~0u);
    }
#pragma unroll
    for (uint32_t h = 0; h < GRAD_HELD; ++h)
        if (n[h]) {
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                const double x = kept(m[h], i) ? v[h][i] : 0.0f;
                sum = fma(x, x, sum);
            }
        }
    const double all = sqrt(sum_of_block<GRAD_SMALL_THREADS>(sum, smem));
    if (threadIdx.x == 0) *norm = (float)all;
    if constexpr (CLIP) {
        const double factor = clip_factor(all, max_norm);
#pragma unroll
        for (uint32_t h = 0; h < GRAD_HELD; ++h) {
            if (n[h] == 0) continue;
            if (dtype[h] == SHIFTER_F32) write_scaled(global<float>(out[h]), n[h], v[h], m[h], factor);
            else if (dtype[h] == SHIFTER_BF16) write_scaled(global<__bf16>(out[h]), n[h], v[h], m[h], factor);
            else write_scaled(global<_Float16>(out[h]), n[h], v[h], m[h], factor);
        }
    }
}

void launch_grad_norm(shifter_ctx* ctx, const std::vector<shifter_grad>& all, bool clip, float max_norm, float* norm, uint8_t* work) {
    uint32_t* ticket = reinterpret_cast<uint32_t*>(work);
    double* norm64 = reinterpret_cast<double*>(work + LEARN_TICKETS);
    double* sums = reinterpret_cast<double*>(work + LEARN_TICKETS + GRAD_HEAD);
    GradList l;
    if (grad_small(all)) {
        ProfileScope ps(ctx, K_GRAD_NORM);
        grad_list(all, 0, 8, &l);
        if (clip) grad_small_kernel<true><<<1, GRAD_SMALL_THREADS, 0, ctx->stream>>>(l, max_norm, norm);
        else grad_small_kernel<false><<<1, GRAD_SMALL_THREADS, 0, ctx->stream>>>(l, max_norm, norm);
        return;
    }
    const uint64_t launches = grad_launches(all.size());
    auto blocks_of = [](const GradList& l) { return l.chunks == 0 ? 1u : std::min(l.chunks, GRAD_BLOCKS); };
    uint32_t before = 0;
    for (uint64_t i = 0; i < launches; ++i) {
        ProfileScope ps(ctx, K_GRAD_NORM);
        grad_list(all, i * GRAD_LIST, GRAD_CHUNK, &l);
        const uint32_t blocks = blocks_of(l);
        grad_norm_kernel<<<blocks, GRAD_THREADS, 0, ctx->stream>>>(l, sums, before, ticket, norm64, i + 1 == launches ? norm : nullptr);
        before += blocks;
    }
    if (!clip) return;
    for (uint64_t i = launches; i-- > 0;) {
        ProfileScope ps(ctx, K_GRAD_CLIP);
        if (i + 1 != launches) grad_list(all, i * GRAD_LIST, GRAD_CHUNK, &l);
        grad_clip_kernel<<<blocks_of(l), GRAD_THREADS, 0, ctx->stream>>>(l, norm64, max_norm);
    }
}

}  // namespace shifter

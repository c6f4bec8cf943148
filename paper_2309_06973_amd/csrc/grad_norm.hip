// The norm of many tensors' elements, and their clipping: N = sqrt(sum g^2) over what the masks keep, then
// min(1, max / (N + 1e-6)) g.
//
// Two streaming passes, a launch each (for up to GRAD_LIST tensors).  Squares are summed in 64 bits: no square overflows or is lost, and a
// sum's error is far below the one rounding of the result, whatever the order.  The order is fixed all the same: each block
// leaves the sum of its chunks, and the last block of the launch adds those up.  The second pass takes the chunks from the
// last to the first, so that what the first pass left in the last-level cache (256 MB) is read from there.
#include <cmath>

#include "dev_common.h"
#include "learn.h"
#include "q8_eight.h"

namespace shifter {

constexpr uint32_t GRAD_THREADS = 256, GRAD_PIECE = 8 * GRAD_THREADS;    // elements of a block at a time

enum GradPart { GRAD_IN, GRAD_OUT, GRAD_MASK };

struct GradChunk {
    uint64_t in, out, mask;            // addresses of its first element
    uint32_t n, dtype;
};

__device__ __forceinline__ GradChunk grad_chunk(const GradList& l, uint32_t chunk) {
    const uint32_t i = find_tensor(l.first, l.n, chunk);
    const uint32_t last = l.last[i], end = i + 1 < l.n ? l.first[i + 1] : l.chunks;
    GradChunk c;
    c.dtype = last >> 13;
    c.n = chunk + 1 == end ? (last & 8191u) + 1 : GRAD_CHUNK;
    const uint64_t at = (uint64_t)(chunk - l.first[i]) * GRAD_CHUNK, size = c.dtype == SHIFTER_F32 ? 4 : 2;
    auto address = [&](int part) { return (uint64_t)l.high[part][i] << 32 | l.low[part][i]; };
    c.in = address(GRAD_IN) + at * size;
    c.out = address(GRAD_OUT) + at * size;
    c.mask = address(GRAD_MASK);
    if (c.mask) c.mask += at;
    return c;
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

// f(first element, elements of it: 8 or fewer, values, kept bytes) for all of a chunk's, U pieces under way.
template <typename T, bool MASK, uint32_t U, typename F>
__device__ __forceinline__ void each8(const GradChunk& c, F f) {
    const T* in = global<const T>(c.in);
    const uint8_t* mask = global<const uint8_t>(c.mask);
    const uint32_t t = threadIdx.x * 8;
    uint32_t at = 0;
    for (; at + U * GRAD_PIECE <= c.n; at += U * GRAD_PIECE) {
        Eight<T> e[U];
        uint2 m[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            e[u].load(in + at + u * GRAD_PIECE + t);
            m[u] = MASK ? mask8(mask + at + u * GRAD_PIECE + t) : make_uint2(~0u, ~0u);
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            float v[8];
            e[u].floats(v);
            f(at + u * GRAD_PIECE + t, 8u, v, m[u]);
        }
    }
    for (at += t; at < c.n; at += GRAD_PIECE) {
        float v[8];
        uint2 m = make_uint2(~0u, ~0u);
        const uint32_t n = min(8u, c.n - at);
        if (n == 8) {
            Eight<T> e;
            e.load(in + at);
            e.floats(v);
            if (MASK) m = mask8(mask + at);
        } else {
            if (MASK) m = make_uint2(0u, 0u);
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                v[i] = i < n ? (float)in[at + i] : 0.0f;
                if (MASK && i < n && mask[at + i]) (i < 4 ? m.x : m.y) |= 255u << (8 * (i % 4));
            }
        }
        f(at, n, v, m);
    }
}

template <typename T>
__device__ __forceinline__ void squares(const GradChunk& c, double (&sum)[4]) {
    auto add = [&](uint32_t, uint32_t, const float (&v)[8], uint2 m) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const double x = kept(m, i) ? v[i] : 0.0f;
            sum[i % 4] = fma(x, x, sum[i % 4]);
        }
    };
    if (c.mask) each8<T, true, 2>(c, add);
    else each8<T, false, 4>(c, add);
}

__device__ __forceinline__ double sum_of_block(double v, double* smem) {
#pragma unroll
    for (uint32_t d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if ((threadIdx.x & 63u) == 0) smem[threadIdx.x / 64] = v;
    __syncthreads();
    return (smem[0] + smem[1]) + (smem[2] + smem[3]);
}

// sums: one a block of this launch, those of earlier launches before them; before: how many of those.  The last launch ends
// with the norm: in 64 bits at `norm64`, rounded at `norm`.
__global__ __launch_bounds__(GRAD_THREADS) void grad_norm_kernel(GradList l, double* sums, uint32_t before, uint32_t* ticket, double* norm64,
                                                                 float* norm) {
    __shared__ double smem[GRAD_THREADS / 64];
    __shared__ uint32_t s_last;
    double part[4] = {0.0, 0.0, 0.0, 0.0};
    for (uint32_t chunk = blockIdx.x; chunk < l.chunks; chunk += gridDim.x) {
        const GradChunk c = grad_chunk(l, chunk);
        if (c.dtype == SHIFTER_F32) squares<float>(c, part);
        else if (c.dtype == SHIFTER_BF16) squares<__bf16>(c, part);
        else squares<_Float16>(c, part);
    }
    const double sum = sum_of_block((part[0] + part[1]) + (part[2] + part[3]), smem);
    auto words = [](double* p) { return reinterpret_cast<unsigned long long*>(p); };
    if (threadIdx.x == 0) __hip_atomic_store(words(sums + before + blockIdx.x), (unsigned long long)__double_as_longlong(sum), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (!norm) return;
    if (!last_block(ticket, gridDim.x, &s_last)) return;
    double all = 0.0;
    for (uint32_t i = threadIdx.x; i < before + gridDim.x; i += GRAD_THREADS)
        all += __longlong_as_double((long long)__hip_atomic_load(words(sums + i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    all = sum_of_block(all, smem);
    if (threadIdx.x == 0) {
        *norm64 = sqrt(all);
        *norm = (float)sqrt(all);
        *ticket = 0;                   // as it was, for the next call
    }
}

template <typename T>
__device__ __forceinline__ void scale_chunk(const GradChunk& c, double factor) {
    T* out = global<T>(c.out);
    auto write = [&](uint32_t at, uint32_t n, const float (&v)[8], uint2 m) {
        float r[8];
        // the product in 64 bits is rounded once, whatever the factor's size
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) r[i] = kept(m, i) ? (float)((double)v[i] * factor) : 0.0f;
        if (n == 8) {
            Eight<T> e;
            e.from(r);
            e.store(out + at);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i)
                if (i < n) out[at + i] = (T)r[i];
        }
    };
    if (c.mask) each8<T, true, 2>(c, write);
    else each8<T, false, 4>(c, write);
}

// Chunks whose result is what they hold already are left: in place, without a mask, with a factor of 1.
__global__ __launch_bounds__(GRAD_THREADS) void grad_clip_kernel(GradList l, const double* norm64, float max_norm) {
    const double by = (double)max_norm / (*norm64 + 1e-6), factor = by >= 1.0 ? 1.0 : by;      // NaN stays
    for (uint32_t i = blockIdx.x; i < l.chunks; i += gridDim.x) {
        const GradChunk c = grad_chunk(l, l.chunks - 1 - i);
        if (factor == 1.0 && c.in == c.out && !c.mask) continue;
        if (c.dtype == SHIFTER_F32) scale_chunk<float>(c, factor);
        else if (c.dtype == SHIFTER_BF16) scale_chunk<__bf16>(c, factor);
        else scale_chunk<_Float16>(c, factor);
    }
}

void launch_grad_norm(shifter_ctx* ctx, const std::vector<shifter_grad>& all, bool clip, float max_norm, float* norm, uint8_t* work) {
    uint32_t* ticket = reinterpret_cast<uint32_t*>(work);
    double* norm64 = reinterpret_cast<double*>(work + LEARN_TICKETS);
    double* sums = reinterpret_cast<double*>(work + LEARN_TICKETS + GRAD_HEAD);
    const uint64_t launches = grad_launches(all.size());
    auto blocks_of = [](const GradList& l) { return l.chunks == 0 ? 1u : std::min(l.chunks, GRAD_BLOCKS); };
    GradList l;
    uint32_t before = 0;
    for (uint64_t i = 0; i < launches; ++i) {
        ProfileScope ps(ctx, K_GRAD_NORM);
        grad_list(all, i * GRAD_LIST, &l);
        const uint32_t blocks = blocks_of(l);
        grad_norm_kernel<<<blocks, GRAD_THREADS, 0, ctx->stream>>>(l, sums, before, ticket, norm64, i + 1 == launches ? norm : nullptr);
        before += blocks;
    }
    if (!clip || all.empty()) return;
    for (uint64_t i = launches; i-- > 0;) {
        ProfileScope ps(ctx, K_GRAD_CLIP);
        if (i + 1 != launches) grad_list(all, i * GRAD_LIST, &l);
        grad_clip_kernel<<<blocks_of(l), GRAD_THREADS, 0, ctx->stream>>>(l, norm64, max_norm);
    }
}

}  // namespace shifter

// Rows to 8 bits and back: plain rows (weights of an output channel, activations of a token),
// and rows behind an RMS norm with the residual's addition.
//
//   a = max |p|,  scale = a / 127,  code = 127 p / a to the nearest whole number, ties to even
//
// p is the row itself, its ReLU, or fl(h * weight) of the norm: the norm's common factor
// 1 / sqrt(mean(h^2) + eps) cancels in the codes and appears in the scale alone, so a row is
// coded without waiting for its sum of squares.  Codes are exact, that is the same on every
// machine and for every order of work: see q8_code.
//
// Streaming work: each row is read once into registers, reduced and written.
#include <algorithm>

#include "dev_common.h"
#include "q8.h"

namespace shifter {

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&f)[8]) {
    if constexpr (sizeof(T) == 4) {
        const uint4 a = load_u4<false>(reinterpret_cast<const float*>(p));
        const uint4 b = load_u4<false>(reinterpret_cast<const float*>(p) + 4);
        f[0] = __uint_as_float(a.x); f[1] = __uint_as_float(a.y); f[2] = __uint_as_float(a.z); f[3] = __uint_as_float(a.w);
        f[4] = __uint_as_float(b.x); f[5] = __uint_as_float(b.y); f[6] = __uint_as_float(b.z); f[7] = __uint_as_float(b.w);
    } else {
        typedef T vec __attribute__((ext_vector_type(8), aligned(2)));
        const vec v = *reinterpret_cast<const vec*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
    }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
    if constexpr (sizeof(T) == 4) {
        store_u4<false>(reinterpret_cast<float*>(p),
                        make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
        store_u4<false>(reinterpret_cast<float*>(p) + 4,
                        make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
    } else {
        typedef T vec __attribute__((ext_vector_type(8), aligned(2)));
        vec v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (T)f[i];
        *reinterpret_cast<vec*>(p) = v;
    }
}

// The first n < 8 elements alone; the others read as zero.
template <typename T>
__device__ __forceinline__ void load_part(const T* p, uint32_t n, float (&f)[8]) {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) f[i] = i < n ? (float)p[i] : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store_part(T* p, uint32_t n, const float (&f)[8]) {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
        if (i < n) p[i] = (T)f[i];
}

// 127 p / a to the nearest whole number, ties to even, exactly.  r = fl(127 / a), or 0 where a is so small
// that it could overflow (every value then takes the long way).  t = fl(p r) is within 127 * 2^-23 = 1.6e-5 of the
// quotient, so the nearest whole number is certain unless t lies within 2e-5 of a half; there one division
// in 64 bits decides: 127 p is exact in them, and the quotient of 24-bit numbers that is no tie is
// further than 2^-32 from one.
__device__ __forceinline__ float q8_code(float p, float a, float r) {
    const float t = __fmul_rn(p, r);
    float n = rintf(t);
    if (fabsf(fabsf(t - n) - 0.5f) < (r > 0.0f ? 4e-5f : 1.0f)) n = (float)rint(127.0 * (double)p / (double)a);
    return n;
}
__device__ __forceinline__ float q8_factor(float a) { return a >= 0x1p-100f ? 127.0f / a : 0.0f; }

// Eight codes as two words.
__device__ __forceinline__ uint2 q8_codes(const float (&p)[8], float a, float r) {
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i / 4] |= ((uint32_t)(int)q8_code(p[i], a, r) & 255u) << (8 * (i % 4));
    return make_uint2(w[0], w[1]);
}

// Largest and sum over the TPR threads of a row, in every one of them.
template <uint32_t TPR, bool SUM>
__device__ __forceinline__ void row_reduce(uint32_t& top, double& sum) {
#pragma unroll
    for (uint32_t d = 32; d > 0; d >>= 1) {
        top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
        if (SUM) sum += __shfl_xor(sum, d, 64);
    }
    if constexpr (TPR > 64) {
        __shared__ uint32_t s_top[TPR / 64];
        __shared__ double s_sum[TPR / 64];
        __syncthreads();                  // the row before has been read
        if ((threadIdx.x & 63u) == 0) {
            s_top[threadIdx.x >> 6] = top;
            if (SUM) s_sum[threadIdx.x >> 6] = sum;
        }
        __syncthreads();
        top = s_top[0];
        if (SUM) sum = s_sum[0];
#pragma unroll
        for (uint32_t i = 1; i < TPR / 64; ++i) {
            top = max(top, s_top[i]);
            if (SUM) sum += s_sum[i];
        }
    }
}

// The row's scale.  A row with a value that is not finite has no codes: its scale is NaN, so that whatever
// reads the row becomes NaN instead of a wrong number.
template <bool NORM>
__device__ __forceinline__ float row_scale(uint32_t top, double sum, const Q8RowsArgs& g) {
    if (top >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
    const float a = __uint_as_float(top);
    if (a == 0.0f) return 0.0f;
    return NORM ? (float)((double)a / (127.0 * sqrt(sum / (double)g.cols + (double)g.eps))) : a / 127.0f;
}

enum Q8Form { Q8_PLAIN, Q8_NORM, Q8_NORM_ADD };

// p of the eight elements from column c on; what lies behind the row's end is zero.  Adds to the sum of squares.
template <typename T, int FORM>
__device__ __forceinline__ void row_values(const Q8RowsArgs& g, uint64_t row, uint32_t c, float (&p)[8], double& sum,
                                           bool again = false) {
    const T* x = (again && FORM == Q8_NORM_ADD ? static_cast<const T*>(g.h) + row * g.ld_h
                                               : static_cast<const T*>(g.x) + row * g.ld_x) + c;
    const uint32_t n = c < g.cols ? min(g.cols - c, 8u) : 0u;
    if (n == 8) load8(x, p); else load_part(x, n, p);
    if constexpr (FORM == Q8_PLAIN) {
        if (g.relu) {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = p[i] < 0.0f ? 0.0f : p[i];
        }
    } else {
        if (FORM == Q8_NORM_ADD && !again) {
            float r[8];
            const T* res = static_cast<const T*>(g.residual) + row * g.ld_r + c;
            T* h = static_cast<T*>(g.h) + row * g.ld_h + c;
            if (n == 8) load8(res, r); else load_part(res, n, r);
            // the stream is held in its own type, and the norm is of what is held; the sum in 32 bits
            // first is rounded as the exact one would be (24 bits are more than twice 11 and two)
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = (float)(T)(p[i] + r[i]);
            if (n == 8) store8(h, p); else store_part(h, n, p);
        }
        float w[8];
        if (n == 8) load8(g.weight + c, w); else load_part(g.weight + c, n, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!again) sum = fma((double)p[i], (double)p[i], sum);
            p[i] = __fmul_rn(p[i], w[i]);
        }
    }
}

__device__ __forceinline__ uint32_t top8(const float (&p)[8], uint32_t top) {
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, key_of(p[i]));      // NaN and infinity come out on top
    return top;
}

// TPR threads a row, NV times eight elements in the registers of each.
template <typename T, int FORM, uint32_t TPR, uint32_t NV>
__global__ __launch_bounds__(TPR < BLOCK ? BLOCK : TPR) void q8_rows_kernel(Q8RowsArgs g) {
    constexpr uint32_t AT_ONCE = TPR < BLOCK ? BLOCK / TPR : 1u;      // rows of a block
    const uint32_t t = threadIdx.x % TPR, pad = (g.cols + Q8_ALIGN - 1u) & ~(Q8_ALIGN - 1u);
    for (uint64_t row = (uint64_t)blockIdx.x * AT_ONCE + threadIdx.x / TPR; row < g.rows;
         row += (uint64_t)gridDim.x * AT_ONCE) {
        float p[NV][8];
        uint32_t top = 0;
        double sum = 0.0;
#pragma unroll
        for (uint32_t v = 0; v < NV; ++v) {
            row_values<T, FORM>(g, row, (v * TPR + t) * 8u, p[v], sum);
            top = top8(p[v], top);
        }
        row_reduce<TPR, FORM != Q8_PLAIN>(top, sum);
        if (t == 0) g.scale[row] = row_scale<FORM != Q8_PLAIN>(top, sum, g);
        const bool none = top == 0u || top >= 0x7f800000u;
        const float a = __uint_as_float(top), r = none ? 0.0f : q8_factor(a);
        uint2* q = reinterpret_cast<uint2*>(g.q + row * g.ld_q);
#pragma unroll
        for (uint32_t v = 0; v < NV; ++v) {
            const uint32_t c = (v * TPR + t) * 8u;
            if (c < pad) q[c / 8u] = none ? make_uint2(0u, 0u) : q8_codes(p[v], a, r);
        }
    }
}

// Rows longer than the registers of a block: read a second time for the codes.
template <typename T, int FORM>
__global__ __launch_bounds__(1024) void q8_long_rows_kernel(Q8RowsArgs g) {
    constexpr uint32_t TPR = 1024;
    const uint32_t pad = (g.cols + Q8_ALIGN - 1u) & ~(Q8_ALIGN - 1u);
    for (uint64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
        uint32_t top = 0;
        double sum = 0.0;
        for (uint32_t c = threadIdx.x * 8u; c < pad; c += TPR * 8u) {
            float p[8];
            row_values<T, FORM>(g, row, c, p, sum);
            top = top8(p, top);
        }
        row_reduce<TPR, FORM != Q8_PLAIN>(top, sum);
        if (threadIdx.x == 0) g.scale[row] = row_scale<FORM != Q8_PLAIN>(top, sum, g);
        const bool none = top == 0u || top >= 0x7f800000u;
        const float a = __uint_as_float(top), r = none ? 0.0f : q8_factor(a);
        uint2* q = reinterpret_cast<uint2*>(g.q + row * g.ld_q);
        for (uint32_t c = threadIdx.x * 8u; c < pad; c += TPR * 8u) {
            float p[8];
            row_values<T, FORM>(g, row, c, p, sum, true);     // the stream comes from what this thread wrote
            q[c / 8u] = none ? make_uint2(0u, 0u) : q8_codes(p, a, r);
        }
    }
}

// A launch holds less than 2^32 threads; blocks take further rows in turn.
constexpr uint32_t Q8_MAX_BLOCKS = 1u << 21;

template <typename T, int FORM, uint32_t TPR, uint32_t NV>
static void launch_rows_as(shifter_ctx* ctx, const Q8RowsArgs& g) {
    constexpr uint32_t AT_ONCE = TPR < BLOCK ? BLOCK / TPR : 1u;
    const uint32_t blocks = std::min((g.rows + AT_ONCE - 1u) / AT_ONCE, Q8_MAX_BLOCKS);
    q8_rows_kernel<T, FORM, TPR, NV><<<blocks, TPR < BLOCK ? BLOCK : TPR, 0, ctx->stream>>>(g);
}

template <typename T, int FORM>
static void launch_rows(shifter_ctx* ctx, const Q8RowsArgs& g) {
    const uint32_t units = (uint32_t)(q8_pad(g.cols) / 8u);
    if (units <= 64) launch_rows_as<T, FORM, 64, 1>(ctx, g);
    else if (units <= 128) launch_rows_as<T, FORM, 64, 2>(ctx, g);
    else if (units <= 256) launch_rows_as<T, FORM, 64, 4>(ctx, g);
    else if (units <= 512) launch_rows_as<T, FORM, 256, 2>(ctx, g);
    else if (units <= 1024) launch_rows_as<T, FORM, 256, 4>(ctx, g);
    else if (units <= 2048) launch_rows_as<T, FORM, 1024, 2>(ctx, g);
    else if (units <= 4096) launch_rows_as<T, FORM, 1024, 4>(ctx, g);
    else q8_long_rows_kernel<T, FORM><<<std::min(g.rows, Q8_MAX_BLOCKS), 1024, 0, ctx->stream>>>(g);
}

template <typename T>
static void launch_rows_of(shifter_ctx* ctx, const Q8RowsArgs& g) {
    if (!g.weight) launch_rows<T, Q8_PLAIN>(ctx, g);
    else if (!g.residual) launch_rows<T, Q8_NORM>(ctx, g);
    else launch_rows<T, Q8_NORM_ADD>(ctx, g);
}

void launch_q8_rows(shifter_ctx* ctx, int dtype, const Q8RowsArgs& g) {
    if (g.rows == 0) return;
    ProfileScope ps(ctx, g.weight ? K_Q8_NORM : K_Q8_ROWS);
    if (dtype == SHIFTER_F32) launch_rows_of<float>(ctx, g);
    else if (dtype == SHIFTER_BF16) launch_rows_of<__bf16>(ctx, g);
    else launch_rows_of<_Float16>(ctx, g);
}

// Eight elements a thread at a time: code * scale, rounded to the element type once.
template <typename T>
__global__ __launch_bounds__(BLOCK) void q8_read_kernel(const int8_t* __restrict__ q, uint64_t ld_q,
                                                        const float* __restrict__ scale, uint32_t rows,
                                                        uint32_t cols, T* __restrict__ x, uint64_t ld_x) {
    const uint32_t units = (cols + 7u) / 8u;
    for (uint64_t i = (uint64_t)blockIdx.x * BLOCK + threadIdx.x; i < (uint64_t)rows * units;
         i += (uint64_t)gridDim.x * BLOCK) {
        const uint64_t row = i / units;
        const uint32_t c = (uint32_t)(i - row * units) * 8u;
        const uint2 w = *reinterpret_cast<const uint2*>(q + row * ld_q + c);
        const float s = scale[row];
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (float)(int8_t)((j < 4 ? w.x : w.y) >> (8 * (j % 4))) * s;
        T* out = x + row * ld_x + c;
        if (c + 8u <= cols) store8(out, f); else store_part(out, cols - c, f);
    }
}

template <typename T>
static void launch_read_as(shifter_ctx* ctx, const int8_t* q, uint64_t ld_q, const float* scale, uint32_t rows,
                           uint32_t cols, void* x, uint64_t ld_x) {
    const uint64_t blocks = ((uint64_t)rows * ((cols + 7u) / 8u) + BLOCK - 1) / BLOCK;
    q8_read_kernel<<<(uint32_t)std::min<uint64_t>(blocks, Q8_MAX_BLOCKS), BLOCK, 0, ctx->stream>>>(
        q, ld_q, scale, rows, cols, static_cast<T*>(x), ld_x);
}

void launch_q8_read(shifter_ctx* ctx, int dtype, const int8_t* q, uint64_t ld_q, const float* scale,
                    uint32_t rows, uint32_t cols, void* x, uint64_t ld_x) {
    if (rows == 0 || cols == 0) return;
    ProfileScope ps(ctx, K_Q8_READ);
    if (dtype == SHIFTER_F32) launch_read_as<float>(ctx, q, ld_q, scale, rows, cols, x, ld_x);
    else if (dtype == SHIFTER_BF16) launch_read_as<__bf16>(ctx, q, ld_q, scale, rows, cols, x, ld_x);
    else launch_read_as<_Float16>(ctx, q, ld_q, scale, rows, cols, x, ld_x);
}

}  // namespace shifter

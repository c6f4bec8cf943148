// The 8-bit operators: what the host hands to the kernels.
#pragma once

#include "internal.h"
#include "q8_plan.h"

namespace shifter {

// Rows to be quantised: as they are, or normed first.
struct Q8RowsArgs {
    const void* x;          // [rows][ld_x]
    const void* residual;   // [rows][ld_r] or nullptr
    const float* weight;    // cols, or nullptr: no norm
    void* h;                // [rows][ld_h]: x + residual, or nullptr
    uint64_t ld_x, ld_r, ld_h;
    uint32_t rows, cols;
    int8_t* q;
    uint64_t ld_q;
    float* scale;
    float eps;
    uint32_t relu;
};
void launch_q8_rows(shifter_ctx* ctx, int dtype, const Q8RowsArgs& a);
void launch_q8_read(shifter_ctx* ctx, int dtype, const int8_t* q, uint64_t ld_q, const float* scale,
                    uint32_t rows, uint32_t cols, void* x, uint64_t ld_x);


// c[m][n] = sum_k a[m][k] b[n][k] * sa[m] * sb[n] (+ bias[n], ReLU).
struct Q8ProductArgs {
    const int8_t *a, *b;
    const float *sa, *sb, *bias;
    uint64_t ld_a, ld_b, ld_c;
    uint32_t m, n, k;
    void* c;
    uint32_t relu;
};
void launch_q8_product(shifter_ctx* ctx, int dtype, const Q8ProductArgs& a);

// dw[n][k] (+)= keep[n][k] * sum_m g[m][n] s[m] q[m][k].
struct Q8GradientArgs {
    const void* g;
    const int8_t* q;
    const float* s;
    const uint8_t* mask;
    uint64_t ld_g, ld_q, ld_mask, ld_dw;
    uint32_t m, n, k;
    float* dw;
    uint32_t accumulate;
    uint8_t* work;
};
void launch_q8_gradient(shifter_ctx* ctx, int dtype, const Q8GradientArgs& a);

}  // namespace shifter

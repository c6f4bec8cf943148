// Log probabilities, gradient norms and adapters: what the host hands to the kernels.
#pragma once

#include "internal.h"
#include "adapters_plan.h"
#include "grad_norm_plan.h"
#include "log_probs_plan.h"

namespace shifter {

struct LogProbsArgs {
    const void* x;             // [rows][ld_x]
    uint64_t ld_x;
    uint32_t rows, cols, top;
    const int64_t* target;     // rows, or nullptr
    float scale, unit, by;     // log_probs_unit(scale); the scale of logits in that unit
    float* norm;               // [rows][2]: max x, log sum e^(z - scale max x)
    float *lse, *logp, *entropy;   // rows; logp nullptr without targets, entropy nullptr: not asked for
    float* top_logp;           // [rows][top]
    int64_t* index;
    uint8_t* work;
};
void launch_log_probs(shifter_ctx* ctx, int dtype, const LogProbsArgs& a);

// dx = scale (g_logp ([v = target] - p) + g_lse p - g_entropy p (log p + entropy)).
struct LogProbsGradArgs {
    const void* x;
    uint64_t ld_x, ld_dx;
    uint32_t rows, cols;
    const int64_t* target;
    float scale, unit, by;
    const float* norm;         // [rows][2]
    const float *entropy, *g_logp, *g_entropy, *g_lse;   // rows each, or nullptr
    void* dx;
};
void launch_log_probs_grad(shifter_ctx* ctx, int dtype, const LogProbsGradArgs& a);

// The norm of all tensors to d_norm; with clip, the tensors times min(1, max_norm / (norm + 1e-6)) as well.
void launch_grad_norm(shifter_ctx* ctx, const std::vector<shifter_grad>& all, bool clip, float max_norm, float* norm, uint8_t* work);

// out_r = y_r + scale[i] (x_r a_i') b_i', i = which[r].
struct AdaptersArgs {
    const void* x;             // [m][ld_x], codes with x_scale
    const float* x_scale;      // m, or nullptr
    const void *a, *b;         // [adapters][rank][k], [adapters][n][rank]
    const int64_t* which;      // m
    const float* scale;        // adapters, or nullptr
    const void* y;
    void* out;
    float* down;               // [m][rank] or nullptr
    uint64_t ld_x, ld_y, ld_out;
    uint32_t m, n, k, rank, adapters;
    uint8_t* work;
};
void launch_adapters(shifter_ctx* ctx, int dtype, int y_dtype, const AdaptersArgs& a);

struct AdaptersGradArgs {
    const void *x, *g;
    const float* x_scale;
    const void *a, *b;
    const int64_t* which;
    const float *scale, *down;
    void* dx;                  // or nullptr
    float *da, *db;
    uint64_t ld_x, ld_g, ld_dx;
    uint32_t m, n, k, rank, adapters;
    uint8_t* work;
};
void launch_adapters_grad(shifter_ctx* ctx, int dtype, const AdaptersGradArgs& a);

// The kernels' own, behind those two.
struct AdaptersDownArgs {
    const void* x;
    const float* x_scale;
    const void* a;
    const int64_t* which;
    const float* scale;
    const uint32_t* order;     // the rows in the order that they are taken in, or nullptr: as they come
    float* s;                  // [parts][m][rank padded to 16], in that order
    uint64_t ld_x;
    uint32_t m, k, rank, adapters, parts;
    uint32_t groups, jobs;     // of up to 64 ranks, a block each; blocks that share a tile's adapters
};
struct AdaptersUpArgs {
    const float* s;
    const uint32_t* order;
    const void* b;
    const int64_t* which;
    const void* y;             // or nullptr: 0
    void* out;
    float* down;               // [m][down_cols], the sum of the parts; or nullptr
    uint64_t ld_y, ld_out;
    uint32_t m, n, rank, adapters, parts, down_cols;
};
struct AdaptersTurnArgs {
    const int64_t* which;
    const void *a, *b;
    void *a_turned, *b_turned;
    uint32_t *rows, *first;
    uint32_t m, n, k, rank, adapters;
};
struct AdaptersSumArgs {
    const void *x, *g;
    const float *x_scale, *up, *down;
    uint64_t ld_x, ld_g, ld_up, ld_down;
    const uint32_t *rows, *first;
    float *da, *db, *partial;
    uint32_t n, k, rank, adapters, parts, rows_each;
};

}  // namespace shifter

// What a network is trained on and answers with: what the host hands to the kernels.
#pragma once

#include "internal.h"
#include "grad_norm_plan.h"
#include "log_probs_plan.h"

namespace shifter {

struct LogProbsArgs {
    const void* x;             // [rows][ld_x]
    uint64_t ld_x;
    uint32_t rows, cols, top;
    const int64_t* target;     // rows, or nullptr
    float scale;
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
    float scale;
    const float* norm;         // [rows][2]
    const float *entropy, *g_logp, *g_entropy, *g_lse;   // rows each, or nullptr
    void* dx;
};
void launch_log_probs_grad(shifter_ctx* ctx, int dtype, const LogProbsGradArgs& a);

// The norm of all tensors to d_norm; with clip, the tensors times min(1, max_norm / (norm + 1e-6)) as well.
void launch_grad_norm(shifter_ctx* ctx, const std::vector<shifter_grad>& all, bool clip, float max_norm, float* norm, uint8_t* work);

}  // namespace shifter

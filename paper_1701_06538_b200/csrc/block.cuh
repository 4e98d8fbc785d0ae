// Launchers of what stands around and beside the layer: the norms of the block, the layer for a few tokens, AdamW
#pragma once

#include "moe_internal.cuh"

namespace moe {

// ----------------------------------------------------------------------------- norms (norms.cu)
struct NormArgs {
    int64_t T;
    int32_t d, act;
    // x: of norm_in, or the residual stream before the block. y: the block's output, or nullptr: norm_in
    const void *x, *y, *gate;
    const float *w, *w_next;
    int64_t rows_per_gate;  // of gate
    float residual_scale, eps;
    void *out, *next;
    float *rstd, *rstd_next;
};
int32_t launch_norms(const NormArgs &a, cudaStream_t st);
struct NormGradArgs {
    int64_t T;
    int32_t d, act;
    const void *dOut, *dNext, *out, *y, *gate;  // dOut: nullptr for zeros; dNext: nullptr, or with out, w_next, rstd_next and dw_next; y: nullptr for norm_in
    const float *w, *w_next, *rstd, *rstd_next;
    int64_t rows_per_gate;
    float residual_scale;
    void *dX, *dY, *dgate;
    float *dw, *dw_next;
    float *ws;  // norm_grad_floats
};
int64_t norm_grad_floats(int64_t T, int32_t d, int32_t act);
int32_t launch_norm_grads(const NormGradArgs &a, cudaStream_t st);

// ----------------------------------------------------------------------------- AdamW (adamw.cu)
int32_t launch_adamw(const moe_adamw_tensor *tensors, int32_t count, const moe_adamw_params &p, const moe_adamw_rates *rates, cudaStream_t st);

// ----------------------------------------------------------------------------- a few tokens (few_tokens.cu)
unsigned long long bounds_violations_few_tokens();  // see moe_internal.cuh
int64_t few_tokens_bytes(const moe_config &c);
int32_t launch_few_tokens(const moe_config &c, const void *x, const float *Wg, const void *W1, const void *b1, const void *W2, const void *b2, void *y,
                          int32_t *topk_idx, float *gates, void *ws, cudaStream_t st);

}  // namespace moe

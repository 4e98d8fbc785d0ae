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

// ----------------------------------------------------------------------------- layer norm (layer_norm.cu)
struct LayerNormArgs {
    int64_t T;
    int32_t d, act;
    const void *x;
    const float *w, *b;  // b: or nullptr
    float eps;
    void *xn;
    float *mean, *rstd;  // each or nullptr
};
int32_t launch_layer_norm(const LayerNormArgs &a, cudaStream_t st);
struct LayerNormGradArgs {
    int64_t T;
    int32_t d, act;
    const void *dxn, *x, *dres;  // dres: or nullptr
    const float *w, *mean, *rstd;
    void *dX;
    float *dw, *db;  // db: or nullptr
    float *part;     // layer_norm_grad_floats
};
int64_t layer_norm_grad_floats(int64_t T, int32_t d, int32_t act);
int32_t launch_layer_norm_grads(const LayerNormGradArgs &a, cudaStream_t st);

// ----------------------------------------------------------------------------- losses of the router (router_losses.cu)
struct RouterLossArgs {
    int64_t T;
    int32_t n, k, S;
    const float *logits;
    const int32_t *topk_idx;
    const uint8_t *keep;      // or nullptr: all tokens
    const int32_t *offsets;   // [S + 1], or nullptr: all tokens are one sequence
    float w_balance, w_z;
    float *losses;
    int32_t *counts;
    float *prob_sums, *dlogits;  // each or nullptr
};
int64_t router_losses_bytes(int64_t T, int32_t n, int32_t S);  // behind the header
int32_t launch_router_losses(const RouterLossArgs &a, void *ws, cudaStream_t st);

// ----------------------------------------------------------------------------- AdamW (adamw.cu)
int32_t launch_adamw(const moe_adamw_tensor *tensors, int32_t count, const moe_adamw_params &p, const moe_adamw_rates *rates, cudaStream_t st);

// ----------------------------------------------------------------------------- Muon (muon.cu)
int32_t muon_check(const moe_muon_tensor *tensors, int32_t count);
int32_t muon_bytes(const moe_muon_tensor *tensors, int32_t count, int64_t *bytes);
int32_t launch_muon(const moe_muon_tensor *tensors, int32_t count, const moe_muon_params &p, const moe_muon_rates *rates, void *ws, cudaStream_t st);

// ----------------------------------------------------------------------------- a few tokens (few_tokens.cu)
unsigned long long bounds_violations_few_tokens();  // see moe_internal.cuh
int64_t few_tokens_bytes(const moe_config &c);
int32_t launch_few_tokens(const moe_config &c, const void *x, const float *Wg, const void *W1, const void *b1, const void *W2, const void *b2, void *y,
                          int32_t *topk_idx, float *gates, void *ws, cudaStream_t st);

}  // namespace moe

// The C ABI of what stands around and beside the layer (include/moe.h): argument checks and the way to the launchers.
#include <float.h>
#include <math.h>

#include "block.cuh"

using namespace moe;

namespace {

bool bad_ptr(const void *p) { return p == nullptr || !aligned16(p); }
#define REQUIRE_PTRS(...)                                             \
    do {                                                              \
        const void *ps_[] = {__VA_ARGS__};                            \
        for (size_t i_ = 0; i_ < sizeof(ps_) / sizeof(ps_[0]); ++i_)  \
            if (bad_ptr(ps_[i_])) return MOE_ERR_INVALID_ARG;         \
    } while (0)

bool bad_float(float v) { return !(fabsf(v) <= FLT_MAX); }

int32_t check_norm(const moe_config *c) {
    MOE_TRY(moe_validate(c));
    return c->d > MOE_NORM_MAX_D ? MOE_ERR_UNSUPPORTED : MOE_OK;
}
int32_t check_few(const moe_config *c) {
    MOE_TRY(moe_validate(c));
    return c->a > 0 || c->T > MOE_FEW_MAX_TOKENS ? MOE_ERR_UNSUPPORTED : MOE_OK;
}

int64_t norm_bytes(const moe_config &c, float **floats, void *ws) {
    Carver cv(ws);
    cv.take_bytes(kWsHeader);
    float *f = cv.take<float>(norm_grad_floats(c.T, c.d, c.act));
    if (floats) *floats = f;
    return (int64_t)cv.off;
}

int64_t layer_norm_bytes(const moe_config &c, float **floats, void *ws) {
    Carver cv(ws);
    cv.take_bytes(kWsHeader);
    float *f = cv.take<float>(layer_norm_grad_floats(c.T, c.d, c.act));
    if (floats) *floats = f;
    return (int64_t)cv.off;
}
int32_t check_router(const moe_config *c, int32_t sequences) {
    MOE_TRY(moe_validate(c));
    if (sequences < 1 || sequences > MOE_MAX_SEQUENCES) return MOE_ERR_INVALID_ARG;
    return c->a > 0 ? MOE_ERR_UNSUPPORTED : MOE_OK;
}

}  // namespace

extern "C" {

int32_t moe_norm_workspace_bytes(const moe_config *cfg, size_t *host_bytes) {
    MOE_TRY(check_norm(cfg));
    if (!host_bytes) return MOE_ERR_INVALID_ARG;
    *host_bytes = (size_t)norm_bytes(*cfg, nullptr, nullptr);
    return MOE_OK;
}

int32_t moe_norm_in(const moe_config *cfg, const void *x, const float *w, float eps, void *xn, float *rstd, void *stream) {
    MOE_TRY(check_norm(cfg));
    REQUIRE_PTRS(x, w, xn);
    if ((rstd && bad_ptr(rstd)) || !(eps > 0.0f) || bad_float(eps)) return MOE_ERR_INVALID_ARG;
    NormArgs a = {};
    a.T = cfg->T; a.d = cfg->d; a.act = cfg->act; a.x = x; a.w_next = w; a.eps = eps; a.next = xn; a.rstd_next = rstd;
    return launch_norms(a, static_cast<cudaStream_t>(stream));
}

int32_t moe_norm_in_bwd(const moe_config *cfg, const void *dxn, const void *x, const float *w, const float *rstd, const void *dres,
                        void *dX, float *dw, void *ws, void *stream) {
    MOE_TRY(check_norm(cfg));
    REQUIRE_PTRS(dxn, x, w, rstd, dX, dw, ws);
    if (dres && bad_ptr(dres)) return MOE_ERR_INVALID_ARG;
    NormGradArgs a = {};
    a.T = cfg->T; a.d = cfg->d; a.act = cfg->act; a.dOut = dres; a.dNext = dxn; a.out = x; a.w_next = w; a.rstd_next = rstd;
    a.residual_scale = 1.0f; a.dX = dX; a.dw_next = dw;
    norm_bytes(*cfg, &a.ws, ws);
    return launch_norm_grads(a, static_cast<cudaStream_t>(stream));
}

int32_t moe_norm_out(const moe_config *cfg, const void *x, const void *y, const float *w, const void *gate, int32_t rows_per_gate,
                     float residual_scale, const float *w_next, float eps, void *out, void *next, float *rstd, float *rstd_next,
                     void *stream) {
    MOE_TRY(check_norm(cfg));
    REQUIRE_PTRS(x, y, w, out, rstd);
    if (gate && (bad_ptr(gate) || rows_per_gate <= 0)) return MOE_ERR_INVALID_ARG;
    if (w_next) REQUIRE_PTRS(w_next, next, rstd_next);
    if (w_next && next == out) return MOE_ERR_INVALID_ARG;
    if (!(eps > 0.0f) || bad_float(eps) || bad_float(residual_scale)) return MOE_ERR_INVALID_ARG;
    NormArgs a = {};
    a.T = cfg->T; a.d = cfg->d; a.act = cfg->act; a.x = x; a.y = y; a.gate = gate; a.w = w; a.w_next = w_next; a.rows_per_gate = rows_per_gate;
    a.residual_scale = residual_scale; a.eps = eps; a.out = out; a.rstd = rstd;
    if (w_next) { a.next = next; a.rstd_next = rstd_next; }
    return launch_norms(a, static_cast<cudaStream_t>(stream));
}

int32_t moe_norm_out_bwd(const moe_config *cfg, const void *dOut, const void *dNext, const void *out, const void *y, const float *w,
                         const void *gate, int32_t rows_per_gate, float residual_scale, const float *w_next, const float *rstd,
                         const float *rstd_next, void *dX, void *dY, float *dw, void *dgate, float *dw_next, void *ws, void *stream) {
    MOE_TRY(check_norm(cfg));
    REQUIRE_PTRS(dOut, y, w, rstd, dX, dY, dw, ws);
    if (gate && (bad_ptr(gate) || bad_ptr(dgate) || rows_per_gate <= 0)) return MOE_ERR_INVALID_ARG;
    if (w_next) REQUIRE_PTRS(w_next, dNext, out, rstd_next, dw_next);
    if (bad_float(residual_scale) || dX == dY) return MOE_ERR_INVALID_ARG;
    NormGradArgs a = {};
    a.T = cfg->T; a.d = cfg->d; a.act = cfg->act; a.dOut = dOut; a.y = y; a.w = w; a.rstd = rstd; a.residual_scale = residual_scale;
    a.dX = dX; a.dY = dY; a.dw = dw;
    if (gate) { a.gate = gate; a.rows_per_gate = rows_per_gate; a.dgate = dgate; }
    if (w_next) { a.dNext = dNext; a.out = out; a.w_next = w_next; a.rstd_next = rstd_next; a.dw_next = dw_next; }
    norm_bytes(*cfg, &a.ws, ws);
    return launch_norm_grads(a, static_cast<cudaStream_t>(stream));
}

int32_t moe_few_workspace_bytes(const moe_config *cfg, size_t *host_bytes) {
    MOE_TRY(check_few(cfg));
    if (!host_bytes) return MOE_ERR_INVALID_ARG;
    *host_bytes = (size_t)few_tokens_bytes(*cfg);
    return MOE_OK;
}

int32_t moe_forward_few(const moe_config *cfg, const void *x, const float *Wg, const void *W1, const void *b1, const void *W2,
                        const void *b2, void *y, int32_t *topk_idx, float *gates, void *ws, void *stream) {
    MOE_TRY(check_few(cfg));
    REQUIRE_PTRS(x, Wg, W1, b1, W2, b2, y, ws);
    if ((topk_idx && bad_ptr(topk_idx)) || (gates && bad_ptr(gates))) return MOE_ERR_INVALID_ARG;
    const int64_t T = cfg->T, d = cfg->d, h = cfg->h, n = cfg->n, act = (int64_t)act_bytes(cfg->act);
    const struct { const void *at; int64_t bytes; } inputs[] = {{x, T * d * act}, {Wg, d * n * 4}, {W1, n * d * h * act}, {b1, n * h * act}, {W2, n * h * d * act}, {b2, n * d * act}};
    for (const auto &in : inputs)  // which are read until the last of y is written
        if (overlap(y, T * d * act, in.at, in.bytes)) return MOE_ERR_INVALID_ARG;
    return launch_few_tokens(*cfg, x, Wg, W1, b1, W2, b2, y, topk_idx, gates, ws, static_cast<cudaStream_t>(stream));
}

int32_t moe_adamw(const moe_adamw_tensor *host_tensors, int32_t count, const moe_adamw_params *host_params, const moe_adamw_rates *rates,
                  void *stream) {
    if (count < 0 || (count > 0 && !host_tensors) || !host_params) return MOE_ERR_INVALID_ARG;
    const moe_adamw_params &p = *host_params;
    if (!(p.beta1 >= 0.0 && p.beta1 < 1.0 && p.beta2 >= 0.0 && p.beta2 < 1.0) || !((float)p.eps >= FLT_MIN) || bad_float((float)p.eps)) return MOE_ERR_INVALID_ARG;
    if (rates ? ((uintptr_t)rates & 3) != 0 : (p.step < 1 || bad_float((float)p.lr) || bad_float((float)p.grad_scale))) return MOE_ERR_INVALID_ARG;
    return launch_adamw(host_tensors, count, p, rates, static_cast<cudaStream_t>(stream));
}

int32_t moe_muon_workspace_bytes(const moe_muon_tensor *host_tensors, int32_t count, size_t *host_bytes) {
    if (count < 0 || (count > 0 && !host_tensors) || !host_bytes) return MOE_ERR_INVALID_ARG;
    MOE_TRY(muon_check(host_tensors, count));
    int64_t bytes = 0;
    MOE_TRY(muon_bytes(host_tensors, count, &bytes));
    *host_bytes = (size_t)bytes;
    return MOE_OK;
}

int32_t moe_muon(const moe_muon_tensor *host_tensors, int32_t count, const moe_muon_params *host_params, const moe_muon_rates *rates, void *ws, void *stream) {
    if (count < 0 || (count > 0 && !host_tensors) || !host_params) return MOE_ERR_INVALID_ARG;
    const moe_muon_params &p = *host_params;
    if (!(p.momentum >= 0.0 && p.momentum < 1.0) || !(p.eps > 0.0) || !((float)p.eps >= FLT_MIN) || bad_float((float)p.eps)) return MOE_ERR_INVALID_ARG;
    if (p.steps < 1 || p.steps > MOE_MUON_MAX_STEPS || (p.nesterov != 0 && p.nesterov != 1)) return MOE_ERR_INVALID_ARG;
    if (rates ? ((uintptr_t)rates & 3) != 0 : (bad_float((float)p.lr) || bad_float((float)p.grad_scale))) return MOE_ERR_INVALID_ARG;
    MOE_TRY(muon_check(host_tensors, count));
    if (!ws || ((uintptr_t)ws & 255) != 0) return MOE_ERR_INVALID_ARG;
    return launch_muon(host_tensors, count, p, rates, ws, static_cast<cudaStream_t>(stream));
}

int32_t moe_router_losses_workspace_bytes(const moe_config *cfg, int32_t sequences, size_t *host_bytes) {
    MOE_TRY(check_router(cfg, sequences));
    if (!host_bytes) return MOE_ERR_INVALID_ARG;
    *host_bytes = (size_t)(kWsHeader + router_losses_bytes(cfg->T, cfg->n, sequences));
    return MOE_OK;
}

int32_t moe_router_losses(const moe_config *cfg, const float *logits, const int32_t *topk_idx, const uint8_t *keep, const int32_t *seq_offsets, int32_t sequences,
                          float w_balance, float w_z, float *losses, int32_t *counts, float *prob_sums, float *dlogits, void *ws, void *stream) {
    MOE_TRY(check_router(cfg, sequences));
    REQUIRE_PTRS(logits, topk_idx, losses, counts, ws);
    if ((keep && bad_ptr(keep)) || (seq_offsets && bad_ptr(seq_offsets)) || (prob_sums && bad_ptr(prob_sums)) || (dlogits && bad_ptr(dlogits))) return MOE_ERR_INVALID_ARG;
    if (!seq_offsets && sequences != 1) return MOE_ERR_INVALID_ARG;
    if (bad_float(w_balance) || bad_float(w_z)) return MOE_ERR_INVALID_ARG;
    const int64_t T = cfg->T, n = cfg->n, k = cfg->k, S = sequences;
    const struct { const void *at; int64_t bytes; } all[] = {{losses, 8}, {counts, S * n * 4}, {prob_sums, S * n * 4}, {dlogits, T * n * 4}, {logits, T * n * 4}, {topk_idx, T * k * 4},
                                                             {keep, T}, {seq_offsets, (S + 1) * 4}};
    for (int i = 0; i < 4; ++i)
        for (int j = i + 1; j < 8; ++j)
            if (all[i].at && all[j].at && overlap(all[i].at, all[i].bytes, all[j].at, all[j].bytes)) return MOE_ERR_INVALID_ARG;
    const RouterLossArgs a = {T, cfg->n, cfg->k, sequences, logits, topk_idx, keep, seq_offsets, w_balance, w_z, losses, counts, prob_sums, dlogits};
    return launch_router_losses(a, static_cast<char *>(ws) + kWsHeader, static_cast<cudaStream_t>(stream));
}

int32_t moe_layer_norm_workspace_bytes(const moe_config *cfg, size_t *host_bytes) {
    MOE_TRY(check_norm(cfg));
    if (!host_bytes) return MOE_ERR_INVALID_ARG;
    *host_bytes = (size_t)layer_norm_bytes(*cfg, nullptr, nullptr);
    return MOE_OK;
}

int32_t moe_layer_norm(const moe_config *cfg, const void *x, const float *w, const float *b, float eps, void *xn, float *mean, float *rstd, void *stream) {
    MOE_TRY(check_norm(cfg));
    REQUIRE_PTRS(x, w, xn);
    if ((b && bad_ptr(b)) || (mean && bad_ptr(mean)) || (rstd && bad_ptr(rstd)) || !(eps > 0.0f) || bad_float(eps)) return MOE_ERR_INVALID_ARG;
    const LayerNormArgs a = {cfg->T, cfg->d, cfg->act, x, w, b, eps, xn, mean, rstd};
    return launch_layer_norm(a, static_cast<cudaStream_t>(stream));
}

int32_t moe_layer_norm_bwd(const moe_config *cfg, const void *dxn, const void *x, const float *w, const float *mean, const float *rstd, const void *dres, void *dX, float *dw,
                           float *db, void *ws, void *stream) {
    MOE_TRY(check_norm(cfg));
    REQUIRE_PTRS(dxn, x, w, mean, rstd, dX, dw, ws);
    if ((dres && bad_ptr(dres)) || (db && bad_ptr(db))) return MOE_ERR_INVALID_ARG;
    LayerNormGradArgs a = {cfg->T, cfg->d, cfg->act, dxn, x, dres, w, mean, rstd, dX, dw, db, nullptr};
    layer_norm_bytes(*cfg, &a.part, ws);
    return launch_layer_norm_grads(a, static_cast<cudaStream_t>(stream));
}

}  // extern "C"

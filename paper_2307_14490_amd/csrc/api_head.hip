// C-ABI host layer of the softmax head's operators: argument checks, then the
// launches.  Nothing here allocates, synchronises or keeps anything from one call
// to the next.
#include <math.h>

#include "api_head.hpp"

using namespace huge;

namespace {

bool softmax_ok(const huge_softmax_config* c) {
    return c != nullptr && c->num_classes >= 1 && c->num_classes <= kMaxRows && c->max_rows >= 1 &&
           c->max_rows <= kMaxRows && c->dim >= 4 && c->dim <= kMaxDim && c->dim % 4 == 0 &&
           dtype_ok(c->dtype) && (c->grad == 0 || c->grad == 1);
}

// The checks that the two softmax calls share.
huge_status softmax_args(const huge_softmax_config* cfg, const void* h, int64_t ld_h, int64_t n,
                         const void* w, int64_t ld_w, const float* bias, const int32_t* labels,
                         const float* weight, const float* lse, const int32_t* status,
                         const void* ws, size_t ws_bytes) {
    if (!softmax_ok(cfg) || n < 0 || n > cfg->max_rows || ld_w < cfg->dim || !w || !status ||
        (n > 0 && (!h || !labels || !lse || ld_h < cfg->dim)) || !on(h, elem(cfg->dtype)) ||
        !on(w, elem(cfg->dtype)) || !on(bias, 4) || !on(labels, 4) || !on(weight, 4) ||
        !on(lse, 4) || !on(status, 4))
        return HUGE_ERR_INVALID_ARG;
    if (!ws || ws_bytes < huge_softmax_workspace_bytes(cfg)) return HUGE_ERR_WORKSPACE;
    if (!on(ws, 256)) return HUGE_ERR_INVALID_ARG;
    return HUGE_OK;
}

SoftmaxArgs softmax_call(const huge_softmax_config* cfg, const void* h, int64_t ld_h, int64_t n,
                         const void* w, int64_t ld_w, const float* bias, const int32_t* labels,
                         const float* weight, int32_t* status, void* ws) {
    SoftmaxArgs a{};
    a.h = h, a.w = w, a.ld_h = ld_h, a.ld_w = ld_w, a.n = n, a.classes = cfg->num_classes;
    a.dim = cfg->dim, a.dtype = cfg->dtype, a.bias = bias, a.labels = labels, a.weight = weight;
    a.status = status, a.ws = static_cast<uint8_t*>(ws);
    return a;
}

bool state_ok(int32_t kind) { return kind == HUGE_STATE_F32 || kind == HUGE_STATE_Q8; }

bool rate_ok(double v) { return v >= 0.0 && isfinite(v); }

// Fills launches of up to kAdamTensors tensors of one pair of types with the
// tensors that have elements, and hands each to `launch`.
template <typename Pick, typename Launch>
huge_status in_launches(AdamArgs& a, int32_t count, Pick pick, Launch launch) {
    int64_t chunks = 0;
    a.count = 0;
    for (int32_t k = 0; k < count; ++k) {
        AdamTensor t{};
        if (!pick(k, t) || t.n == 0) continue;
        const int64_t more = (t.n + kAdamChunk - 1) / kAdamChunk;
        if (a.count == kAdamTensors || chunks + more > kMaxRows) {
            HEAD_TRY(launch(a, chunks));
            a.count = 0;
            chunks = 0;
        }
        t.first = (uint32_t)chunks;
        a.t[a.count++] = t;
        chunks += more;
    }
    if (a.count > 0) HEAD_TRY(launch(a, chunks));
    return HUGE_OK;
}

huge_status state_call(const huge_adamw_tensor* ts, int32_t count, int32_t kind,
                       const float* const* m, const float* const* v, bool write, void* stream) {
    if (count < 0 || !state_ok(kind) || (count > 0 && (!ts || !m || !v)))
        return HUGE_ERR_INVALID_ARG;
    for (int32_t k = 0; k < count; ++k)
        if (ts[k].n < 0 || ts[k].n > kAdamMaxElements ||
            (ts[k].n > 0 && (!ts[k].d_state || !on(ts[k].d_state, 16) || !m[k] || !v[k] ||
                             !on(m[k], 4) || !on(v[k], 4))))
            return HUGE_ERR_INVALID_ARG;
    AdamArgs a{};
    return in_launches(
        a, count,
        [&](int32_t k, AdamTensor& t) {
            t.p = const_cast<float*>(m[k]), t.g = v[k], t.n = ts[k].n;
            t.state = static_cast<uint8_t*>(ts[k].d_state);
            t.vec = on(m[k], 16) && on(v[k], 16);
            return true;
        },
        [&](const AdamArgs& b, int64_t chunks) {
            return launch_adamw_state(b, chunks, kind, write, static_cast<hipStream_t>(stream));
        });
}

}  // namespace

namespace huge {

huge_status adamw_args(const huge_adamw_config* cfg, const huge_adamw_tensor* h_tensors,
                       int32_t count, const int32_t* d_status) {
    if (!cfg || count < 0 || (count > 0 && !h_tensors) || !d_status || !on(d_status, 4) ||
        !state_ok(cfg->state_kind) || cfg->step < 1 || !rate_ok(cfg->lr) ||
        !rate_ok(cfg->weight_decay) || !isfinite(cfg->grad_scale) ||
        !(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0) ||
        !(cfg->eps >= 1e-30 && isfinite((float)cfg->eps)))
        return HUGE_ERR_INVALID_ARG;
    for (int32_t k = 0; k < count; ++k) {
        const huge_adamw_tensor& t = h_tensors[k];
        if (t.n < 0 || t.n > kAdamMaxElements || !dtype_ok(t.param_dtype) ||
            !dtype_ok(t.grad_dtype) ||
            (t.n > 0 && (!t.d_param || !t.d_grad || !t.d_state || !on(t.d_state, 16) ||
                         !on(t.d_param, elem(t.param_dtype)) ||
                         !on(t.d_grad, elem(t.grad_dtype)))))
            return HUGE_ERR_INVALID_ARG;
    }
    return HUGE_OK;
}

huge_status adamw_step(const huge_adamw_config* cfg, const huge_adamw_tensor* h_tensors,
                       int32_t count, const float* d_factor, int32_t* d_status, void* stream) {
    AdamArgs a{};
    const double b1 = cfg->beta1, b2 = cfg->beta2, steps = (double)cfg->step;
    a.beta1 = (float)b1, a.one_beta1 = (float)(1.0 - b1);
    a.beta2 = (float)b2, a.one_beta2 = (float)(1.0 - b2);
    a.rate = (float)(cfg->lr / (1.0 - pow(b1, steps)));
    a.fix = (float)(1.0 / sqrt(1.0 - pow(b2, steps)));
    a.eps = (float)cfg->eps;
    a.keep = (float)(1.0 - cfg->lr * cfg->weight_decay);
    a.grad_scale = (float)cfg->grad_scale;
    a.factor = d_factor;
    a.status = d_status;
    for (int32_t types = 0; types < 4; ++types) {
        const int32_t pt = types >> 1, gt = types & 1;
        const huge_status st = in_launches(
            a, count,
            [&](int32_t k, AdamTensor& t) {
                const huge_adamw_tensor& u = h_tensors[k];
                if (u.param_dtype != pt || u.grad_dtype != gt) return false;
                t.p = u.d_param, t.g = u.d_grad, t.n = u.n;
                t.state = static_cast<uint8_t*>(u.d_state);
                t.vec = on(u.d_param, 4 * elem(pt)) && on(u.d_grad, 4 * elem(gt));
                return true;
            },
            [&](const AdamArgs& b, int64_t chunks) {
                return launch_adamw(b, chunks, pt, gt, cfg->state_kind,
                                    static_cast<hipStream_t>(stream));
            });
        if (st != HUGE_OK) return st;
    }
    return HUGE_OK;
}

}  // namespace huge

extern "C" {

huge_status huge_layer_norm(const void* d_x, int64_t ld_x, int64_t n, int32_t dim, int32_t dtype,
                            const float* d_gamma, const float* d_beta, float eps, void* d_y,
                            int64_t ld_y, float* d_mean, float* d_rstd, void* stream) {
    if (n < 0 || n > kMaxRows || dim < 1 || dim > kNormMaxDim || !dtype_ok(dtype) ||
        !(eps > 0.f && eps < INFINITY) || !d_gamma || !d_beta || !on(d_gamma, 4) ||
        !on(d_beta, 4) || (!d_mean != !d_rstd) || !on(d_mean, 4) || !on(d_rstd, 4) ||
        !on(d_x, elem(dtype)) || !on(d_y, elem(dtype)) ||
        (n > 0 && (!d_x || !d_y || ld_x < dim || ld_y < dim)))
        return HUGE_ERR_INVALID_ARG;
    if (n == 0) return HUGE_OK;
    NormArgs a{};
    a.x = d_x, a.y = d_y, a.ld_x = ld_x, a.ld_y = ld_y, a.n = n, a.dim = dim, a.dtype = dtype;
    a.gamma = d_gamma, a.beta = d_beta, a.eps = eps, a.mean = d_mean, a.rstd = d_rstd;
    a.vec = dim % 4 == 0 && fours(d_x, ld_x, dtype) && fours(d_y, ld_y, dtype) &&
            on(d_gamma, 16) && on(d_beta, 16);
    HEAD_TRY(launch_norm(a, static_cast<hipStream_t>(stream)));
    return HUGE_OK;
}

size_t huge_layer_norm_workspace_bytes(int64_t n, int32_t dim) {
    if (n < 0 || n > kMaxRows || dim < 1 || dim > kNormMaxDim) return 0;
    const size_t bytes = (size_t)norm_blocks(n, dim) * 2 * dim * sizeof(float);
    return bytes > 0 ? bytes : 16;
}

huge_status huge_layer_norm_backward(const void* d_dy, int64_t ld_dy, const void* d_x,
                                     int64_t ld_x, int64_t n, int32_t dim, int32_t dtype,
                                     const float* d_gamma, const float* d_mean,
                                     const float* d_rstd, void* d_dx, int64_t ld_dx,
                                     float* d_dgamma, float* d_dbeta, void* d_workspace,
                                     size_t ws_bytes, void* stream) {
    if (n < 0 || n > kMaxRows || dim < 1 || dim > kNormMaxDim || !dtype_ok(dtype) || !d_gamma ||
        !on(d_gamma, 4) || !on(d_mean, 4) || !on(d_rstd, 4) || (!d_dgamma != !d_dbeta) ||
        !on(d_dgamma, 4) || !on(d_dbeta, 4) || !on(d_x, elem(dtype)) || !on(d_dy, elem(dtype)) ||
        !on(d_dx, elem(dtype)) ||
        (n > 0 && (!d_x || !d_dy || !d_mean || !d_rstd || ld_x < dim || ld_dy < dim ||
                   (d_dx && ld_dx < dim))))
        return HUGE_ERR_INVALID_ARG;
    if (d_dgamma && (!d_workspace || ws_bytes < huge_layer_norm_workspace_bytes(n, dim)))
        return HUGE_ERR_WORKSPACE;
    if (!on(d_workspace, 16)) return HUGE_ERR_INVALID_ARG;
    if (!d_dgamma && (n == 0 || !d_dx)) return HUGE_OK;
    NormArgs a{};
    a.x = d_x, a.dy = d_dy, a.y = d_dx, a.ld_x = ld_x, a.ld_dy = ld_dy, a.ld_y = ld_dx, a.n = n;
    a.dim = dim, a.dtype = dtype, a.gamma = d_gamma;
    a.mean = const_cast<float*>(d_mean), a.rstd = const_cast<float*>(d_rstd);
    a.partial = d_dgamma ? static_cast<float*>(d_workspace) : nullptr;
    a.vec = dim % 4 == 0 && fours(d_x, ld_x, dtype) && fours(d_dy, ld_dy, dtype) &&
            (!d_dx || fours(d_dx, ld_dx, dtype)) && on(d_gamma, 16);
    HEAD_TRY(launch_norm_backward(a, d_dgamma, d_dbeta, static_cast<hipStream_t>(stream)));
    return HUGE_OK;
}

size_t huge_softmax_workspace_bytes(const huge_softmax_config* cfg) {
    if (!softmax_ok(cfg)) return 0;
    return softmax_plan(cfg->num_classes, cfg->max_rows, cfg->dim, cfg->dtype, cfg->grad != 0)
        .total;
}

huge_status huge_softmax_loss(const huge_softmax_config* cfg, const void* d_h, int64_t ld_h,
                              int64_t n, const void* d_w, int64_t ld_w, const float* d_bias,
                              const int32_t* d_labels, const float* d_weight, float* d_loss,
                              float* d_lse, double* d_loss_sum, int32_t* d_status,
                              void* d_workspace, size_t ws_bytes, void* stream) {
    const huge_status st = softmax_args(cfg, d_h, ld_h, n, d_w, ld_w, d_bias, d_labels, d_weight,
                                        d_lse, d_status, d_workspace, ws_bytes);
    if (st != HUGE_OK) return st;
    if ((n > 0 && !d_loss) || !on(d_loss, 4) || !on(d_loss_sum, 8)) return HUGE_ERR_INVALID_ARG;
    SoftmaxArgs a = softmax_call(cfg, d_h, ld_h, n, d_w, ld_w, d_bias, d_labels, d_weight,
                                 d_status, d_workspace);
    a.loss = d_loss, a.lse = d_lse, a.loss_sum = d_loss_sum;
    HEAD_TRY(launch_softmax_loss(a, static_cast<hipStream_t>(stream)));
    return HUGE_OK;
}

huge_status huge_softmax_grad(const huge_softmax_config* cfg, const void* d_h, int64_t ld_h,
                              int64_t n, const void* d_w, int64_t ld_w, const float* d_bias,
                              const int32_t* d_labels, const float* d_weight, const float* d_lse,
                              float scale, void* d_dh, void* d_dw, float* d_dbias,
                              int32_t* d_status, void* d_workspace, size_t ws_bytes,
                              void* stream) {
    const huge_status st = softmax_args(cfg, d_h, ld_h, n, d_w, ld_w, d_bias, d_labels, d_weight,
                                        d_lse, d_status, d_workspace, ws_bytes);
    if (st != HUGE_OK) return st;
    if (cfg->grad == 0 || !isfinite(scale) || !on(d_dh, elem(cfg->dtype)) ||
        !on(d_dw, elem(cfg->dtype)) || !on(d_dbias, 4))
        return HUGE_ERR_INVALID_ARG;
    SoftmaxArgs a = softmax_call(cfg, d_h, ld_h, n, d_w, ld_w, d_bias, d_labels, d_weight,
                                 d_status, d_workspace);
    a.lse = const_cast<float*>(d_lse), a.scale = scale;
    a.dh = n > 0 ? d_dh : nullptr, a.dw = d_dw, a.dbias = d_dbias;
    HEAD_TRY(launch_softmax_grad(a, static_cast<hipStream_t>(stream)));
    return HUGE_OK;
}

size_t huge_adamw_state_bytes(int64_t n, int32_t state_kind) {
    if (n < 0 || n > kAdamMaxElements || !state_ok(state_kind)) return 0;
    const int64_t padded = adam_padded(n);
    return (size_t)(state_kind == HUGE_STATE_F32 ? 8 * padded
                                                 : 2 * padded + padded / kAdamBlock * 8);
}

huge_status huge_adamw_step(const huge_adamw_config* cfg, const huge_adamw_tensor* h_tensors,
                            int32_t count, int32_t* d_status, void* stream) {
    const huge_status st = adamw_args(cfg, h_tensors, count, d_status);
    return st != HUGE_OK ? st : adamw_step(cfg, h_tensors, count, nullptr, d_status, stream);
}

huge_status huge_adamw_get_state(const huge_adamw_tensor* h_tensors, int32_t count,
                                 int32_t state_kind, float* const* h_m, float* const* h_v,
                                 void* stream) {
    return state_call(h_tensors, count, state_kind, h_m, h_v, false, stream);
}

huge_status huge_adamw_set_state(const huge_adamw_tensor* h_tensors, int32_t count,
                                 int32_t state_kind, const float* const* h_m,
                                 const float* const* h_v, void* stream) {
    return state_call(h_tensors, count, state_kind, h_m, h_v, true, stream);
}

}  // extern "C"

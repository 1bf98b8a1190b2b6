// C-ABI host layer of RMS norm, rows in 8 bits, log probabilities and clipped gradients:
// argument checks, then the launches.  Nothing here allocates, synchronises or keeps
// anything from one call to the next.
#include <math.h>

#include "api_head.hpp"

using namespace huge;

namespace {

bool rows_ok(int64_t n, int32_t dim, int32_t dtype) {
    return n >= 0 && n <= kMaxRows && dim >= 1 && dim <= kNormMaxDim && dtype_ok(dtype);
}

// Rows that a call reads or writes: there, aligned for their element, not overlapping.
bool matrix_ok(const void* p, int64_t ld, int32_t dim, size_t size) {
    return p != nullptr && on(p, size) && ld >= dim;
}

// Whether rows start on a number of bytes, that many at a time being whole rows.
bool starts_on(const void* p, int64_t ld, size_t size, size_t bytes) {
    return p == nullptr || (on(p, bytes) && ld * size % bytes == 0);
}

// Codes and scales of rows in 8 bits.
bool bytes_ok(const uint8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t ld_scales,
              int32_t dim) {
    return codes != nullptr && scales != nullptr && ld_codes >= dim &&
           ld_scales >= (dim + kByteBlock - 1) / kByteBlock;
}

bool answer_ok(const huge_log_probs_config* c) {
    return c != nullptr && c->num_classes >= 1 && c->num_classes <= kMaxRows && c->max_rows >= 1 &&
           c->max_rows <= kMaxRows && c->dim >= 4 && c->dim <= kMaxDim && c->dim % 4 == 0 &&
           dtype_ok(c->dtype) && c->top >= 0 && c->top <= kMostTop && c->top <= c->num_classes &&
           (c->grad == 0 || c->grad == 1) &&
           (c->table_dtype == c->dtype ||
            (c->table_dtype == HUGE_DTYPE_Q8 && c->dtype == HUGE_DTYPE_BF16 && c->grad == 0));
}

size_t table_elem(const huge_log_probs_config* c) {
    return c->table_dtype == HUGE_DTYPE_Q8 ? 1 : elem(c->dtype);
}

// The checks that the two calls of log probabilities share.
huge_status answer_args(const huge_log_probs_config* c, const void* h, int64_t ld_h, int64_t n,
                        const void* w, int64_t ld_w, const uint8_t* scales, int64_t ld_scales,
                        const float* bias, const int32_t* labels, const float* lse,
                        const float* entropy, const int32_t* status, const void* ws,
                        size_t ws_bytes) {
    if (!answer_ok(c) || n < 0 || n > c->max_rows || !matrix_ok(w, ld_w, c->dim, table_elem(c)) ||
        (n > 0 && (!matrix_ok(h, ld_h, c->dim, elem(c->dtype)) || !lse)) || !status ||
        !on(bias, 4) || !on(labels, 4) || !on(lse, 4) || !on(entropy, 4) || !on(status, 4))
        return HUGE_ERR_INVALID_ARG;
    if (c->table_dtype == HUGE_DTYPE_Q8
            ? !bytes_ok(static_cast<const uint8_t*>(w), ld_w, scales, ld_scales, c->dim)
            : scales != nullptr)
        return HUGE_ERR_INVALID_ARG;
    if (!ws || ws_bytes < huge_log_probs_workspace_bytes(c)) return HUGE_ERR_WORKSPACE;
    if (!on(ws, 256)) return HUGE_ERR_INVALID_ARG;
    return HUGE_OK;
}

SoftmaxArgs answer_call(const huge_log_probs_config* c, const void* h, int64_t ld_h, int64_t n,
                        const void* w, int64_t ld_w, const uint8_t* scales, int64_t ld_scales,
                        const float* bias, const int32_t* labels, int32_t* status, void* ws) {
    SoftmaxArgs a{};
    a.h = h, a.w = w, a.ld_h = ld_h, a.ld_w = ld_w, a.n = n, a.classes = c->num_classes;
    a.dim = c->dim, a.dtype = c->dtype, a.bias = bias, a.labels = labels;
    a.w_scales = scales, a.ld_scales = ld_scales;
    a.status = status, a.ws = static_cast<uint8_t*>(ws);
    return a;
}

// A launch's tensors and what goes on with each full one.
template <typename Tensor, typename Launch>
huge_status clip_launches(int32_t count, Tensor tensor, Launch launch) {
    ClipArgs a;
    a.count = 0, a.chunks = 0;
    auto go = [&] {
        if (a.count == 0) return hipSuccess;
        const hipError_t e = launch(a);
        a.count = 0, a.chunks = 0;
        return e;
    };
    for (int32_t k = 0; k < count; ++k) {
        const huge_grad_tensor g = tensor(k);
        if (g.n == 0) continue;
        const int64_t more = (g.n + kClipChunk - 1) / kClipChunk;
        if (a.count == kClipTensors || (int64_t)a.chunks + more > kMaxRows) HEAD_TRY(go());
        a.t[a.count] = {g.d_grad, 2 * g.n + (g.dtype == HUGE_DTYPE_BF16 ? 1 : 0)};
        a.first[a.count++] = a.chunks;
        a.chunks += (uint32_t)more;
    }
    HEAD_TRY(go());
    return HUGE_OK;
}

bool grads_ok(const huge_grad_tensor* ts, int32_t count) {
    if (count < 0 || (count > 0 && !ts)) return false;
    for (int32_t k = 0; k < count; ++k)
        if (ts[k].n < 0 || ts[k].n > kAdamMaxElements || !dtype_ok(ts[k].dtype) ||
            (ts[k].n > 0 && (!ts[k].d_grad || !on(ts[k].d_grad, elem(ts[k].dtype)))))
            return false;
    return true;
}

// The workspace: the factor, then the partial sums.
constexpr size_t kFactorBytes = 16;

huge_status norm_ws(int32_t count, const void* ws, size_t ws_bytes) {
    if (!ws || ws_bytes < huge_grad_norm_workspace_bytes(count)) return HUGE_ERR_WORKSPACE;
    return on(ws, 16) ? HUGE_OK : HUGE_ERR_INVALID_ARG;
}

template <typename Tensor>
huge_status norm_factor(int32_t count, Tensor tensor, double scale, double max_norm, float* d_norm,
                        void* ws, hipStream_t s) {
    float* factor = static_cast<float*>(ws);
    double* part = reinterpret_cast<double*>(static_cast<uint8_t*>(ws) + kFactorBytes);
    int parts = 0, left = 0;
    for (int32_t k = 0; k < count; ++k) left += tensor(k).n > 0;
    bool done = false;
    const huge_status st = clip_launches(count, tensor, [&](const ClipArgs& a) {
        left -= a.count;
        if (parts == 0 && left == 0 && a.chunks <= kClipSmall) {
            done = true;
            return launch_norm_small(a, scale, max_norm, d_norm, factor, s);
        }
        int more = 0;
        const hipError_t e = launch_squares(a, part + parts, &more, s);
        parts += more;
        return e;
    });
    if (st != HUGE_OK || done) return st;
    HEAD_TRY(launch_norm_factor(part, parts, scale, max_norm, d_norm, factor, s));
    return HUGE_OK;
}

}  // namespace

extern "C" {

huge_status huge_rms_norm(const void* d_x, int64_t ld_x, const void* d_residual, int64_t ld_residual,
                          int64_t n, int32_t dim, int32_t dtype, const float* d_gamma, float eps,
                          void* d_total, int64_t ld_total, void* d_y, int64_t ld_y,
                          uint8_t* d_codes, int64_t ld_codes, uint8_t* d_scales, int64_t ld_scales,
                          float* d_rstd, void* stream) {
    if (!rows_ok(n, dim, dtype) || !(eps > 0.f && eps < INFINITY) || !d_gamma || !on(d_gamma, 4) ||
        !on(d_rstd, 4) || (!d_residual != !d_total) || (!d_codes != !d_scales))
        return HUGE_ERR_INVALID_ARG;
    const size_t e = elem(dtype);
    if (n > 0) {
        if (!matrix_ok(d_x, ld_x, dim, e) || !d_y == !d_codes ||
            (d_residual && (!matrix_ok(d_residual, ld_residual, dim, e) ||
                            !matrix_ok(d_total, ld_total, dim, e))) ||
            (d_y && !matrix_ok(d_y, ld_y, dim, e)) ||
            (d_codes && !bytes_ok(d_codes, ld_codes, d_scales, ld_scales, dim)))
            return HUGE_ERR_INVALID_ARG;
    }
    if (n == 0) return HUGE_OK;
    RmsArgs a{};
    a.x = d_x, a.res = d_residual, a.total = d_total, a.y = d_y, a.codes = d_codes;
    a.scales = d_scales, a.ld_x = ld_x, a.ld_res = ld_residual, a.ld_total = ld_total;
    a.ld_y = ld_y, a.ld_codes = ld_codes, a.ld_scales = ld_scales, a.n = n, a.dim = dim;
    a.dtype = dtype, a.gamma = d_gamma, a.eps = eps, a.rstd = d_rstd;
    a.vec = dim % 4 == 0 && fours(d_x, ld_x, dtype) && on(d_gamma, 16) &&
            (!d_residual || (fours(d_residual, ld_residual, dtype) && fours(d_total, ld_total, dtype))) &&
            (d_y ? fours(d_y, ld_y, dtype) : on(d_codes, 4) && ld_codes % 4 == 0);
    a.eights = dtype == HUGE_DTYPE_BF16 && dim % 8 == 0 && on(d_gamma, 16) &&
               starts_on(d_x, ld_x, e, 16) && starts_on(d_residual, ld_residual, e, 16) &&
               starts_on(d_total, ld_total, e, 16) && starts_on(d_y, ld_y, e, 16) &&
               starts_on(d_codes, ld_codes, 1, 8);
    HEAD_TRY(launch_rms(a, static_cast<hipStream_t>(stream)));
    return HUGE_OK;
}

size_t huge_rms_norm_workspace_bytes(int64_t n, int32_t dim) {
    if (!rows_ok(n, dim, HUGE_DTYPE_F32)) return 0;
    const size_t bytes = (size_t)norm_blocks(n, dim) * dim * sizeof(float);
    return bytes > 0 ? bytes : 16;
}

huge_status huge_rms_norm_backward(const void* d_dy, int64_t ld_dy, const void* d_total,
                                   int64_t ld_total, const void* d_dtotal, int64_t ld_dtotal,
                                   int64_t n, int32_t dim, int32_t dtype, const float* d_gamma,
                                   const float* d_rstd, void* d_dx, int64_t ld_dx, float* d_dgamma,
                                   void* d_workspace, size_t ws_bytes, void* stream) {
    if (!rows_ok(n, dim, dtype) || !d_gamma || !on(d_gamma, 4) || !on(d_rstd, 4) ||
        !on(d_dgamma, 4))
        return HUGE_ERR_INVALID_ARG;
    const size_t e = elem(dtype);
    if (n > 0 && (!matrix_ok(d_dy, ld_dy, dim, e) || !matrix_ok(d_total, ld_total, dim, e) || !d_rstd ||
                  (d_dtotal && !matrix_ok(d_dtotal, ld_dtotal, dim, e)) ||
                  (d_dx && !matrix_ok(d_dx, ld_dx, dim, e))))
        return HUGE_ERR_INVALID_ARG;
    if (d_dgamma && (!d_workspace || ws_bytes < huge_rms_norm_workspace_bytes(n, dim)))
        return HUGE_ERR_WORKSPACE;
    if (!on(d_workspace, 16)) return HUGE_ERR_INVALID_ARG;
    if (!d_dgamma && (n == 0 || !d_dx)) return HUGE_OK;
    RmsArgs a{};
    a.x = d_total, a.dy = d_dy, a.res = d_dtotal, a.y = n > 0 ? d_dx : nullptr;
    a.ld_x = ld_total, a.ld_dy = ld_dy, a.ld_res = ld_dtotal, a.ld_y = ld_dx, a.n = n, a.dim = dim;
    a.dtype = dtype, a.gamma = d_gamma, a.rstd = const_cast<float*>(d_rstd);
    a.partial = d_dgamma ? static_cast<float*>(d_workspace) : nullptr;
    a.vec = dim % 4 == 0 && fours(d_total, ld_total, dtype) && fours(d_dy, ld_dy, dtype) &&
            (!d_dtotal || fours(d_dtotal, ld_dtotal, dtype)) &&
            (!d_dx || fours(d_dx, ld_dx, dtype)) && on(d_gamma, 16);
    a.eights = dtype == HUGE_DTYPE_BF16 && dim % 8 == 0 && on(d_gamma, 16) &&
               starts_on(d_total, ld_total, e, 16) && starts_on(d_dy, ld_dy, e, 16) &&
               starts_on(d_dtotal, ld_dtotal, e, 16) && starts_on(d_dx, ld_dx, e, 16);
    HEAD_TRY(launch_rms_backward(a, d_dgamma, static_cast<hipStream_t>(stream)));
    return HUGE_OK;
}

huge_status huge_quantise_rows(const void* d_x, int64_t ld_x, int64_t n, int32_t dim, int32_t dtype,
                               uint8_t* d_codes, int64_t ld_codes, uint8_t* d_scales,
                               int64_t ld_scales, void* stream) {
    if (!rows_ok(n, dim, dtype) ||
        (n > 0 && (!matrix_ok(d_x, ld_x, dim, elem(dtype)) ||
                   !bytes_ok(d_codes, ld_codes, d_scales, ld_scales, dim))))
        return HUGE_ERR_INVALID_ARG;
    if (n == 0) return HUGE_OK;
    RmsArgs a{};
    a.x = d_x, a.ld_x = ld_x, a.codes = d_codes, a.ld_codes = ld_codes, a.scales = d_scales;
    a.ld_scales = ld_scales, a.n = n, a.dim = dim, a.dtype = dtype;
    a.vec = dim % 4 == 0 && fours(d_x, ld_x, dtype) && on(d_codes, 4) && ld_codes % 4 == 0;
    a.eights = dim % 8 == 0 && starts_on(d_x, ld_x, elem(dtype), 16) &&
               starts_on(d_codes, ld_codes, 1, 8);
    HEAD_TRY(launch_to_bytes(a, static_cast<hipStream_t>(stream)));
    return HUGE_OK;
}

huge_status huge_dequantise_rows(const uint8_t* d_codes, int64_t ld_codes, const uint8_t* d_scales,
                                 int64_t ld_scales, int64_t n, int32_t dim, void* d_y, int64_t ld_y,
                                 int32_t dtype, void* stream) {
    if (!rows_ok(n, dim, dtype) ||
        (n > 0 && (!matrix_ok(d_y, ld_y, dim, elem(dtype)) ||
                   !bytes_ok(d_codes, ld_codes, d_scales, ld_scales, dim))))
        return HUGE_ERR_INVALID_ARG;
    if (n == 0) return HUGE_OK;
    RmsArgs a{};
    a.y = d_y, a.ld_y = ld_y, a.codes = const_cast<uint8_t*>(d_codes), a.ld_codes = ld_codes;
    a.scales = const_cast<uint8_t*>(d_scales), a.ld_scales = ld_scales;
    a.n = n, a.dim = dim, a.dtype = dtype;
    a.vec = dim % 4 == 0 && fours(d_y, ld_y, dtype) && on(d_codes, 4) && ld_codes % 4 == 0;
    a.eights = dim % 8 == 0 && starts_on(d_y, ld_y, elem(dtype), 16) &&
               starts_on(d_codes, ld_codes, 1, 8);
    HEAD_TRY(launch_from_bytes(a, static_cast<hipStream_t>(stream)));
    return HUGE_OK;
}

size_t huge_log_probs_workspace_bytes(const huge_log_probs_config* cfg) {
    if (!answer_ok(cfg)) return 0;
    const bool codes = cfg->table_dtype == HUGE_DTYPE_Q8;
    size_t most = 0;
    auto at_least = [&](size_t bytes) { most = bytes > most ? bytes : most; };
    // few rows are laid out otherwise
    for (int64_t few : {16, 32, 48, 64, 0}) {
        const int64_t n = few == 0 || few > cfg->max_rows ? cfg->max_rows : few;
        at_least(answer_plan(cfg->num_classes, n, cfg->dim, cfg->dtype, codes, cfg->top).total);
    }
    if (cfg->grad)
        at_least(softmax_plan(cfg->num_classes, cfg->max_rows, cfg->dim, cfg->dtype, true).total);
    return most;
}

huge_status huge_log_probs(const huge_log_probs_config* cfg, const void* d_h, int64_t ld_h,
                           int64_t n, const void* d_w, int64_t ld_w, const uint8_t* d_w_scales,
                           int64_t ld_scales, const float* d_bias, const int32_t* d_labels,
                           float* d_logp, float* d_entropy, float* d_lse, int32_t* d_ids,
                           float* d_top_logp, int32_t* d_status, void* d_workspace, size_t ws_bytes,
                           void* stream) {
    const huge_status st = answer_args(cfg, d_h, ld_h, n, d_w, ld_w, d_w_scales, ld_scales, d_bias,
                                       d_labels, d_lse, d_entropy, d_status, d_workspace, ws_bytes);
    if (st != HUGE_OK) return st;
    if (n == 0) return HUGE_OK;
    if (!d_labels != !d_logp || !on(d_logp, 4) ||
        (cfg->top > 0 ? !d_ids || !d_top_logp || !on(d_ids, 4) || !on(d_top_logp, 4)
                      : d_ids || d_top_logp))
        return HUGE_ERR_INVALID_ARG;
    SoftmaxArgs a = answer_call(cfg, d_h, ld_h, n, d_w, ld_w, d_w_scales, ld_scales, d_bias,
                                d_labels, d_status, d_workspace);
    a.logp = d_logp, a.entropy = d_entropy, a.lse = d_lse;
    a.top = cfg->top, a.ids = d_ids, a.top_logp = d_top_logp;
    HEAD_TRY(launch_log_probs(a, static_cast<hipStream_t>(stream)));
    return HUGE_OK;
}

huge_status huge_log_probs_grad(const huge_log_probs_config* cfg, const void* d_h, int64_t ld_h,
                                int64_t n, const void* d_w, int64_t ld_w, const float* d_bias,
                                const int32_t* d_labels, const float* d_lse, const float* d_entropy,
                                const float* d_dlogp, const float* d_dentropy, void* d_dh,
                                void* d_dw, float* d_dbias, int32_t* d_status, void* d_workspace,
                                size_t ws_bytes, void* stream) {
    const huge_status st = answer_args(cfg, d_h, ld_h, n, d_w, ld_w, nullptr, 0, d_bias, d_labels,
                                       d_lse, d_entropy, d_status, d_workspace, ws_bytes);
    if (st != HUGE_OK) return st;
    if (cfg->grad == 0 || (n > 0 && ((d_dlogp && !d_labels) || (d_dentropy && !d_entropy))) ||
        !on(d_dlogp, 4) || !on(d_dentropy, 4) || !on(d_dh, elem(cfg->dtype)) ||
        !on(d_dw, elem(cfg->dtype)) || !on(d_dbias, 4))
        return HUGE_ERR_INVALID_ARG;
    SoftmaxArgs a = answer_call(cfg, d_h, ld_h, n, d_w, ld_w, nullptr, 0, d_bias, d_labels, d_status,
                                d_workspace);
    a.lse = const_cast<float*>(d_lse), a.entropy = const_cast<float*>(d_entropy), a.scale = 1.f;
    a.dlogp = d_dlogp, a.dentropy = d_dentropy;
    a.dh = n > 0 ? d_dh : nullptr, a.dw = d_dw, a.dbias = d_dbias;
    HEAD_TRY(launch_log_probs_grad(a, static_cast<hipStream_t>(stream)));
    return HUGE_OK;
}

size_t huge_grad_norm_workspace_bytes(int32_t count) {
    if (count < 0) return 0;
    const size_t launches = ((size_t)count + kClipTensors - 1) / kClipTensors;
    // a launch is cut short where it would have 2^31 chunks: a tensor has fewer than 2^27
    const size_t cut = (size_t)count / 8;
    return kFactorBytes + (launches + cut + 1) * kClipBlocks * sizeof(double);
}

huge_status huge_grad_norm(const huge_grad_tensor* h_tensors, int32_t count, float* d_norm,
                           void* d_workspace, size_t ws_bytes, void* stream) {
    if (!grads_ok(h_tensors, count) || !d_norm || !on(d_norm, 4)) return HUGE_ERR_INVALID_ARG;
    const huge_status st = norm_ws(count, d_workspace, ws_bytes);
    if (st != HUGE_OK) return st;
    return norm_factor(count, [&](int32_t k) { return h_tensors[k]; }, 1.0, INFINITY, d_norm,
                       d_workspace, static_cast<hipStream_t>(stream));
}

huge_status huge_clip_grads(const huge_grad_tensor* h_tensors, int32_t count, double max_norm,
                            float* d_norm, void* d_workspace, size_t ws_bytes, void* stream) {
    if (!grads_ok(h_tensors, count) || !(max_norm > 0.0) || !on(d_norm, 4))
        return HUGE_ERR_INVALID_ARG;
    huge_status st = norm_ws(count, d_workspace, ws_bytes);
    if (st != HUGE_OK) return st;
    auto tensor = [&](int32_t k) { return h_tensors[k]; };
    hipStream_t s = static_cast<hipStream_t>(stream);
    st = norm_factor(count, tensor, 1.0, max_norm, d_norm, d_workspace, s);
    if (st != HUGE_OK) return st;
    return clip_launches(count, tensor, [&](const ClipArgs& a) {
        return launch_scale(a, static_cast<const float*>(d_workspace), s);
    });
}

huge_status huge_adamw_step_clipped(const huge_adamw_config* cfg, const huge_adamw_tensor* h_tensors,
                                    int32_t count, double max_norm, float* d_norm,
                                    int32_t* d_status, void* d_workspace, size_t ws_bytes,
                                    void* stream) {
    huge_status st = adamw_args(cfg, h_tensors, count, d_status);
    if (st != HUGE_OK) return st;
    if (!(max_norm > 0.0) || !on(d_norm, 4)) return HUGE_ERR_INVALID_ARG;
    st = norm_ws(count, d_workspace, ws_bytes);
    if (st != HUGE_OK) return st;
    auto tensor = [&](int32_t k) {
        const huge_adamw_tensor& t = h_tensors[k];
        return huge_grad_tensor{const_cast<void*>(t.d_grad), t.n, t.grad_dtype};
    };
    st = norm_factor(count, tensor, cfg->grad_scale, max_norm, d_norm, d_workspace,
                     static_cast<hipStream_t>(stream));
    if (st != HUGE_OK) return st;
    return adamw_step(cfg, h_tensors, count, static_cast<const float*>(d_workspace), d_status,
                      stream);
}

}  // extern "C"

// C ABI of include/gns_layers.h: argument checks and launches.
#include "gns_checks.hpp"
#include "gns_layers.hpp"
#include <math.h>

using namespace gns;

namespace {

// What is wrong with a norm of rows of this width; null if nothing.
const char* norm_fault(const gns_norm* n, int32_t width)
{
    if (!n) return "null norm";
    if (n->groups < 1 || width % n->groups) return "groups must divide the width";
    if (n->activation < GNS_ACT_NONE || n->activation > GNS_ACT_GELU) return "no such activation";
    if (!(n->eps > 0.f) || !isfinite(n->eps)) return "eps must be positive and finite";
    if (n->segments_dev ? n->num_segments < 0 || n->num_segments > GNS_MAX_SEGMENTS : n->segment_rows < 1) return "segments out of range";
    if (misaligned(n->segments_dev, 4) || misaligned(n->gamma_dev, 4) || misaligned(n->beta_dev, 4)) return "segments, gamma and beta must be aligned";
    return nullptr;
}

// Rows that a call writes and may share with others of it: the same rows, or none of them.
bool same_rows(const gns_rows* a, const gns_rows* b) { return a->stride == b->stride && a->type == b->type; }

NormArgs norm_args(const gns_norm* n)
{
    NormArgs a = {};
    a.segments = n->segments_dev; a.num_segments = n->num_segments; a.segment_rows = n->segment_rows;
    a.groups = n->groups; a.activation = n->activation; a.eps = n->eps;
    a.gamma = n->gamma_dev; a.beta = n->beta_dev;
    return a;
}

size_t norm_bytes(const gns_ctx* ctx, int32_t width, const gns_norm* norm, int32_t num_rows, bool backward)
{
    if (!ctx || width < 1 || width > GNS_MAX_WIDTH || norm_fault(norm, width)) return 0;
    const int32_t rows = worst_rows(ctx, num_rows);
    return rows < 1 ? 0 : align256(norm_workspace(ctx, width, norm, rows, backward));
}

// [x1 | x2] of a quantising call
gns_status quantize_args(gns_ctx* ctx, const gns_rows* x1, const gns_rows* x2, int32_t num_rows, QuantizeFp8Args* a)
{
    GNS_REQUIRE_ROWS(x1);
    a->x1 = as_const(x1);
    a->x2 = ConstRows{nullptr, 0, 0};
    int64_t k = x1->width;
    if (x2) {
        GNS_REQUIRE_ROWS(x2);
        GNS_REQUIRE(x2->type == x1->type, "both inputs must be of one type");
        a->x2 = as_const(x2);
        k += x2->width;
    }
    GNS_REQUIRE(k <= GNS_FP8_MAX_K, "more columns than GNS_FP8_MAX_K");
    a->stride = GNS_FP8_STRIDE(k);
    a->exponent_stride = GNS_FP8_EXPONENTS(k);
    GNS_REQUIRE(row_count(ctx, num_rows, &a->count), "bad device-count placeholder");
    return GNS_OK;
}

gns_status dense_fp8_args(gns_ctx* ctx, int32_t k, const uint8_t* wq, const uint8_t* w_exponents, const float* bias, int32_t relu,
                          const gns_rows* out, int32_t num_rows, DenseFp8Args* a)
{
    GNS_REQUIRE_ROWS(out);
    GNS_REQUIRE(wq && w_exponents, "null weights or exponents");
    GNS_REQUIRE(!misaligned(wq, 16) && !misaligned(w_exponents, 4), "weights in 8 bits must be 16-byte aligned, their exponents 4-byte");
    GNS_REQUIRE(!misaligned(bias, 4), "bias must be aligned");
    a->wq = wq; a->w_exponents = w_exponents; a->bias = bias;
    a->out = as_mut(out);
    a->stride = GNS_FP8_STRIDE(k);
    a->exponent_stride = GNS_FP8_EXPONENTS(k);
    a->k = k; a->relu = relu;
    return GNS_OK;
}

}  // namespace

extern "C" {

size_t gns_group_norm_workspace_bytes(const gns_ctx* ctx, int32_t width, const gns_norm* norm, int32_t num_rows)
{
    return norm_bytes(ctx, width, norm, num_rows, false);
}

gns_status gns_group_norm(gns_ctx* ctx, const gns_rows* x, const gns_norm* norm, const gns_rows* out, float* stats_dev,
                          int32_t num_rows, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    GNS_REQUIRE_ROWS(x);
    GNS_REQUIRE_ROWS(out);
    GNS_REQUIRE(out->width == x->width && out->type == x->type, "out must have the width and type of x");
    GNS_REQUIRE_OF_ROWS(out->data != x->data || same_rows(out, x), "out may only be x's own rows");
    if (const char* fault = norm_fault(norm, x->width)) return ctx_fail(ctx, GNS_EINVAL, fault);
    GNS_REQUIRE(!misaligned(stats_dev, 8), "stats must be 8-byte aligned");
    NormArgs a = norm_args(norm);
    GNS_REQUIRE(row_count(ctx, num_rows, &a.count), "bad device-count placeholder");
    if (a.count.rows > 0) {
        const size_t need = norm_need(ctx, x->width, norm, x->type, a.count.rows, false);
        if (need) {
            GNS_REQUIRE(workspace && !misaligned(workspace, 256), "workspace is null or not 256-byte aligned");
            if (workspace_bytes < need) return ctx_fail(ctx, GNS_ECAPACITY, "workspace is too small");
        }
    }
    a.x = as_const(x);
    a.out = as_mut(out);
    a.stats = stats_dev;
    a.workspace = workspace;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_NORM, s);
    const hipError_t e = launch_norm(ctx, a, x->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "norm launch", e);
}

size_t gns_group_norm_backward_workspace_bytes(const gns_ctx* ctx, int32_t width, const gns_norm* norm, int32_t num_rows)
{
    return norm_bytes(ctx, width, norm, num_rows, true);
}

gns_status gns_group_norm_backward(gns_ctx* ctx, const gns_rows* d_out, const gns_rows* x, const gns_norm* norm,
                                   const float* stats_dev, const gns_rows* dx, float* dgamma_dev, float* dbeta_dev,
                                   int32_t num_rows, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    GNS_REQUIRE_ROWS(x);
    GNS_REQUIRE_ROWS(d_out);
    GNS_REQUIRE(d_out->width == x->width && d_out->type == x->type, "d_out must have the width and type of x");
    if (const char* fault = norm_fault(norm, x->width)) return ctx_fail(ctx, GNS_EINVAL, fault);
    GNS_REQUIRE(dx || dgamma_dev || dbeta_dev, "no gradient is wanted");
    GNS_REQUIRE_OF_ROWS(stats_dev || (norm->segments_dev && norm->num_segments == 0), "null stats");
    GNS_REQUIRE(!misaligned(stats_dev, 8), "stats must be 8-byte aligned");
    GNS_REQUIRE(!misaligned(dgamma_dev, 4) && !misaligned(dbeta_dev, 4), "dgamma and dbeta must be aligned");
    NormArgs a = norm_args(norm);
    if (dx) {
        GNS_REQUIRE_ROWS(dx);
        GNS_REQUIRE(dx->width == x->width && dx->type == x->type, "dx must have the width and type of x");
        GNS_REQUIRE_OF_ROWS((dx->data != x->data || same_rows(dx, x)) && (dx->data != d_out->data || same_rows(dx, d_out)),
                            "dx may only be the own rows of x or d_out");
        a.out = as_mut(dx);
    }
    GNS_REQUIRE(row_count(ctx, num_rows, &a.count), "bad device-count placeholder");
    if (a.count.rows > 0) {
        const size_t need = norm_need(ctx, x->width, norm, x->type, a.count.rows, true);
        if (need) {
            GNS_REQUIRE(workspace && !misaligned(workspace, 256), "workspace is null or not 256-byte aligned");
            if (workspace_bytes < need) return ctx_fail(ctx, GNS_ECAPACITY, "workspace is too small");
        }
    }
    a.x = as_const(x);
    a.d_out = as_const(d_out);
    a.stats = const_cast<float*>(stats_dev);
    a.dgamma = dgamma_dev; a.dbeta = dbeta_dev;
    a.workspace = workspace;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_NORM, s);
    const hipError_t e = launch_norm_backward(ctx, a, x->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "norm backward launch", e);
}

size_t gns_orthogonal_update_workspace_bytes(const gns_ctx* ctx, int32_t width, int32_t num_rows)
{
    if (!ctx || width < 1 || width > GNS_ORTHOGONAL_MAX || num_rows < 1 || num_rows > GNS_ORTHOGONAL_MAX) return 0;
    return align256(orthogonal_workspace(ctx, width, num_rows));
}

gns_status gns_orthogonal_update(gns_ctx* ctx, const gns_rows* grad, const gns_rows* momentum, const gns_orthogonal* how,
                                 const gns_rows* w, const gns_rows* momentum_out, const gns_rows* out, int32_t num_rows,
                                 void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    GNS_REQUIRE(num_rows >= 0 && num_rows <= GNS_ORTHOGONAL_MAX, "rows of a matrix of weights out of range");
    GNS_REQUIRE_ROWS(grad);
    GNS_REQUIRE_ROWS(out);
    GNS_REQUIRE(grad->width <= GNS_ORTHOGONAL_MAX, "width of a matrix of weights out of range");
    GNS_REQUIRE(out->width == grad->width, "out must have the width of the gradient");
    GNS_REQUIRE(!momentum == !momentum_out, "momentum and momentum_out go together");
    GNS_REQUIRE(how, "null coefficients");
    GNS_REQUIRE(how->steps >= 0 && how->steps <= GNS_MAX_STEPS, "steps out of range");
    GNS_REQUIRE(how->eps >= 0.f && isfinite(how->eps) && isfinite(how->mu) && isfinite(how->keep) && isfinite(how->rate), "eps, mu, keep and rate must be finite");
    for (int i = 0; i < how->steps; ++i)
        for (int j = 0; j < 3; ++j) GNS_REQUIRE(isfinite(how->coefficients[i][j]), "coefficients must be finite");
    OrthogonalArgs a = {};
    if (momentum) {
        GNS_REQUIRE_ROWS(momentum);
        GNS_REQUIRE_ROWS(momentum_out);
        GNS_REQUIRE(momentum->width == grad->width && momentum_out->width == grad->width, "momentum must have the width of the gradient");
        GNS_REQUIRE_OF_ROWS(momentum_out->data != momentum->data || same_rows(momentum_out, momentum), "momentum_out may only be momentum's own rows");
        GNS_REQUIRE_OF_ROWS(momentum_out->data != out->data && momentum_out->data != grad->data && momentum->data != out->data, "momentum and the others must not overlap");
        a.momentum = as_const(momentum); a.momentum_type = momentum->type;
        a.momentum_out = as_mut(momentum_out); a.momentum_out_type = momentum_out->type;
    }
    if (w) {
        GNS_REQUIRE_ROWS(w);
        GNS_REQUIRE(w->width == grad->width, "weights must have the width of the gradient");
        GNS_REQUIRE_OF_ROWS(out->data != w->data || same_rows(out, w), "out may only be the weights' own rows");
        GNS_REQUIRE_OF_ROWS(!momentum || momentum_out->data != w->data, "momentum and the others must not overlap");
        a.w = as_const(w); a.w_type = w->type;
    }
    GNS_REQUIRE_OF_ROWS(out->data != grad->data || same_rows(out, grad), "out may only be the gradient's own rows");
    if (num_rows == 0) return GNS_OK;
    GNS_REQUIRE(workspace && !misaligned(workspace, 256), "workspace is null or not 256-byte aligned");
    if (workspace_bytes < orthogonal_workspace(ctx, grad->width, num_rows)) return ctx_fail(ctx, GNS_ECAPACITY, "workspace is too small");
    a.grad = as_const(grad); a.grad_type = grad->type;
    a.out = as_mut(out); a.out_type = out->type;
    a.rows = num_rows;
    a.how = how;
    a.workspace = workspace;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_ORTHOGONAL, s);
    const hipError_t e = launch_orthogonal(ctx, a, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "orthogonal update launch", e);
}

gns_status gns_quantize_fp8(gns_ctx* ctx, const gns_rows* x1, const gns_rows* x2, uint8_t* q_dev, uint8_t* exponents_dev,
                            int32_t num_rows, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    QuantizeFp8Args a;
    const gns_status st = quantize_args(ctx, x1, x2, num_rows, &a);
    if (st != GNS_OK) return st;
    GNS_REQUIRE_OF_ROWS(q_dev && exponents_dev, "null output");
    GNS_REQUIRE(!misaligned(q_dev, 16) && !misaligned(exponents_dev, 4), "rows in 8 bits must be 16-byte aligned, their exponents 4-byte");
    a.q = q_dev; a.exponents = exponents_dev;
    if (a.count.rows == 0) return GNS_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_FP8, s);
    const hipError_t e = launch_quantize_fp8(ctx, a, x1->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "quantize launch", e);
}

gns_status gns_dense_fp8(gns_ctx* ctx, const uint8_t* q_dev, const uint8_t* exponents_dev, int32_t k, const uint8_t* wq_dev,
                         const uint8_t* w_exponents_dev, const float* bias_dev, int32_t relu, const gns_rows* out,
                         int32_t num_rows, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    GNS_REQUIRE_OF_ROWS(q_dev && exponents_dev, "null rows in 8 bits");
    GNS_REQUIRE(!misaligned(q_dev, 16) && !misaligned(exponents_dev, 4), "rows in 8 bits must be 16-byte aligned, their exponents 4-byte");
    GNS_REQUIRE(k >= 1 && k <= GNS_FP8_MAX_K, "k out of range");
    DenseFp8Args a;
    const gns_status st = dense_fp8_args(ctx, k, wq_dev, w_exponents_dev, bias_dev, relu, out, num_rows, &a);
    if (st != GNS_OK) return st;
    GNS_REQUIRE(row_count(ctx, num_rows, &a.count), "bad device-count placeholder");
    a.q = q_dev; a.exponents = exponents_dev;
    if (a.count.rows == 0) return GNS_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_FP8, s);
    const hipError_t e = launch_dense_fp8(ctx, a, out->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "fp8 product launch", e);
}

size_t gns_sage_dense_fp8_workspace_bytes(const gns_ctx* ctx, int32_t k, int32_t num_rows)
{
    if (!ctx || k < 1 || k > GNS_FP8_MAX_K) return 0;
    const int32_t rows = worst_rows(ctx, num_rows);
    if (rows < 1) return 0;
    return align256((size_t) rows * GNS_FP8_STRIDE(k)) + align256((size_t) rows * GNS_FP8_EXPONENTS(k));
}

gns_status gns_sage_dense_fp8(gns_ctx* ctx, const gns_rows* x1, const gns_rows* x2, const uint8_t* wq_dev,
                              const uint8_t* w_exponents_dev, const float* bias_dev, int32_t relu, const gns_rows* out,
                              int32_t num_rows, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    QuantizeFp8Args x;
    gns_status st = quantize_args(ctx, x1, x2, num_rows, &x);
    if (st != GNS_OK) return st;
    const int32_t k = x.x1.width + x.x2.width;
    DenseFp8Args a;
    st = dense_fp8_args(ctx, k, wq_dev, w_exponents_dev, bias_dev, relu, out, num_rows, &a);
    if (st != GNS_OK) return st;
    a.count = x.count;
    if (a.count.rows == 0) return GNS_OK;
    GNS_REQUIRE(workspace && !misaligned(workspace, 256), "workspace is null or not 256-byte aligned");
    if (workspace_bytes < gns_sage_dense_fp8_workspace_bytes(ctx, k, num_rows)) return ctx_fail(ctx, GNS_ECAPACITY, "workspace is too small");
    x.q = static_cast<uint8_t*>(workspace);
    x.exponents = x.q + align256((size_t) a.count.rows * (size_t) x.stride);
    a.q = x.q; a.exponents = x.exponents;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_FP8, s);
    const hipError_t e = launch_sage_dense_fp8(ctx, x, a, x1->type, out->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "fp8 update launch", e);
}

}  // extern "C"

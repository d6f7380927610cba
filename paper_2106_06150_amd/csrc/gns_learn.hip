// C ABI of include/gns_learn.h: argument checks and launches.
#include "gns_learn.hpp"

using namespace gns;

namespace {

constexpr size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// Reads num_rows: a count, or the placeholder of a layer whose count is on the device.
bool row_count(gns_ctx* c, int32_t num_rows, RowCount* out)
{
    out->rows = num_rows;
    out->rows_dev = nullptr;
    if (num_rows >= 0) return true;
    const int layer = -1 - num_rows;
    if (layer >= c->config.num_layers) return false;
    out->rows = (int32_t) c->lay.rows[layer];
    out->rows_dev = &c->d_state->num_dst[layer];
    return true;
}

int32_t worst_rows(const gns_ctx* c, int32_t num_rows)
{
    if (num_rows >= 0) return num_rows;
    return -1 - num_rows < c->config.num_layers ? (int32_t) c->lay.rows[-1 - num_rows] : -1;
}

// What is wrong with rows of a call of num_rows; null if nothing.  Without rows there need be no data.
const char* rows_fault(const gns_rows* x, int32_t num_rows)
{
    if (!x || (!x->data && num_rows)) return "null rows";
    if (x->type != GNS_FP32 && x->type != GNS_BF16) return "rows are of no known type";
    if (x->width < 1 || x->width > GNS_MAX_WIDTH) return "width of rows out of range";
    if (x->stride < x->width || x->stride > GNS_MAX_STRIDE) return "stride of rows out of range";
    if (reinterpret_cast<uintptr_t>(x->data) % (x->type == GNS_FP32 ? 4 : 2)) return "rows are not aligned to their element";
    return nullptr;
}

bool misaligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

ConstRows as_const(const gns_rows* x) { return ConstRows{x->data, x->stride, x->width}; }
MutRows as_mut(const gns_rows* x) { return MutRows{x->data, x->stride, x->width}; }

#define GNS_REQUIRE(cond, message) \
    do { if (!(cond)) return ctx_fail(ctx, GNS_EINVAL, message); } while (0)
// what belongs to the rows of a call: its buffers have no address where there are none
#define GNS_REQUIRE_OF_ROWS(cond, message) GNS_REQUIRE((cond) || num_rows == 0, message)
#define GNS_REQUIRE_ROWS(x) \
    do { if (const char* fault = rows_fault(x, num_rows)) return ctx_fail(ctx, GNS_EINVAL, fault); } while (0)

// [x1 | x2] of a quantising call
gns_status quantize_args(gns_ctx* ctx, const gns_rows* x1, const gns_rows* x2, int32_t num_rows, QuantizeArgs* a)
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
    GNS_REQUIRE(k <= GNS_INT8_MAX_K, "more columns than an exact sum holds");
    a->stride = GNS_INT8_STRIDE(k);
    GNS_REQUIRE(row_count(ctx, num_rows, &a->count), "bad device-count placeholder");
    return GNS_OK;
}

gns_status dense_int8_args(gns_ctx* ctx, int32_t k, const int8_t* wq, const float* w_scale, const float* bias, int32_t relu,
                           const gns_rows* out, int32_t num_rows, DenseInt8Args* a)
{
    GNS_REQUIRE_ROWS(out);
    GNS_REQUIRE(wq && w_scale, "null weights or scales");
    GNS_REQUIRE(!misaligned(wq, 16), "weights in 8 bits must be 16-byte aligned");
    GNS_REQUIRE(!misaligned(w_scale, 4) && !misaligned(bias, 4), "scales and bias must be aligned");
    a->wq = wq; a->w_scale = w_scale; a->bias = bias;
    a->out = as_mut(out);
    a->stride = GNS_INT8_STRIDE(k);
    a->k = k; a->relu = relu;
    return GNS_OK;
}

}  // namespace

extern "C" {

gns_status gns_quantize_rows(gns_ctx* ctx, const gns_rows* x1, const gns_rows* x2, int8_t* q_dev, float* scale_dev,
                             int32_t num_rows, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    QuantizeArgs a;
    const gns_status st = quantize_args(ctx, x1, x2, num_rows, &a);
    if (st != GNS_OK) return st;
    GNS_REQUIRE_OF_ROWS(q_dev && scale_dev, "null output");
    GNS_REQUIRE(!misaligned(q_dev, 16) && !misaligned(scale_dev, 4), "rows in 8 bits must be 16-byte aligned");
    a.q = q_dev; a.scale = scale_dev;
    if (a.count.rows == 0) return GNS_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_INT8, s);
    const hipError_t e = launch_quantize(ctx, a, x1->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "quantize launch", e);
}

gns_status gns_dense_int8(gns_ctx* ctx, const int8_t* q_dev, const float* scale_dev, int32_t k, const int8_t* wq_dev,
                          const float* w_scale_dev, const float* bias_dev, int32_t relu, const gns_rows* out,
                          int32_t num_rows, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    GNS_REQUIRE_OF_ROWS(q_dev && scale_dev, "null rows in 8 bits");
    GNS_REQUIRE(!misaligned(q_dev, 16) && !misaligned(scale_dev, 4), "rows in 8 bits must be 16-byte aligned");
    GNS_REQUIRE(k >= 1 && k <= GNS_INT8_MAX_K, "k out of range");
    DenseInt8Args a;
    const gns_status st = dense_int8_args(ctx, k, wq_dev, w_scale_dev, bias_dev, relu, out, num_rows, &a);
    if (st != GNS_OK) return st;
    GNS_REQUIRE(row_count(ctx, num_rows, &a.count), "bad device-count placeholder");
    a.q = q_dev; a.scale = scale_dev;
    if (a.count.rows == 0) return GNS_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_INT8, s);
    const hipError_t e = launch_dense_int8(ctx, a, out->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "int8 product launch", e);
}

size_t gns_sage_dense_int8_workspace_bytes(const gns_ctx* ctx, int32_t k, int32_t num_rows)
{
    if (!ctx || k < 1 || k > GNS_INT8_MAX_K) return 0;
    const int32_t rows = worst_rows(ctx, num_rows);
    if (rows < 1) return 0;
    return align256((size_t) rows * GNS_INT8_STRIDE(k)) + align256((size_t) rows * 4);
}

gns_status gns_sage_dense_int8(gns_ctx* ctx, const gns_rows* x1, const gns_rows* x2, const int8_t* wq_dev,
                               const float* w_scale_dev, const float* bias_dev, int32_t relu, const gns_rows* out,
                               int32_t num_rows, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    QuantizeArgs x;
    gns_status st = quantize_args(ctx, x1, x2, num_rows, &x);
    if (st != GNS_OK) return st;
    const int32_t k = x.x1.width + x.x2.width;
    DenseInt8Args a;
    st = dense_int8_args(ctx, k, wq_dev, w_scale_dev, bias_dev, relu, out, num_rows, &a);
    if (st != GNS_OK) return st;
    a.count = x.count;
    if (a.count.rows == 0) return GNS_OK;
    GNS_REQUIRE(workspace && !misaligned(workspace, 256), "workspace is null or not 256-byte aligned");
    if (workspace_bytes < gns_sage_dense_int8_workspace_bytes(ctx, k, num_rows))
        return ctx_fail(ctx, GNS_ECAPACITY, "workspace is too small");
    x.q = static_cast<int8_t*>(workspace);
    x.scale = reinterpret_cast<float*>(static_cast<char*>(workspace) + align256((size_t) a.count.rows * (size_t) x.stride));
    a.q = x.q; a.scale = x.scale;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_INT8, s);
    const hipError_t e = launch_sage_dense_int8(ctx, x, a, x1->type, out->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "int8 update launch", e);
}

gns_status gns_checkpoint_save(gns_ctx* ctx, const gns_rows* x, int8_t* q_dev, uint8_t* exponents_dev,
                               uint32_t* positive_dev, int32_t num_rows, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    GNS_REQUIRE_ROWS(x);
    GNS_REQUIRE_OF_ROWS(q_dev && exponents_dev, "null checkpoint");
    GNS_REQUIRE(!misaligned(q_dev, 16) && !misaligned(positive_dev, 4), "checkpoints must be 16-byte aligned");
    CheckpointArgs a = {};
    GNS_REQUIRE(row_count(ctx, num_rows, &a.count), "bad device-count placeholder");
    a.x = as_const(x);
    a.q = q_dev; a.exponents = exponents_dev; a.positive = positive_dev;
    a.width = x->width; a.groups = (int32_t) (((int64_t) x->width + 31) / 32);
    if (a.count.rows == 0) return GNS_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_CHECKPOINT, s);
    const hipError_t e = launch_checkpoint_save(ctx, a, x->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "checkpoint launch", e);
}

gns_status gns_checkpoint_load(gns_ctx* ctx, const int8_t* q_dev, const uint8_t* exponents_dev, const gns_rows* x,
                               int32_t num_rows, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    GNS_REQUIRE_ROWS(x);
    GNS_REQUIRE_OF_ROWS(q_dev && exponents_dev, "null checkpoint");
    GNS_REQUIRE(!misaligned(q_dev, 16), "checkpoints must be 16-byte aligned");
    CheckpointArgs a = {};
    GNS_REQUIRE(row_count(ctx, num_rows, &a.count), "bad device-count placeholder");
    a.out = as_mut(x);
    a.q = const_cast<int8_t*>(q_dev); a.exponents = const_cast<uint8_t*>(exponents_dev);
    a.width = x->width; a.groups = (int32_t) (((int64_t) x->width + 31) / 32);
    if (a.count.rows == 0) return GNS_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_CHECKPOINT, s);
    const hipError_t e = launch_checkpoint_load(ctx, a, x->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "checkpoint launch", e);
}

size_t gns_sage_dense_backward_workspace_bytes(const gns_ctx* ctx, int32_t f1, int32_t f2, int32_t hdim, int32_t num_rows)
{
    if (!ctx || f1 < 1 || f2 < 0 || hdim < 1 || (int64_t) f1 + f2 > GNS_MAX_WIDTH || hdim > GNS_MAX_WIDTH) return 0;
    const int32_t rows = worst_rows(ctx, num_rows);
    return rows < 0 ? 0 : align256(backward_workspace(ctx, f1, f2, hdim, rows));
}

gns_status gns_sage_dense_backward(gns_ctx* ctx, const gns_rows* d_out, const uint32_t* positive_dev,
                                   const int8_t* q1_dev, const uint8_t* exponents1_dev, int32_t f1,
                                   const int8_t* q2_dev, const uint8_t* exponents2_dev, int32_t f2, const float* w_dev,
                                   float* dw_dev, float* db_dev, const gns_rows* dx, int32_t num_rows, void* workspace,
                                   size_t workspace_bytes, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    GNS_REQUIRE_ROWS(d_out);
    GNS_REQUIRE(f1 >= 1 && f2 >= 0 && (int64_t) f1 + f2 <= GNS_MAX_WIDTH, "f1 or f2 out of range");
    GNS_REQUIRE(dw_dev || dx, "no gradient is wanted");
    GNS_REQUIRE(dw_dev || !db_dev, "db comes with dw only");
    GNS_REQUIRE(!misaligned(positive_dev, 4) && !misaligned(db_dev, 4), "positive and db must be aligned");
    if (dw_dev) {
        GNS_REQUIRE_OF_ROWS(q1_dev && exponents1_dev && (!f2 || (q2_dev && exponents2_dev)), "null checkpoint");
        GNS_REQUIRE(!misaligned(q1_dev, 16) && (!f2 || !misaligned(q2_dev, 16)), "checkpoints must be 16-byte aligned");
        GNS_REQUIRE(!misaligned(dw_dev, 4), "dw must be aligned");
    }
    BackwardArgs a = {};
    if (dx) {
        GNS_REQUIRE_ROWS(dx);
        GNS_REQUIRE(dx->width == f1 + f2, "dx must have f1 + f2 columns");
        GNS_REQUIRE(dx->type == d_out->type, "dx must be of the type of d_out");
        GNS_REQUIRE(w_dev && !misaligned(w_dev, 4), "null or misaligned weights");
        a.dx = as_mut(dx);
    }
    GNS_REQUIRE(row_count(ctx, num_rows, &a.count), "bad device-count placeholder");
    GNS_REQUIRE(workspace && !misaligned(workspace, 256), "workspace is null or not 256-byte aligned");
    if (workspace_bytes < align256(backward_need(ctx, f1, f2, d_out->width, a.count.rows)))
        return ctx_fail(ctx, GNS_ECAPACITY, "workspace is too small");
    a.d_out = as_const(d_out);
    a.positive = positive_dev;
    a.x1 = PackedRows{q1_dev, exponents1_dev, f1, (int32_t) (((int64_t) f1 + 31) / 32)};
    a.x2 = PackedRows{q2_dev, exponents2_dev, f2, (int32_t) (((int64_t) f2 + 31) / 32)};
    a.w = w_dev; a.dw = dw_dev; a.db = db_dev;
    a.hdim = d_out->width;
    a.workspace = workspace;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_BACKWARD, s);
    const hipError_t e = launch_backward(ctx, a, d_out->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "backward launch", e);
}

size_t gns_log_probs_workspace_bytes(const gns_ctx* ctx, int32_t num_classes, int32_t top, int32_t num_rows)
{
    if (!ctx || num_classes < 1 || top < 0 || top > GNS_MAX_TOP) return 0;
    const int32_t rows = worst_rows(ctx, num_rows);
    return rows < 1 ? 0 : align256(log_probs_workspace(ctx, num_classes, top, rows));
}

gns_status gns_log_probs(gns_ctx* ctx, const gns_rows* logits, const int32_t* labels_dev, float* logp_dev,
                         float* entropy_dev, float* stats_dev, int32_t top, int32_t* top_index_dev, float* top_logp_dev,
                         int32_t num_rows, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    GNS_REQUIRE_ROWS(logits);
    GNS_REQUIRE_OF_ROWS(!labels_dev == !logp_dev, "labels and logp go together");
    GNS_REQUIRE(top >= 0 && top <= GNS_MAX_TOP, "top out of range");
    GNS_REQUIRE_OF_ROWS(top ? top_index_dev && top_logp_dev : !top_index_dev && !top_logp_dev, "top and its outputs do not agree");
    GNS_REQUIRE_OF_ROWS(logp_dev || entropy_dev || stats_dev || top, "no output is wanted");
    GNS_REQUIRE(!misaligned(labels_dev, 4) && !misaligned(logp_dev, 4) && !misaligned(entropy_dev, 4) &&
                !misaligned(top_index_dev, 4) && !misaligned(top_logp_dev, 4), "labels and outputs must be aligned");
    GNS_REQUIRE(!misaligned(stats_dev, 8), "stats must be 8-byte aligned");
    LogProbsArgs a = {};
    GNS_REQUIRE(row_count(ctx, num_rows, &a.count), "bad device-count placeholder");
    if (a.count.rows == 0) return GNS_OK;
    const size_t need = log_probs_need(ctx, logits->width, top, a.count.rows);
    if (need) {
        GNS_REQUIRE(workspace && !misaligned(workspace, 256), "workspace is null or not 256-byte aligned");
        if (workspace_bytes < need) return ctx_fail(ctx, GNS_ECAPACITY, "workspace is too small");
    }
    a.logits = as_const(logits);
    a.labels = labels_dev; a.logp = logp_dev; a.entropy = entropy_dev; a.stats = stats_dev;
    a.top = top; a.top_index = top_index_dev; a.top_logp = top_logp_dev;
    a.workspace = workspace;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_LOG_PROBS, s);
    const hipError_t e = launch_log_probs(ctx, a, logits->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "log probs launch", e);
}

gns_status gns_log_probs_backward(gns_ctx* ctx, const gns_rows* logits, const int32_t* labels_dev, const float* stats_dev,
                                  const float* entropy_dev, const float* g_logp_dev, const float* g_entropy_dev,
                                  const gns_rows* d_logits, int32_t num_rows, void* hip_stream)
{
    if (!ctx) return GNS_EINVAL;
    GNS_REQUIRE_ROWS(logits);
    GNS_REQUIRE_ROWS(d_logits);
    GNS_REQUIRE(d_logits->width == logits->width, "d_logits must have the width of the logits");
    GNS_REQUIRE_OF_ROWS(d_logits->data != logits->data || (d_logits->stride == logits->stride && d_logits->type == logits->type),
                "d_logits may only be the logits' own rows");
    GNS_REQUIRE_OF_ROWS(stats_dev, "null stats");
    GNS_REQUIRE(!misaligned(stats_dev, 8), "stats must be 8-byte aligned");
    GNS_REQUIRE_OF_ROWS(!g_logp_dev || labels_dev, "g_logp needs the labels");
    GNS_REQUIRE_OF_ROWS(!g_entropy_dev || entropy_dev, "g_entropy needs the entropy");
    GNS_REQUIRE_OF_ROWS(g_logp_dev || g_entropy_dev, "no gradient is given");
    GNS_REQUIRE(!misaligned(labels_dev, 4) && !misaligned(g_logp_dev, 4) && !misaligned(entropy_dev, 4) && !misaligned(g_entropy_dev, 4),
                "labels and gradients must be aligned");
    LogProbsBackwardArgs a = {};
    GNS_REQUIRE(row_count(ctx, num_rows, &a.count), "bad device-count placeholder");
    if (a.count.rows == 0) return GNS_OK;
    a.logits = as_const(logits);
    a.labels = g_logp_dev ? labels_dev : nullptr;
    a.entropy = g_entropy_dev ? entropy_dev : nullptr;
    a.stats = stats_dev; a.g_logp = g_logp_dev; a.g_entropy = g_entropy_dev;
    a.d_logits = as_mut(d_logits);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    StageTimer t(ctx, GNS_STAGE_LOG_PROBS, s);
    const hipError_t e = launch_log_probs_backward(ctx, a, logits->type, d_logits->type, s);
    return e == hipSuccess ? GNS_OK : ctx_fail(ctx, GNS_EHIP, "log probs backward launch", e);
}

}  // extern "C"

// Checks of arguments that the entry points of training and answering share.
#pragma once
#include "gns_learn.hpp"

namespace gns {

constexpr size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// Reads num_rows: a count, or the placeholder of a layer whose count is on the device.
inline bool row_count(gns_ctx* c, int32_t num_rows, RowCount* out)
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

inline int32_t worst_rows(const gns_ctx* c, int32_t num_rows)
{
    if (num_rows >= 0) return num_rows;
    return -1 - num_rows < c->config.num_layers ? (int32_t) c->lay.rows[-1 - num_rows] : -1;
}

// What is wrong with rows of a call of num_rows; null if nothing.  Without rows there need be no data.
inline const char* rows_fault(const gns_rows* x, int32_t num_rows)
{
    if (!x || (!x->data && num_rows)) return "null rows";
    if (x->type != GNS_FP32 && x->type != GNS_BF16) return "rows are of no known type";
    if (x->width < 1 || x->width > GNS_MAX_WIDTH) return "width of rows out of range";
    if (x->stride < x->width || x->stride > GNS_MAX_STRIDE) return "stride of rows out of range";
    if (reinterpret_cast<uintptr_t>(x->data) % (x->type == GNS_FP32 ? 4 : 2)) return "rows are not aligned to their element";
    return nullptr;
}

inline bool misaligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

inline ConstRows as_const(const gns_rows* x) { return ConstRows{x->data, x->stride, x->width}; }
inline MutRows as_mut(const gns_rows* x) { return MutRows{x->data, x->stride, x->width}; }

}  // namespace gns

#define GNS_REQUIRE(cond, message) \
    do { if (!(cond)) return ctx_fail(ctx, GNS_EINVAL, message); } while (0)
// what belongs to the rows of a call: its buffers have no address where there are none
#define GNS_REQUIRE_OF_ROWS(cond, message) GNS_REQUIRE((cond) || num_rows == 0, message)
#define GNS_REQUIRE_ROWS(x) \
    do { if (const char* fault = rows_fault(x, num_rows)) return ctx_fail(ctx, GNS_EINVAL, fault); } while (0)

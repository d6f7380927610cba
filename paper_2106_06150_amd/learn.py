"""ctypes binding of include/gns_learn.h (argument marshalling only): the update step in 8-bit integers, activation
checkpoints in 8 bits and the backward pass from them, log probabilities with their gradient.

Matrices of floats are 2-D torch tensors on the device, fp32 or bf16, whose columns are adjacent; rows may be any stride
apart.  num_rows is a count, or -1 - i for the dst rows of layer index i of the context's last mini-batch (read on the
device).  Errors are binding.GnsError.
"""
import ctypes

import torch

from .binding import _check, _stream_ptr, lib

GNS_FP32, GNS_BF16 = 0, 1
GNS_MAX_WIDTH, GNS_MAX_STRIDE = 1 << 22, 1 << 24
GNS_INT8_MAX_K = 131072
GNS_MAX_TOP = 32
GNS_STAGE_INT8, GNS_STAGE_CHECKPOINT, GNS_STAGE_BACKWARD, GNS_STAGE_LOG_PROBS = 22, 23, 24, 25
CHECKPOINT_GROUP = 32

EXPORTED = ["gns_quantize_rows", "gns_dense_int8", "gns_sage_dense_int8", "gns_sage_dense_int8_workspace_bytes",
            "gns_checkpoint_save", "gns_checkpoint_load", "gns_sage_dense_backward",
            "gns_sage_dense_backward_workspace_bytes", "gns_log_probs", "gns_log_probs_workspace_bytes",
            "gns_log_probs_backward"]


class gns_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64), ("width", ctypes.c_int32), ("type", ctypes.c_int32)]


def _declare():
    vp, i32, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    R = ctypes.POINTER(gns_rows)
    for name, args in dict(
            gns_quantize_rows=[vp, R, R, vp, vp, i32, vp],
            gns_dense_int8=[vp, vp, vp, i32, vp, vp, vp, i32, R, i32, vp],
            gns_sage_dense_int8=[vp, R, R, vp, vp, vp, i32, R, i32, vp, size, vp],
            gns_checkpoint_save=[vp, R, vp, vp, vp, i32, vp],
            gns_checkpoint_load=[vp, vp, vp, R, i32, vp],
            gns_sage_dense_backward=[vp, R, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp, R, i32, vp, size, vp],
            gns_log_probs=[vp, R, vp, vp, vp, vp, i32, vp, vp, i32, vp, size, vp],
            gns_log_probs_backward=[vp, R, vp, vp, vp, vp, vp, R, i32, vp]).items():
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = ctypes.c_int
    for name, args in dict(gns_sage_dense_int8_workspace_bytes=[vp, i32, i32],
                           gns_sage_dense_backward_workspace_bytes=[vp, i32, i32, i32, i32],
                           gns_log_probs_workspace_bytes=[vp, i32, i32, i32]).items():
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = size


_declare()


def int8_stride(k):
    """Bytes between rows in 8 bits of k columns."""
    return (k + 63) // 64 * 64


def checkpoint_groups(width):
    return (width + CHECKPOINT_GROUP - 1) // CHECKPOINT_GROUP


_TYPES = {torch.float32: GNS_FP32, torch.bfloat16: GNS_BF16}


def _rows(t, num_rows):
    """gns_rows of a 2-D tensor, or None of None."""
    if t is None:
        return None
    count, width = t.shape
    stride, step = t.stride()
    assert t.is_cuda and count >= num_rows and (step == 1 or width == 1)
    return gns_rows(t.data_ptr(), stride if count > 1 else max(width, stride), width, _TYPES[t.dtype])


def _flat(t, dtype, count):
    """Address of a contiguous tensor of at least `count` elements, or None of None."""
    if t is None:
        return None
    assert t.is_cuda and t.dtype is dtype and t.numel() >= count and t.is_contiguous()
    return t.data_ptr()


def _space(workspace):
    return (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())


def alloc_workspace(nbytes, device="cuda:0"):
    """A workspace of nbytes, or None if none is needed."""
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def gns_quantize_rows(ctx, x1, x2, q, scale, num_rows, stream=None):
    """q int8 [rows, int8_stride(k)], scale fp32 [rows]; x2 may be None."""
    k = x1.shape[1] + (0 if x2 is None else x2.shape[1])
    _check(lib.gns_quantize_rows(ctx, _rows(x1, num_rows), _rows(x2, num_rows), _flat(q, torch.int8, num_rows * int8_stride(k)),
                                 _flat(scale, torch.float32, num_rows), num_rows, _stream_ptr(stream)), ctx)


def gns_dense_int8(ctx, q, scale, k, wq, w_scale, bias, relu, out, num_rows, stream=None):
    """wq int8 [out.shape[1], int8_stride(k)], w_scale fp32 [out.shape[1]], bias fp32 or None."""
    n = out.shape[1]
    _check(lib.gns_dense_int8(ctx, _flat(q, torch.int8, num_rows * int8_stride(k)), _flat(scale, torch.float32, num_rows), k,
                              _flat(wq, torch.int8, n * int8_stride(k)), _flat(w_scale, torch.float32, n),
                              _flat(bias, torch.float32, n), 1 if relu else 0, _rows(out, num_rows), num_rows,
                              _stream_ptr(stream)), ctx)


def gns_sage_dense_int8_workspace_bytes(ctx, k, num_rows):
    return lib.gns_sage_dense_int8_workspace_bytes(ctx, k, num_rows)


def gns_sage_dense_int8(ctx, x1, x2, wq, w_scale, bias, relu, out, num_rows, workspace, stream=None):
    n, k = out.shape[1], x1.shape[1] + (0 if x2 is None else x2.shape[1])
    space, nbytes = _space(workspace)
    _check(lib.gns_sage_dense_int8(ctx, _rows(x1, num_rows), _rows(x2, num_rows), _flat(wq, torch.int8, n * int8_stride(k)),
                                   _flat(w_scale, torch.float32, n), _flat(bias, torch.float32, n), 1 if relu else 0,
                                   _rows(out, num_rows), num_rows, space, nbytes, _stream_ptr(stream)), ctx)


def gns_checkpoint_save(ctx, x, q, exponents, positive, num_rows, stream=None):
    """q int8 [rows, 32 * groups], exponents uint8 [rows, groups], positive int32 [rows, groups] or None."""
    cells = max(num_rows, 0) * checkpoint_groups(x.shape[1])
    _check(lib.gns_checkpoint_save(ctx, _rows(x, num_rows), _flat(q, torch.int8, cells * CHECKPOINT_GROUP),
                                   _flat(exponents, torch.uint8, cells), _flat(positive, torch.int32, cells), num_rows,
                                   _stream_ptr(stream)), ctx)


def gns_checkpoint_load(ctx, q, exponents, x, num_rows, stream=None):
    cells = max(num_rows, 0) * checkpoint_groups(x.shape[1])
    _check(lib.gns_checkpoint_load(ctx, _flat(q, torch.int8, cells * CHECKPOINT_GROUP), _flat(exponents, torch.uint8, cells),
                                   _rows(x, num_rows), num_rows, _stream_ptr(stream)), ctx)


def gns_sage_dense_backward_workspace_bytes(ctx, f1, f2, hdim, num_rows):
    return lib.gns_sage_dense_backward_workspace_bytes(ctx, f1, f2, hdim, num_rows)


def gns_sage_dense_backward(ctx, d_out, positive, one, f1, two, f2, w, dw, db, dx, num_rows, workspace, stream=None):
    """one, two: (q, exponents) of the checkpoints of the f1 and f2 input columns (two None with f2 = 0; both None with dw None);
    w, dw fp32 [f1 + f2, hdim]; db fp32 [hdim]; dx [rows, f1 + f2] of d_out's type.  positive, dw, db, dx may be None."""
    hdim, k, rows = d_out.shape[1], f1 + f2, max(num_rows, 0)
    space, nbytes = _space(workspace)

    def packed(p, f):
        if p is None:
            return None, None
        cells = rows * checkpoint_groups(f)
        return _flat(p[0], torch.int8, cells * CHECKPOINT_GROUP), _flat(p[1], torch.uint8, cells)

    q1, e1 = packed(one, f1)
    q2, e2 = packed(two, f2)
    _check(lib.gns_sage_dense_backward(ctx, _rows(d_out, num_rows), _flat(positive, torch.int32, rows * checkpoint_groups(hdim)),
                                       q1, e1, f1, q2, e2, f2, _flat(w, torch.float32, k * hdim),
                                       _flat(dw, torch.float32, k * hdim), _flat(db, torch.float32, hdim), _rows(dx, num_rows),
                                       num_rows, space, nbytes, _stream_ptr(stream)), ctx)


def gns_log_probs_workspace_bytes(ctx, num_classes, top, num_rows):
    return lib.gns_log_probs_workspace_bytes(ctx, num_classes, top, num_rows)


def gns_log_probs(ctx, logits, labels, logp, entropy, stats, top_index, top_logp, num_rows, workspace=None, stream=None):
    """labels int32 [rows], logp, entropy fp32 [rows], stats fp32 [rows, 2], top_index int32 and top_logp fp32 [rows, top];
    each may be None (labels with logp, top_index with top_logp)."""
    rows, top = max(num_rows, 0), 0 if top_index is None else top_index.shape[1]
    assert top_logp is None or top_logp.shape[1] == top
    space, nbytes = _space(workspace)
    _check(lib.gns_log_probs(ctx, _rows(logits, num_rows), _flat(labels, torch.int32, rows), _flat(logp, torch.float32, rows),
                             _flat(entropy, torch.float32, rows), _flat(stats, torch.float32, 2 * rows), top,
                             _flat(top_index, torch.int32, rows * top), _flat(top_logp, torch.float32, rows * top), num_rows,
                             space, nbytes, _stream_ptr(stream)), ctx)


def gns_log_probs_backward(ctx, logits, labels, stats, entropy, g_logp, g_entropy, d_logits, num_rows, stream=None):
    """g_logp (which needs labels) or g_entropy (which needs entropy) may be None; d_logits may be logits itself."""
    rows = max(num_rows, 0)
    _check(lib.gns_log_probs_backward(ctx, _rows(logits, num_rows), _flat(labels, torch.int32, rows),
                                      _flat(stats, torch.float32, 2 * rows), _flat(entropy, torch.float32, rows),
                                      _flat(g_logp, torch.float32, rows), _flat(g_entropy, torch.float32, rows),
                                      _rows(d_logits, num_rows), num_rows, _stream_ptr(stream)), ctx)

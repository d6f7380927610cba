"""The operators of include/gns_learn.h where a tolerance that grows with the size would hide a fault: sums that are exact in fp32,
infinities, sizes at which a kernel takes over from another, buffers made for more rows than a call has.

U = 2^-24 is one rounding to fp32.  Where every sum on the way is an fp32 value, results are compared to the bit.
"""
import math

import numpy as np
import pytest
import torch

from test_gpu_learn import BF16, FP32, TYPES, U, ctx, f64, gen, layout, save, within  # noqa: F401

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2106_06150_amd import binding as B
    from paper_2106_06150_amd import learn

# rows, f1, f2, hdim, whether the weights' gradient is wanted too: every way the input's gradient is made in (plain sums of few
# columns, few rows, tiles with the weights as they are, these with hdim split, both gradients in one launch, tiles with the
# weights cut beforehand, large tiles), with hdim a multiple of eight and not
WAYS = [(50, 33, 0, 5, False), (4, 64, 0, 40, False), (13, 70, 0, 41, False), (16, 2080, 0, 1030, True), (9000, 64, 0, 40, False),
        (9000, 64, 0, 41, False), (300, 64, 0, 2048, False), (300, 100, 0, 40, True), (300, 64, 0, 1031, True), (70001, 40, 0, 72, True),
        (70001, 33, 7, 73, True), (33000, 100, 0, 72, False), (33000, 100, 30, 73, False), (8193, 520, 0, 304, True), (8200, 520, 0, 301, True)]


def words_of(mask):
    """The `positive` words of a mask."""
    rows, hdim = mask.shape
    bits = torch.nn.functional.pad(mask.long(), (0, -hdim % 32)).view(rows, -1, 32)
    return (bits << torch.arange(32, device=mask.device)).sum(2).to(torch.uint32).view(torch.int32)


def backward(ctx, d_out, positive, one, f1, two, f2, w, dw, dx, space=None):
    """dw, db (None where dw is not wanted) and dx (or None)."""
    rows, hdim = d_out.shape
    out = torch.full((f1 + f2, hdim), 3.0, device="cuda") if dw else None
    db = torch.full((hdim,), 3.0, device="cuda") if dw else None
    grad = torch.full((rows, f1 + f2), 3.0, dtype=d_out.dtype, device="cuda") if dx else None
    if space is None:
        space = learn.alloc_workspace(learn.gns_sage_dense_backward_workspace_bytes(ctx, f1, f2, hdim, rows))
    learn.gns_sage_dense_backward(ctx, d_out, positive, one if dw else None, f1, two if dw else None, f2, w, out, db, grad, rows, space)
    return out, db, grad


def two_checkpoints(ctx, x, f1, f2):
    return save(ctx, x[:, :f1])[:2], save(ctx, x[:, f1:])[:2] if f2 else None


@TYPES
@pytest.mark.parametrize("rows,f1,f2,hdim,dw", WAYS)
def test_input_gradient_sees_every_bit_of_the_weights(ctx, rows, f1, f2, hdim, dw, dtype):
    """Weights in pairs that differ in their last eight bits alone, gradients of 1 and -1: the leading bits cancel, and what is left
    is a sum of small multiples of 2^-23 that fp32 holds.  Sixteen columns of a row count, so the partial sums, below four, cost
    at most a bit of 2^-22 each."""
    k = f1 + f2
    g = gen("bits", rows, k, hdim)
    pairs = hdim // 2
    base = 1.0 + torch.randint(0, 64, (k, pairs), generator=g).float() / 128 + torch.randint(128, 256, (k, pairs), generator=g).float() * 2.0 ** -15
    low = torch.randint(1, 256, (k, pairs), generator=g).float() * 2.0 ** -23
    w = torch.ones(k, hdim)
    w[:, 0:2 * pairs:2], w[:, 1:2 * pairs:2] = base + low, base
    first = torch.randint(0, max(1, pairs - 7), (rows, 1), generator=g)
    counts = (torch.arange(pairs)[None, :] >= first) & (torch.arange(pairs)[None, :] < first + 8)
    sign = torch.where(torch.rand(rows, pairs, generator=g) < 0.5, 1.0, -1.0) * counts
    d_out = torch.zeros(rows, hdim)
    d_out[:, 0:2 * pairs:2], d_out[:, 1:2 * pairs:2] = sign, -sign
    one, two = two_checkpoints(ctx, torch.zeros(rows, k), f1, f2) if dw else (None, None)
    dx = backward(ctx, d_out.to(dtype).cuda(), None, one, f1, two, f2, w.cuda(), dw, True)[2]
    want = (sign.cuda() @ low.cuda().t().contiguous()).double()          # small integers times 2^-23: exact
    bound = 16 * 2.0 ** -22 + (2.0 ** -8 * want.abs() if dtype == BF16 else 0.0)
    within(f64(dx), f64(want), bound if isinstance(bound, float) else f64(bound))

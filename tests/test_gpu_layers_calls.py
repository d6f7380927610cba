"""How the operators of include/gns_layers.h are called: refusals, calls of no rows, streams, captured graphs, rows counted on the device,
and every kernel at a size that reaches it."""
import math

import numpy as np
import pytest
import torch

from conftest import random_symmetric_csr

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2106_06150_amd import binding as B
    from paper_2106_06150_amd import layers, learn, synth
    from gpu_harness import GpuGns

from test_gpu_layers import (BF16, FP32, QUINTIC, TABLE, TYPES, U, check_norm, check_norm_grad, check_update, f64, fp8_values, gen, parameters, random_fp8,  # noqa: E402
                             stored, within)
from test_gpu_layers import ctx  # noqa: E402,F401  (the module's context)


# ---- refusals ---------------------------------------------------------------------------------------------------------
def test_refusals(ctx):  # noqa: F811
    lib = B.lib
    x = torch.randn(4, 64, device="cuda")
    y = torch.randn(4, 64, device="cuda")
    f = torch.zeros(64 * 64, device="cuda")
    b = torch.zeros(64 * 128, dtype=torch.uint8, device="cuda")
    e = torch.zeros(64 * 4, dtype=torch.uint8, device="cuda")
    offsets = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    space = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    s, p, p2 = torch.cuda.current_stream().cuda_stream, x.data_ptr(), y.data_ptr()
    fp, bp, ep, op, wp, size = f.data_ptr(), b.data_ptr(), e.data_ptr(), offsets.data_ptr(), space.data_ptr(), space.numel()
    einval, small = B.GNS_EINVAL, B.GNS_ECAPACITY

    def rows(data=p, stride=64, width=64, type=0):
        return learn.gns_rows(data, stride, width, type)

    def norm(segments=None, gamma=None, beta=None, count=0, per=1, groups=4, act=0, eps=1e-5):
        return layers.gns_norm(segments, gamma, beta, count, per, groups, act, eps)

    def how(mu=0.9, nesterov=1, eps=1e-7, keep=1.0, rate=1.0, steps=1, coefficient=1.0):
        h = layers.gns_orthogonal(mu, nesterov, eps, keep, rate, steps)
        h.coefficients[0][:] = (coefficient, -1.0, 0.5)
        return h

    def refused(status, name, *args):
        assert getattr(lib, name)(ctx, *args) == status, (name, args)
        assert lib.gns_last_error(ctx)

    bad_rows = [None, rows(data=None), rows(stride=63), rows(width=0), rows(width=-1), rows(type=2), rows(type=-1), rows(data=p + 2), rows(data=p + 1, type=1),
                rows(stride=learn.GNS_MAX_STRIDE, width=learn.GNS_MAX_WIDTH + 1), rows(stride=learn.GNS_MAX_STRIDE + 1), rows(stride=-64)]
    for r in bad_rows:
        refused(einval, "gns_group_norm", r, norm(), rows(p2), None, 4, wp, size, s)
        refused(einval, "gns_group_norm", rows(), norm(), r, None, 4, wp, size, s)
        refused(einval, "gns_group_norm_backward", r, rows(), norm(), fp, rows(p2), None, None, 4, wp, size, s)
        refused(einval, "gns_group_norm_backward", rows(), r, norm(), fp, rows(p2), None, None, 4, wp, size, s)
        refused(einval, "gns_orthogonal_update", r, None, how(), None, None, rows(p2), 4, wp, size, s)
        refused(einval, "gns_orthogonal_update", rows(), None, how(), None, None, r, 4, wp, size, s)
        refused(einval, "gns_quantize_fp8", r, None, bp, ep, 4, s)
        refused(einval, "gns_dense_fp8", bp, ep, 64, bp, ep, None, 0, r, 4, s)
        refused(einval, "gns_sage_dense_fp8", r, None, bp, ep, None, 0, rows(), 4, wp, size, s)
        refused(einval, "gns_sage_dense_fp8", rows(), None, bp, ep, None, 0, r, 4, wp, size, s)
        if r is not None:
            refused(einval, "gns_group_norm_backward", rows(), rows(), norm(), fp, r, None, None, 4, wp, size, s)
            refused(einval, "gns_orthogonal_update", rows(), r, how(), None, rows(p2), rows(fp), 4, wp, size, s)
            refused(einval, "gns_orthogonal_update", rows(), rows(p2), how(), None, r, rows(fp), 4, wp, size, s)
            refused(einval, "gns_orthogonal_update", rows(), None, how(), r, None, rows(p2), 4, wp, size, s)
            refused(einval, "gns_quantize_fp8", rows(), r, bp, ep, 4, s)
    bad_norms = [None, norm(groups=0), norm(groups=-1), norm(groups=5), norm(groups=128), norm(act=-1), norm(act=4), norm(eps=0.0), norm(eps=-1.0), norm(eps=math.inf),
                 norm(eps=math.nan), norm(per=0), norm(per=-3), norm(segments=op, count=-1), norm(segments=op, count=layers.GNS_MAX_SEGMENTS + 1), norm(segments=op + 2, count=1),
                 norm(gamma=fp + 1), norm(beta=fp + 2)]
    for n in bad_norms:
        refused(einval, "gns_group_norm", rows(), n, rows(p2), None, 4, wp, size, s)
        refused(einval, "gns_group_norm_backward", rows(), rows(), n, fp, rows(p2), None, None, 4, wp, size, s)
        assert lib.gns_group_norm_workspace_bytes(ctx, 64, n, 4) == 0
        assert lib.gns_group_norm_backward_workspace_bytes(ctx, 64, n, 4) == 0
    for n in (-2, -9):                                            # layers that the context does not have
        refused(einval, "gns_group_norm", rows(), norm(), rows(p2), None, n, wp, size, s)
        refused(einval, "gns_group_norm_backward", rows(), rows(), norm(), fp, rows(p2), None, None, n, wp, size, s)
        refused(einval, "gns_quantize_fp8", rows(), None, bp, ep, n, s)
        refused(einval, "gns_dense_fp8", bp, ep, 64, bp, ep, None, 0, rows(), n, s)
        refused(einval, "gns_sage_dense_fp8", rows(), None, bp, ep, None, 0, rows(), n, wp, size, s)
    # norm: shapes that do not agree, rows that overlap otherwise than as the same, workspaces
    tiled = norm(offsets.data_ptr(), count=1)
    refused(einval, "gns_group_norm", rows(), norm(), rows(p2, width=32), None, 4, wp, size, s)
    refused(einval, "gns_group_norm", rows(), norm(), rows(p2, type=1), None, 4, wp, size, s)
    refused(einval, "gns_group_norm", rows(width=32), norm(), rows(width=32, stride=32), None, 4, wp, size, s)
    refused(einval, "gns_group_norm", rows(), norm(), rows(p2), fp + 4, 4, wp, size, s)
    refused(einval, "gns_group_norm", rows(), tiled, rows(p2), None, 4, None, size, s)
    refused(einval, "gns_group_norm", rows(), tiled, rows(p2), None, 4, wp + 128, size, s)
    refused(small, "gns_group_norm", rows(), tiled, rows(p2), None, 4, wp, 64, s)
    refused(einval, "gns_group_norm_backward", rows(), rows(), norm(), None, rows(p2), None, None, 4, wp, size, s)
    refused(einval, "gns_group_norm_backward", rows(), rows(), norm(), fp + 4, rows(p2), None, None, 4, wp, size, s)
    refused(einval, "gns_group_norm_backward", rows(), rows(), norm(), fp, None, None, None, 4, wp, size, s)
    refused(einval, "gns_group_norm_backward", rows(), rows(), norm(), fp, None, fp + 2, None, 4, wp, size, s)
    refused(einval, "gns_group_norm_backward", rows(), rows(), norm(), fp, None, None, fp + 1, 4, wp, size, s)
    refused(einval, "gns_group_norm_backward", rows(type=1), rows(), norm(), fp, rows(p2), None, None, 4, wp, size, s)
    refused(einval, "gns_group_norm_backward", rows(width=32), rows(), norm(), fp, rows(p2), None, None, 4, wp, size, s)
    refused(einval, "gns_group_norm_backward", rows(), rows(p2), norm(), fp, rows(p2, stride=128), None, None, 4, wp, size, s)
    refused(einval, "gns_group_norm_backward", rows(), rows(p2), norm(), fp, rows(stride=128), None, None, 4, wp, size, s)
    refused(einval, "gns_group_norm_backward", rows(), rows(), tiled, fp, rows(p2), None, None, 4, None, size, s)
    refused(small, "gns_group_norm_backward", rows(), rows(), tiled, fp, rows(p2), None, None, 4, wp, 64, s)
    # orthogonal update
    for h in (None, how(steps=-1), how(steps=layers.GNS_MAX_STEPS + 1), how(mu=math.nan), how(eps=-1.0), how(eps=math.inf), how(keep=math.inf), how(rate=math.nan), how(coefficient=math.inf)):
        refused(einval, "gns_orthogonal_update", rows(), None, h, None, None, rows(p2), 4, wp, size, s)
    for n in (-1, layers.GNS_ORTHOGONAL_MAX + 1):
        refused(einval, "gns_orthogonal_update", rows(), None, how(), None, None, rows(p2), n, wp, size, s)
        assert layers.gns_orthogonal_update_workspace_bytes(ctx, 64, n) == 0
        assert layers.gns_orthogonal_update_workspace_bytes(ctx, n, 64) == 0
    wide = layers.GNS_ORTHOGONAL_MAX + 1
    refused(einval, "gns_orthogonal_update", rows(width=wide, stride=wide), None, how(), None, None, rows(p2, width=wide, stride=wide), 1, wp, size, s)
    refused(einval, "gns_orthogonal_update", rows(), rows(p2), how(), None, None, rows(fp), 4, wp, size, s)          # momentum without its output
    refused(einval, "gns_orthogonal_update", rows(), None, how(), None, rows(p2), rows(fp), 4, wp, size, s)
    refused(einval, "gns_orthogonal_update", rows(), None, how(), None, None, rows(p2, width=32), 4, wp, size, s)
    refused(einval, "gns_orthogonal_update", rows(), None, how(), rows(fp, width=32), None, rows(p2), 4, wp, size, s)
    refused(einval, "gns_orthogonal_update", rows(), rows(p2), how(), None, rows(p2, stride=128), rows(fp), 4, wp, size, s)
    refused(einval, "gns_orthogonal_update", rows(), rows(p2), how(), None, rows(p2), rows(p2), 4, wp, size, s)
    refused(einval, "gns_orthogonal_update", rows(), rows(p2), how(), None, rows(), rows(fp), 4, wp, size, s)        # the momentum over the gradient
    refused(einval, "gns_orthogonal_update", rows(), rows(p2), how(), rows(fp), rows(fp), rows(fp + 8192), 4, wp, size, s)
    refused(einval, "gns_orthogonal_update", rows(), None, how(), rows(fp), None, rows(fp, stride=128), 4, wp, size, s)
    refused(einval, "gns_orthogonal_update", rows(), None, how(), None, None, rows(type=1), 4, wp, size, s)
    refused(einval, "gns_orthogonal_update", rows(), None, how(), None, None, rows(p2), 4, None, size, s)
    refused(einval, "gns_orthogonal_update", rows(), None, how(), None, None, rows(p2), 4, wp + 64, size, s)
    refused(small, "gns_orthogonal_update", rows(), None, how(), None, None, rows(p2), 4, wp, 1024, s)
    # 8-bit floats
    refused(einval, "gns_quantize_fp8", rows(), rows(type=1), bp, ep, 4, s)
    refused(einval, "gns_quantize_fp8", rows(width=layers.GNS_FP8_MAX_K, stride=1 << 21), rows(), bp, ep, 4, s)
    for q_, e_ in ((None, ep), (bp, None), (bp + 8, ep), (bp, ep + 2)):
        refused(einval, "gns_quantize_fp8", rows(), None, q_, e_, 4, s)
        refused(einval, "gns_dense_fp8", q_, e_, 64, bp, ep, None, 0, rows(), 4, s)
        refused(einval, "gns_dense_fp8", bp, ep, 64, q_, e_, None, 0, rows(), 4, s)
        refused(einval, "gns_sage_dense_fp8", rows(), None, q_, e_, None, 0, rows(p2), 4, wp, size, s)
    for k in (0, -1, layers.GNS_FP8_MAX_K + 1):
        refused(einval, "gns_dense_fp8", bp, ep, k, bp, ep, None, 0, rows(), 4, s)
        assert layers.gns_sage_dense_fp8_workspace_bytes(ctx, k, 4) == 0
    refused(einval, "gns_dense_fp8", bp, ep, 64, bp, ep, fp + 1, 0, rows(), 4, s)
    refused(einval, "gns_sage_dense_fp8", rows(), None, bp, ep, None, 0, rows(p2), 4, None, size, s)
    refused(einval, "gns_sage_dense_fp8", rows(), None, bp, ep, None, 0, rows(p2), 4, wp + 16, size, s)
    refused(small, "gns_sage_dense_fp8", rows(), None, bp, ep, None, 0, rows(p2), 4, wp, 256, s)
    torch.cuda.synchronize()


def test_calls_of_no_rows(ctx):  # noqa: F811
    """No row is read or written; sums over no rows are zero, and so are the statistics of segments without rows."""
    empty = torch.empty(0, 12, device="cuda")
    norm = layers.Norm(3, segments=torch.tensor([0, 0, 0], dtype=torch.int32, device="cuda"))
    stats = torch.full((2, 3, 2), 5.0, device="cuda")
    layers.gns_group_norm(ctx, empty, norm, empty, stats, 0)
    assert not stats.any()
    dgamma, dbeta = torch.full((12,), 5.0, device="cuda"), torch.full((12,), 5.0, device="cuda")
    layers.gns_group_norm_backward(ctx, empty, empty, norm, stats, empty, dgamma, dbeta, 0)
    assert not dgamma.any() and not dbeta.any()
    single = layers.Norm(3)
    layers.gns_group_norm(ctx, empty, single, empty, None, 0)
    dgamma.fill_(5.0)
    layers.gns_group_norm_backward(ctx, empty, empty, single, torch.empty(0, 3, 2, device="cuda"), None, dgamma, None, 0)
    assert not dgamma.any()
    layers.gns_orthogonal_update(ctx, empty, None, layers.Orthogonal([QUINTIC]), None, None, empty, 0, None)
    q, e = torch.empty(0, 128, dtype=torch.uint8, device="cuda"), torch.empty(0, 4, dtype=torch.uint8, device="cuda")
    layers.gns_quantize_fp8(ctx, empty, None, q, e, 0)
    wq, we = torch.zeros(5, 128, dtype=torch.uint8, device="cuda"), torch.zeros(5, 4, dtype=torch.uint8, device="cuda")
    out = torch.empty(0, 5, device="cuda")
    layers.gns_dense_fp8(ctx, q, e, 12, wq, we, None, False, out, 0)
    layers.gns_sage_dense_fp8(ctx, empty, None, wq, we, None, False, out, 0, None)
    torch.cuda.synchronize()


def test_offsets_out_of_order_stay_inside_the_rows(ctx):  # noqa: F811
    """Offsets that do not ascend, or lie outside: unspecified values in the outputs' rows, nothing behind or before them."""
    rows, width, groups = 100, 24, 3
    for offsets in ([0, 50, 20, 100], [-5, 10, 400], [100, 0], [70, 70, 3, 2, 1], [-9, -3], [500, 600]):
        seg = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        norm = layers.Norm(groups, segments=seg, activation=layers.GNS_ACT_SILU)
        n = len(offsets) - 1
        wide = torch.full((rows + 20, width), 7.0, device="cuda")
        x = torch.randn(rows, width, device="cuda")
        stats = torch.full((n + 2, groups, 2), 5.0, device="cuda")
        layers.gns_group_norm(ctx, x, norm, wide[10:10 + rows], stats[1:1 + n].contiguous(), rows, layers.alloc_workspace(layers.gns_group_norm_workspace_bytes(ctx, width, norm, rows)))
        layers.gns_group_norm_backward(ctx, x, x, norm, torch.ones(n, groups, 2, device="cuda"), wide[10:10 + rows], torch.empty(width, device="cuda"), None, rows,
                                       layers.alloc_workspace(layers.gns_group_norm_backward_workspace_bytes(ctx, width, norm, rows)))
        torch.cuda.synchronize()
        assert bool((wide[:10] == 7).all()) and bool((wide[10 + rows:] == 7).all())


# ---- streams, graphs, counts on the device -----------------------------------------------------------------------------
class Everything:
    """All calls on one set of inputs, with outputs and workspaces of their own."""

    def __init__(self, ctx, seed=0):  # noqa: F811
        g = gen("everything", seed)
        self.ctx, self.rows = ctx, 300
        new = lambda *shape: torch.randn(*shape, generator=g).cuda()
        self.x, self.d, self.gamma, self.beta = new(300, 96), new(300, 96), new(96), new(96)
        self.w, self.grad, self.momentum = new(96, 160), new(96, 160), new(96, 160)
        self.norms = [layers.Norm(8, activation=layers.GNS_ACT_SILU, gamma=self.gamma, beta=self.beta),
                      layers.Norm(8, segments=torch.tensor([0, 100, 100, 290], dtype=torch.int32, device="cuda"), activation=layers.GNS_ACT_GELU, gamma=self.gamma, beta=self.beta)]
        self.how = layers.Orthogonal([QUINTIC] * 3, mu=0.9, nesterov=True, keep=0.99, rate=-0.1)
        self.q, self.e = torch.empty(160, 128, dtype=torch.uint8, device="cuda"), torch.empty(160, 4, dtype=torch.uint8, device="cuda")
        layers.gns_quantize_fp8(ctx, self.w.t().contiguous(), None, self.q, self.e, 160)
        zero = lambda *shape: torch.zeros(*shape, device="cuda")
        self.outs = [zero(300, 96), zero(300, 8, 2), zero(300, 96), zero(96), zero(96), zero(300, 96), zero(3, 8, 2), zero(300, 96), zero(96), zero(96),
                     zero(96, 160), zero(96, 160), zero(300, 160)]
        space = layers.alloc_workspace
        self.spaces = [space(layers.gns_group_norm_backward_workspace_bytes(ctx, 96, self.norms[0], 300)), space(layers.gns_group_norm_workspace_bytes(ctx, 96, self.norms[1], 300)),
                       space(layers.gns_group_norm_backward_workspace_bytes(ctx, 96, self.norms[1], 300)), space(layers.gns_orthogonal_update_workspace_bytes(ctx, 160, 96)),
                       space(layers.gns_sage_dense_fp8_workspace_bytes(ctx, 96, 300))]
        torch.cuda.synchronize()

    def run(self, stream=None):
        c, o, n = self.ctx, self.outs, self.rows
        layers.gns_group_norm(c, self.x, self.norms[0], o[0], o[1], n, None, stream)
        layers.gns_group_norm_backward(c, self.d, self.x, self.norms[0], o[1], o[2], o[3], o[4], n, self.spaces[0], stream)
        layers.gns_group_norm(c, self.x, self.norms[1], o[5], o[6], n, self.spaces[1], stream)
        layers.gns_group_norm_backward(c, self.d, self.x, self.norms[1], o[6], o[7], o[8], o[9], n, self.spaces[2], stream)
        layers.gns_orthogonal_update(c, self.grad, self.momentum, self.how, self.w, o[10], o[11], 96, self.spaces[3], stream)
        layers.gns_sage_dense_fp8(c, self.x, None, self.q, self.e, None, True, o[12], n, self.spaces[4], stream)


def test_captured_calls_replay_with_the_same_results(ctx):  # noqa: F811
    work = Everything(ctx)
    work.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work.run()
    for turn in range(4):
        work.x.mul_(1.25).add_(0.1 * turn)
        work.grad.add_(0.5)
        work.run()
        torch.cuda.synchronize()
        eager = [t.clone() for t in work.outs]
        for t in work.outs:
            t.zero_()
        for t in work.spaces:
            t.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, work.outs)), turn


def test_calls_on_two_streams_at_once(ctx):  # noqa: F811
    """Each with its own buffers, all on one context."""
    works = [Everything(ctx, seed) for seed in range(2)]
    want = []
    for w in works:
        w.run()
        torch.cuda.synchronize()
        want.append([t.clone() for t in w.outs])
        for t in w.outs:
            t.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in works]
    for _ in range(5):
        for w, s in zip(works, streams):
            w.run(s)
    torch.cuda.synchronize()
    for w, outs in zip(works, want):
        assert all(torch.equal(a, b) for a, b in zip(outs, w.outs))


def test_stage_timer_counts_the_calls(ctx):  # noqa: F811
    work = Everything(ctx)
    B.gns_profile_begin(ctx, 1 << layers.GNS_STAGE_NORM | 1 << layers.GNS_STAGE_ORTHOGONAL | 1 << layers.GNS_STAGE_FP8, 16)
    work.run()
    assert [B.gns_profile_collect(ctx, s)[1] for s in (layers.GNS_STAGE_NORM, layers.GNS_STAGE_ORTHOGONAL, layers.GNS_STAGE_FP8)] == [4, 1, 1]
    B.gns_profile_begin(ctx, 0, 0)


@TYPES
def test_rows_counted_on_the_device(dtype):
    """num_rows as a layer's placeholder: results of as many rows as the layer has, nothing behind them."""
    indptr, indices = random_symmetric_csr(3000, 10, np.random.default_rng(5))
    gns = GpuGns(torch.from_numpy(indptr), torch.from_numpy(indices), None, fanouts=(6, 4), policies=(0, 0), cache_size=0, max_seeds=100)
    try:
        c, layer = gns.ctx, 1
        B.gns_sample_blocks(c, 3, synth.uniform_seed_batch(3000, 60, 9).cuda(), gns.blocks.array)
        count, cap = gns.blocks.array[layer].num_dst, gns.blocks.array[layer].cap_dst
        assert 60 < count < cap
        g = gen("device")
        x, d = (torch.randn(cap, 96, generator=g).to(dtype).cuda() for _ in range(2))
        w = torch.randn(72, 96, generator=g).cuda()
        gamma, beta = (t.cuda() for t in parameters(96, g))
        wq, we = torch.empty(72, 128, dtype=torch.uint8, device="cuda"), torch.empty(72, 4, dtype=torch.uint8, device="cuda")
        layers.gns_quantize_fp8(c, w, None, wq, we, 72)
        ragged = torch.tensor([0, 10, 10, 50, cap], dtype=torch.int32, device="cuda")          # the last one ends where the rows do

        def everything(rows):
            new = lambda *shape, t=FP32: torch.full(shape, 42, dtype=t, device="cuda")
            by_row, sums = [], []
            for norm, segments in ((layers.Norm(8, activation=2, gamma=gamma, beta=beta), cap), (layers.Norm(8, segment_rows=7, activation=3, gamma=gamma, beta=beta), (cap + 6) // 7),
                                   (layers.Norm(8, segments=ragged, activation=0, gamma=gamma, beta=beta), 4)):
                out, stats, dx, dgamma, dbeta = new(cap, 96, t=dtype), new(segments, 8, 2), new(cap, 96, t=dtype), new(96), new(96)
                layers.gns_group_norm(c, x, norm, out, stats, rows, layers.alloc_workspace(layers.gns_group_norm_workspace_bytes(c, 96, norm, rows)))
                layers.gns_group_norm_backward(c, d, x, norm, stats, dx, dgamma, dbeta, rows,
                                               layers.alloc_workspace(layers.gns_group_norm_backward_workspace_bytes(c, 96, norm, rows)))
                by_row += [out, dx]
                sums += [stats, dgamma, dbeta]
            q, e, out, both = new(cap, 128, t=torch.uint8), new(cap, 4, t=torch.uint8), new(cap, 72, t=dtype), new(cap, 72, t=dtype)
            layers.gns_quantize_fp8(c, x, None, q, e, rows)
            layers.gns_dense_fp8(c, q, e, 96, wq, we, None, True, out, rows)
            layers.gns_sage_dense_fp8(c, x, None, wq, we, None, True, both, rows, layers.alloc_workspace(layers.gns_sage_dense_fp8_workspace_bytes(c, 96, rows)))
            torch.cuda.synchronize()
            return by_row + [q, e, out, both], sums

        got, got_sums = everything(-1 - layer)
        want, want_sums = everything(count)
        tol = 2.0 ** -7 if dtype == BF16 else 1e-5
        for i, (a, b) in enumerate(zip(got, want)):
            assert bool((a[count:] == 42).all()), i
            if a.dtype == torch.uint8:
                assert torch.equal(a[:count], b[:count]), i
            else:
                within(f64(a[:count]), f64(b[:count]), tol * (np.abs(f64(b[:count])) + float(b[:count].abs().float().mean())))
        for a, b in zip(got_sums, want_sums):
            within(f64(a), f64(b), 1e-5 * (np.abs(f64(b)) + float(b.abs().mean())))
    finally:
        gns.close()


def test_a_workspace_serves_every_smaller_call(ctx):  # noqa: F811
    """Bytes needed do not grow when rows go: a buffer for the most rows is enough for each remainder."""
    rng = np.random.default_rng(3)
    for _ in range(40):
        width, groups = int(rng.integers(1, 40)) * 8, int(2 ** rng.integers(0, 4))
        most = int(rng.integers(2, 300000))
        norms = [layers.Norm(groups), layers.Norm(groups, segment_rows=int(rng.integers(2, 5000))),
                 layers.Norm(groups, segments=torch.zeros(int(rng.integers(2, 50)), dtype=torch.int32, device="cuda"))]
        for call in (layers.gns_group_norm_workspace_bytes, layers.gns_group_norm_backward_workspace_bytes):
            for norm in norms:
                top = call(ctx, width, norm, most)
                assert all(call(ctx, width, norm, int(r)) <= top for r in rng.integers(1, most, 30))
        rows = int(rng.integers(2, 9000))
        top = layers.gns_orthogonal_update_workspace_bytes(ctx, width, rows)
        assert all(layers.gns_orthogonal_update_workspace_bytes(ctx, width, int(r)) <= top for r in rng.integers(1, rows, 30))


# ---- every kernel ----------------------------------------------------------------------------------------------------------
@TYPES
@pytest.mark.parametrize("rows,width,groups,segments", [(3300, 128, 64, [0, 3300]), (3300, 512, 64, [0, 3300]), (900, 64, 4, list(range(0, 901, 3))), (900, 36, 4, list(range(0, 901, 3))),
                                                        (6000, 2600, 2, [0, 6000])])
def test_norm_whose_parts_are_joined_in_a_launch_of_their_own(ctx, rows, width, groups, segments, dtype):  # noqa: F811
    g = gen(rows, width)
    x = (torch.randn(rows, width, generator=g) * 2 + torch.randn(1, width, generator=g)).to(dtype)
    gamma, beta = parameters(width, g)
    check_norm(ctx, x, groups, 2, segments=segments, gamma=gamma, beta=beta)
    check_norm_grad(ctx, x, torch.randn(rows, width, generator=g).to(dtype), groups, 2, segments=segments, gamma=gamma, beta=beta)


def exact_rows(rows, k, g):
    """Rows in 8-bit floats of values -2 .. 2 with scales 1, 2, 4: (q, exponents, values)."""
    small = torch.tensor(np.nonzero(np.isin(TABLE, (-2, -1, 0, 1, 2)))[0], dtype=torch.uint8)
    q = small[torch.randint(0, len(small), (rows, layers.fp8_stride(k)), generator=g)]
    q[:, k:] = 0
    e = torch.zeros(rows, layers.fp8_exponents(k), dtype=torch.uint8)
    blocks = (k + 127) // 128
    e[:, :blocks] = 127 + torch.randint(0, 3, (rows, blocks), generator=g, dtype=torch.uint8)
    return q, e, fp8_values(q, e, k)


@TYPES
@pytest.mark.parametrize("rows,k,n", [(2600, 1100, 4000), (4200, 640, 1000), (700, 1153, 300), (50, 5000, 33), (2, 9000, 70), (5200, 1300, 2100)])
def test_fp8_tiles_of_every_size_are_exact(ctx, rows, k, n, dtype):  # noqa: F811
    """Sums of whole numbers below 2^24 (5000 products of up to 64), whose products lie within 2^13 of each other."""
    g = gen("tiles", rows, k, n)
    q, e, x = exact_rows(rows, k, g)
    wq, we, w = exact_rows(n, k, g)
    out = torch.empty(rows, n, dtype=dtype, device="cuda")
    layers.gns_dense_fp8(ctx, q.cuda(), e.cuda(), k, wq.cuda(), we.cuda(), None, False, out, rows)
    want = torch.from_numpy(x).cuda() @ torch.from_numpy(w).cuda().t().contiguous()
    assert torch.equal(out, want.to(dtype))


@TYPES
@pytest.mark.parametrize("rows,f1,f2,n", [(8200, 256, 0, 500), (8193, 64, 64, 1000), (8195, 256, 0, 301), (8333, 128, 0, 33), (8192, 512, 0, 300), (8450, 24, 8, 64), (8500, 8, 0, 5)])
def test_fp8_rows_in_registers_are_exact(ctx, rows, f1, f2, n, dtype):  # noqa: F811
    """Rows of whole numbers up to 8, which 8-bit floats hold: what is quantised on the way is exact, whatever the block's scale."""
    g = gen("rows", rows, f1, f2, n)
    k = f1 + f2
    x = torch.randint(-8, 9, (rows, k), generator=g).to(dtype)
    wq, we, w = exact_rows(n, k, g)
    bias = torch.randint(-3, 4, (n,), generator=g).float()
    for pad in (0, 3):
        out = torch.full((rows, n + pad), 9.0, dtype=dtype, device="cuda")[:, :n]
        space = layers.alloc_workspace(layers.gns_sage_dense_fp8_workspace_bytes(ctx, k, rows))
        layers.gns_sage_dense_fp8(ctx, x[:, :f1].contiguous().cuda(), x[:, f1:].contiguous().cuda() if f2 else None, wq.cuda(), we.cuda(), bias.cuda(), False, out, rows, space)
        want = x.double().cuda() @ torch.from_numpy(w).cuda().t().contiguous() + bias.double().cuda()
        assert torch.equal(out, want.to(dtype))


@pytest.mark.parametrize("rows,width,steps", [(900, 900, 2), (1000, 2500, 2), (2500, 1000, 2), (1500, 1500, 1), (4100, 4096, 2), (4096, 4160, 2), (5632, 5632, 1), (2304, 9000, 1), (600, 32000, 1),
                                              (3000, 70, 2), (70, 3000, 2), (1024, 1024, 2), (64, 512, 2), (512, 64, 2), (64, 513, 2), (513, 64, 2),
                                              (65, 512, 2), (1, 512, 3), (64, 256, 2), (257, 20, 3), (64, 5000, 2), (20000, 33, 1), (1, 4097, 2), (47, 300, 5), (33, 31, 5), (2, 1, 1)])
def test_orthogonal_updates_of_every_size(ctx, rows, width, steps):  # noqa: F811
    """One block for all, blocks of 128, 256 and 512 columns, tiles of 32, 64, 128 and 256, whole and in parts, wide and tall, against 64 bits on the GPU.  In the 2-norm: 22 bits of each factor and
    sums' roundings, which are as good as random, and every step lets the errors before it grow by its slope, at most 5 below norm 1."""
    g = torch.Generator(device="cuda").manual_seed(rows * 7 + width)
    grad = torch.randn(rows, width, device="cuda", generator=g)
    w = torch.randn(rows, width, device="cuda", generator=g)
    out = torch.empty_like(w)
    space = layers.alloc_workspace(layers.gns_orthogonal_update_workspace_bytes(ctx, width, rows))
    space.fill_(255)
    layers.gns_orthogonal_update(ctx, grad, None, layers.Orthogonal([QUINTIC] * steps, keep=0.5, rate=2.0), w, None, out, rows, space)
    x = grad.double()
    x = x / (x.norm() + 1e-7)
    if rows > width:
        x = x.t().contiguous()
    a, b, c = (float(np.float32(v)) for v in QUINTIC)
    for _ in range(steps):
        gram = x @ x.t().contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    if rows > width:
        x = x.t()
    want = 0.5 * w.double() + 2.0 * x
    off = float((out.double() - want).norm())
    bound = 2.0 * steps * 5.0 ** steps * (8 * 2.0 ** -22 + math.sqrt(max(rows, width)) * U) * 1.0 + 4 * U * float(want.norm())
    assert off <= bound, (off, bound)
    # element by element: an element in a wrong place is off by as much as elements are large, an error by a few times the mean one
    assert float((out.double() - want).abs().max()) <= 64 * (bound / math.sqrt(rows * width) + U * float(want.abs().max()))


@pytest.mark.parametrize("rows,width", [(40, 60), (512, 33), (64, 512), (130, 150)])
def test_orthogonal_updates_of_nothing_of_any_size_and_of_what_is_not_finite(ctx, rows, width):  # noqa: F811
    """In one block and in many."""
    conf = layers.Orthogonal([QUINTIC] * 3, keep=0.5, rate=1.0, eps=0.0)
    space = layers.alloc_workspace(layers.gns_orthogonal_update_workspace_bytes(ctx, width, rows))
    w = torch.randn(rows, width, generator=gen("w", rows)).cuda()
    out = torch.empty_like(w)
    layers.gns_orthogonal_update(ctx, torch.zeros(rows, width, device="cuda"), None, conf, w, None, out, rows, space)
    assert torch.equal(out, 0.5 * w)
    for bad in (math.inf, math.nan):
        grad = torch.randn(rows, width, generator=gen("g", rows)).cuda()
        grad[13, 7] = bad
        layers.gns_orthogonal_update(ctx, grad, None, conf, w, None, out, rows, space)
        assert out.isnan().all()
    for scale in (1e-30, 1e30):
        check_update(ctx, rows, width, (FP32, FP32, FP32), [QUINTIC] * 3, momentum=False, scale=scale, eps=0.0)
    # over the gradient, and the same bits from a graph that is replayed
    grad = torch.randn(rows, width, generator=gen("in place", rows)).cuda()
    alone = torch.empty_like(grad)
    layers.gns_orthogonal_update(ctx, grad, None, conf, None, None, alone, rows, space)
    moved, m = grad.clone(), torch.zeros_like(grad)
    layers.gns_orthogonal_update(ctx, moved, None, conf, None, None, moved, rows, space)
    assert torch.equal(moved, alone)
    first = torch.empty_like(grad)
    layers.gns_orthogonal_update(ctx, grad, m, conf, w, m, first, rows, space)
    again, kept = torch.empty_like(grad), torch.zeros_like(grad)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        layers.gns_orthogonal_update(ctx, grad, kept, conf, w, kept, again, rows, space)
    for _ in range(3):
        kept.zero_()
        again.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(again, first) and torch.equal(kept, m)


@TYPES
@pytest.mark.parametrize("rows,width,groups,per", [(999, 11, 11, 18), (998, 2048, 2048, 2), (1, 2048, 2048, 7), (1, 2049, 3, 7), (71, 2049, 3, 2), (5, 37, 1, 1000), (8193, 1, 1, 4096),
                                                   (8193, 1, 1, 4097), (300, 64, 8, 64), (300, 65, 5, 63), (300, 65, 5, 64), (203, 512, 32, 20), (503, 1024, 32, 5), (2000, 3, 3, 2), (777, 100, 4, 40)])
def test_norm_of_short_segments(ctx, rows, width, groups, per, dtype):  # noqa: F811
    """Several segments to a block, a segment that just fits one and that just does not, tiles that are segments, the last one shorter."""
    g = gen(rows, width, per)
    x = (torch.randn(rows, width, generator=g) * 2 + torch.randn(1, width, generator=g)).to(dtype)
    d_out = torch.randn(rows, width, generator=g).to(dtype)
    gamma, beta = parameters(width, g)
    for act in (1, 3):
        check_norm(ctx, x, groups, act, segment_rows=per, gamma=gamma, beta=beta, inplace=act == 3)
        check_norm_grad(ctx, x, d_out, groups, act, segment_rows=per, gamma=gamma, beta=beta)


@TYPES
@pytest.mark.parametrize("rows,width,how", [(53, 19, dict()), (53, 64, dict()), (53, 19, dict(segments=True)), (53, 64, dict(segments=True)), (40, 2600, dict(segments=True)), (1, 19, dict(segment_rows=7)),
                                            (1, 2600, dict(segment_rows=7))])
def test_the_gradient_of_a_group_of_one_value_is_zero(ctx, rows, width, how, dtype):  # noqa: F811
    """x is its mean whatever it is; what rounding leaves would be multiplied by 1 / sqrt(eps)."""
    g = gen(rows, width, len(how))
    x, d_out = torch.randn(rows, width, generator=g).to(dtype).cuda(), torch.randn(rows, width, generator=g).to(dtype).cuda()
    gamma, beta = (t.cuda() for t in parameters(width, g))
    if "segments" in how:
        how = dict(segments=torch.arange(rows + 1, dtype=torch.int32, device="cuda"))
    for act in range(4):
        norm = layers.Norm(width, activation=act, gamma=gamma, beta=beta, **how)
        sizes = [layers.gns_group_norm_workspace_bytes(ctx, width, norm, rows), layers.gns_group_norm_backward_workspace_bytes(ctx, width, norm, rows)]
        space = layers.alloc_workspace(max(sizes))
        stats, out, dx = torch.empty(rows, width, 2, device="cuda"), torch.empty_like(x), torch.full_like(x, 7.0)
        layers.gns_group_norm(ctx, x, norm, out, stats, rows, space)
        layers.gns_group_norm_backward(ctx, d_out, x, norm, stats, dx, None, None, rows, space)
        assert torch.equal(stats[..., 0], x.float()) and bool((dx == 0).all())

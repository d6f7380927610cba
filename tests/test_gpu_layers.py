"""The operators of include/gns_layers.h on the GPU against plain implementations in 64 bits, through the C ABI.

Error bounds follow from the arithmetic: u = 2^-24 is one rounding to fp32.  A sum of n values in fp32, in any order, is off by
at most n roundings of the sum of magnitudes.  A result stored in bf16 is off by 2^-8 of itself besides.
"""
import math
import zlib

import numpy as np
import pytest
import torch

from conftest import random_symmetric_csr

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2106_06150_amd import binding as B
    from paper_2106_06150_amd import layers, learn, synth
    from gpu_harness import GpuGns

U = 2.0 ** -24
FP32, BF16 = torch.float32, torch.bfloat16
TYPES = pytest.mark.parametrize("dtype", [FP32, BF16], ids=["fp32", "bf16"])
LAYOUTS = ("packed", "strided", "odd")
EPS = 1e-5


@pytest.fixture(scope="module")
def ctx():
    dev = torch.device("cuda:0")
    graph = B.make_graph(torch.tensor([0, 1, 2], dtype=torch.int32, device=dev), torch.tensor([1, 0], dtype=torch.int32, device=dev))
    config = B.make_config([1], [B.GNS_UNIFORM], 0, 1)
    workspace = B.alloc_workspace(graph, config, dev)
    c = B.gns_create(graph, config, workspace)
    yield c
    torch.cuda.synchronize()
    B.gns_destroy(c)


def layout(t, how):
    """The 2-D tensor on the GPU with its rows adjacent, further apart, or off the 16-byte marks."""
    t = t.cuda()
    if how == "packed":
        return t.contiguous()
    rows, width = t.shape
    pad, first = (16, 0) if how == "strided" else (3, 1)
    wide = torch.full((rows, width + pad + first), float("nan"), dtype=t.dtype, device="cuda")
    view = wide[:, first:first + width]
    view.copy_(t)
    return view


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def f64(t):
    return t.detach().cpu().double().numpy()


def within(got, want, bound):
    got, want, bound = (np.asarray(v, dtype=np.float64) for v in (got, want, bound))
    bound = np.broadcast_to(bound, want.shape)
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True)
    off = np.abs(got[~odd] - want[~odd])
    assert np.all(off <= bound[~odd]), (float(np.max(off / np.maximum(bound[~odd], 1e-300))), int(np.argmax(off / np.maximum(bound[~odd], 1e-300))))


def stored(dtype, value):
    """What rounding a value to its type may take away."""
    return (2.0 ** -8 if dtype == BF16 else 2.0 ** -24) * np.abs(value) * 1.01 + 2.0 ** -126


# ---- group norm -----------------------------------------------------------------------------------------------------
ACTS = {0: "none", 1: "relu", 2: "silu", 3: "gelu"}


def normal_cdf(y):
    return np.asarray(torch.special.erfc(torch.from_numpy(np.asarray(-y / math.sqrt(2.0))))) / 2.0


def ref_act(y, act):
    """Value and slope in 64 bits."""
    if act == 0:
        return y, np.ones_like(y)
    if act == 1:
        return np.where(y < 0, 0.0, y), np.where(np.isnan(y), y, (y > 0).astype(float))
    if act == 2:
        s = 1.0 / (1.0 + np.exp(-np.clip(y, -700, None)))
        return y * s, s * (1.0 + y * (1.0 - s))
    cdf = normal_cdf(y)
    return y * cdf, cdf + y * np.exp(-y * y / 2.0) / math.sqrt(2.0 * math.pi)


def ranges_of(rows, segments, segment_rows):
    if segments is not None:
        return list(zip(segments[:-1], segments[1:]))
    return [(a, min(a + segment_rows, rows)) for a in range(0, rows, segment_rows)]


def ref_norm(x, ranges, groups, gamma, beta, eps):
    """h, y, mean, rstd, count per value and stats, in 64 bits; rows of no segment are NaN."""
    rows, width = x.shape
    w = width // groups
    h, mean_of, rstd_of, n_of = (np.full((rows, width), np.nan) for _ in range(4))
    stats = np.zeros((len(ranges), groups, 2))
    for s, (a, b) in enumerate(ranges):
        if b <= a:
            continue
        v = x[a:b].reshape(b - a, groups, w)
        mean = v.mean((0, 2))
        with np.errstate(invalid="ignore", over="ignore"):
            var = ((v - mean[None, :, None]) ** 2).mean((0, 2))
            rstd = 1.0 / np.sqrt(var + eps)
            h[a:b] = ((v - mean[None, :, None]) * rstd[None, :, None]).reshape(b - a, width)
        stats[s, :, 0], stats[s, :, 1] = mean, rstd
        mean_of[a:b], rstd_of[a:b] = np.repeat(mean, w)[None], np.repeat(rstd, w)[None]
        n_of[a:b] = (b - a) * w
    return h, h * gamma + beta, mean_of, rstd_of, n_of, stats


def check_norm(ctx, x, groups, act, segments=None, segment_rows=1, how="packed", gamma=None, beta=None, inplace=False, eps=EPS):
    """x on the CPU.  Returns the statistics on the GPU."""
    rows, width = x.shape
    seg = None if segments is None else torch.tensor(segments, dtype=torch.int32, device="cuda")
    norm = layers.Norm(groups, segments=seg, segment_rows=segment_rows, activation=act, eps=eps,
                       gamma=None if gamma is None else gamma.cuda(), beta=None if beta is None else beta.cuda())
    ranges = ranges_of(rows, segments, segment_rows)
    xd = layout(x, how)
    out = xd if inplace else layout(torch.full((rows, width), 7.0, dtype=x.dtype), how)
    stats = torch.full((len(ranges), groups, 2), 5.0, device="cuda")
    nbytes = layers.gns_group_norm_workspace_bytes(ctx, width, norm, rows)
    layers.gns_group_norm(ctx, xd, norm, out, stats, rows, layers.alloc_workspace(nbytes))
    g64 = np.ones(width) if gamma is None else f64(gamma)
    b64 = np.zeros(width) if beta is None else f64(beta)
    h, y, mean, rstd, n, want_stats = ref_norm(f64(x), ranges, groups, g64, b64, eps)
    # mean: a tree of sums (registers, lanes, tiles), 64 roundings of the mean magnitude at most; the variance is a sum of squares of
    # distances (each off by the mean's error and a rounding), rstd half of its relative error
    w = width // groups
    size, spread = np.zeros_like(want_stats[..., 0]), np.zeros_like(want_stats[..., 0])
    for s, (a, b) in enumerate(ranges):
        if b > a:
            size[s] = np.abs(f64(x)[a:b]).reshape(b - a, groups, w).mean((0, 2))
            spread[s] = f64(x)[a:b].reshape(b - a, groups, w).std((0, 2))
    mean_bound = 64 * U * size + 2.0 ** -126
    within(f64(stats)[..., 0], want_stats[..., 0], mean_bound)
    rel = 64 * U + 2 * mean_bound * spread * want_stats[..., 1] ** 2 + mean_bound ** 2 * want_stats[..., 1] ** 2
    within(f64(stats)[..., 1], want_stats[..., 1], rel * want_stats[..., 1])
    # y: the distance is off by the mean's error and a rounding, the scale by rstd's, and the sum rounds
    covered = ~np.isnan(n) if segments is not None else np.ones(x.shape, dtype=bool)
    bound = np.zeros(x.shape)
    for s, (a, b) in enumerate(ranges):
        if b > a:
            bound[a:b] = np.repeat(mean_bound[s] * want_stats[s, :, 1], w)[None] * np.abs(g64) + np.abs(h[a:b] * g64) * np.repeat(rel[s] + 4 * U, w)[None]
    bound = bound + 4 * U * np.abs(b64)
    value, slope = ref_act(y, act)
    # slopes are at most 1.13; the activation itself costs a dozen roundings of the value, and of y where it is nearly 0
    bound = 1.13 * bound + 16 * U * np.abs(value) + (0 if act < 2 else 2.0 ** -126)
    got = f64(out)
    keep = f64(x) if inplace else np.full(x.shape, 7.0)
    assert np.array_equal(got[~covered], keep[~covered], equal_nan=True)
    within(got[covered], value[covered], (bound + stored(x.dtype, value))[covered])
    # without statistics, and once more to the bit
    if not inplace:
        again = layout(torch.full((rows, width), 7.0, dtype=x.dtype), how)
        layers.gns_group_norm(ctx, xd, norm, again, None, rows, layers.alloc_workspace(nbytes))
        assert torch.equal(again, out)
    return stats


def parameters(width, g):
    return 1.0 + 0.3 * torch.randn(width, generator=g), 0.3 * torch.randn(width, generator=g)


UNIT_SHAPES = [(1, 1, 1), (3, 5, 5), (7, 6, 3), (2, 16, 1), (9, 24, 3), (5, 33, 1), (1, 4096, 32), (70, 100, 4), (31, 128, 1), (33, 256, 8),
               (17, 250, 1), (5, 512, 2), (3, 1000, 1), (130, 64, 16), (4, 2050, 2), (2, 2049, 1), (3, 4100, 1), (2, 8192, 1), (1, 9000, 1), (2, 16384, 1),
               (1, 20001, 1), (600, 8, 8), (257, 37 * 4, 37), (5, 3 * 700, 3), (4000, 32, 2)]


@TYPES
@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("rows,width,groups", UNIT_SHAPES)
def test_norm_of_single_rows(ctx, rows, width, groups, how, dtype):
    g = gen(rows, width, groups)
    x = (torch.randn(rows, width, generator=g) * torch.exp(torch.randn(1, width, generator=g)) + torch.randn(1, width, generator=g)).to(dtype)
    gamma, beta = parameters(width, g)
    for act in (rows % 4, (rows + 1) % 4):
        check_norm(ctx, x, groups, act, how=how, gamma=gamma, beta=beta if rows % 3 else None)


SEGMENTED = [(1, 1, 1, [0, 1]), (10, 7, 1, [0, 0, 3, 3, 10]), (64, 32, 4, [0, 1, 2, 40, 64]), (100, 100, 4, [5, 17, 17, 90]), (300, 33, 11, [0, 300]),
             (257, 64, 64, [0, 100, 257]), (50, 2500, 5, [0, 20, 50]), (40, 3000, 1, [3, 40]), (1000, 16, 2, [0, 16, 32, 500, 1000]), (2000, 8, 1, [0] + list(range(3, 2000, 7))),
             (5000, 24, 3, [0, 4999, 5000]), (33, 5, 5, [0, 33]), (20, 12, 2, [7, 7]), (20, 12, 2, [0])]


@TYPES
@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("rows,width,groups,segments", SEGMENTED)
def test_norm_of_ragged_segments(ctx, rows, width, groups, segments, how, dtype):
    g = gen(rows, width, groups)
    x = (torch.randn(rows, width, generator=g) * torch.exp(torch.randn(1, width, generator=g)) + torch.randn(1, width, generator=g)).to(dtype)
    gamma, beta = parameters(width, g)
    check_norm(ctx, x, groups, rows % 4, segments=segments, how=how, gamma=gamma, beta=beta)
    check_norm(ctx, x, groups, (rows + 1) % 4, segments=segments, how=how, inplace=True)


EQUAL = [(1, 5, 5, 9), (10, 16, 2, 3), (100, 64, 8, 2), (128, 100, 4, 32), (77, 300, 3, 10), (3000, 8, 1, 1000), (4096, 32, 4, 256), (513, 48, 48, 100), (64, 2100, 2, 7),
         (9000, 16, 16, 4500), (300, 40, 5, 16), (2, 9000, 1, 2)]


@TYPES
@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("rows,width,groups,segment_rows", EQUAL)
def test_norm_of_equal_segments(ctx, rows, width, groups, segment_rows, how, dtype):
    g = gen(rows, width, groups, segment_rows)
    x = (torch.randn(rows, width, generator=g) * 2 + torch.randn(1, width, generator=g)).to(dtype)
    gamma, beta = parameters(width, g)
    check_norm(ctx, x, groups, (rows + groups) % 4, segment_rows=segment_rows, how=how, gamma=gamma, beta=beta)


@pytest.mark.parametrize("rows,width,groups,segment_rows", [(64, 256, 4, 1), (5000, 64, 2, 2500), (300, 100, 1, 300), (40, 3000, 1, 40), (8, 9000, 1, 1)])
def test_norm_far_from_zero(ctx, rows, width, groups, segment_rows):
    """Means a thousand times the spread: the variance comes from distances, not from squares of the values."""
    x = 1000.0 + torch.randn(rows, width, generator=gen(rows, width))
    check_norm(ctx, x, groups, 0, segment_rows=segment_rows)


@pytest.mark.parametrize("segment_rows", [1, 50])
def test_norm_of_constants_and_of_what_is_not_finite(ctx, segment_rows):
    rows, width, groups = 200, 48, 3
    x = torch.randn(rows, width, generator=gen("odd"))
    x[0:50, :16] = 3.0                                    # no spread: out is beta
    x[50, 20], x[100, 0], x[150, 47], x[199, 16] = math.inf, math.nan, -math.inf, 3e38
    norm = layers.Norm(groups, segment_rows=segment_rows, activation=layers.GNS_ACT_RELU)
    out, stats = torch.empty(rows, width, device="cuda"), torch.empty((rows + segment_rows - 1) // segment_rows, groups, 2, device="cuda")
    layers.gns_group_norm(ctx, x.cuda(), norm, out, stats, rows, layers.alloc_workspace(layers.gns_group_norm_workspace_bytes(ctx, width, norm, rows)))
    out, stats = out.cpu(), stats.cpu()
    assert torch.equal(out[0:50 if segment_rows == 50 else 1, :16], torch.zeros(50 if segment_rows == 50 else 1, 16))
    spoilt = torch.zeros(rows, width, dtype=torch.bool)
    for r, c in ((50, 20), (100, 0), (150, 47), (199, 16)):
        s = r // segment_rows
        spoilt[s * segment_rows:(s + 1) * segment_rows, c // 16 * 16:c // 16 * 16 + 16] = True
        assert stats[s, c // 16].isnan().all()
    assert out[spoilt].isnan().all() and out[~spoilt].isfinite().all()


def ref_norm_grad(d_out, x, ranges, groups, gamma, beta, act, stats):
    """dx, dgamma, dbeta in 64 bits from the statistics, and the magnitudes that go into each."""
    rows, width = x.shape
    w = width // groups
    dx, size = np.full((rows, width), np.nan), np.zeros((rows, width))
    dgamma, dbeta, sg, sb = (np.zeros(width) for _ in range(4))
    for s, (a, b) in enumerate(ranges):
        if b <= a:
            continue
        mean, rstd = np.repeat(stats[s, :, 0], w)[None], np.repeat(stats[s, :, 1], w)[None]
        h = (x[a:b] - mean) * rstd
        slope = ref_act(h * gamma + beta, act)[1]
        dy = d_out[a:b] * slope
        dbeta += dy.sum(0)
        dgamma += (dy * h).sum(0)
        # h is off by two roundings of the distance's terms
        h_size = (np.abs(x[a:b]) + np.abs(mean)) * rstd
        reach = np.abs(d_out[a:b]) * (1.13 + (0 if act < 2 else 1.0) * h_size * np.abs(gamma))
        sb += reach.sum(0)
        sg += (reach * (h_size + 1)).sum(0)
        g = dy * gamma
        m1 = g.reshape(b - a, groups, w).mean((0, 2))
        m2 = (g * h).reshape(b - a, groups, w).mean((0, 2))
        dx[a:b] = rstd * (g - np.repeat(m1, w)[None] - h * np.repeat(m2, w)[None])
        g_size = reach * np.abs(gamma)
        m1_size = np.repeat(g_size.reshape(b - a, groups, w).mean((0, 2)), w)[None]
        m2_size = np.repeat((g_size * (h_size + 1)).reshape(b - a, groups, w).mean((0, 2)), w)[None]
        size[a:b] = rstd * (g_size + m1_size + (h_size + 1) * m2_size)
    return dx, dgamma, dbeta, size, sg, sb


def check_norm_grad(ctx, x, d_out, groups, act, segments=None, segment_rows=1, how="packed", gamma=None, beta=None, inplace=None):
    rows, width = x.shape
    seg = None if segments is None else torch.tensor(segments, dtype=torch.int32, device="cuda")
    norm = layers.Norm(groups, segments=seg, segment_rows=segment_rows, activation=act, eps=EPS,
                       gamma=None if gamma is None else gamma.cuda(), beta=None if beta is None else beta.cuda())
    ranges = ranges_of(rows, segments, segment_rows)
    g64 = np.ones(width) if gamma is None else f64(gamma)
    b64 = np.zeros(width) if beta is None else f64(beta)
    stats = torch.tensor(ref_norm(f64(x), ranges, groups, g64, b64, EPS)[5], dtype=FP32)
    stats64 = f64(stats)
    # a ReLU's slope jumps at zero: values whose y is within its own error of it are moved away
    if act == 1:
        x = x.clone()
        for s, (a, b) in enumerate(ranges):
            w = width // groups
            h = (f64(x)[a:b] - np.repeat(stats64[s, :, 0], w)) * np.repeat(stats64[s, :, 1], w)
            near = np.abs(h * g64 + b64) < 1e-4 * (1 + np.abs(f64(x)[a:b]) * np.repeat(stats64[s, :, 1], w))
            d_out = d_out.clone()
            d_out[a:b][torch.from_numpy(near)] = 0.0
    want, want_gamma, want_beta, size, sg, sb = ref_norm_grad(f64(d_out), f64(x), ranges, groups, g64, b64, act, stats64)
    xd, dd = layout(x, how), layout(d_out, how)
    dx = {None: layout(torch.full((rows, width), 7.0, dtype=x.dtype), how), "x": xd, "d_out": dd}[inplace]
    dgamma, dbeta = torch.full((width,), 3.0, device="cuda"), torch.full((width,), 3.0, device="cuda")
    nbytes = layers.gns_group_norm_backward_workspace_bytes(ctx, width, norm, rows)
    keep = f64(dx)
    layers.gns_group_norm_backward(ctx, dd, xd, norm, stats.cuda(), dx, dgamma, dbeta, rows, layers.alloc_workspace(nbytes))
    covered = ~np.isnan(want)
    assert np.array_equal(f64(dx)[~covered], keep[~covered], equal_nan=True)
    # 24 roundings of each value's parts, and a sum's: registers, lanes, tiles, 96 more
    within(f64(dx)[covered], want[covered], (128 * U * size + stored(x.dtype, np.nan_to_num(want)))[covered])
    within(f64(dgamma), want_gamma, 128 * U * sg + 2.0 ** -126)
    within(f64(dbeta), want_beta, 128 * U * sb + 2.0 ** -126)
    if inplace is None:                                   # each output alone, the same to the bit
        other = [torch.full_like(t, 9.0) for t in (dgamma, dbeta)]
        layers.gns_group_norm_backward(ctx, dd, xd, norm, stats.cuda(), None, other[0], None, rows, layers.alloc_workspace(nbytes))
        layers.gns_group_norm_backward(ctx, dd, xd, norm, stats.cuda(), None, None, other[1], rows, layers.alloc_workspace(nbytes))
        assert torch.equal(other[0], dgamma) and torch.equal(other[1], dbeta)
        alone = layout(torch.full((rows, width), 7.0, dtype=x.dtype), how)
        layers.gns_group_norm_backward(ctx, dd, xd, norm, stats.cuda(), alone, None, None, rows, layers.alloc_workspace(nbytes))
        assert torch.equal(alone, dx)


@TYPES
@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("rows,width,groups", UNIT_SHAPES)
def test_norm_gradient_of_single_rows(ctx, rows, width, groups, how, dtype):
    g = gen(rows, width, groups, "grad")
    x = (torch.randn(rows, width, generator=g) * torch.exp(torch.randn(1, width, generator=g))).to(dtype)
    d_out = torch.randn(rows, width, generator=g).to(dtype)
    gamma, beta = parameters(width, g)
    check_norm_grad(ctx, x, d_out, groups, rows % 4, how=how, gamma=gamma, beta=beta)
    check_norm_grad(ctx, x, d_out, groups, (rows + 1) % 4, how=how, gamma=gamma, inplace="x" if rows % 2 else "d_out")


@TYPES
@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("rows,width,groups,segments", SEGMENTED)
def test_norm_gradient_of_ragged_segments(ctx, rows, width, groups, segments, how, dtype):
    g = gen(rows, width, groups, "grad")
    x = (torch.randn(rows, width, generator=g) * torch.exp(torch.randn(1, width, generator=g))).to(dtype)
    d_out = torch.randn(rows, width, generator=g).to(dtype)
    gamma, beta = parameters(width, g)
    check_norm_grad(ctx, x, d_out, groups, rows % 4, segments=segments, how=how, gamma=gamma, beta=beta)
    check_norm_grad(ctx, x, d_out, groups, (rows + 1) % 4, segments=segments, how=how, inplace="x" if rows % 2 else "d_out")


@TYPES
@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("rows,width,groups,segment_rows", EQUAL)
def test_norm_gradient_of_equal_segments(ctx, rows, width, groups, segment_rows, how, dtype):
    g = gen(rows, width, groups, segment_rows, "grad")
    x = (torch.randn(rows, width, generator=g) * 2).to(dtype)
    d_out = torch.randn(rows, width, generator=g).to(dtype)
    gamma, beta = parameters(width, g)
    check_norm_grad(ctx, x, d_out, groups, (rows + groups) % 4, segment_rows=segment_rows, how=how, gamma=gamma, beta=beta)


@pytest.mark.parametrize("act", [0, 2, 3])
@pytest.mark.parametrize("segment_rows", [1, 5])
def test_norm_gradient_against_differences(ctx, act, segment_rows):
    """The gradient of sum(out * d) against central differences of the kernel's own forward pass."""
    rows, width, groups = 10, 24, 2
    g = gen("differences", act)
    x, d = torch.randn(rows, width, generator=g), torch.randn(rows, width, generator=g)
    gamma, beta = parameters(width, g)
    seg = (rows + segment_rows - 1) // segment_rows

    def forward(x, gamma, beta):
        norm = layers.Norm(groups, segment_rows=segment_rows, activation=act, gamma=gamma.cuda(), beta=beta.cuda())
        out, stats = torch.empty(rows, width, device="cuda"), torch.empty(seg, groups, 2, device="cuda")
        layers.gns_group_norm(ctx, x.cuda(), norm, out, stats, rows, layers.alloc_workspace(layers.gns_group_norm_workspace_bytes(ctx, width, norm, rows)))
        return float((f64(out) * f64(d)).sum()), norm, stats

    _, norm, stats = forward(x, gamma, beta)
    dx, dgamma, dbeta = torch.empty(rows, width, device="cuda"), torch.empty(width, device="cuda"), torch.empty(width, device="cuda")
    layers.gns_group_norm_backward(ctx, d.cuda(), x.cuda(), norm, stats, dx, dgamma, dbeta, rows,
                                   layers.alloc_workspace(layers.gns_group_norm_backward_workspace_bytes(ctx, width, norm, rows)))
    # steps of 2^-6: the third derivative's term is of 2^-12, the sums' roundings, 240 values of 2^-22 each, over 2^-5 of 2^-9
    step = 2.0 ** -6
    for name, t, grad in (("x", x, dx), ("gamma", gamma, dgamma), ("beta", beta, dbeta)):
        for i in range(0, t.numel(), 7):
            ends = []
            for sign in (1, -1):
                moved = t.clone()
                moved.view(-1)[i] += sign * step
                args = {"x": x, "gamma": gamma, "beta": beta}
                args[name] = moved
                ends.append(forward(**args)[0])
            want = (ends[0] - ends[1]) / (2 * step)
            assert abs(float(grad.view(-1)[i]) - want) < 0.02 * (1 + abs(want)), (name, i)


# ---- orthogonalised updates -------------------------------------------------------------------------------------------
QUINTIC = (3.4445, -4.7750, 2.0315)
EXACT = (1.875, -1.25, 0.375)


def ref_orthogonal(u, coefficients, eps):
    """X in 64 bits, and how far an error of 1 in X's elements can grow."""
    norm = np.sqrt((u.astype(np.float64) ** 2).sum())
    x = u / (norm + eps) if norm else np.zeros_like(u)
    turned = x.shape[0] > x.shape[1]
    if turned:
        x = x.T
    growth = 1.0
    for a, b, c in coefficients:
        a, b, c = (float(np.float32(v)) for v in (a, b, c))
        gram = x @ x.T
        top = float(np.linalg.norm(gram, 2))
        x = a * x + (b * gram + c * gram @ gram) @ x
        growth *= max(1.0, abs(a) + 3 * abs(b) * top + 5 * abs(c) * top * top)
    return (x.T if turned else x), growth


def check_update(ctx, rows, width, types, coefficients, how="packed", weights=True, momentum=True, nesterov=True, inplace=False, scale=1e-3, eps=1e-7):
    g = gen(rows, width, len(coefficients))
    grad_t, mom_t, w_t = types
    rank = max(1, min(rows, width) // 4)
    low = torch.randn(rows, rank, generator=g) @ torch.randn(rank, width, generator=g) / math.sqrt(rank)
    grad = (scale * (low + torch.randn(rows, width, generator=g))).to(grad_t)
    mom = (scale * 4 * torch.randn(rows, width, generator=g)).to(mom_t) if momentum else None
    w = (torch.randn(rows, width, generator=g) / math.sqrt(rows)).to(w_t) if weights else None
    mu, keep, rate = 0.9, 0.99, -0.05
    conf = layers.Orthogonal(coefficients, mu=mu, nesterov=nesterov, eps=eps, keep=keep, rate=rate)
    mu, keep, rate = (float(np.float32(v)) for v in (mu, keep, rate))
    gd, md, wd = layout(grad, how), layout(mom, how) if momentum else None, layout(w, how) if weights else None
    out = (wd if weights else gd) if inplace else layout(torch.full((rows, width), 7.0, dtype=w_t), how)
    mo = None if not momentum else md if inplace else layout(torch.full((rows, width), 7.0, dtype=mom_t), how)
    space = layers.alloc_workspace(layers.gns_orthogonal_update_workspace_bytes(ctx, width, rows))
    space.fill_(255)
    layers.gns_orthogonal_update(ctx, gd, md, conf, wd, mo, out, rows, space)
    m64 = mu * f64(mom) + f64(grad) if momentum else f64(grad)
    if momentum:
        within(f64(mo), m64, 3 * U * (np.abs(mu * f64(mom)) + np.abs(f64(grad))) + stored(mom_t, m64))
    u64 = f64(grad) + mu * m64 if nesterov else m64
    x, growth = ref_orthogonal(u64, coefficients, float(np.float32(eps)))
    # In the 2-norm: X is off by a few roundings of 22 bits at first and at each step, and by the sums' roundings, which are
    # as good as random: (sqrt(k) of them) of rows' and columns' norms; every step lets the errors before it grow.
    steps = max(len(coefficients), 1)
    first = np.linalg.norm(u64) and 1.0
    bound = steps * growth * (8 * 2.0 ** -22 + math.sqrt(max(rows, width)) * U) * first
    want = keep * f64(w) + rate * x if weights else rate * x
    off = np.linalg.norm(f64(out) - want)
    room = abs(rate) * bound + np.linalg.norm(stored(out.dtype, want)) + 4 * U * np.linalg.norm(want)
    assert off <= room, (off, room)
    return x


MATRICES = [(1, 1), (1, 40), (40, 1), (5, 7), (7, 5), (32, 32), (64, 200), (127, 129), (129, 127), (128, 128), (200, 64), (256, 256), (130, 700), (700, 130), (300, 1000), (515, 515)]


@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("rows,width", MATRICES)
def test_orthogonal_update(ctx, rows, width, how):
    check_update(ctx, rows, width, (FP32, FP32, FP32), [QUINTIC] * 5, how)
    check_update(ctx, rows, width, (BF16, BF16, BF16), [QUINTIC] * 5, how, nesterov=False)
    check_update(ctx, rows, width, (BF16, FP32, FP32), [QUINTIC, EXACT], how, weights=False)
    check_update(ctx, rows, width, (FP32, BF16, FP32), [EXACT], how, momentum=False)
    check_update(ctx, rows, width, (FP32, FP32, FP32), [QUINTIC] * 2, how, inplace=True)
    check_update(ctx, rows, width, (FP32, FP32, BF16), [], how)


def test_orthogonal_update_makes_singular_values_one(ctx):
    rows, width = 192, 320
    g = gen("singular")
    grad = torch.randn(rows, width, generator=g)
    conf = layers.Orthogonal([QUINTIC] * 4 + [EXACT] * 8)
    out = torch.empty(rows, width, device="cuda")
    space = layers.alloc_workspace(layers.gns_orthogonal_update_workspace_bytes(ctx, width, rows))
    layers.gns_orthogonal_update(ctx, grad.cuda(), None, conf, None, None, out, rows, space)
    # each Gram entry is a sum of products of the last step's roundings: 320 products of 22-bit values
    within(f64(out) @ f64(out).T, np.eye(rows), 1e-5)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e30])
def test_orthogonal_update_of_gradients_of_any_size(ctx, scale):
    check_update(ctx, 96, 160, (FP32, FP32, FP32), [QUINTIC] * 3, momentum=False, scale=scale, eps=0.0)


def test_orthogonal_update_of_nothing_and_of_what_is_not_finite(ctx):
    conf = layers.Orthogonal([QUINTIC] * 3, keep=0.5, rate=1.0, eps=0.0)
    space = layers.alloc_workspace(layers.gns_orthogonal_update_workspace_bytes(ctx, 50, 60))
    w = torch.randn(60, 50, generator=gen("w")).cuda()
    out = torch.empty_like(w)
    layers.gns_orthogonal_update(ctx, torch.zeros(60, 50, device="cuda"), None, conf, w, None, out, 60, space)
    assert torch.equal(out, 0.5 * w)
    for bad in (math.inf, math.nan):
        grad = torch.randn(60, 50, generator=gen("g")).cuda()
        grad[13, 7] = bad
        layers.gns_orthogonal_update(ctx, grad, None, conf, w, None, out, 60, space)
        assert out.isnan().all()


def test_orthogonal_update_repeats_to_the_bit(ctx):
    grad = torch.randn(700, 500, generator=gen("repeat")).cuda()
    conf = layers.Orthogonal([QUINTIC] * 5)
    space = layers.alloc_workspace(layers.gns_orthogonal_update_workspace_bytes(ctx, 500, 700))
    outs = [torch.empty_like(grad) for _ in range(3)]
    for o in outs:
        layers.gns_orthogonal_update(ctx, grad, None, conf, None, None, o, 700, space)
        space.fill_(255)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


# ---- 8-bit floats -------------------------------------------------------------------------------------------------------
def e4m3_table():
    codes = np.arange(256)
    e, m = (codes >> 3) & 15, codes & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * np.exp2(e.astype(float) - 7))
    v = np.where((codes & 127) == 127, np.nan, v)
    return np.where(codes >= 128, -v, v)


TABLE = e4m3_table()


def ref_fp8(x):
    """Values (64 bits) of rows in 8-bit floats, q's values and exponent bytes, from the definition."""
    x = x.double().numpy()
    rows, k = x.shape
    blocks = (k + 127) // 128
    padded = np.zeros((rows, blocks * 128))
    padded[:, :k] = x
    g = padded.reshape(rows, blocks, 128)
    with np.errstate(invalid="ignore"):
        a = np.abs(g).max(2)
        bad, none = ~np.isfinite(a), a < 2.0 ** -100
        safe = np.where(bad | none, 1.0, a)
        e = np.floor(np.log2(safe)).astype(int) - 11
        for _ in range(6):
            e = e + (safe > 464.0 * np.exp2(e))
        v = np.where((bad | none)[:, :, None], 0.0, g) / np.exp2(e)[:, :, None]
        place = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
        step = np.exp2(np.maximum(place, -6) - 3)
        q = np.clip(np.rint(v / step) * step, -448, 448)
    inside = (np.arange(blocks * 128) < k).reshape(1, blocks, 128)
    q = np.where(bad[:, :, None] & inside, np.nan, q)
    byte = np.zeros((rows, (k + 511) // 512 * 4), dtype=np.uint8)
    byte[:, :blocks] = np.where(bad, 255, np.where(none, 0, e + 127))
    values = q * np.where(none, 1.0, np.exp2(e))[:, :, None]
    return values.reshape(rows, -1)[:, :k], q.reshape(rows, -1), byte


def odd_rows(x):
    """Rows with blocks of zeros, of tiny values, of the least that counts, of the largest, not finite, and on the borders of rounding."""
    rows, k = x.shape
    special = (0.0, 2.0 ** -101, 2.0 ** -100, float(torch.finfo(x.dtype).max), math.inf, math.nan, 464.0, 466.0, 232.0, 1.0)
    for i, v in enumerate(special):
        if rows > i + 1:
            c = 128 * (i % ((k + 127) // 128))
            if i < 3:
                x[i + 1, c:c + 128] = v
            elif i < 6:
                x[i + 1, c] = v
            else:
                x[i + 1, c:c + 128] = torch.linspace(-1, 1, 128)[:x[i + 1, c:c + 128].numel()].to(x.dtype) * v
                x[i + 1, c] = v
    return x


@TYPES
@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("rows,f1,f2", [(1, 1, 0), (3, 5, 0), (9, 127, 1), (12, 128, 128), (33, 65, 64), (130, 100, 28), (7, 4096, 0), (6, 1000, 3001), (300, 128, 128), (2, 20000, 0)])
def test_quantize_fp8(ctx, rows, f1, f2, how, dtype):
    k = f1 + f2
    g = gen(rows, f1, f2)
    x = odd_rows((torch.randn(rows, k, generator=g) * torch.exp2(torch.randint(-12, 12, (rows, k), generator=g).float())).to(dtype))
    q = torch.full((rows, layers.fp8_stride(k)), 77, dtype=torch.uint8, device="cuda")
    e = torch.full((rows, layers.fp8_exponents(k)), 99, dtype=torch.uint8, device="cuda")
    layers.gns_quantize_fp8(ctx, layout(x[:, :f1], how), layout(x[:, f1:], how) if f2 else None, q, e, rows)
    _, want_q, want_e = ref_fp8(x)
    assert np.array_equal(e.cpu().numpy(), want_e)
    assert np.array_equal(TABLE[q.cpu().numpy()], want_q, equal_nan=True)


def random_fp8(rows, k, g, spread=3):
    """Rows in 8-bit floats of any finite values: (q, exponents) on the CPU and their values in 64 bits."""
    q = torch.randint(0, 256, (rows, layers.fp8_stride(k)), generator=g, dtype=torch.uint8)
    q[(q & 127) == 127] -= 1
    q[:, k:] = 0
    e = torch.zeros(rows, layers.fp8_exponents(k), dtype=torch.uint8)
    blocks = (k + 127) // 128
    e[:, :blocks] = torch.randint(120 - spread, 121 + spread, (rows, blocks), generator=g, dtype=torch.uint8)
    return q, e, fp8_values(q, e, k)


def fp8_values(q, e, k):
    blocks = (k + 127) // 128
    scale = np.where(e.cpu().numpy()[:, :blocks] == 255, np.nan, np.exp2(e.cpu().numpy()[:, :blocks].astype(float) - 127))
    return (TABLE[q.cpu().numpy()] * np.repeat(scale, 128, 1))[:, :k]


def check_dense(out, x, w, bias, relu):
    with np.errstate(invalid="ignore", over="ignore"):
        b = np.zeros(w.shape[0]) if bias is None else f64(bias)
        y = x @ w.T + b
        size = np.abs(x) @ np.abs(w.T) + np.abs(b)
        if relu:
            y = np.where(y < 0, 0.0, y)
        # products are exact; matrix cores may cut where they add, two roundings a step of 16 products, and splits are joined
        rows, k = x.shape
        bound = (2 * (k // 16 + 1) + 16) * U * size
        if out.dtype == BF16:
            # each product of 128 columns may lose 2^-13 of their largest
            blocks = (k + 127) // 128
            most = [np.abs(np.pad(v, ((0, 0), (0, blocks * 128 - k))).reshape(-1, blocks, 128)).max(2) for v in (x, w)]
            bound = bound + 128 * 2.0 ** -13 * (most[0] @ most[1].T)
        bound = bound + stored(out.dtype, np.nan_to_num(y, posinf=0, neginf=0)) + 2.0 ** -120
        # What is larger than the type's largest value is an infinity, but for values within the error of that border: 2^128 (1 - d), d below
        # 2^-24, is above the largest fp32 value, 2^128 (1 - 2^-24), and two roundings away is that value itself.
        got, most = f64(out), float(torch.finfo(out.dtype).max)
        border = (np.abs(np.abs(y) - most) <= bound) & (got * y > 0) & (np.abs(got) >= most - 2 * bound)
        y = np.where(border, got, np.where(np.abs(y) > most, np.sign(y) * np.inf, y))
    within(got, y, bound)


@TYPES
@pytest.mark.parametrize("rows,k,n", [(1, 1, 1), (1, 128, 7), (1, 4096, 515), (2, 1000, 33), (5, 257, 64), (16, 512, 129), (17, 96, 96), (64, 2048, 40), (65, 65, 65),
                                      (130, 300, 47), (257, 128, 256), (1000, 256, 172), (300, 1024, 1027), (520, 1100, 600)])
def test_fp8_product(ctx, rows, k, n, dtype):
    g = gen(rows, k, n)
    q, e, x = random_fp8(rows, k, g)
    wq, we, w = random_fp8(n, k, g)
    wq[:, k:] = 3                                         # padding of the weights of any finite content
    bias = torch.randn(n, generator=g) if n % 2 else None
    relu = rows % 2 == 0
    for how in LAYOUTS:
        out = layout(torch.full((rows, n), 9.0, dtype=dtype), how)
        layers.gns_dense_fp8(ctx, q.cuda(), e.cuda(), k, wq.cuda(), we.cuda(), None if bias is None else bias.cuda(), relu, out, rows)
        check_dense(out, x, w, bias, relu)


@TYPES
@pytest.mark.parametrize("rows,k,n", [(1, 700, 40), (40, 700, 40), (300, 1500, 200), (9000, 256, 40), (9000, 400, 40)])
def test_fp8_products_of_whole_numbers_are_exact(ctx, rows, k, n, dtype):
    """Values whose sums fp32 holds (up to 1500 products of up to 4 times 16) and whose products lie within 2^13 of each other: any wrong
    place of a value or an exponent shows."""
    g = gen("whole", rows, k, n)
    q, e, _ = random_fp8(rows, k, g, 0)
    wq, we, _ = random_fp8(n, k, g, 0)
    small = torch.tensor(np.nonzero(np.isin(TABLE, (-2, -1, 0, 1, 2)))[0], dtype=torch.uint8)
    q, wq = small[q.long() % len(small)], small[wq.long() % len(small)]
    q[:, k:] = 0
    blocks = (k + 127) // 128
    e[:, :blocks] = 127 + torch.randint(0, 3, (rows, blocks), generator=g, dtype=torch.uint8)
    we[:, :blocks] = 127 + torch.randint(0, 3, (n, blocks), generator=g, dtype=torch.uint8)
    out = torch.empty(rows, n, dtype=dtype, device="cuda")
    layers.gns_dense_fp8(ctx, q.cuda(), e.cuda(), k, wq.cuda(), we.cuda(), None, False, out, rows)
    want = torch.from_numpy(fp8_values(q, e, k) @ fp8_values(wq, we, k).T)
    assert torch.equal(out.cpu(), want.to(dtype))


@TYPES
@pytest.mark.parametrize("rows,f1,f2,n", [(1, 3, 0, 5), (1, 4096, 0, 300), (1, 100, 28, 47), (4, 700, 0, 130), (7, 256, 256, 48), (8, 64, 0, 1), (16, 1024, 1, 64), (33, 129, 0, 65),
                                          (200, 128, 128, 256), (700, 300, 212, 100), (9000, 32, 28, 47), (8200, 100, 28, 48), (8300, 128, 128, 100), (8195, 256, 200, 36),
                                          (8192, 512, 0, 40)])
@pytest.mark.parametrize("how", LAYOUTS)
def test_update_step_in_fp8(ctx, rows, f1, f2, n, how, dtype):
    g = gen(rows, f1, f2, n)
    k = f1 + f2
    x = odd_rows((torch.randn(rows, k, generator=g) * 2).to(dtype))
    wq, we, w = random_fp8(n, k, g)
    bias = torch.randn(n, generator=g)
    out = layout(torch.zeros(rows, n, dtype=dtype), how)
    space = layers.alloc_workspace(layers.gns_sage_dense_fp8_workspace_bytes(ctx, k, rows))
    layers.gns_sage_dense_fp8(ctx, layout(x[:, :f1], how), layout(x[:, f1:], how) if f2 else None, wq.cuda(), we.cuda(), bias.cuda(), True, out, rows, space)
    check_dense(out, ref_fp8(x)[0], w, bias, True)


@pytest.mark.parametrize("rows", [1, 40, 200])
def test_fp8_exponents_far_apart(ctx, rows):
    """Blocks whose exponents leave fp32's range in the product with one factor alone."""
    k, n = 256, 64
    g = gen("far", rows)
    q, e, _ = random_fp8(rows, k, g, 0)
    wq, we, _ = random_fp8(n, k, g, 0)
    e[:, 0], we[:, 0] = 247, 20
    e[:, 1], we[:, 1] = 27, 220
    out = torch.empty(rows, n, device="cuda")
    layers.gns_dense_fp8(ctx, q.cuda(), e.cuda(), k, wq.cuda(), we.cuda(), None, False, out, rows)
    check_dense(out, fp8_values(q, e, k), fp8_values(wq, we, k), None, False)

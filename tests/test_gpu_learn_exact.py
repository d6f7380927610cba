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


@pytest.mark.parametrize("rows,f1,f2,hdim,dw", [s for s in WAYS if s[3] >= 8])
def test_input_gradient_of_values_that_cut_badly(ctx, rows, f1, f2, hdim, dw):
    """Eight products of one fp32 value with itself whose bits below the leading ones are all set.  The sum's magnitude is met by one
    rounding and what products of the last terms leave out: 2^-22 of it is more than both."""
    v = np.uint32(0x3F80FFFF).view(np.float32)
    w = torch.full((f1 + f2, hdim), float(v), device="cuda")
    d_out = torch.zeros(rows, hdim, device="cuda")
    d_out[:, :8] = float(v)
    one, two = two_checkpoints(ctx, torch.zeros(rows, f1 + f2), f1, f2) if dw else (None, None)
    dx = backward(ctx, d_out, None, one, f1, two, f2, w, dw, True)[2]
    want = np.full(dx.shape, 8 * float(v) ** 2)
    within(f64(dx), want, 2.0 ** -22 * want)



@pytest.mark.parametrize("rows,f1,hdim,dw", [(3000, 256, 256, True), (12, 500, 256, False), (30000, 128, 256, False), (400, 96, 256, True)])
def test_input_gradient_rounds_its_sums_once_per_sixteen_columns(ctx, rows, f1, hdim, dw):
    """A sum's error in the 2-norm: each rounding costs 2.5e-8 (an ulp over the root of twelve, of a value anywhere in its binade) of the
    part summed so far, which grows like the root; 16 of them and what joins the rest come to 8e-8, and twice that is allowed."""
    g = gen("norm", rows, f1)
    d_out, w = torch.randn(rows, hdim, generator=g).cuda(), torch.randn(f1, hdim, generator=g).cuda()
    one = save(ctx, torch.zeros(rows, f1))[:2] if dw else None
    dx = backward(ctx, d_out, None, one, f1, None, 0, w, dw, True)[2].double()
    want = d_out.double() @ w.double().t().contiguous()
    assert float((dx - want).norm() / want.norm()) < 1.6e-7


@pytest.mark.parametrize("scale", [2.0 ** -118, 1.0, 2.0 ** 100])
@pytest.mark.parametrize("rows,f1,f2,hdim,dw", WAYS)
def test_gradients_of_single_products_are_exact(ctx, rows, f1, f2, hdim, dw, scale):
    """One column of a row and one row of a column count, inputs are 0, 1 and -1 and weights powers of two: each result is one
    gradient of 24 bits, small and large ones too."""
    k = f1 + f2
    g = gen("single", rows, k, hdim)
    value = (torch.randint(2 ** 23, 2 ** 24, (rows,), generator=g).double() * 2.0 ** -23 * scale).float()
    value = torch.where(torch.rand(rows, generator=g) < 0.5, value, -value)
    w = torch.exp2(torch.randint(-3, 4, (k, hdim), generator=g).float())
    column = torch.randint(0, hdim, (rows,), generator=g)
    d_out = torch.zeros(rows, hdim)
    d_out[torch.arange(rows), column] = value
    x = torch.randint(-1, 2, (rows, k), generator=g).float()
    one, two = two_checkpoints(ctx, x, f1, f2) if dw else (None, None)
    dx = backward(ctx, d_out.cuda(), None, one, f1, two, f2, w.cuda(), dw, True)[2]
    assert torch.equal(dx.cpu(), value[:, None] * w[:, column].t())


@TYPES
@pytest.mark.parametrize("least", [-30, -120])
@pytest.mark.parametrize("rows,f1,f2,hdim", [(1, 5, 0, 3), (70, 40, 0, 33), (600, 300, 100, 129), (4000, 100, 28, 40), (20000, 128, 128, 256),
                                             (3000, 1024, 0, 1024), (2500, 257, 0, 385), (9001, 512, 0, 1030), (40001, 64, 36, 41)])
def test_weights_gradient_keeps_every_bit(ctx, rows, f1, f2, hdim, least, dtype):
    """In each column of d_out one row counts (the rest is masked or zero) and inputs are 0, 1 and -1: a gradient of the weights is one
    of d_out's values, of all bits its type has, or zero, and the bias's is the value."""
    k = f1 + f2
    g = gen("dw", rows, k, hdim)
    x = torch.randint(-1, 2, (rows, k), generator=g).float()
    row = torch.randint(0, rows, (hdim,), generator=g)
    value = ((1 + torch.rand(hdim, generator=g)) * torch.exp2(torch.randint(least, least + 60, (hdim,), generator=g).float())).to(dtype)
    n = torch.arange(hdim)
    one, two = two_checkpoints(ctx, x, f1, f2)
    w = torch.zeros(k, hdim, device="cuda")
    want = (x[row].t() * value.float()[None, :])
    for masked in (False, True):
        d_out = torch.randn(rows, hdim, generator=g).to(dtype) if masked else torch.zeros(rows, hdim, dtype=dtype)
        d_out[row, n] = value
        mask = torch.zeros(rows, hdim, dtype=torch.bool)
        mask[row, n] = True
        dw, db, _ = backward(ctx, d_out.cuda(), words_of(mask).cuda() if masked else None, one, f1, two, f2, w, True, False)
        assert torch.equal(dw.cpu(), want) and torch.equal(db.cpu(), value.float())


@TYPES
@pytest.mark.parametrize("classes", [11, 47, 200, 300, 4097])
def test_probabilities_far_below_the_largest(ctx, classes, dtype):
    """The gradient is -p with p = e^z, of logits that are log probabilities as they are: the exponential is good to a unit in the last
    place and two roundings wherever z is, not to |z| of them."""
    z = -torch.linspace(0.0, 80.0, 3 * classes).view(3, classes)
    z = z.to(dtype)
    stats = torch.zeros(3, 2, device="cuda")
    labels = torch.zeros(3, dtype=torch.int32, device="cuda")
    for how in ("packed", "odd"):
        out = layout(torch.zeros(3, classes), how)
        learn.gns_log_probs_backward(ctx, layout(z, how), labels, stats, None, torch.ones(3, device="cuda"), None, out, 3)
        want = -np.exp(f64(z))
        within(f64(out)[:, 1:], want[:, 1:], 4 * U * np.abs(want[:, 1:]))


def times(a, b):
    """a @ b in 64 bits, with each product's infinities and NaN."""
    y = a @ b
    odd_rows, odd_cols = ~np.isfinite(a).all(1), ~np.isfinite(b).all(0)
    with np.errstate(invalid="ignore"):
        for r in np.flatnonzero(odd_rows):
            y[r] = (a[r][:, None] * b).sum(0)
        for c in np.flatnonzero(odd_cols):
            y[:, c] = (a * b[:, c][None, :]).sum(1)
    return y


@TYPES
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("rows,f1,f2,hdim,dw", [s for s in WAYS if s[0] < 10000] + [(33000, 100, 0, 72, True), (17, 300, 0, 64, True)])
def test_backward_of_infinities(ctx, rows, f1, f2, hdim, dw, masked, dtype):
    """Infinities and NaN in d_out, the weights and the inputs go where the formulas take them, whatever kernel runs: an infinity stays
    one unless it meets a zero or its opposite."""
    k = f1 + f2
    g = gen("inf", rows, k, hdim)
    d_out, w, x = torch.randn(rows, hdim, generator=g).to(dtype), torch.randn(k, hdim, generator=g), torch.randn(rows, k, generator=g)
    x[torch.rand(rows, k, generator=g) < 0.3] = 0.0
    big = torch.finfo(dtype).max
    d_out[0, 0], d_out[rows // 2, hdim - 1], d_out[rows - 1, hdim // 2] = math.inf, -math.inf, math.inf
    if rows > 8:
        d_out[3, 1], d_out[5, 2], d_out[6, 1], d_out[7, 0] = math.nan, math.inf, -math.inf, -math.inf
    w[k // 2, hdim // 3], w[k - 1, 0] = math.inf, -math.inf
    if k > 40:
        w[3, hdim - 1], w[39, 1] = math.nan, math.inf
        w[39, 2] = math.inf
    if rows > 20 and dw:
        x[9, 1] = math.nan                               # spoils a group of its row
    mask = torch.rand(rows, hdim, generator=g) < 0.6
    if masked:
        mask[0, 0] = mask[rows - 1, hdim // 2] = True
        if rows > 8:
            mask[5, 2] = False
    one, two = two_checkpoints(ctx, x, f1, f2) if dw else (None, None)
    for value in (None, big):
        if value is not None:                            # large values, whose sums do not overflow
            d_out = torch.where(torch.isfinite(d_out), d_out, torch.zeros_like(d_out))
            d_out[0, 0] = d_out[rows - 1, hdim // 2] = value
            w = torch.where(torch.isfinite(w), w, torch.zeros_like(w)).clamp(-3, 3) / 64
        got_dw, db, dx = backward(ctx, d_out.cuda(), words_of(mask).cuda() if masked else None, one, f1, two, f2, w.cuda(), dw, True)
        dz = np.where(mask.numpy() if masked else True, f64(d_out), 0.0)
        w64 = f64(w)
        with np.errstate(invalid="ignore", over="ignore"):
            want, size = times(dz, w64.T.copy()), np.abs(dz) @ np.abs(w64).T
            size[~np.isfinite(want)] = 0.0
            limit = float(torch.finfo(dtype).max)
            want = np.where(np.abs(want) > limit, np.sign(want) * np.inf, want)
            bound = (hdim + 8) * 2 * U * size + (2.0 ** -8 * np.abs(want) if dtype == BF16 else 0.0) + 2.0 ** -126
            within(f64(dx), want, np.nan_to_num(bound, posinf=0.0))
        if dw:
            values = []
            for p, f in ((one, f1), (two, f2)):
                if f:
                    out = torch.empty(rows, f, device="cuda")
                    learn.gns_checkpoint_load(ctx, *p, out, rows)
                    values.append(f64(out))
            x64 = np.concatenate(values, 1)
            with np.errstate(invalid="ignore", over="ignore"):
                want, size = times(x64.T.copy(), dz), np.abs(x64).T @ np.abs(dz)
                want = np.where(np.abs(want) > float(torch.finfo(FP32).max), np.sign(want) * np.inf, want)
                size[~np.isfinite(want)] = 0.0
                within(f64(got_dw), want, np.nan_to_num((rows + 8) * 2 * U * size, posinf=0.0) + 2.0 ** -126)
                want = dz.sum(0)
                within(f64(db), want, np.nan_to_num((rows + 8) * 2 * U * np.abs(dz).sum(0), posinf=0.0))


ROWS = [0, 1, 2, 15, 16, 17, 31, 33, 64, 100, 127, 129, 200, 255, 257, 300, 400, 511, 512, 513, 600, 700, 1000, 1023, 1025, 1400, 1500, 2000, 2047, 2048, 2049,
        3000, 4000, 4096, 4097, 5000, 6982, 8192, 8193, 10000, 12000, 16384, 20000, 32746, 40000, 65536, 85000, 100000, 300000, 1000000]


def test_workspaces_grow_with_the_rows(ctx):
    """A workspace for some rows serves any call of fewer."""
    def grows(bytes_of):
        sizes = [bytes_of(r) for r in ROWS]
        assert sizes == sorted(sizes), [(r, s) for r, s in zip(ROWS, sizes)]
    for classes in (47, 257, 1000, 2100, 5003, 10000, 100003, 131072):
        for top in (0, 1, 5, 20, 32):
            grows(lambda r: learn.gns_log_probs_workspace_bytes(ctx, classes, top, r))
    for f1, f2, hdim in ((1, 0, 1), (40, 0, 72), (100, 28, 47), (128, 128, 256), (400, 0, 256), (64, 64, 2048), (1024, 0, 1024), (4096, 0, 4096), (300, 0, 5),
                         (2141, 0, 1102), (1000, 0, 1000), (40000, 0, 64), (64, 0, 40000)):
        grows(lambda r: learn.gns_sage_dense_backward_workspace_bytes(ctx, f1, f2, hdim, r))
    for k in (1, 64, 1000, 4096):
        grows(lambda r: learn.gns_sage_dense_int8_workspace_bytes(ctx, k, r))


@TYPES
@pytest.mark.parametrize("most,classes,top", [(4096, 100003, 20), (4096, 10000, 5), (5000, 5003, 20), (1500, 2100, 32)])
def test_log_probs_of_fewer_rows_in_the_same_workspace(ctx, most, classes, top, dtype):
    z = torch.randn(512, classes, generator=gen("fewer", classes), dtype=torch.float32).to(dtype).cuda()
    space = learn.alloc_workspace(learn.gns_log_probs_workspace_bytes(ctx, classes, top, most))
    for rows in (512, 300, 129, 17, 2, 1):
        results = []
        for s in (space, learn.alloc_workspace(learn.gns_log_probs_workspace_bytes(ctx, classes, top, rows))):
            if s is not None:
                s.fill_(255)
            entropy, index, value = torch.zeros(rows, device="cuda"), torch.zeros(rows, top, dtype=torch.int32, device="cuda"), torch.zeros(rows, top, device="cuda")
            learn.gns_log_probs(ctx, z[:rows], None, None, entropy, None, index, value, rows, s)
            results.append((entropy, index, value))
        assert all(torch.equal(a, b) for a, b in zip(*results))


@TYPES
@pytest.mark.parametrize("most,f1,f2,hdim", [(10000, 400, 0, 256), (8192, 1024, 0, 1024), (40000, 64, 64, 2048), (20000, 300, 0, 47), (6000, 600, 9, 1001)])
def test_backward_of_fewer_rows_in_the_same_workspace(ctx, most, f1, f2, hdim, dtype):
    g = gen("fewer", most, f1, hdim)
    rows0 = min(most, 7000)
    x = torch.randn(rows0, f1 + f2, generator=g)
    d_out, w = torch.randn(rows0, hdim, generator=g).to(dtype).cuda(), torch.randn(f1 + f2, hdim, generator=g).cuda()
    one, two = two_checkpoints(ctx, x, f1, f2)
    space = learn.alloc_workspace(learn.gns_sage_dense_backward_workspace_bytes(ctx, f1, f2, hdim, most))
    for rows in (rows0, 6982, 4096, 2000, 1104, 500, 129, 64, 9, 1):
        if rows > rows0:
            continue
        results = []
        for s in (space, None):
            if s is not None:
                s.fill_(255)
            results.append(backward(ctx, d_out[:rows], None, one, f1, two, f2, w, True, True, s))
        assert all(torch.equal(a, b) for a, b in zip(*results)), rows


@TYPES
def test_calls_with_empty_tensors(ctx, dtype):
    """No rows: their buffers have no address.  The gradients of the weights and the bias are zero all the same."""
    def none(*shape, t=FP32):
        return torch.empty((0,) + shape, dtype=t, device="cuda")

    x, weights, scales = none(40, t=dtype), torch.zeros(24, 64, dtype=torch.int8, device="cuda"), torch.ones(24, device="cuda")
    q, scale = none(64, t=torch.int8), none()
    learn.gns_quantize_rows(ctx, x, none(3, t=dtype), q, scale, 0)
    learn.gns_dense_int8(ctx, q, scale, 40, weights, scales, None, False, none(24, t=dtype), 0)
    learn.gns_sage_dense_int8(ctx, x, none(3, t=dtype), weights, scales, None, True, none(24, t=dtype), 0, None)
    one, two = (none(64, t=torch.int8), none(2, t=torch.uint8)), (none(32, t=torch.int8), none(1, t=torch.uint8))
    learn.gns_checkpoint_save(ctx, x, *one, none(2, t=torch.int32), 0)
    learn.gns_checkpoint_load(ctx, *one, x, 0)
    labels, logp, stats = none(t=torch.int32), none(), none(2)
    for top in (0, 3):
        learn.gns_log_probs(ctx, x, labels, logp, logp, stats, none(top, t=torch.int32) if top else None, none(top) if top else None, 0)
    learn.gns_log_probs_backward(ctx, x, labels, stats, logp, logp, logp, none(40, t=dtype), 0)
    w, dw, db = torch.ones(43, 24, device="cuda"), torch.full((43, 24), 3.0, device="cuda"), torch.full((24,), 3.0, device="cuda")
    space = learn.alloc_workspace(learn.gns_sage_dense_backward_workspace_bytes(ctx, 40, 3, 24, 0))
    learn.gns_sage_dense_backward(ctx, none(24, t=dtype), none(1, t=torch.int32), one, 40, two, 3, w, dw, db, none(43, t=dtype), 0, space)
    torch.cuda.synchronize()
    assert not dw.any() and not db.any()
    learn.gns_sage_dense_backward(ctx, none(24, t=dtype), None, None, 40, None, 3, w, None, None, none(43, t=dtype), 0, space)
    # what does not belong to the rows is asked for as ever
    with pytest.raises(B.GnsError):
        learn.gns_dense_int8(ctx, q, scale, 40, None, scales, None, False, none(24, t=dtype), 0)
    with pytest.raises(B.GnsError):
        learn.gns_sage_dense_backward(ctx, none(24, t=dtype), None, one, 40, two, 3, w, None, None, None, 0, space)


@TYPES
@pytest.mark.parametrize("rows,k,n", [(3, 64, 40), (20, 100, 33), (50, 64, 64), (100, 300, 47), (2100, 64, 2051), (2600, 1100, 4099)])
def test_product_of_scales_far_apart(ctx, rows, k, n, dtype):
    """A large scale of one side and a small one of the other: what is finite comes out finite, whichever is which."""
    q = torch.full((rows, learn.int8_stride(k)), 0, dtype=torch.int8)
    q[:, :k] = 127
    wq = q[:1].repeat(n, 1)
    for row_scale, channel_scale in ((2.0 ** -100, 2.0 ** 118), (2.0 ** 118, 2.0 ** -100)):
        out = torch.zeros(rows, n, dtype=dtype, device="cuda")
        learn.gns_dense_int8(ctx, q.cuda(), torch.full((rows,), row_scale, device="cuda"), k, wq.cuda(), torch.full((n,), channel_scale, device="cuda"),
                             None, False, out, rows)
        want = 127.0 * 127.0 * k * 2.0 ** 18
        within(f64(out), np.full((rows, n), want), (2.0 ** -8 if dtype == BF16 else 2 * U) * want)


@TYPES
@pytest.mark.parametrize("rows", [5, 100, 9000])
def test_update_step_of_scales_far_apart(ctx, rows, dtype):
    k, n = 64, 48
    x = torch.full((rows, k), 127 * 2.0 ** -100, dtype=dtype, device="cuda")
    x[1] = math.nan                                          # a spoilt row stays one
    wq = torch.full((n, k), 127, dtype=torch.int8, device="cuda")
    out = torch.zeros(rows, n, dtype=dtype, device="cuda")
    space = learn.alloc_workspace(learn.gns_sage_dense_int8_workspace_bytes(ctx, k, rows))
    learn.gns_sage_dense_int8(ctx, x, None, wq, torch.full((n,), 2.0 ** 118, device="cuda"), None, False, out, rows, space)
    want = np.full((rows, n), 127.0 * 127.0 * k * 2.0 ** 18)
    want[1] = math.nan
    within(f64(out), want, (2.0 ** -8 if dtype == BF16 else 2 * U) * np.nan_to_num(want))


def test_product_of_very_many_rows(ctx):
    """More tiles than the 2^22 that one dimension of a grid is given."""
    rows, k, n = (1 << 29) + 12345, 16, 1
    q = torch.zeros(rows, learn.int8_stride(k), dtype=torch.int8, device="cuda")
    scale, out = torch.ones(rows, device="cuda"), torch.full((rows, n), 9.0, device="cuda")
    at = torch.tensor([0, 1, 127, 128, 4097, (1 << 29) - 1, 1 << 29, (1 << 29) + 200, rows - 1], device="cuda")
    q[at, 0] = torch.arange(1, at.numel() + 1, dtype=torch.int8, device="cuda")
    wq = torch.zeros(n, learn.int8_stride(k), dtype=torch.int8, device="cuda")
    wq[0, 0] = 3
    learn.gns_dense_int8(ctx, q, scale, k, wq, torch.ones(n, device="cuda"), None, False, out, rows)
    assert torch.equal(out[at, 0], 3.0 * torch.arange(1, at.numel() + 1, device="cuda"))
    out[at] = 0.0
    assert int(torch.count_nonzero(out)) == 0
    del q, scale, out
    torch.cuda.empty_cache()                                 # 39 GB


# ---- sizes at which a kernel takes over -----------------------------------------------------------------------------
@TYPES
@pytest.mark.parametrize("rows,f1,f2", [(5, 4100, 0), (70, 8000, 191), (3, 8191, 0), (40, 8195, 0), (9, 16384, 0), (600, 6000, 0)])
def test_quantize_rows_of_a_block(ctx, rows, f1, f2, dtype):
    """Rows that a whole block has: each value half a step off at most (and the inverse's two roundings), the largest 127 steps."""
    k = f1 + f2
    x = (torch.randn(rows, k, generator=gen("block", rows, k)) * torch.exp(torch.randn(rows, 1, generator=gen(rows)))).to(dtype)
    x[0, k - 1] = 100.0
    if rows > 4:
        x[1], x[2, k // 2], x[3, 0] = 0.0, math.inf, math.nan
    for how in ("packed", "odd"):
        q = torch.full((rows, learn.int8_stride(k)), 77, dtype=torch.int8, device="cuda")
        scale = torch.full((rows,), -1.0, device="cuda")
        learn.gns_quantize_rows(ctx, layout(x[:, :f1], how), layout(x[:, f1:], how) if f2 else None, q, scale, rows)
        a = x.cuda().double().abs().amax(1, keepdim=True)
        good = torch.isfinite(a[:, 0]) & (a[:, 0] > 0)
        steps = x.cuda().double()[good] * 127.0 / a[good]
        assert float((q[good][:, :k].double() - steps).abs().max()) <= 0.5 + 127 * 4 * U
        assert bool((q[good][:, :k].abs().amax(1) == 127).all())
        assert not q[:, k:].any() and not q[~good].any()
        want = f64(a[:, 0] / 127.0)
        want[f64(~good) > 0] = np.where(f64(a[:, 0])[f64(~good) > 0] == 0, 0.0, np.nan)
        within(f64(scale), want, U * np.nan_to_num(np.abs(want)))


# 128 x 128 and 256 x 256 outputs a block, the longest sums
@TYPES
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("rows,k,n", [(2100, 300, 2051), (2049, 1000, 2048), (3001, 1100, 4099), (10000, 1500, 1030), (65, 131072, 70),
                                      (1, 131072, 40), (20, 131071, 20), (33, 100000, 100)])
def test_int8_product_of_large_tiles_and_long_sums(ctx, rows, k, n, relu, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + k + n)
    q = torch.randint(-127, 128, (rows, learn.int8_stride(k)), generator=g, dtype=torch.int8, device="cuda")
    w = torch.randint(-127, 128, (n, learn.int8_stride(k)), generator=g, dtype=torch.int8, device="cuda")
    q[:, k:] = 0
    q[rows // 2, :k], w[n // 2, :k], w[0, :k] = 127, -127, 127
    scale, w_scale = torch.rand(rows, generator=g, device="cuda") * 0.05, torch.rand(n, generator=g, device="cuda") * 0.01
    bias = torch.randn(n, generator=g, device="cuda") if rows % 2 else None
    y = (q[:, :k].double() @ w[:, :k].double().t().contiguous()) * scale.double()[:, None] * w_scale.double()
    size = y.abs() + (0.0 if bias is None else bias.double().abs())
    y = y if bias is None else y + bias.double()
    y = y.relu() if relu else y
    bound = 4 * U * size + (2.0 ** -8 * y.abs() if dtype == BF16 else 0.0) + 2.0 ** -133
    for how in ("packed", "odd"):
        out = layout(torch.full((rows, n), 9.0, dtype=dtype), how)
        learn.gns_dense_int8(ctx, q, scale, k, w, w_scale, bias, relu, out, rows)
        off = (out.double() - y).abs() - bound
        assert float(off.max()) <= 0.0, int(off.argmax())


@TYPES
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("rows,f1,f2,hdim,dw", WAYS + [(17000, 300, 0, 264, True), (16385, 300, 0, 520, False)])
def test_backward_in_every_way(ctx, rows, f1, f2, hdim, dw, relu, dtype):
    """Normal values.  Errors of sums of so many roundings add up as a random walk: eight of its standard deviations at most."""
    k = f1 + f2
    g = torch.Generator(device="cuda").manual_seed(rows + k + hdim)
    x = torch.randn(rows, k, generator=g, device="cuda")
    d_out = (torch.randn(rows, hdim, generator=g, device="cuda") * 1e-2).to(dtype)
    w = torch.randn(k, hdim, generator=g, device="cuda") / math.sqrt(k)
    mask = torch.rand(rows, hdim, generator=g, device="cuda") < 0.5
    dz = d_out.double() * mask if relu else d_out.double()
    one, two = two_checkpoints(ctx, x, f1, f2) if dw else (None, None)
    if relu:
        d_out = torch.where(mask, d_out, torch.full_like(d_out, math.nan))
    for how in ("packed", "odd"):
        got_dw, db, dx = backward(ctx, layout(d_out, how), words_of(mask) if relu else None, one, f1, two, f2, w, dw, True)
        want = dz @ w.double().t().contiguous()
        size = ((dz * dz) @ (w.double() ** 2).t().contiguous()).sqrt()
        bound = 8 * U * size * math.sqrt(hdim + 8) + (2.0 ** -8 * want.abs() if dtype == BF16 else 0.0) + 2.0 ** -126
        assert float(((dx.double() - want).abs() - bound).max()) <= 0.0
        if dw:
            values = []
            for p, f in ((one, f1), (two, f2)):
                if f:
                    values.append(torch.empty(rows, f, device="cuda"))
                    learn.gns_checkpoint_load(ctx, *p, values[-1], rows)
            x64 = torch.cat(values, 1).double()
            want, size = x64.t().contiguous() @ dz, ((x64 * x64).t().contiguous() @ (dz * dz)).sqrt()
            assert float(((got_dw.double() - want).abs() - 8 * U * size * math.sqrt(rows + 8) - 2.0 ** -126).max()) <= 0.0
            want, size = dz.sum(0), (dz * dz).sum(0).sqrt()
            assert float(((db.double() - want).abs() - 8 * U * size * math.sqrt(rows + 8) - 2.0 ** -126).max()) <= 0.0


@TYPES
@pytest.mark.parametrize("rows,classes,top", [(1500, 2100, 20), (4200, 5003, 20), (9000, 1025, 3), (700, 30011, 32), (5000, 300, 0)])
def test_log_probs_of_many_long_rows(ctx, rows, classes, top, dtype):
    """Whole rows of several tiles a wave, against 64 bits on the device."""
    g = torch.Generator(device="cuda").manual_seed(rows + classes)
    z = (torch.randn(rows, classes, generator=g, device="cuda") * 3).to(dtype)
    z[5::16] = torch.where(torch.rand(z[5::16].shape, generator=g, device="cuda") < 0.5, torch.full((), -math.inf, dtype=dtype, device="cuda"), z[5::16])
    z[7] = -math.inf
    z[9] = 0.25
    labels = torch.randint(0, classes, (rows,), generator=g, dtype=torch.int32, device="cuda")
    labels[::17] = -1
    z64 = z.double()
    m = z64.amax(1)
    safe = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    d = z64 - safe[:, None]
    p = d.exp()
    s = p.sum(1)
    none = torch.isinf(m)
    log_s = torch.where(none, torch.zeros_like(s), s.log())
    entropy = torch.where(none, torch.zeros_like(s), log_s - torch.where(p > 0, p * d, torch.zeros_like(p)).sum(1) / s.clamp(min=1e-300))
    at = d.gather(1, labels.clamp(min=0).long()[:, None])[:, 0] - log_s
    logp = torch.where(labels < 0, torch.zeros_like(at), at)
    logp[none & (labels >= 0)] = -math.inf
    order = torch.sort(z64, dim=1, descending=True, stable=True)
    index = torch.where(torch.isinf(order.values[:, :top]), torch.full((), -1, device="cuda"), order.indices[:, :top])
    chain = 64 + classes / 64 + 16
    tol = 2 * U * (chain + 2 * log_s.abs())
    for how in ("packed", "odd"):
        out = dict(logp=torch.full((rows,), 9.0, device="cuda"), entropy=torch.full((rows,), 9.0, device="cuda"), stats=torch.full((rows, 2), 9.0, device="cuda"))
        best, value = (torch.full((rows, top), 9, dtype=t, device="cuda") if top else None for t in (torch.int32, FP32))
        space = learn.alloc_workspace(learn.gns_log_probs_workspace_bytes(ctx, classes, top, rows))
        learn.gns_log_probs(ctx, layout(z, how), labels, out["logp"], out["entropy"], out["stats"], best, value, rows, space)
        within(f64(out["logp"]), f64(logp), f64(tol + 4 * U * torch.nan_to_num(logp.abs(), posinf=0.0)))
        within(f64(out["entropy"]), f64(entropy), f64(2 * U * chain * (1 + entropy.abs() + log_s.abs())))
        within(f64(out["stats"][:, 0]), f64(m), 0.0)
        within(f64(out["stats"][:, 1]), f64(log_s), f64(tol))
        if top:
            assert torch.equal(best.long(), index)
            want = order.values[:, :top] - (safe + log_s)[:, None]
            within(f64(value), f64(want), f64(tol[:, None] + 4 * U * torch.nan_to_num(want.abs(), posinf=0.0)))


@TYPES
@pytest.mark.parametrize("rows,f1,f2", [(40, 50, 0), (200, 7, 57), (30, 1500, 0), (9, 1025, 900), (33, 513, 0), (5, 2048, 0)])
def test_quantize_rows_of_a_few_lanes_or_a_wave(ctx, rows, f1, f2, dtype):
    """Half a step off at most (and the inverse's two roundings), the largest 127 steps."""
    k = f1 + f2
    x = (torch.randn(rows, k, generator=gen("lanes", rows, k)) * torch.exp(torch.randn(rows, 1, generator=gen(rows)))).to(dtype)
    for how in ("packed", "odd"):
        q = torch.full((rows, learn.int8_stride(k)), 77, dtype=torch.int8, device="cuda")
        scale = torch.full((rows,), -1.0, device="cuda")
        learn.gns_quantize_rows(ctx, layout(x[:, :f1], how), layout(x[:, f1:], how) if f2 else None, q, scale, rows)
        a = x.cuda().double().abs().amax(1, keepdim=True)
        assert float((q[:, :k].double() - x.cuda().double() * 127.0 / a).abs().max()) <= 0.5 + 127 * 4 * U
        assert bool((q[:, :k].abs().amax(1) == 127).all()) and not q[:, k:].any()
        want = f64(a[:, 0] / 127.0)
        within(f64(scale), want, U * want)


# inputs of one type and outputs of the other; weights that leave eight waves' room in LDS and not sixteen's
@pytest.mark.parametrize("rows,f1,f2,n", [(1, 300, 0, 70), (7, 100, 29, 33), (16, 1024, 0, 40), (100, 200, 0, 65), (9001, 128, 0, 900), (8300, 256, 0, 400),
                                          (8192, 504, 0, 100), (8250, 64, 0, 1650), (9000, 100, 28, 908)])
@pytest.mark.parametrize("x_type,out_type", [(FP32, FP32), (FP32, BF16), (BF16, FP32), (BF16, BF16)])
def test_update_step_of_mixed_types_and_wide_weights(ctx, rows, f1, f2, n, x_type, out_type):
    k = f1 + f2
    g = torch.Generator(device="cuda").manual_seed(rows + k + n)
    x = torch.randn(rows, k, generator=g, device="cuda").to(x_type)
    w = torch.randint(-127, 128, (n, learn.int8_stride(k)), generator=g, dtype=torch.int8, device="cuda")
    w_scale, bias = torch.rand(n, generator=g, device="cuda") * 0.01, torch.randn(n, generator=g, device="cuda")
    q = torch.empty(rows, learn.int8_stride(k), dtype=torch.int8, device="cuda")
    scale = torch.empty(rows, device="cuda")
    learn.gns_quantize_rows(ctx, x, None, q, scale, rows)
    y = (q[:, :k].double() @ w[:, :k].double().t().contiguous()) * scale.double()[:, None] * w_scale.double()
    size = y.abs() + bias.double().abs()
    y = (y + bias.double()).relu()
    bound = 4 * U * size + (2.0 ** -8 * y.abs() if out_type == BF16 else 0.0)
    space = learn.alloc_workspace(learn.gns_sage_dense_int8_workspace_bytes(ctx, k, rows))
    for how in ("packed", "odd"):
        out = layout(torch.full((rows, n), 9.0, dtype=out_type), how)
        one, two = layout(x[:, :f1], how), layout(x[:, f1:], how) if f2 else None
        learn.gns_sage_dense_int8(ctx, one, two, w, w_scale, bias, True, out, rows, space)
        assert float(((out.double() - y).abs() - bound).max()) <= 0.0


@TYPES
@pytest.mark.parametrize("entropy_term", [False, True])
@pytest.mark.parametrize("classes", [300, 4099])
def test_gradient_that_lies_unlike_its_logits(ctx, classes, entropy_term, dtype):
    """Logits and gradients at different places against the 16-byte marks: the same results as at like ones, but for the order in which
    a product is rounded."""
    rows = 40
    g = gen("unlike", classes)
    z = (torch.randn(rows, classes, generator=g) * 3).to(dtype)
    labels = torch.randint(0, classes, (rows,), generator=g, dtype=torch.int32).cuda()
    g_logp, g_entropy = torch.randn(rows, generator=g).cuda(), torch.randn(rows, generator=g).cuda()
    log_p = torch.log_softmax(z.double(), 1)
    stats = torch.stack([z.double().amax(1), torch.logsumexp(z.double(), 1) - z.double().amax(1)], 1).float().cuda()
    entropy = -(log_p.exp() * log_p).sum(1).float().cuda()
    want_log_p = z.cuda().double() - stats[:, :1].double() - stats[:, 1:].double()
    p = want_log_p.exp()
    one = torch.nn.functional.one_hot(labels.long(), classes).double()
    want = g_logp.double()[:, None] * (one - p)
    size = g_logp.double().abs()[:, None] * (one + p * (8 + want_log_p.abs()))
    if entropy_term:
        want = want - g_entropy.double()[:, None] * p * (want_log_p + entropy.double()[:, None])
        size = size + g_entropy.double().abs()[:, None] * p * (8 + want_log_p.abs()) * (1 + want_log_p.abs() + entropy.double()[:, None])
    bound = 4 * U * size + (2.0 ** -8 * want.abs() if dtype == BF16 else 0.0) + 2.0 ** -126
    for how, out_how in (("packed", "odd"), ("odd", "packed"), ("odd", "odd")):
        out = layout(torch.full((rows, classes), 9.0, dtype=dtype), out_how)
        learn.gns_log_probs_backward(ctx, layout(z, how), labels, stats, entropy if entropy_term else None, g_logp, g_entropy if entropy_term else None, out, rows)
        assert float(((out.double() - want).abs() - bound).max()) <= 0.0


def test_entropy_of_long_rows_in_the_two_norm(ctx):
    """Its own rounding, log S's and T / S's, an ulp of 2^-20 over the root of twelve each for values of 8 to 16, are 4.8e-7 together, 5.1e-8
    of an entropy of 9.5; a lane's hundred sums of tiles, in 64 lanes, add 2e-8 of T / S.  A quarter more is allowed."""
    rows, classes = 4096, 100003
    g = torch.Generator(device="cuda").manual_seed(5)
    z = (2.0 * torch.randn(rows, classes, generator=g, device="cuda") + 3.0 * torch.randn(rows, 1, generator=g, device="cuda")).to(BF16)
    entropy = torch.zeros(rows, device="cuda")
    space = learn.alloc_workspace(learn.gns_log_probs_workspace_bytes(ctx, classes, 0, rows))
    learn.gns_log_probs(ctx, z, None, None, entropy, None, None, None, rows, space)
    want = []
    for part in z.split(250):
        log_p = torch.log_softmax(part.double(), 1)
        want.append(-(log_p.exp() * log_p).sum(1))
    want = torch.cat(want)
    assert float((entropy.double() - want).norm() / want.norm()) < 6.5e-8

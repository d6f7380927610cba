"""Cases of the operators of deeper classifiers to be timed: group norm with an activation over segments of rows and its
backward pass, the orthogonalised update of a weight matrix, the update step in 8-bit floats.

A case is a dict of plain values; "kind" names the operator:
  norm       rows x width of fp32 or bf16, normalised over each segment of rows and group of columns, scaled, shifted and put
             through an activation; with the statistics.  Segments are equally long ("segment_rows") or ragged ("segments")
  norm_grad  gradients of the rows, the scales and the shifts, from those statistics
  update     momentum, its Newton-Schulz orthogonalisation, and where "weights" is set the weights moved along it
  fp8        rows x (f1 [+ f2]) of fp32 or bf16, quantised to 8-bit floats with a power of two per row and block of 128 columns,
             times weights held so (laid out once), plus a bias: rows x hdim in the inputs' type

With `own` false everything is computed in plain torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

FLOAT = {"fp32": torch.float32, "bf16": torch.bfloat16}
ACTIVATIONS = ("none", "relu", "silu", "gelu")
BLOCK = 128                     # columns that share a power of two in 8-bit floats
EPS = 1e-5
MU = 0.95
STEPS = 5
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
KEEP, RATE = 0.999, -0.02       # weight decay and step of an update


def _norm(name, rows, width, groups, dtype, activation, segment_rows=0, segments=0, kind="norm"):
    return dict(name=name, kind=kind, rows=rows, width=width, groups=groups, dtype=dtype, activation=activation,
                segment_rows=segment_rows, segments=segments)


def _update(name, rows, width, dtype, weights, nesterov=True):
    return dict(name=name, kind="update", rows=rows, width=width, dtype=dtype, weights=weights, nesterov=nesterov)


def _fp8(name, rows, f1, f2, hdim, dtype, relu=True):
    return dict(name=name, kind="fp8", rows=rows, f1=f1, f2=f2, hdim=hdim, dtype=dtype, relu=relu)


def listed():
    return [
        # one row between two wide layers: answering one request, latency
        _norm("norm-one-row", 1, 4096, 32, "bf16", "silu", segment_rows=1),
        # the hidden layer of a mini-batch's input nodes, each node by itself
        _norm("norm-nodes", 85_000, 256, 8, "fp32", "relu", segment_rows=1),
        # gathered rows of a group of sixteen mini-batches of different sizes, each normalised over its nodes
        _norm("norm-batches", 168_003, 100, 4, "fp32", "gelu", segments=16),
        # sixteen maps of 64 x 64 positions with 512 channels
        _norm("norm-maps", 65_536, 512, 32, "bf16", "silu", segment_rows=4096),
        # backward passes of the second and the fourth, and of ragged ones
        _norm("norm-grad-nodes", 85_000, 256, 8, "fp32", "relu", segment_rows=1, kind="norm_grad"),
        _norm("norm-grad-maps", 65_536, 512, 32, "bf16", "silu", segment_rows=4096, kind="norm_grad"),
        # the weights of a hidden layer (128 features and their neighbors' mean, 256 hidden units): latency
        _update("update-hidden", 256, 256, "fp32", True),
        # the weights of a wide layer in bf16, of odd sizes and tall
        _update("update-odd", 2709, 1433, "bf16", True),
        # the weights of a very wide layer, the orthogonal matrix itself
        _update("update-wide", 4096, 4096, "fp32", False),
        # one row through a wide layer: answering one request, all of it reading weights
        _fp8("fp8-one-row", 1, 4096, 0, 4096, "bf16"),
        # the hidden layer of a mini-batch's input nodes (128 features, 256 hidden units)
        _fp8("fp8-hidden", 85_000, 128, 128, 256, "fp32"),
        # a long batch through a wide layer
        _fp8("fp8-wide", 8192, 8192, 0, 8192, "bf16", relu=False),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(("norm", "norm", "norm_grad", "norm_grad", "update", "update", "fp8", "fp8"))
    dtype = rng.choice(("fp32", "bf16"))
    if kind in ("norm", "norm_grad"):
        groups = log_int(1, 64)
        width = groups * max(1, log_int(8, 8192) // groups)
        rows = max(1, min(log_int(1, 200_000), 30_000_000 // width))
        activation = rng.choice(ACTIVATIONS)
        if rng.random() < 0.4:
            case = _norm("", rows, width, groups, dtype, activation, segments=log_int(1, 64), kind=kind)
        else:
            case = _norm("", rows, width, groups, dtype, activation, segment_rows=rng.choice((1, log_int(1, 8192))), kind=kind)
    elif kind == "update":
        case = _update("", log_int(1, 4096), log_int(16, 4096), dtype, rng.random() < 0.7, rng.random() < 0.7)
    else:
        k, hdim = log_int(16, 8192), log_int(16, 8192)
        if rng.random() < 0.5:
            k, hdim = (1 << round(math.log2(v)) for v in (k, hdim))
        rows = max(1, min(log_int(1, 100_000), int(5e11 / (k * hdim)), int(4e8 / max(k, hdim))))
        two = rng.random() < 0.5
        f1 = max(1, k // 2) if two else k
        case = _fp8("", rows, f1, k - f1 if two else 0, hdim, dtype, rng.random() < 0.5)
    del case["name"]
    return case


def _segment_count(case):
    return case["segments"] or (case["rows"] + case["segment_rows"] - 1) // case["segment_rows"]


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    rows, kind = case["rows"], case["kind"]
    if kind in ("norm", "norm_grad"):
        values, stats = rows * case["width"] * size, 8 * _segment_count(case) * case["groups"]
        small = 8 * case["width"] + 4 * case["segments"]
        if kind == "norm":
            return {"bytes": 2 * values + stats + small, "flops": 0}
        return {"bytes": 3 * values + stats + small + 8 * case["width"], "flops": 0}
    if kind == "update":
        short, long = sorted((rows, case["width"]))
        # gradient and momentum in, momentum and result out; of the symmetric products half is enough
        return {"bytes": rows * case["width"] * size * (5 if case["weights"] else 4),
                "flops": STEPS * (3 * short * short * long + short ** 3)}
    k, n = case["f1"] + case["f2"], case["hdim"]
    return {"bytes": rows * k * size + n * k + n * ((k + BLOCK - 1) // BLOCK) + 4 * n + rows * n * size, "flops": 2 * rows * k * n}


# ---------------------------------------------------------------------------------------------------------------
# Plain forms.

def _ranges(rows, offsets, segment_rows):
    if offsets is not None:
        return list(zip(offsets[:-1], offsets[1:]))
    return [(i, min(rows, i + segment_rows)) for i in range(0, rows, segment_rows)]


def _by_length(state, function, rows):
    """function(rows of equally long segments as [segments, length, width], first segment) for all segments: equally long
    ones at once, ragged ones one after the other."""
    if state["offsets"] is None:
        length = state["segment_rows"]
        whole = rows // length
        if whole:
            function(0, whole * length, whole, length, 0)
        if rows % length:
            function(whole * length, rows, 1, rows % length, whole)
        return
    for i, (a, b) in enumerate(_ranges(rows, state["offsets"], 0)):
        if b > a:
            function(a, b, 1, b - a, i)


def _act(y, activation):
    if activation == "relu":
        return torch.clamp(y, min=0.0)
    if activation == "silu":
        return y / (1.0 + torch.exp(-y))
    if activation == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    return y


def _act_slope(y, activation):
    if activation == "relu":
        return (y > 0).to(y.dtype)
    if activation == "silu":
        s = 1.0 / (1.0 + torch.exp(-y))
        return s * (1.0 + y * (1.0 - s))
    if activation == "gelu":
        return 0.5 * (1.0 + torch.erf(y * math.sqrt(0.5))) + y * torch.exp(-0.5 * y * y) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(y)


def _plain_norm(state):
    x, groups = state["x"], state["groups"]
    rows, width = x.shape
    w = width // groups
    out = torch.empty((rows, width), dtype=x.dtype, device=x.device)
    stats = torch.zeros((state["count"], groups, 2), dtype=torch.float32, device=x.device)

    def part(a, b, count, length, first):
        v = x[a:b].float().view(count, length, groups, w)
        mean = v.mean((1, 3), keepdim=True)
        centred = v - mean
        rstd = 1.0 / torch.sqrt((centred * centred).mean((1, 3), keepdim=True) + EPS)
        y = (centred * rstd).reshape(b - a, width) * state["gamma"] + state["beta"]
        out[a:b] = _act(y, state["activation"]).to(x.dtype)
        stats[first:first + count, :, 0] = mean[:, 0, :, 0]
        stats[first:first + count, :, 1] = rstd[:, 0, :, 0]

    _by_length(state, part, rows)
    return [out, stats]


def _plain_norm_grad(state):
    x, groups, stats, gamma = state["x"], state["groups"], state["stats"], state["gamma"]
    rows, width = x.shape
    w = width // groups
    dx = torch.empty_like(x)
    dgamma, dbeta = torch.zeros_like(gamma), torch.zeros_like(gamma)

    def part(a, b, count, length, first):
        s = stats[first:first + count]
        mean, rstd = s[:, None, :, None, 0], s[:, None, :, None, 1]
        xhat = (x[a:b].float().view(count, length, groups, w) - mean) * rstd
        y = xhat.view(b - a, width) * gamma + state["beta"]
        dy = state["d_out"][a:b].float() * _act_slope(y, state["activation"])
        dbeta.add_(dy.sum(0))
        dgamma.add_((dy * xhat.view(b - a, width)).sum(0))
        dh = (dy * gamma).view(count, length, groups, w)
        m1, m2 = dh.mean((1, 3), keepdim=True), (dh * xhat).mean((1, 3), keepdim=True)
        dx[a:b] = (rstd * (dh - m1 - xhat * m2)).view(b - a, width).to(x.dtype)

    _by_length(state, part, rows)
    return [dx, dgamma, dbeta]


def _plain_update(state):
    grad = state["grad"].float()
    momentum = MU * state["momentum"].float() + grad
    u = grad + MU * momentum if state["nesterov"] else momentum
    tall = u.shape[0] > u.shape[1]
    if tall:
        u = u.t().contiguous()
    x = u / (torch.sqrt((u * u).sum()) + 1e-7)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    if tall:
        x = x.t()
    if state["w"] is None:
        return [x.to(state["grad"].dtype).contiguous(), momentum.to(state["grad"].dtype)]
    return [(KEEP * state["w"].float() + RATE * x).to(state["w"].dtype), momentum.to(state["grad"].dtype)]


def _two(e):
    """2^e in fp32 for integers -126 <= e <= 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _plain_blocks(x):
    """Rows (fp32) in 8-bit floats: their values before scaling [rows, blocks * 128] and the exponent of each block; -127 for
    blocks of nothing but zeros."""
    rows, k = x.shape
    blocks = (k + BLOCK - 1) // BLOCK
    x = torch.nn.functional.pad(x, (0, blocks * BLOCK - k)).view(rows, blocks, BLOCK)
    mantissa, exponent = torch.frexp(x.abs().amax(2))               # mantissa in [0.5, 1)
    # the largest value is 448, and what is up to 464 rounds to it
    e = exponent - 9 + (mantissa > 464.0 / 512.0).to(exponent.dtype)
    none = (mantissa == 0) | (exponent - 1 < -100)
    v = x * torch.where(none, torch.zeros_like(mantissa), _two(-e))[:, :, None]
    # four bits from the leading one on, or down to 2^-9
    _, place = torch.frexp(v)
    step = _two(torch.clamp(place - 4, min=-9))
    return (torch.round(v / step) * step).view(rows, blocks * BLOCK), torch.where(none, torch.full_like(e, -127), e)


def _block_values(q, e, k):
    rows, blocks = e.shape
    power = torch.where(e == -127, torch.zeros_like(e, dtype=torch.float32), _two(torch.clamp(e, min=-126)))
    return (q.view(rows, blocks, BLOCK) * power[:, :, None]).view(rows, blocks * BLOCK)[:, :k]


# ---------------------------------------------------------------------------------------------------------------
_kept = {}


def _context():
    """A context on a graph of two nodes: these operators take from it the device and the place of errors alone."""
    if "ctx" not in _kept:
        from paper_2106_06150_amd import binding as B
        dev = torch.device("cuda:0")
        graph = B.make_graph(torch.tensor([0, 1, 2], dtype=torch.int32, device=dev), torch.tensor([1, 0], dtype=torch.int32, device=dev))
        config = B.make_config([1], [B.GNS_UNIFORM], 0, 1)
        workspace = B.alloc_workspace(graph, config, dev)
        _kept.update(graph=graph, workspace=workspace, ctx=B.gns_create(graph, config, workspace))
    return _kept["ctx"]


def _activations(rows, width, gen, dtype):
    """Outputs of a layer: columns of different mean and spread, rows of different size."""
    x = torch.randn((rows, width), device="cuda:0", generator=gen)
    x *= torch.exp(0.5 * torch.randn((1, width), device="cuda:0", generator=gen))
    x += torch.randn((1, width), device="cuda:0", generator=gen)
    x *= torch.exp(0.5 * torch.randn((rows, 1), device="cuda:0", generator=gen))
    return x.to(dtype)


def _gradient(rows, width, gen):
    """A weight gradient: a few strong directions over a floor of weak ones."""
    rank = max(1, min(rows, width) // 8)
    strong = torch.randn((rows, rank), device="cuda:0", generator=gen) @ torch.randn((rank, width), device="cuda:0", generator=gen)
    return 1e-3 * (strong / math.sqrt(rank) + torch.randn((rows, width), device="cuda:0", generator=gen))


def _offsets(rows, segments, seed):
    """Ragged segments that cover all rows: one of no rows and one of a single row among them where there are enough."""
    gen = torch.Generator().manual_seed(int(seed) + 17)
    cuts = torch.sort(torch.randint(0, rows + 1, (segments - 1,), generator=gen)).values.tolist()
    if segments > 4 and rows > 4:
        cuts[1] = cuts[0]
        cuts[2] = min(rows, max(cuts[0] + 1, 1))
        cuts.sort()
    return [0] + cuts + [rows]


def prepare(case, seed):
    gen = torch.Generator(device="cuda:0").manual_seed(int(seed))
    kind, rows, dtype = case["kind"], case["rows"], FLOAT[case["dtype"]]
    state = {"kind": kind, "kept": {}}

    def normal(*shape):
        return torch.randn(shape, device="cuda:0", generator=gen)

    if kind in ("norm", "norm_grad"):
        width = case["width"]
        offsets = _offsets(rows, case["segments"], seed) if case["segments"] else None
        state.update(x=_activations(rows, width, gen, dtype), groups=case["groups"], activation=case["activation"],
                     offsets=offsets, segment_rows=case["segment_rows"], count=_segment_count(case),
                     segments=None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda:0"),
                     gamma=1.0 + 0.2 * normal(width), beta=0.2 * normal(width))
        if kind == "norm_grad":
            state.update(d_out=(1e-3 * normal(rows, width)).to(dtype), stats=_plain_norm(state)[1])
    elif kind == "update":
        width = case["width"]
        state.update(grad=_gradient(rows, width, gen).to(dtype), momentum=(6.0 * _gradient(rows, width, gen)).to(dtype),
                     w=(normal(rows, width) / math.sqrt(rows)).to(dtype) if case["weights"] else None, nesterov=case["nesterov"])
    else:
        f1, f2, n = case["f1"], case["f2"], case["hdim"]
        k = f1 + f2
        x = _activations(rows, k, gen, dtype)
        q, e = _plain_blocks(normal(n, k) / math.sqrt(k))
        # exponents are stored as bytes e + 127, a multiple of four a row
        state.update(x1=x[:, :f1].contiguous(), x2=x[:, f1:].contiguous() if f2 else None, k=k, relu=case["relu"], bias=normal(n), dtype=dtype,
                     w=q.to(torch.float8_e4m3fn).view(torch.uint8),
                     w_exponents=torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -e.shape[1] % 4)))
    return state


def _run_own(state):
    from paper_2106_06150_amd import layers
    ctx, kind, kept = _context(), state["kind"], state["kept"]

    def empty(name, shape, dtype):
        """Output buffers and workspaces are a program's own and serve every pass."""
        if name not in kept:
            kept[name] = torch.empty(shape, dtype=dtype, device="cuda:0")
        return kept[name]

    def space(function, *args):
        if "workspace" not in kept:
            kept["workspace"] = layers.alloc_workspace(function(ctx, *args))
        return kept["workspace"]

    if kind in ("norm", "norm_grad"):
        x = state["x"]
        rows, width = x.shape
        if "norm" not in kept:
            kept["norm"] = layers.Norm(state["groups"], segments=state["segments"], segment_rows=state["segment_rows"],
                                       activation=ACTIVATIONS.index(state["activation"]), eps=EPS, gamma=state["gamma"], beta=state["beta"])
        norm = kept["norm"]
        if kind == "norm":
            out, stats = empty("out", (rows, width), x.dtype), empty("stats", (state["count"], state["groups"], 2), torch.float32)
            layers.gns_group_norm(ctx, x, norm, out, stats, rows, space(layers.gns_group_norm_workspace_bytes, width, norm, rows))
            return [out, stats]
        dx, dgamma, dbeta = empty("dx", (rows, width), x.dtype), empty("dgamma", (width,), torch.float32), empty("dbeta", (width,), torch.float32)
        layers.gns_group_norm_backward(ctx, state["d_out"], x, norm, state["stats"], dx, dgamma, dbeta, rows,
                                       space(layers.gns_group_norm_backward_workspace_bytes, width, norm, rows))
        return [dx, dgamma, dbeta]
    if kind == "update":
        grad, w = state["grad"], state["w"]
        rows, width = grad.shape
        if "how" not in kept:
            kept["how"] = layers.Orthogonal([COEFFICIENTS] * STEPS, mu=MU, nesterov=state["nesterov"], eps=1e-7,
                                            keep=0.0 if w is None else KEEP, rate=1.0 if w is None else RATE)
        out, momentum = empty("out", (rows, width), grad.dtype), empty("momentum", (rows, width), grad.dtype)
        layers.gns_orthogonal_update(ctx, grad, state["momentum"], kept["how"], w, momentum, out, rows,
                                     space(layers.gns_orthogonal_update_workspace_bytes, width, rows))
        return [out, momentum]
    x1, x2, w = state["x1"], state["x2"], state["w"]
    out = empty("out", (x1.shape[0], w.shape[0]), state["dtype"])
    layers.gns_sage_dense_fp8(ctx, x1, x2, w, state["w_exponents"], state["bias"], state["relu"], out, x1.shape[0],
                              space(layers.gns_sage_dense_fp8_workspace_bytes, state["k"], x1.shape[0]))
    return out


def run(state):
    if own:
        return _run_own(state)
    kind = state["kind"]
    if kind == "norm":
        return _plain_norm(state)
    if kind == "norm_grad":
        return _plain_norm_grad(state)
    if kind == "update":
        return _plain_update(state)
    x = state["x1"] if state["x2"] is None else torch.cat([state["x1"], state["x2"]], 1)
    k = state["k"]
    w = _block_values(state["w"].view(torch.float8_e4m3fn).float(), state["w_exponents"][:, :(k + BLOCK - 1) // BLOCK].to(torch.int32) - 127, k)
    y = _block_values(*_plain_blocks(x.float()), k) @ w.t() + state["bias"]
    return (torch.clamp(y, min=0.0) if state["relu"] else y).to(state["dtype"])


# ---------------------------------------------------------------------------------------------------------------
def _pieces(rows, per_row):
    """Row ranges of at most 2^26 values: 64-bit copies of the large cases are made piece by piece."""
    step = max(1, (1 << 26) // per_row)
    return [(i, min(rows, i + step)) for i in range(0, rows, step)]


def _activation64(y, name):
    """Value and slope in 64 bits."""
    if name == "none":
        return y, torch.ones_like(y)
    if name == "relu":
        return y.relu(), (y > 0).double()
    if name == "silu":
        s = torch.sigmoid(y)
        return y * s, s + y * s * torch.sigmoid(-y)
    cdf = 0.5 * torch.erfc(-y / math.sqrt(2.0))
    return y * cdf, cdf + y * torch.exp(-y * y / 2.0) / math.sqrt(2.0 * math.pi)


def _exact_norm(state, case):
    x, groups = state["x"], case["groups"]
    rows, width = x.shape
    if state["offsets"] is None:
        index = torch.arange(rows, device="cuda:0") // case["segment_rows"]
    else:
        lengths = torch.tensor(state["offsets"], device="cuda:0").diff()
        index = torch.repeat_interleave(torch.arange(lengths.numel(), device="cuda:0"), lengths)
    count, per = state["count"], width // groups
    n = torch.bincount(index, minlength=count).double()[:, None].clamp(min=1) * per

    def sums(values):
        """Of a function's values (rows [a, b) -> [b - a, groups] each) by segment."""
        total = torch.zeros((count, groups), dtype=torch.float64, device="cuda:0")
        for a, b in _pieces(rows, width):
            total.index_add_(0, index[a:b], values(a, b))
        return total

    def grouped(t):
        return t.view(t.shape[0], groups, per)

    if case["kind"] == "norm":
        mean = sums(lambda a, b: grouped(x[a:b].double()).sum(2)) / n
        var = sums(lambda a, b: (grouped(x[a:b].double()) - mean[index[a:b], :, None]).square().sum(2)) / n
        rstd = torch.where(torch.bincount(index, minlength=count)[:, None] > 0, (var + EPS).rsqrt(), 0.0)
    else:
        mean, rstd = state["stats"][:, :, 0].double(), state["stats"][:, :, 1].double()
    gamma, beta = state["gamma"].double(), state["beta"].double()

    def normalised(a, b):
        i = index[a:b]
        return ((grouped(x[a:b].double()) - mean[i][:, :, None]) * rstd[i][:, :, None]).view(b - a, width)

    if case["kind"] == "norm":
        out = [_activation64(normalised(a, b) * gamma + beta, case["activation"])[0] for a, b in _pieces(rows, width)]
        return [torch.cat(out), torch.stack([mean, rstd], 2)]

    def through(a, b):
        xhat = normalised(a, b)
        return xhat, state["d_out"][a:b].double() * _activation64(xhat * gamma + beta, case["activation"])[1]

    dgamma, dbeta = (torch.zeros(width, dtype=torch.float64, device="cuda:0") for _ in range(2))
    for a, b in _pieces(rows, width):
        xhat, dy = through(a, b)
        dgamma += (dy * xhat).sum(0)
        dbeta += dy.sum(0)
    m1 = sums(lambda a, b: grouped(through(a, b)[1] * gamma).sum(2)) / n
    m2 = sums(lambda a, b: grouped(through(a, b)[0] * through(a, b)[1] * gamma).sum(2)) / n
    dx = []
    for a, b in _pieces(rows, width):
        xhat, dy = through(a, b)
        i = index[a:b]
        inner = grouped(dy * gamma) - m1[i][:, :, None] - grouped(xhat) * m2[i][:, :, None]
        dx.append((inner * rstd[i][:, :, None]).view(b - a, width))
    return [torch.cat(dx), dgamma, dbeta]


def exact(case, seed):
    state = prepare(case, seed)
    kind, rows = case["kind"], case["rows"]
    if kind in ("norm", "norm_grad"):
        return _exact_norm(state, case)
    if kind == "update":
        grad, old = state["grad"].double(), state["momentum"].double()
        momentum = grad + MU * old
        u = MU * momentum + grad if state["nesterov"] else momentum
        x = u / (torch.linalg.vector_norm(u) + 1e-7)
        wide = x.shape[0] <= x.shape[1]
        a, b, c = COEFFICIENTS
        for _ in range(STEPS):
            # from the side whose Gram matrix is the smaller one
            xt = x.t().contiguous()
            gram = x @ xt if wide else xt @ x
            poly = torch.addmm(b * gram, gram, gram, alpha=c)
            x = a * x + (poly @ x if wide else x @ poly)
        return [x if state["w"] is None else KEEP * state["w"].double() + RATE * x, momentum]
    k = state["k"]
    blocks = (k + BLOCK - 1) // BLOCK
    codes = torch.arange(256, device="cuda:0")
    sign, ex, fraction = codes >> 7, (codes >> 3) & 15, codes & 7
    magnitude = torch.where(ex == 0, fraction.double() / 8 * 2.0 ** -6, (1 + fraction.double() / 8) * torch.exp2((ex - 7).double()))
    table = torch.where(sign == 1, -magnitude, magnitude)
    scale = torch.exp2(state["w_exponents"][:, :blocks].double() - 127)
    w = (table[state["w"].long()] * scale.repeat_interleave(BLOCK, 1))[:, :k].t().contiguous()
    out = []
    for a, b in _pieces(rows, max(k, case["hdim"])):
        x = state["x1"][a:b].double()
        if state["x2"] is not None:
            x = torch.cat([x, state["x2"][a:b].double()], 1)
        x = torch.nn.functional.pad(x, (0, blocks * BLOCK - k)).view(b - a, blocks, BLOCK)
        largest = x.abs().max(2, keepdim=True).values
        power = torch.exp2(torch.ceil(torch.log2(largest.clamp(min=2.0 ** -101) / 464.0)))
        power = torch.where(largest > 464.0 * power, 2 * power, torch.where(largest <= 232.0 * power, power / 2, power))
        v = torch.where(largest < 2.0 ** -100, 0.0, x / power)
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        value = (torch.round(v / step) * step * power).view(b - a, blocks * BLOCK)[:, :k]
        y = value @ w + state["bias"].double()
        out.append(y.relu() if state["relu"] else y)
    return torch.cat(out)

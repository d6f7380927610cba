"""Cases of the operators around the update step to be timed: the update in 8-bit integers, activation checkpoints in
8 bits, the update's backward pass from such checkpoints, log probabilities of given classes and their gradient.

A case is a dict of plain values; "kind" names the operator:
  int8        rows x (f1 [+ f2]) of fp32 or bf16, quantised row by row, times an 8-bit weight matrix with a scale per output
              channel (laid out once), plus a bias: rows x hdim in the inputs' type
  checkpoint  rows x f1 saved in 8 bits with one power of two per 32 columns and a bit per positive value, and loaded again
  backward    gradients of the weights, the bias and the input of relu([x1 | x2] W + b), x1 and x2 from their checkpoints
  logprobs    log probability of each row's label, entropy, softmax statistics and the `top` best classes
  loss_grad   the gradient with respect to the logits, from those statistics

With `own` false everything is computed in plain torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

FLOAT = {"fp32": torch.float32, "bf16": torch.bfloat16}
GROUP = 32                      # columns that share a power of two in a checkpoint


def _int8(name, rows, f1, f2, hdim, dtype, relu=True):
    return dict(name=name, kind="int8", rows=rows, f1=f1, f2=f2, hdim=hdim, dtype=dtype, relu=relu)


def _checkpoint(name, rows, f1, dtype):
    return dict(name=name, kind="checkpoint", rows=rows, f1=f1, dtype=dtype)


def _backward(name, rows, f1, f2, hdim, dtype, relu=True):
    return dict(name=name, kind="backward", rows=rows, f1=f1, f2=f2, hdim=hdim, dtype=dtype, relu=relu)


def _logprobs(name, rows, classes, dtype, top):
    return dict(name=name, kind="logprobs", rows=rows, classes=classes, dtype=dtype, top=top)


def _loss_grad(name, rows, classes, dtype, entropy):
    return dict(name=name, kind="loss_grad", rows=rows, classes=classes, dtype=dtype, entropy=entropy)


def listed():
    return [
        # one row through a wide layer: answering one request, all of it reading weights
        _int8("int8-one-row", 1, 4096, 0, 4096, "bf16"),
        # the hidden layer of a mini-batch's input nodes (128 features, 256 hidden units)
        _int8("int8-hidden", 85_000, 128, 128, 256, "fp32"),
        # a long batch through a wide layer
        _int8("int8-wide", 8192, 8192, 0, 8192, "bf16", relu=False),
        # gathered rows of the products-shaped graph kept for the backward pass (100 features: the last group is short)
        _checkpoint("checkpoint-features", 168_003, 100, "fp32"),
        # activations of a wide layer
        _checkpoint("checkpoint-wide", 16_384, 4096, "bf16"),
        # backward pass of the hidden layer of a mini-batch
        _backward("backward-hidden", 85_000, 128, 128, 256, "fp32"),
        # backward pass of a wide layer in bf16
        _backward("backward-wide", 16_384, 4096, 0, 4096, "bf16", relu=False),
        # one answer over many classes, with alternatives
        _logprobs("logprobs-one-row", 1, 131_072, "fp32", 20),
        # all nodes of a large mini-batch over 172 classes
        _logprobs("logprobs-classes", 85_000, 172, "fp32", 5),
        # a long batch over very many classes, an odd number of them
        _logprobs("logprobs-many", 4096, 100_003, "bf16", 20),
        # the seeds of a mini-batch over 47 classes: latency
        _loss_grad("grad-seeds", 1000, 47, "fp32", False),
        # a long batch over very many classes, with an entropy term in the loss
        _loss_grad("grad-many", 4096, 100_003, "bf16", True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(("int8", "int8", "checkpoint", "backward", "backward", "logprobs", "logprobs", "loss_grad"))
    dtype = rng.choice(("fp32", "bf16"))
    rows = log_int(1, 100_000)
    if kind in ("int8", "backward"):
        # widths up to 8192 for the product, 4096 for the backward pass; the work stays below that of the wide cases
        most, room = (8192, 5e11) if kind == "int8" else (4096, 2.5e11)
        k, hdim = log_int(16, most), log_int(16, most)
        if rng.random() < 0.5:
            k, hdim = (1 << round(math.log2(v)) for v in (k, hdim))
        rows = max(1, min(rows, int(room / (k * hdim)), int(4e8 / max(k, hdim))))
        two = rng.random() < 0.5
        f1 = max(1, k // 2) if two else k
        make = _int8 if kind == "int8" else _backward
        case = make("", rows, f1, k - f1 if two else 0, hdim, dtype, rng.random() < 0.5)
    elif kind == "checkpoint":
        f1 = log_int(1, 8192)
        case = _checkpoint("", max(1, min(rows, 60_000_000 // f1)), f1, dtype)
    else:
        classes = log_int(2, 200_000)
        rows = max(1, min(rows, 400_000_000 // classes))
        if kind == "logprobs":
            case = _logprobs("", rows, classes, dtype, rng.choice((0, 1, 5, 10, 20, rng.randint(1, 32))))
        else:
            case = _loss_grad("", rows, classes, dtype, rng.random() < 0.5)
    del case["name"]
    return case


def work(case):
    size = 4 if case.get("dtype") == "fp32" else 2
    rows, kind = case["rows"], case["kind"]
    if kind == "int8":
        k, n = case["f1"] + case["f2"], case["hdim"]
        return {"bytes": rows * k * size + n * k + 8 * n + rows * n * size, "flops": 2 * rows * k * n}
    if kind == "checkpoint":
        groups = (case["f1"] + GROUP - 1) // GROUP
        packed = rows * (case["f1"] + groups + 4 * groups)
        return {"bytes": 2 * rows * case["f1"] * size + packed + packed - rows * 4 * groups, "flops": 0}
    if kind == "backward":
        k, n = case["f1"] + case["f2"], case["hdim"]
        groups = (k + GROUP - 1) // GROUP
        bits = rows * ((n + 31) // 32) * 4 if case["relu"] else 0
        return {"bytes": rows * n * size + bits + rows * (k + groups) + 2 * 4 * k * n + 4 * n + rows * k * size, "flops": 4 * rows * k * n}
    read = rows * case["classes"] * size
    if kind == "logprobs":
        return {"bytes": read + rows * (4 + 4 + 4 + 8 + 8 * case["top"]), "flops": 0}
    return {"bytes": 2 * read + rows * (4 + 4 + 8 + 4 + 4), "flops": 0}


# ---------------------------------------------------------------------------------------------------------------
# Plain forms.

def _plain_quantize(x):
    """int8 values (as fp32) and scales of the rows of x (fp32)."""
    amax = x.abs().amax(1, keepdim=True)
    inv = torch.where(amax >= 2.0 ** -120, 127.0 / amax, torch.zeros_like(amax))
    return torch.round(x * inv), torch.where(amax >= 2.0 ** -120, amax / 127.0, torch.zeros_like(amax))


def _two(e):
    """2^e in fp32 for integers -126 <= e <= 127; 0 for -127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _pack(x):
    """Checkpoint of x (fp32): int8 [rows, groups * 32] and exponent bytes [rows, groups], where 0 stands for no value but 0."""
    rows, dim = x.shape
    groups = (dim + GROUP - 1) // GROUP
    x = torch.nn.functional.pad(x, (0, groups * GROUP - dim)).view(rows, groups, GROUP)
    mantissa, exponent = torch.frexp(x.abs().amax(2))              # in [0.5, 1)
    e = exponent - 7 + (mantissa >= 127.5 / 128.0).to(exponent.dtype)
    e = torch.clamp(e, max=121)
    none = (mantissa == 0) | (exponent - 1 < -100)
    inverse = torch.where(none, torch.zeros_like(mantissa), _two(-e))
    q = torch.clamp(torch.round(x * inverse[:, :, None]), -127, 127).to(torch.int8).view(rows, groups * GROUP)
    return q, torch.where(none, torch.zeros_like(e), e + 127).to(torch.uint8)


def _unpack(q, exponents, dim):
    """fp32 values of a checkpoint."""
    rows, groups = exponents.shape
    return (q.view(rows, groups, GROUP).float() * _two(exponents.to(torch.int32) - 127)[:, :, None]).reshape(rows, groups * GROUP)[:, :dim]


def _positive(x):
    """Bit j of word g of a row: whether column 32 g + j is positive; int32 words."""
    rows, dim = x.shape
    groups = (dim + 31) // 32
    bits = torch.nn.functional.pad((x > 0).to(torch.int64), (0, groups * 32 - dim)).view(rows, groups, 32)
    words = (bits << torch.arange(32, device=x.device)).sum(2)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)


def _masked(dout, positive):
    """dout where the bits are set, 0 elsewhere (fp32)."""
    dout = dout.float()
    if positive is None:
        return dout
    shift = torch.arange(32, device=dout.device, dtype=torch.int32)
    bits = ((positive[:, :, None] >> shift) & 1).reshape(dout.shape[0], -1)[:, :dout.shape[1]]
    return torch.where(bits != 0, dout, torch.zeros_like(dout))


def _plain_top(z, k):
    """Indices of the k largest of each row of z (fp32), largest first, ties to the lowest index."""
    classes = z.shape[1]
    bits = (z + 0.0).view(torch.int32).to(torch.int64)
    order = torch.where(bits < 0, -1 - (bits & 0x7FFFFFFF), bits)
    key = (order << 32) | (classes - 1 - torch.arange(classes, device=z.device))
    return torch.topk(key, k, dim=1).indices


def _plain_logprobs(state):
    z, labels, top = state["logits"].float(), state["labels"].long(), state["top"]
    m = z.amax(1, keepdim=True)
    d = z - m
    p = torch.exp(d)
    total = p.sum(1)
    log_total = torch.log(total)
    terms = p * torch.where(p > 0, d, torch.zeros_like(d))
    entropy = log_total - terms.sum(1) / total
    at = d.gather(1, labels.clamp(min=0)[:, None])[:, 0] - log_total
    logp = torch.where(labels >= 0, at, torch.zeros_like(at))
    out = [logp, entropy, torch.stack([m[:, 0], log_total], 1)]
    if top:
        k = min(top, z.shape[1])
        index = _plain_top(z, k)
        value = d.gather(1, index) - log_total[:, None]
        # a class that is masked is no alternative, and a row has no more alternatives than classes
        gone = value == -math.inf
        index = torch.where(gone, torch.full_like(index, -1), index).to(torch.int32)
        out += [torch.nn.functional.pad(index, (0, top - k), value=-1), torch.nn.functional.pad(value, (0, top - k), value=-math.inf)]
    return out


def _plain_loss_grad(state):
    z, labels, stats = state["logits"].float(), state["labels"].long(), state["stats"]
    log_p = (z - stats[:, :1]) - stats[:, 1:]
    p = torch.exp(log_p)
    grad = -state["g_logp"][:, None] * p
    grad[labels < 0] = 0.0
    rows = torch.nonzero(labels >= 0)[:, 0]
    grad[rows, labels[rows]] += state["g_logp"][rows]
    if state["g_entropy"] is not None:
        weight = torch.where(p > 0, log_p + state["entropy"][:, None], torch.zeros_like(p))
        grad -= state["g_entropy"][:, None] * p * weight
    return grad.to(state["logits"].dtype)


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


def _features(rows, dim, gen, dtype):
    """Activations: magnitudes that differ from row to row and a few columns that stand out."""
    x = torch.randn((rows, dim), device="cuda:0", generator=gen)
    x *= torch.exp(0.5 * torch.randn((rows, 1), device="cuda:0", generator=gen))
    x *= torch.exp(0.7 * torch.randn((1, dim), device="cuda:0", generator=gen))
    return x.to(dtype)


def _logits(rows, classes, gen, dtype):
    """Scores with a few high ones a row; every sixteenth row has about half of its classes masked."""
    z = 2.0 * torch.randn((rows, classes), device="cuda:0", generator=gen)
    z += 3.0 * torch.randn((rows, 1), device="cuda:0", generator=gen)
    some = z[5::16]
    if some.numel():
        masked = torch.rand(some.shape, device="cuda:0", generator=gen) < 0.5
        masked[:, 0] = False
        some.masked_fill_(masked, -math.inf)
    return z.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda:0").manual_seed(int(seed))
    kind, rows = case["kind"], case["rows"]
    dtype = FLOAT[case["dtype"]]
    state = {"kind": kind, "kept": {}}

    def normal(*shape):
        return torch.randn(shape, device="cuda:0", generator=gen)

    if kind == "int8":
        f1, f2, n = case["f1"], case["f2"], case["hdim"]
        k = f1 + f2
        x = _features(rows, k, gen, dtype)
        state.update(x1=x[:, :f1].contiguous(), x2=x[:, f1:].contiguous() if f2 else None, k=k, relu=case["relu"], bias=normal(n))
        q, scale = _plain_quantize(normal(n, k) / math.sqrt(k))
        # weight rows are stored with a stride of a multiple of 64, zeros behind
        state.update(w=torch.nn.functional.pad(q, (0, -k % 64)).to(torch.int8), w_scale=scale[:, 0].contiguous(), dtype=dtype)
    elif kind == "checkpoint":
        state.update(x=_features(rows, case["f1"], gen, dtype))
    elif kind == "backward":
        f1, f2, n = case["f1"], case["f2"], case["hdim"]
        for name, f in (("one", f1), ("two", f2)):
            state[name] = _pack(_features(rows, f, gen, dtype).float()) if f else None
        state.update(f1=f1, f2=f2, w=normal(f1 + f2, n) / math.sqrt(f1 + f2),
                     dout=(1e-3 * normal(rows, n) * torch.exp(normal(rows, 1))).to(dtype),
                     positive=_positive(normal(rows, n)) if case["relu"] else None)
    else:
        classes = case["classes"]
        z = _logits(rows, classes, gen, dtype)
        labels = torch.randint(0, classes, (rows,), device="cuda:0", generator=gen, dtype=torch.int32)
        if rows > 1:
            labels[::16] = -1                                       # nodes without a label
        state.update(logits=z, labels=labels)
        if kind == "logprobs":
            state.update(top=case["top"])
        else:
            _, entropy, stats = _plain_logprobs(dict(logits=z, labels=labels, top=0))
            state.update(entropy=entropy, stats=stats, g_logp=-(0.5 + torch.rand(rows, device="cuda:0", generator=gen)) / rows,
                         g_entropy=0.01 * normal(rows) / rows if case["entropy"] else None)
    return state


def _run_own(state):
    from paper_2106_06150_amd import learn
    ctx, kind, kept = _context(), state["kind"], state["kept"]

    def empty(name, shape, dtype):
        """Output buffers and workspaces are a program's own and serve every pass."""
        if name not in kept:
            kept[name] = torch.empty(shape, dtype=dtype, device="cuda:0")
        return kept[name]

    if kind == "int8":
        x1, x2, w = state["x1"], state["x2"], state["w"]
        out = empty("out", (x1.shape[0], w.shape[0]), state["dtype"])
        if "workspace" not in kept:
            kept["workspace"] = learn.alloc_workspace(learn.gns_sage_dense_int8_workspace_bytes(ctx, state["k"], x1.shape[0]))
        learn.gns_sage_dense_int8(ctx, x1, x2, w, state["w_scale"], state["bias"], state["relu"], out, x1.shape[0], kept["workspace"])
        return out
    if kind == "checkpoint":
        x = state["x"]
        rows, dim = x.shape
        groups = (dim + GROUP - 1) // GROUP
        q, e = empty("q", (rows, groups * GROUP), torch.int8), empty("e", (rows, groups), torch.uint8)
        positive = empty("positive", (rows, groups), torch.int32)
        out = empty("out", (rows, dim), x.dtype)
        learn.gns_checkpoint_save(ctx, x, q, e, positive, rows)
        learn.gns_checkpoint_load(ctx, q, e, out, rows)
        return [out, positive]
    if kind == "backward":
        dout, w = state["dout"], state["w"]
        rows, f1, f2 = dout.shape[0], state["f1"], state["f2"]
        dw, db = empty("dw", w.shape, torch.float32), empty("db", (w.shape[1],), torch.float32)
        dx = empty("dx", (rows, f1 + f2), dout.dtype)
        if "workspace" not in kept:
            kept["workspace"] = learn.alloc_workspace(learn.gns_sage_dense_backward_workspace_bytes(ctx, f1, f2, w.shape[1], rows))
        learn.gns_sage_dense_backward(ctx, dout, state["positive"], state["one"], f1, state["two"], f2, w, dw, db, dx, rows, kept["workspace"])
        return [dw, db, dx]
    z, labels = state["logits"], state["labels"]
    rows, classes = z.shape
    if kind == "logprobs":
        top = state["top"]
        logp, entropy = empty("logp", (rows,), torch.float32), empty("entropy", (rows,), torch.float32)
        stats = empty("stats", (rows, 2), torch.float32)
        index = empty("index", (rows, top), torch.int32) if top else None
        value = empty("value", (rows, top), torch.float32) if top else None
        if "workspace" not in kept:
            kept["workspace"] = learn.alloc_workspace(learn.gns_log_probs_workspace_bytes(ctx, classes, top, rows))
        learn.gns_log_probs(ctx, z, labels, logp, entropy, stats, index, value, rows, kept["workspace"])
        return [logp, entropy, stats] + ([index, value] if top else [])
    out = empty("out", (rows, classes), z.dtype)
    learn.gns_log_probs_backward(ctx, z, labels, state["stats"], state["entropy"], state["g_logp"], state["g_entropy"], out, rows)
    return out


def run(state):
    if own:
        return _run_own(state)
    kind = state["kind"]
    if kind == "int8":
        x = state["x1"] if state["x2"] is None else torch.cat([state["x1"], state["x2"]], 1)
        q, scale = _plain_quantize(x.float())
        y = q @ state["w"][:, :state["k"]].float().t()
        y = y * scale * state["w_scale"] + state["bias"]
        return (torch.clamp(y, min=0.0) if state["relu"] else y).to(state["dtype"])
    if kind == "checkpoint":
        x = state["x"].float()
        q, e = _pack(x)
        return [_unpack(q, e, x.shape[1]).to(state["x"].dtype), _positive(x)]
    if kind == "backward":
        dz = _masked(state["dout"], state["positive"])
        x = _unpack(*state["one"], state["f1"])
        if state["two"] is not None:
            x = torch.cat([x, _unpack(*state["two"], state["f2"])], 1)
        return [x.t() @ dz, dz.sum(0), (dz @ state["w"].t()).to(state["dout"].dtype)]
    return _plain_logprobs(state) if kind == "logprobs" else _plain_loss_grad(state)


# ---------------------------------------------------------------------------------------------------------------
def _slices(rows, per_row):
    """Row ranges of at most 2^26 values: 64-bit copies of the large cases are made piece by piece."""
    step = max(1, (1 << 26) // per_row)
    return [(i, min(rows, i + step)) for i in range(0, rows, step)]


def _power64(e):
    return ((e + 1023) << 52).view(torch.float64)


def _checkpoint_values64(packed, dim):
    q, e = packed
    power = _power64(e.long() - 127)
    power[e == 0] = 0.0
    return (q.double() * power.repeat_interleave(GROUP, 1))[:, :dim]


def exact(case, seed):
    state = prepare(case, seed)
    kind, rows = case["kind"], case["rows"]
    if kind == "int8":
        w = state["w"][:, :state["k"]].double() * state["w_scale"].double()[:, None]
        out = []
        for a, b in _slices(rows, max(state["k"], case["hdim"])):
            x = state["x1"][a:b].double()
            if state["x2"] is not None:
                x = torch.cat([x, state["x2"][a:b].double()], 1)
            largest = x.abs().max(1, keepdim=True).values
            keep = largest >= 2.0 ** -120
            rounded = torch.where(keep, torch.round(x * 127.0 / largest), 0.0)
            y = (rounded @ w.t()) * (largest / 127.0) + state["bias"].double()
            out.append(y.relu() if state["relu"] else y)
        return torch.cat(out)
    if kind == "checkpoint":
        out = []
        groups = (case["f1"] + GROUP - 1) // GROUP
        for a, b in _slices(rows, groups * GROUP):
            x = torch.zeros((b - a, groups * GROUP), dtype=torch.float64, device="cuda:0")
            x[:, :case["f1"]] = state["x"][a:b].double()
            x = x.view(b - a, groups, GROUP)
            largest = x.abs().max(2, keepdim=True).values
            # the smallest power of two whose 127.5-fold exceeds the largest magnitude of the group
            power = torch.floor(torch.log2(largest.clamp(min=2.0 ** -101) / 127.5)).long()
            power = torch.where(largest < 127.5 * _power64(power), power, power + 1).clamp(max=121)
            steps = torch.round(x / _power64(power)).clamp(-127, 127)
            steps = torch.where(largest < 2.0 ** -100, 0.0, steps)
            out.append((steps * _power64(power)).view(b - a, groups * GROUP)[:, :case["f1"]])
        return [torch.cat(out), None]
    if kind == "backward":
        w = state["w"].double()
        dw = torch.zeros(w.shape, dtype=torch.float64, device="cuda:0")
        db = torch.zeros(w.shape[1], dtype=torch.float64, device="cuda:0")
        dx = []
        for a, b in _slices(rows, max(w.shape)):
            dz = state["dout"][a:b].double()
            if state["positive"] is not None:
                word = state["positive"][a:b].repeat_interleave(32, 1)[:, :w.shape[1]]
                dz = dz * ((word >> (torch.arange(w.shape[1], device="cuda:0", dtype=torch.int32) % 32)) & 1)
            parts = [_checkpoint_values64((p[0][a:b], p[1][a:b]), f) for p, f in ((state["one"], case["f1"]), (state["two"], case["f2"])) if p is not None]
            dw += torch.cat(parts, 1).t().contiguous() @ dz
            db += dz.sum(0)
            dx.append(dz @ w.t().contiguous())
        return [dw, db, torch.cat(dx)]
    labels = state["labels"].long()
    pieces = []
    for a, b in _slices(rows, case["classes"]):
        z, y = state["logits"][a:b].double(), labels[a:b]
        index = torch.arange(b - a, device="cuda:0")
        if kind == "logprobs":
            log_p = torch.log_softmax(z, 1)
            p = log_p.exp()
            highest = z.max(1).values
            piece = [torch.where(y >= 0, log_p[index, y.clamp(min=0)], 0.0), -torch.special.xlogy(p, p).sum(1),
                     torch.stack([highest, torch.logsumexp(z, 1) - highest], 1)]
            if case["top"]:
                k = min(case["top"], case["classes"])
                best = torch.full((b - a, case["top"]), -math.inf, dtype=torch.float64, device="cuda:0")
                best[:, :k] = torch.topk(log_p, k, 1).values
                piece += [best]
        else:
            norm = (state["stats"][a:b, 0].double() + state["stats"][a:b, 1].double())[:, None]
            p = torch.exp(z - norm)
            g = torch.where(y >= 0, state["g_logp"][a:b].double(), 0.0)
            grad = -g[:, None] * p
            grad[index, y.clamp(min=0)] += g
            if state["g_entropy"] is not None:
                grad -= state["g_entropy"][a:b].double()[:, None] * (torch.special.xlogy(p, p) + p * state["entropy"][a:b].double()[:, None])
            piece = [grad]
        pieces.append(piece)
    whole = [torch.cat(c) for c in zip(*pieces)]
    if kind == "loss_grad":
        return whole[0]
    return whole[:3] + ([None, whole[3]] if case["top"] else [])

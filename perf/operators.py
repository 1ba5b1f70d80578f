"""The calls around a compressed gradient in a training step of a language model, over the sizes they come in: the
embedding's lookup and its gradient (what a sender compresses begins there), and the orthogonalised update of weight
matrices from the gradient that a receiver leaves.

A case is a dict of plain values.  Its "call" says which operator one pass goes through:

  "embedding"  out[t] = scale * table[tokens[t]]; a token outside the table (padding is -1) gives a row of zeros.
  "gradient"   out[v] = base[v] + scale * (sum of grad[t] over the t with tokens[t] == v); without a base, 0 instead.
  "orthogonal" every matrix G of a list: X = G / (|G|_F + eps), then five times X <- a X + (b A + c A A) X with
               A = X X^T (on the transposed matrix where it is taller than wide); out = gain * X.
  "step"       the same on momentum: M <- beta M + G, U = G + beta M, O = the above of U,
               W <- (1 - lr decay) W - lr gain O, for the matrices of a flat gradient, momentum and weight vector.

Where `own` is true, run() makes the framework's calls; otherwise it computes the same with elementary torch operations.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
COEFFICIENTS = [(3.4445, -4.7750, 2.0315)] * 5
EPS = 1e-7
LR, BETA, DECAY = 0.02, 0.95, 0.1


def listed():
    return [
        # Serving: the newest token of one sequence.
        {"name": "lookup_one_token", "call": "embedding", "rows": 32000, "width": 1024, "tokens": 1, "index": 64,
         "type": "bf16", "out": "bf16", "padding": 0.0},
        # Odd sizes in 32 bits, a fifth of the batch is padding.
        {"name": "lookup_odd", "call": "embedding", "rows": 10007, "width": 771, "tokens": 4099, "index": 32,
         "type": "fp32", "out": "fp32", "padding": 0.2},
        # A training batch from a table in 32 bits into activations in 16.
        {"name": "lookup_batch", "call": "embedding", "rows": 50000, "width": 2048, "tokens": 16384, "index": 64,
         "type": "fp32", "out": "bf16", "padding": 0.0},
        # A small table's gradient, odd sizes: latency.
        {"name": "gradient_small", "call": "gradient", "rows": 5003, "width": 257, "tokens": 700, "index": 64,
         "type": "fp32", "out": "fp32", "padding": 0.0, "base": False},
        # A training batch's gradient into the flat gradient in 32 bits: most rows of the table have no token.
        {"name": "gradient_batch", "call": "gradient", "rows": 50000, "width": 2048, "tokens": 8192, "index": 64,
         "type": "bf16", "out": "fp32", "padding": 0.0, "base": False},
        # Many short sequences, padded, on a table that the output's product shares: its gradient is added.  The most
        # frequent token has thousands of places.
        {"name": "gradient_shared_table", "call": "gradient", "rows": 32000, "width": 768, "tokens": 65536, "index": 32,
         "type": "bf16", "out": "fp32", "padding": 0.3, "base": True},
        # Two small matrices, odd sizes: latency.
        {"name": "orthogonal_small", "call": "orthogonal", "count": 2, "height": 193, "breadth": 317, "type": "fp16"},
        # The square projections of a layer or two.
        {"name": "orthogonal_square", "call": "orthogonal", "count": 8, "height": 1024, "breadth": 1024, "type": "bf16"},
        # Tall matrices, as of a feed-forward block.
        {"name": "orthogonal_tall", "call": "orthogonal", "count": 4, "height": 4096, "breadth": 1024, "type": "fp32"},
        # The matrices of the repository's three smaller networks, their convolutions' kernels as one row per output channel:
        # many small ones (latency),
        {"name": "step_resnet20", "call": "step", "shapes": "resnet20", "count": 0, "height": 0, "breadth": 0, "type": "fp32"},
        # fifty-four of all sizes, weights in 16 bits,
        {"name": "step_resnet50", "call": "step", "shapes": "resnet50", "count": 0, "height": 0, "breadth": 0, "type": "bf16"},
        # and a few with most of the work in two of them: the largest.
        {"name": "step_alexnet", "call": "step", "shapes": "alexnet", "count": 0, "height": 0, "breadth": 0, "type": "fp32"},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    call = rng.choice(["embedding", "gradient", "gradient", "orthogonal", "orthogonal", "step"])
    if call in ("embedding", "gradient"):
        rows = _log_uniform(rng, 1000, 131072)
        case = {"call": call, "rows": rows, "width": _log_uniform(rng, 64, min(8192, (1 << 28) // rows)),
                "tokens": _log_uniform(rng, 1, 65536), "index": rng.choice([32, 64]), "type": rng.choice(["fp32", "bf16", "fp16"]),
                "out": rng.choice(["fp32", "fp32", "bf16"]), "padding": rng.choice([0.0, 0.0, round(rng.uniform(0.0, 0.9), 2)])}
        if rng.random() < 0.5:
            case["width"] = (case["width"] + 63) // 64 * 64
        case["tokens"] = min(case["tokens"], (1 << 28) // case["width"])
        if call == "gradient":
            case["base"] = rng.random() < 0.4
        return case
    height, breadth = _log_uniform(rng, 16, 4096), _log_uniform(rng, 16, 4096)
    if rng.random() < 0.5:
        height, breadth = (height + 63) // 64 * 64, (breadth + 63) // 64 * 64
    case = {"call": call, "count": _log_uniform(rng, 1, 24), "height": height, "breadth": breadth,
            "type": rng.choice(["fp32", "bf16", "fp16"])}
    most = work(listed()[-1])["flops"]
    while case["count"] > 1 and work(case)["flops"] > most:
        case["count"] //= 2
    if call == "step":
        case["shapes"] = ""
        case["type"] = rng.choice(["fp32", "bf16"])
    return case


def _resnet20():
    got, cin = [(16, 27)], 16
    for cout in (16, 32, 64):
        for _ in range(3):
            got += [(cout, cin * 9), (cout, cout * 9)]
            cin = cout
    return got + [(10, 64)]


def _resnet50():
    got, cin = [(64, 147)], 64
    for width, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
        for b in range(blocks):
            got += [(width, cin), (width, width * 9), (4 * width, width)]
            if b == 0:
                got.append((4 * width, cin))
            cin = 4 * width
    return got + [(1000, 2048)]


def _alexnet():
    return [(96, 363), (256, 2400), (384, 2304), (384, 3456), (256, 3456), (4096, 9216), (4096, 4096), (1000, 4096)]


def _shapes(case):
    """(height, breadth) of every matrix, in the order they lie behind each other in the flat vectors."""
    known = {"resnet20": _resnet20, "resnet50": _resnet50, "alexnet": _alexnet}
    return known[case["shapes"]]() if case.get("shapes") else [(case["height"], case["breadth"])] * case["count"]


def _gain(height, breadth):
    return math.sqrt(max(1.0, height / breadth))


def _gradient_like(height, breadth, gen):
    """A weight matrix's gradient: a sum of a few outer products of falling size, and noise."""
    r = max(1, min(height, breadth) // 8)
    size = torch.arange(1, r + 1, device="cuda", dtype=torch.float32).pow_(-0.7)
    left = torch.randn(height, r, device="cuda", generator=gen).mul_(size)
    right = torch.randn(r, breadth, device="cuda", generator=gen)
    return (left @ right).add_(torch.randn(height, breadth, device="cuda", generator=gen), alpha=0.5).mul_(1e-3)


def _tokens(case, gen):
    """Falling frequencies, as words have: the v-th row is met about 1 / v as often as the first."""
    t = torch.rand(case["tokens"], device="cuda", generator=gen, dtype=torch.float64).mul_(math.log(case["rows"] + 1)).exp_()
    t = t.long().sub_(1).clamp_(0, case["rows"] - 1)
    order = torch.randperm(case["rows"], device="cuda", generator=gen)
    t = order[t]
    if case["padding"]:
        t[torch.rand(case["tokens"], device="cuda", generator=gen) < case["padding"]] = -1
    return t.to(torch.int32 if case["index"] == 32 else torch.int64)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"case": case}
    if case["call"] in ("embedding", "gradient"):
        st["tokens"] = _tokens(case, gen)
        st["scale"] = math.sqrt(case["width"]) if case["call"] == "embedding" else 1.0
        tall = case["rows"] if case["call"] == "embedding" else case["tokens"]
        st["source"] = torch.randn(tall, case["width"], device="cuda", generator=gen).mul_(0.02).to(TYPES[case["type"]])
        deep = case["tokens"] if case["call"] == "embedding" else case["rows"]
        st["out"] = torch.empty(deep, case["width"], device="cuda", dtype=TYPES[case["out"]])
        if case.get("base"):
            st["base"] = torch.randn(deep, case["width"], device="cuda", generator=gen).mul_(0.02).to(TYPES[case["out"]])
        if own and case["call"] == "gradient":
            from paper_1811_08596_amd import fftsp
            st["workspace"] = torch.empty(fftsp.workspace_bytes_embedding(case["rows"], case["width"], case["tokens"]),
                                          dtype=torch.uint8, device="cuda")
        return st
    st["shapes"] = _shapes(case)
    grad = torch.cat([_gradient_like(h, w, gen).reshape(-1) for h, w in st["shapes"]])
    if case["call"] == "step":
        st["grad"] = grad
        st["momentum"] = torch.cat([_gradient_like(h, w, gen).reshape(-1) for h, w in st["shapes"]])
        st["weights"] = torch.randn(grad.numel(), device="cuda", generator=gen).mul_(0.02).to(TYPES[case["type"]])
        st["momentum_out"], st["weights_out"] = torch.empty_like(st["momentum"]), torch.empty_like(st["weights"])
    else:
        st["grad"] = grad.to(TYPES[case["type"]])
        st["out"] = torch.empty_like(st["grad"])
    if own:                                  # the list of matrices and the workspace, which a user's program keeps
        from paper_1811_08596_amd import fftsp
        at, listing = 0, []
        for h, w in st["shapes"]:
            listing.append(fftsp.Matrix(at, h, w, w, _gain(h, w)))
            at += h * w
        st["matrices"] = fftsp.matrices(listing)
        st["workspace"] = torch.empty(fftsp.workspace_bytes_orthogonal(st["matrices"]), dtype=torch.uint8, device="cuda")
    return st


def _orthogonal(g):
    """Newton-Schulz on the last two axes."""
    x = g.float()
    turned = x.shape[-2] > x.shape[-1]
    if turned:
        x = x.transpose(-2, -1)
    norm = x.double().square().sum((-2, -1), keepdim=True).sqrt()
    x = x / (norm + EPS).float()
    for a, b, c in COEFFICIENTS:
        gram = x @ x.transpose(-2, -1)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(-2, -1) if turned else x


def _run_plain(st):
    case = st["case"]
    if case["call"] == "embedding":
        inside = (st["tokens"] >= 0) & (st["tokens"] < case["rows"])
        rows = st["source"][torch.where(inside, st["tokens"], 0)].float() * st["scale"]
        st["out"].copy_(torch.where(inside[:, None], rows, 0.0))
        return st["out"]
    if case["call"] == "gradient":
        inside = (st["tokens"] >= 0) & (st["tokens"] < case["rows"])
        total = torch.zeros(case["rows"], case["width"], device="cuda")
        total.index_add_(0, torch.where(inside, st["tokens"], 0), torch.where(inside[:, None], st["source"].float(), 0.0))
        total.mul_(st["scale"])
        st["out"].copy_(total + st["base"].float() if case["base"] else total)
        return st["out"]
    if case["call"] == "orthogonal":         # equal shapes: one batch
        h, w = st["shapes"][0]
        st["out"].view(-1, h, w).copy_(_gain(h, w) * _orthogonal(st["grad"].view(-1, h, w)))
        return st["out"]
    torch.add(st["grad"], st["momentum"], alpha=BETA, out=st["momentum_out"])
    update = st["grad"] + BETA * st["momentum_out"]
    at = 0
    for h, w in st["shapes"]:                # a matrix at a time: their shapes differ
        part = slice(at, at + h * w)
        o = _orthogonal(update[part].view(h, w)).reshape(-1)
        st["weights_out"][part] = ((1.0 - LR * DECAY) * st["weights"][part].float() - LR * _gain(h, w) * o).to(st["weights"].dtype)
        at += h * w
    return {"momentum": st["momentum_out"], "weights": st["weights_out"]}


def _run_own(st):
    from paper_1811_08596_amd import fftsp
    case = st["case"]
    if case["call"] == "embedding":
        fftsp.embedding(st["source"], st["tokens"], st["out"], scale=st["scale"])
        return st["out"]
    if case["call"] == "gradient":
        fftsp.embedding_gradient(st["source"], st["tokens"], st["out"], st["workspace"], scale=st["scale"], base=st.get("base"))
        return st["out"]
    if case["call"] == "orthogonal":
        fftsp.orthogonal(st["grad"], st["out"], st["matrices"], st["workspace"], eps=EPS)
        return st["out"]
    fftsp.orthogonal_step(st["grad"], st["momentum"], st["weights"], st["matrices"], st["workspace"], lr=LR, beta=BETA,
                          weight_decay=DECAY, eps=EPS, momentum_out=st["momentum_out"], weights_out=st["weights_out"])
    return {"momentum": st["momentum_out"], "weights": st["weights_out"]}


def run(st):
    return _run_own(st) if own else _run_plain(st)


def work(case):
    """Bytes: every input read and every output written once.  Operations of the iteration on n x m matrices, n <= m: the
    products with symmetric results are counted by half, and the five steps by their least form, which keeps to n x n
    products between one n x n product of the matrix with itself and one of the whole polynomial with the matrix."""
    if case["call"] in ("embedding", "gradient"):
        t, d, v = case["tokens"], case["width"], case["rows"]
        read = t * case["index"] // 8 + (min(t, v) if case["call"] == "embedding" else t) * d * BYTES[case["type"]]
        written = (t if case["call"] == "embedding" else v) * d * BYTES[case["out"]]
        return {"bytes": read + written * (2 if case.get("base") else 1), "flops": t * d}
    flops = values = 0
    for h, w in _shapes(case):
        n, m = min(h, w), max(h, w)
        values += n * m
        flops += 3 * n * n * m + (4 * len(COEFFICIENTS) - 3) * n ** 3
    each = 12 + 2 * BYTES[case["type"]] if case["call"] == "step" else 2 * BYTES[case["type"]]
    return {"bytes": values * each, "flops": flops}


def _exact_orthogonal(g):
    """In 64 bits, with the update written as a polynomial in the Gram matrix that multiplies X once."""
    tall = g.size(0) > g.size(1)
    x = g.t().contiguous() if tall else g
    x = x / (torch.linalg.vector_norm(x) + EPS)
    one = torch.eye(x.size(0), dtype=torch.float64, device=x.device)
    for a, b, c in COEFFICIENTS:
        s = torch.mm(x, x.t())
        x = torch.mm(torch.addmm(a * one, s, b * one + c * s), x)
    return x.t() if tall else x


def exact(case, seed):
    st = prepare(case, seed)
    if case["call"] == "embedding":
        table = torch.cat([st["source"].double(), torch.zeros(1, case["width"], dtype=torch.float64, device="cuda")])
        at = st["tokens"].long()
        at[(at < 0) | (at >= case["rows"])] = case["rows"]
        return table.index_select(0, at).mul_(st["scale"])
    if case["call"] == "gradient":
        order = torch.argsort(st["tokens"].long(), stable=True)
        at, start = torch.unique_consecutive(st["tokens"].long()[order], return_counts=True)
        ends = torch.cumsum(start, 0)
        out = st["base"].double() if case["base"] else torch.zeros(case["rows"], case["width"], dtype=torch.float64, device="cuda")
        for c in range(0, case["width"], 256):   # running sums in 64 bits, and their differences at the ends of every token's run
            sums = torch.cumsum(st["source"][:, c:c + 256][order].double(), 0)[ends - 1]
            sums[1:] -= sums[:-1].clone()
            fits = (at >= 0) & (at < case["rows"])
            out[at[fits], c:c + 256] += st["scale"] * sums[fits]
        return out
    if case["call"] == "orthogonal":
        h, w = st["shapes"][0]
        return torch.cat([_gain(h, w) * _exact_orthogonal(g.view(h, w)).reshape(-1) for g in st["grad"].double().view(-1, h * w)])
    momentum = BETA * st["momentum"].double() + st["grad"].double()
    update = st["grad"].double() + BETA * momentum
    weights, at = [], 0
    for h, w in st["shapes"]:
        o = _exact_orthogonal(update[at:at + h * w].view(h, w)).reshape(-1)
        weights.append((1 - LR * DECAY) * st["weights"][at:at + h * w].double() - LR * _gain(h, w) * o)
        at += h * w
    return {"momentum": momentum, "weights": torch.cat(weights)}

"""The losses over a large vocabulary, as cases that a timer can prepare and run.

Three operators of `paper_2007_10412_amd.binding`, for training (the loss with its gradients) and for answering (what a
token costs, forward only):

    rad_linear_ce       softmax cross entropy of a linear layer's outputs, which are never kept whole
    rad_linear_distill  the same layer against the most likely tokens of a teacher
    rad_distill_ce      that loss of logits that the caller has in hand

    listed()            the fixed cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a program has in hand before the call, on the GPU
    run(state)          one pass; returns its outputs
    work(case)          bytes and operations one pass cannot do without
    exact(case, seed)   the outputs by the operators' definition, in 64 bits

`own` false: elementary torch operations in fp32, rounded once at the end.  `own` true: the library's calls.
"""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # The last layer and the loss of the small MNIST network (784-300-300-10), fp32 with biases: launches are all
        # there is.
        {"name": "ce_step_150x300x10_f32", "op": "linear_ce", "dtype": "f32", "rows": 150, "d_in": 300, "classes": 10,
         "train": True, "bias": True, "ignored": 0.0},
        # The last layer and the loss of the wide bf16 network (4096-4096-4096-1000) that the benchmark trains.
        {"name": "ce_step_4096x4096x1000_bf16", "op": "linear_ce", "dtype": "bf16", "rows": 4096, "d_in": 4096,
         "classes": 1000, "train": True, "bias": False, "ignored": 0.0},
        # The head of a language model in training: a large vocabulary over a batch of 4096 tokens.
        {"name": "ce_step_4096x4096x128000_bf16", "op": "linear_ce", "dtype": "bf16", "rows": 4096, "d_in": 4096,
         "classes": 128000, "train": True, "bias": False, "ignored": 0.0},
        # A vocabulary and a packed batch of odd lengths, a third of its tokens belonging to prompts that are not trained on.
        {"name": "ce_step_1999x1000x50257_bf16", "op": "linear_ce", "dtype": "bf16", "rows": 1999, "d_in": 1000,
         "classes": 50257, "train": True, "bias": False, "ignored": 0.33},
        # A character or byte-pair model trained in fp32, biases included.
        {"name": "ce_step_1024x512x8003_f32", "op": "linear_ce", "dtype": "f32", "rows": 1024, "d_in": 512, "classes": 8003,
         "train": True, "bias": True, "ignored": 0.1},
        # One answered token's log-probability: the weights are read once, for one row.
        {"name": "ce_score_1x4096x128000_bf16", "op": "linear_ce", "dtype": "bf16", "rows": 1, "d_in": 4096,
         "classes": 128000, "train": False, "bias": False, "ignored": 0.0},
        # The log-probabilities of a whole answer of 300 tokens.
        {"name": "ce_score_300x2048x32000_bf16", "op": "linear_ce", "dtype": "bf16", "rows": 300, "d_in": 2048,
         "classes": 32000, "train": False, "bias": True, "ignored": 0.0},
        # Distillation of a student whose logits are there already, a batch of tokens.
        {"name": "distill_4096x32000_bf16_k64", "op": "distill", "dtype": "bf16", "rows": 4096, "classes": 32000, "k": 64,
         "temperature": 1.0, "missing": 0.0},
        # A few tokens of a large vocabulary: the rows have to be shared by the chip.
        {"name": "distill_4x128000_f32_k128", "op": "distill", "dtype": "f32", "rows": 4, "classes": 128000, "k": 128,
         "temperature": 2.0, "missing": 0.0},
        # Odd rows, whose teacher's lists end early (some are empty).
        {"name": "distill_777x50257_bf16_k20", "op": "distill", "dtype": "bf16", "rows": 777, "classes": 50257, "k": 20,
         "temperature": 1.5, "missing": 0.3},
        # The same loss with the head in it: a language model that learns from a larger one's stored top tokens.
        {"name": "linear_distill_4096x2048x32000_bf16_k32", "op": "linear_distill", "dtype": "bf16", "rows": 4096,
         "d_in": 2048, "classes": 32000, "k": 32, "temperature": 1.0, "missing": 0.0, "bias": False},
        # A small fp32 student with a bias and short lists.
        {"name": "linear_distill_200x768x10007_f32_k16", "op": "linear_distill", "dtype": "f32", "rows": 200, "d_in": 768,
         "classes": 10007, "k": 16, "temperature": 2.0, "missing": 0.2, "bias": True},
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of the range: as it comes, or (every other time) a multiple of a power of two."""
    n = _log_between(rng, lo, hi)
    if rng.random() < 0.5:
        unit = 1 << rng.randint(3, 7)
        n = max(lo, min(hi, (n + unit - 1) // unit * unit))
    return n


def draw(rng):
    op = rng.choice(["linear_ce", "linear_ce", "distill", "linear_distill"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    while True:
        case = {"op": op, "dtype": dtype, "rows": _size(rng, 1, 8192), "classes": _size(rng, 1000, 131072)}
        if op == "distill":
            if case["rows"] * case["classes"] > 4096 * 32000:
                continue
        else:
            case["d_in"] = _size(rng, 256, 4096)
            most = 4096 * 4096 * 128000 // (16 if dtype == "f32" else 1)
            if case["rows"] * case["d_in"] * case["classes"] > most:
                continue
        break
    if op == "linear_ce":
        # (the bias gradient is a sum in fp32 of what the layer's type rounds, so bf16 training is drawn without one)
        case["train"] = rng.random() < 0.7
        case["bias"] = rng.random() < 0.5 and (dtype == "f32" or not case["train"])
        case["ignored"] = rng.choice([0.0, 0.0, 0.2, 0.6])
    else:
        case["k"] = _log_between(rng, 1, 256)
        case["temperature"] = rng.choice([1.0, 1.0, 0.7, 2.0, 4.0])
        case["missing"] = rng.choice([0.0, 0.0, 0.3])
        if op == "linear_distill":
            case["bias"] = rng.random() < 0.5 and dtype == "f32"
    return case


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, classes, dtype = case["rows"], case["classes"], TORCH[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def numbers(high, *shape):
        return torch.randint(0, high, shape, device="cuda", generator=gen)

    state = {"case": case}
    # logits with a standard deviation of 3: some tokens are a thousand times as likely as others
    if case["op"] == "distill":
        state["logits"] = (3.0 * normal(rows, classes)).to(dtype)
    else:
        d_in = case["d_in"]
        state["x"] = normal(rows, d_in).to(dtype)
        state["W"] = (normal(d_in, classes) * (3.0 / math.sqrt(d_in))).to(dtype)
        state["bias"] = normal(classes) if case["bias"] else None
    if case["op"] == "linear_ce":
        labels = numbers(classes, rows)
        if case["ignored"]:
            # sequences of 64 tokens whose first part is a prompt, of one length or another; the last token is an answer's
            at = torch.arange(rows, device="cuda")
            share = torch.rand((rows + 63) // 64, device="cuda", generator=gen) * 2 * case["ignored"]
            prompt = ((at % 64).float() < 64 * share[at // 64]) & (at < rows - 1)
            labels = torch.where(prompt, torch.full_like(labels, -1), labels)
        state["labels"] = labels.to(torch.int32)
    else:
        # a teacher's likeliest tokens, best first: as many different ones as the list is long
        k = case["k"]
        first = numbers(classes, rows, 1)
        index = (first + torch.arange(k, device="cuda") * (classes // k)) % classes
        logit = (3.0 + 3.0 * normal(rows, k)).sort(dim=1, descending=True).values
        if case["missing"]:
            length = (torch.rand(rows, 1, device="cuda", generator=gen) * (1.0 + case["missing"]) - case["missing"]).clamp(0.0, 1.0)
            index = torch.where(torch.arange(k, device="cuda") < torch.ceil(length * k), index, torch.full_like(index, -1))
        state["index"], state["logit"] = index.to(torch.int32), logit
    return state


_contexts = {}


def _context():
    """The context that a program makes once and keeps (on the default stream)."""
    from paper_2007_10412_amd import binding as B
    if "default" not in _contexts:
        _contexts["default"] = B.rad_ctx_create()
    return B, _contexts["default"]


def _run_own(state):
    B, ctx = _context()
    case = state["case"]
    f32 = dict(device="cuda", dtype=torch.float32)
    kind = B.RAD_F32 if case["dtype"] == "f32" else B.RAD_BF16
    if case["op"] == "distill":
        out = {"row_loss": torch.empty(case["rows"], **f32), "loss": torch.empty(1, **f32),
               "dlogits": torch.empty_like(state["logits"])}
        teacher = B.make_teacher(state["index"], state["logit"], case["temperature"])
        B.rad_distill_ce(ctx, state["logits"], teacher, kind, out["dlogits"], row_loss=out["row_loss"], loss=out["loss"])
        return out
    layer = B.make_layer(case["rows"], case["d_in"], case["classes"], dtype=kind, relu=False, has_bias=case["bias"])
    out = {"row_loss": torch.empty(case["rows"], **f32), "loss": torch.empty(1, **f32)}
    if case.get("train", True):
        out["dX"], out["dW"] = torch.empty_like(state["x"]), torch.empty_like(state["W"])
        if case["bias"]:
            out["dbias"] = torch.empty(case["classes"], **f32)
    if case["op"] == "linear_ce":
        B.rad_linear_ce(ctx, layer, state["x"], state["W"], state["bias"], state["labels"], **out)
    else:
        teacher = B.make_teacher(state["index"], state["logit"], case["temperature"])
        B.rad_linear_distill(ctx, layer, state["x"], state["W"], state["bias"], teacher, **out)
    return out


def _softmax_loss(z, targets, weights, temperature):
    """Loss of each row of z against (index, probability) lists, and the gradient of the mean over the rows that count:
    z and what it returns in fp32.  A row without targets counts for nothing."""
    index, prob = targets
    counts = weights > 0
    scaled = z / temperature
    top = scaled.max(dim=1, keepdim=True).values
    e = torch.exp(scaled - top)
    total = e.sum(dim=1, keepdim=True)
    log_q = scaled.gather(1, index) - top - torch.log(total)
    entropy = torch.where(prob > 0, prob * torch.log(torch.where(prob > 0, prob, torch.ones_like(prob))), torch.zeros_like(prob))
    row_loss = temperature ** 2 * (entropy - prob * log_q).sum(dim=1)
    row_loss = torch.where(counts, row_loss, torch.zeros_like(row_loss))
    share = counts.float() / counts.sum().clamp(min=1)
    g = e / total
    g.scatter_add_(1, index, -prob)
    g *= (temperature * share)[:, None]
    return row_loss, (row_loss * share).sum().reshape(1), g


def _targets(state):
    case = state["case"]
    if case["op"] == "linear_ce":
        counts = (state["labels"] >= 0) & (state["labels"] < case["classes"])
        index = torch.where(counts, state["labels"], torch.zeros_like(state["labels"])).long()[:, None]
        return (index, counts.float()[:, None]), counts.float(), 1.0
    there = state["index"] >= 0
    index = torch.where(there, state["index"], torch.zeros_like(state["index"])).long()
    t = torch.where(there, state["logit"] / case["temperature"], torch.full_like(state["logit"], -math.inf))
    top = t.max(dim=1, keepdim=True).values
    e = torch.where(there, torch.exp(t - torch.where(torch.isfinite(top), top, torch.zeros_like(top))), torch.zeros_like(t))
    prob = e / e.sum(dim=1, keepdim=True).clamp(min=1e-30)
    return (index, prob), there.any(dim=1).float(), case["temperature"]


def _run_plain(state):
    case, dtype = state["case"], TORCH[state["case"]["dtype"]]
    targets, weights, temperature = _targets(state)
    if case["op"] == "distill":
        row_loss, loss, g = _softmax_loss(state["logits"].float(), targets, weights, temperature)
        return {"row_loss": row_loss, "loss": loss, "dlogits": g.to(dtype)}
    x, W = state["x"].float(), state["W"].float()
    z = x @ W
    if case["bias"]:
        z += state["bias"]
    row_loss, loss, g = _softmax_loss(z, targets, weights, temperature)
    out = {"row_loss": row_loss, "loss": loss}
    if case.get("train", True):
        out["dX"], out["dW"] = (g @ W.t()).to(dtype), (x.t() @ g).to(dtype)
        if case["bias"]:
            out["dbias"] = g.sum(dim=0)
    return out


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


def work(case):
    """Each input read once, each output written once; two operations per multiply-add of the products, and per logit what a
    softmax needs: a maximum, a difference, an exponential, a sum, and, with a gradient, a product and a difference."""
    rows, classes, size = case["rows"], case["classes"], SIZE[case["dtype"]]
    train = case.get("train", True)
    nbytes = rows * 4 + 4
    nbytes += rows * 4 if case["op"] == "linear_ce" else rows * case["k"] * 8
    if case["op"] == "distill":
        return {"bytes": nbytes + 2 * rows * classes * size, "flops": 6 * rows * classes}
    d_in = case["d_in"]
    nbytes += (rows * d_in + d_in * classes) * size * (2 if train else 1)
    nbytes += classes * 4 * (2 if train else 1) if case["bias"] else 0
    return {"bytes": nbytes, "flops": (6 if train else 2) * rows * d_in * classes + (6 if train else 4) * rows * classes}


def exact(case, seed):
    """By the definition, in 64 bits, a block of rows at a time: q = softmax(z / T), the loss T^2 sum_j p_j log(p_j / q_j),
    its mean over the rows that have a target, and dz = T (q - p) / rows that count."""
    if 6.0 * case["rows"] * case.get("d_in", 1) * case["classes"] > 1.5e13:
        return None
    state = prepare(case, seed)
    rows, classes = case["rows"], case["classes"]
    T = case.get("temperature", 1.0)
    if case["op"] == "linear_ce":
        ids, lists = state["labels"].long()[:, None], torch.zeros(rows, 1, device="cuda", dtype=torch.float64)
    else:
        ids, lists = state["index"].long(), state["logit"].double() / T
    valid = (ids >= 0) & (ids < classes)
    counted = valid.any(dim=1)
    n = max(1, int(counted.sum()))
    log_p = torch.log_softmax(lists.masked_fill(~valid, -1e300), dim=1)
    p = torch.exp(log_p).masked_fill(~valid, 0.0)
    train = case.get("train", True)
    out = {"row_loss": torch.zeros(rows, device="cuda", dtype=torch.float64)}
    if case["op"] == "distill":
        out["dlogits"] = torch.zeros(rows, classes, device="cuda", dtype=torch.float64)
    else:
        W = state["W"].double()
        if train:
            out["dX"] = torch.zeros(rows, case["d_in"], device="cuda", dtype=torch.float64)
            out["dW"] = torch.zeros_like(W)
            if case["bias"]:
                out["dbias"] = torch.zeros(classes, device="cuda", dtype=torch.float64)
    block = 1024
    for r in range(0, rows, block):
        at = slice(r, min(rows, r + block))
        if case["op"] == "distill":
            z = state["logits"][at].double()
        else:
            xb = state["x"][at].double()
            z = xb @ W
            if case["bias"]:
                z += state["bias"].double()
        log_q = torch.log_softmax(z / T, dim=1)
        where = ids[at].clamp(0, classes - 1)
        pb, use = p[at], counted[at].double()
        out["row_loss"][at] = T * T * use * torch.where(pb > 0, pb * (log_p[at] - torch.gather(log_q, 1, where)), torch.zeros_like(pb)).sum(dim=1)
        if not train:
            continue
        dz = torch.exp(log_q) * use[:, None]
        dz.scatter_add_(1, where, -pb)
        dz *= T / n
        if case["op"] == "distill":
            out["dlogits"][at] = dz
            continue
        out["dX"][at] = dz @ W.t()
        out["dW"] += xb.t() @ dz
        if case["bias"]:
            out["dbias"] += dz.sum(dim=0)
    out["loss"] = (out["row_loss"].sum() / n).reshape(1)
    return out

"""What a model's answer is worth, token by token, and the step that follows, as cases that a timer can prepare and run.

The operators of `paper_2007_10412_amd.binding`:

    rad_token_logprobs         log probabilities of given tokens, entropies and the likeliest tokens, of logits in hand
    rad_token_logprobs_grad    the logits' gradient from those of log probabilities and entropies
    rad_linear_logprobs        the first with the last layer in it, whose logits are never kept
    rad_linear_logprobs_grad   its gradients: rows, weights and biases
    rad_gradient_norm          the norm of many gradients together, and the factor that clips it
    rad_clip_gradients         gradients under that factor
    rad_optimizer_step_scaled  the parameters' step from gradients under that factor

    listed()            the fixed cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a program has in hand before the call, on the GPU
    run(state)          one pass; returns its outputs
    work(case)          bytes and operations one pass cannot do without
    exact(case, seed)   the outputs by the operators' definition, in 64 bits

`own` false: elementary torch operations in fp32 (norms in 64 bits), rounded once at the end.  `own` true: the library's calls.
"""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
LR, L2, BETA1, BETA2, EPS, STEP = 1e-3, 1e-4, 0.9, 0.999, 1e-8, 10


def listed():
    return [
        # One answered token with its 20 likeliest alternatives: latency is all there is.
        {"name": "token_1x128000_bf16_k20", "op": "token", "dtype": "bf16", "rows": 1, "classes": 128000, "k": 20,
         "temperature": 1.0, "ignored": 0.0, "masked": 0.0},
        # A batch of answers scored, with a few alternatives each, as a server returns them.
        {"name": "token_4096x32000_bf16_k5", "op": "token", "dtype": "bf16", "rows": 4096, "classes": 32000, "k": 5,
         "temperature": 1.0, "ignored": 0.0, "masked": 0.0},
        # A teacher's lists made of fp32 logits of odd width, half of whose tokens a grammar forbids; some rows are prompts.
        {"name": "token_777x50257_f32_k64", "op": "token", "dtype": "f32", "rows": 777, "classes": 50257, "k": 64,
         "temperature": 2.0, "ignored": 0.3, "masked": 0.5},
        # The objective's gradient for logits that are there: advantages on tokens and a reward for entropy.
        {"name": "token_grad_4096x32000_bf16", "op": "token_grad", "dtype": "bf16", "rows": 4096, "classes": 32000,
         "temperature": 1.0, "ignored": 0.0, "masked": 0.0},
        {"name": "token_grad_333x50257_f32", "op": "token_grad", "dtype": "f32", "rows": 333, "classes": 50257,
         "temperature": 0.7, "ignored": 0.2, "masked": 0.0},
        # One token of a large model's answer: the weights are read once, for one row.
        {"name": "linear_1x4096x128000_bf16_k20", "op": "linear", "dtype": "bf16", "rows": 1, "d_in": 4096, "classes": 128000,
         "k": 20, "temperature": 1.0, "ignored": 0.0, "bias": False},
        # A whole answer of 300 tokens, with alternatives.
        {"name": "linear_300x2048x32000_bf16_k5", "op": "linear", "dtype": "bf16", "rows": 300, "d_in": 2048, "classes": 32000,
         "k": 5, "temperature": 1.0, "ignored": 0.0, "bias": True},
        # A batch of answers behind prompts of odd lengths, fine-tuned by their advantages.
        {"name": "linear_grad_4096x2048x32000_bf16", "op": "linear_grad", "dtype": "bf16", "rows": 4096, "d_in": 2048,
         "classes": 32000, "temperature": 1.0, "ignored": 0.3, "bias": False},
        # A small fp32 model with a bias.
        {"name": "linear_grad_200x768x10007_f32", "op": "linear_grad", "dtype": "f32", "rows": 200, "d_in": 768, "classes": 10007,
         "temperature": 1.0, "ignored": 0.0, "bias": True},
        # The small MNIST network's six tensors, clipped and stepped: launches are all there is.
        {"name": "clip_step_784-300-300-10_f32", "op": "clip_step", "dtype": "f32", "dims": "784-300-300-10", "bias": True,
         "kind": "adam", "clip": 0.1},
        # The wide bf16 network's (fp32 gradients and master copies).
        {"name": "clip_step_4096-4096-4096-1000_bf16", "op": "clip_step", "dtype": "bf16", "dims": "4096-4096-4096-1000",
         "bias": False, "kind": "adam", "clip": 0.5},
        # Gradients of odd layers clipped before something else takes them.
        {"name": "clip_1023-4097-1000-50257_bf16", "op": "clip", "dtype": "bf16", "dims": "1023-4097-1000-50257", "bias": True,
         "clip": 0.3},
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
    op = rng.choice(["token", "token", "token_grad", "linear", "linear", "linear_grad", "clip_step", "clip"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    if op in ("clip_step", "clip"):
        while True:
            widths = [_size(rng, 10, 8192) for _ in range(rng.randint(2, 25))]
            if sum(a * b for a, b in zip(widths, widths[1:])) <= 4096 * (4096 + 4096 + 1000):
                break
        case = {"op": op, "dtype": dtype, "dims": "-".join(map(str, widths)), "bias": rng.random() < 0.5,
                "clip": rng.choice([0.01, 0.5, 0.9, 2.0])}
        if op == "clip_step":
            case["kind"] = rng.choice(["adam", "adam", "sgd"])
        return case
    while True:
        case = {"op": op, "dtype": dtype, "rows": _size(rng, 1, 8192), "classes": _size(rng, 1000, 131072)}
        if op.startswith("token"):
            if case["rows"] * case["classes"] > 4096 * 32000:
                continue
        else:
            case["d_in"] = _size(rng, 256, 4096)
            most = 4096 * 2048 * 32000 // (16 if dtype == "f32" else 1)
            if case["rows"] * case["d_in"] * case["classes"] > most or case["d_in"] * case["classes"] > 4096 * 128000:
                continue
        break
    case["temperature"] = rng.choice([1.0, 1.0, 0.7, 2.0])
    case["ignored"] = rng.choice([0.0, 0.0, 0.2, 0.6])
    if op in ("token", "linear"):
        case["k"] = 0 if rng.random() < 0.2 else _log_between(rng, 1, 256)
    if op.startswith("token"):
        case["masked"] = rng.choice([0.0, 0.0, 0.5])
    else:
        # (the bias gradient is a sum in fp32 of what the layer's type rounds, so bf16 training is drawn without one)
        case["bias"] = rng.random() < 0.5 and (dtype == "f32" or op == "linear")
    return case


def _shapes(case):
    """Shapes of a network's parameters, weights and biases in turn, and where each begins in one buffer of all of them (at a
    multiple of 16 bytes also where an element has two)."""
    widths = [int(w) for w in case["dims"].split("-")]
    shapes, starts, at = [], [], 0
    for a, b in zip(widths, widths[1:]):
        for shape in [(a, b)] + ([(b,)] if case["bias"] else []):
            shapes.append(shape)
            starts.append(at)
            at += (math.prod(shape) + 7) // 8 * 8
    return shapes, starts, at


def _parameters(case):
    return sum(math.prod(s) for s in _shapes(case)[0])


def _views(flat, case):
    shapes, starts, _ = _shapes(case)
    return [flat[a:a + math.prod(s)].view(s) for s, a in zip(shapes, starts)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = TORCH[case["dtype"]]
    state = {"case": case}

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def numbers(high, *shape):
        return torch.randint(0, high, shape, device="cuda", generator=gen)

    if case["op"] in ("clip_step", "clip"):
        total, n = _shapes(case)[2], _parameters(case)
        there = torch.zeros(total, device="cuda")
        for t in _views(there, case):
            t.fill_(1.0)

        def buffer(values, kind=torch.float32):
            flat = (values * there).to(kind)              # (zeros between the tensors)
            return flat, _views(flat, case)

        # gradients of very different layers: sizes over three powers of ten
        raw = normal(total)
        for i, t in enumerate(_views(raw, case)):
            t.mul_(10.0 ** -(i % 4))
        state["grads_flat"], state["grads"] = buffer(raw, dtype if case["op"] == "clip" else torch.float32)
        state["max_norm"] = case["clip"] * math.sqrt(sum(math.prod(s) * 100.0 ** -(i % 4) for i, s in enumerate(_shapes(case)[0])))
        if case["op"] == "clip":
            state["clipped_flat"], state["clipped"] = buffer(there, dtype)
            return state
        master = 0.05 * normal(total)
        state["params_flat"], state["params"] = buffer(master, dtype)
        if case["dtype"] == "bf16":
            state["master_flat"], state["master"] = buffer(master)
        if case["kind"] == "adam":
            state["m_flat"], state["m"] = buffer(0.1 * raw)
            state["v_flat"], state["v"] = buffer(raw.square() * (0.5 + torch.rand(total, device="cuda", generator=gen)))
        return state

    rows, classes = case["rows"], case["classes"]
    tokens = numbers(classes, rows)
    # logits with a standard deviation of 3: some tokens are a thousand times as likely as others
    if case["op"].startswith("token"):
        logits = 3.0 * normal(rows, classes)
        # every other token is the likeliest one
        tokens = torch.where(numbers(2, rows) == 0, logits.argmax(dim=1), tokens)
        if case["masked"]:
            # a grammar that leaves some tokens, the given ones among them
            gone = torch.rand(rows, classes, device="cuda", generator=gen) < case["masked"]
            gone.scatter_(1, tokens[:, None], False)
            logits = logits.masked_fill_(gone, -math.inf)
        state["logits"] = logits.to(dtype)
    else:
        # Rows and weights of a few bits each, so that sums of their products are exact in fp32 in any order: which of two tokens
        # is the likelier one is then no matter of rounding, and equal logits are equal.
        d_in = case["d_in"]
        step = 2.0 ** round(math.log2(3.0 / math.sqrt(d_in))) / 32.0
        state["x"] = ((normal(rows, d_in) * 16.0).round().clamp(-64, 64) / 16.0).to(dtype)
        state["W"] = ((normal(d_in, classes) * (3.0 / math.sqrt(d_in) / step)).round().clamp(-128, 128) * step).to(dtype)
        state["bias"] = (normal(classes) * 16.0).round() / 16.0 if case["bias"] else None
    if case["ignored"]:
        # sequences of 64 tokens whose first part is a prompt, of one length or another; the last token is an answer's
        at = torch.arange(rows, device="cuda")
        share = torch.rand((rows + 63) // 64, device="cuda", generator=gen) * 2 * case["ignored"]
        prompt = ((at % 64).float() < 64 * share[at // 64]) & (at < rows - 1)
        tokens = torch.where(prompt, torch.full_like(tokens, -1), tokens)
    state["tokens"] = tokens.to(torch.int32)
    if case["op"].endswith("grad"):
        # advantages, over the number of tokens, and a tenth of that for a token's entropy
        state["d_logprob"] = normal(rows) / rows
        state["d_entropy"] = (0.05 + 0.1 * torch.rand(rows, device="cuda", generator=gen)) / rows
    return state


_contexts = {}


def _context():
    """The context that a program makes once and keeps (on the default stream)."""
    from paper_2007_10412_amd import binding as B
    if "default" not in _contexts:
        _contexts["default"] = B.rad_ctx_create()
    return B, _contexts["default"]


def _run_own_clip(state):
    B, ctx = _context()
    case = state["case"]
    norm = torch.empty(1, device="cuda")
    if case["op"] == "clip":
        B.rad_clip_gradients(ctx, state["grads"], state["max_norm"], clipped=state["clipped"], norm=norm)
        return {"norm": norm, "clipped": state["clipped_flat"]}
    scale = torch.empty(1, device="cuda")
    B.rad_gradient_norm(ctx, state["grads"], state["max_norm"], norm=norm, scale=scale)
    opt = B.make_optimizer(B.RAD_ADAM if case["kind"] == "adam" else B.RAD_SGD, LR, L2, BETA1, BETA2, EPS)
    B.rad_optimizer_step_scaled(ctx, opt, STEP, B.RAD_F32 if case["dtype"] == "f32" else B.RAD_BF16, state["params"],
                                state["grads"], scale, m=state.get("m"), v=state.get("v"), master=state.get("master"))
    return {"norm": norm, **{name: state[name] for name in ("params_flat", "master_flat", "m_flat", "v_flat") if name in state}}


def _run_own(state):
    if state["case"]["op"] in ("clip_step", "clip"):
        return _run_own_clip(state)
    B, ctx = _context()
    case = state["case"]
    f32 = dict(device="cuda", dtype=torch.float32)
    kind = B.RAD_F32 if case["dtype"] == "f32" else B.RAD_BF16
    rows = case["rows"]
    given = {"tokens": state["tokens"], "temperature": case["temperature"]}
    if case["op"] in ("token", "linear"):
        out = {"logprob": torch.empty(rows, **f32), "entropy": torch.empty(rows, **f32)}
        if case["k"]:
            out["top_index"] = torch.empty(rows, case["k"], device="cuda", dtype=torch.int32)
            out["top_logprob"] = torch.empty(rows, case["k"], **f32)
    else:
        given["d_logprob"], given["d_entropy"] = state["d_logprob"], state["d_entropy"]
    if case["op"] == "token":
        B.rad_token_logprobs(ctx, state["logits"], kind, **given, **out)
        return out
    if case["op"] == "token_grad":
        out = {"dlogits": torch.empty_like(state["logits"])}
        B.rad_token_logprobs_grad(ctx, state["logits"], kind, **given, **out)
        return out
    layer = B.make_layer(rows, case["d_in"], case["classes"], dtype=kind, relu=False, has_bias=case["bias"])
    if case["op"] == "linear":
        B.rad_linear_logprobs(ctx, layer, state["x"], state["W"], state["bias"], **given, **out)
        return out
    out = {"dX": torch.empty_like(state["x"]), "dW": torch.empty_like(state["W"])}
    if case["bias"]:
        out["dbias"] = torch.empty(case["classes"], **f32)
    B.rad_linear_logprobs_grad(ctx, layer, state["x"], state["W"], state["bias"], **given, **out)
    return out


def _run_plain_clip(state):
    case = state["case"]
    grads = state["grads_flat"].float()
    norm = grads.double().square().sum().sqrt()
    scale = torch.clamp(state["max_norm"] / norm, max=1.0).float()
    g = grads * scale
    norm = norm.float().reshape(1)
    if case["op"] == "clip":
        state["clipped_flat"].copy_(g)
        return {"norm": norm, "clipped": state["clipped_flat"]}
    w = state["master_flat"] if case["dtype"] == "bf16" else state["params_flat"]
    g = g + L2 * w
    if case["kind"] == "adam":
        m, v = state["m_flat"], state["v_flat"]
        m.mul_(BETA1).add_((1.0 - BETA1) * g)
        v.mul_(BETA2).add_((1.0 - BETA2) * g * g)
        w.sub_(LR * (m / (1.0 - BETA1 ** STEP)) / ((v / (1.0 - BETA2 ** STEP)).sqrt() + EPS))
    else:
        w.sub_(LR * g)
    if case["dtype"] == "bf16":
        state["params_flat"].copy_(w)
    return {"norm": norm, **{name: state[name] for name in ("params_flat", "master_flat", "m_flat", "v_flat") if name in state}}


def _order(z):
    """Whole numbers in the order of z, equal logits' in the descending order of their places: the largest are the likeliest
    tokens, ties to the lowest one."""
    bits = (z + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    return bits * (1 << 32) - torch.arange(z.shape[1], device=z.device)


def _run_plain(state):
    case = state["case"]
    if case["op"] in ("clip_step", "clip"):
        return _run_plain_clip(state)
    dtype, classes, T = TORCH[case["dtype"]], case["classes"], case["temperature"]
    if case["op"].startswith("token"):
        z = state["logits"].float()
    else:
        x, W = state["x"].float(), state["W"].float()
        z = x @ W
        if case["bias"]:
            z += state["bias"]
    counts = (state["tokens"] >= 0) & (state["tokens"] < classes)
    token = torch.where(counts, state["tokens"], torch.zeros_like(state["tokens"])).long()[:, None]
    below = (z - z.max(dim=1, keepdim=True).values) / T
    e = torch.exp(below)
    total = e.sum(dim=1, keepdim=True)
    log_q = below - torch.log(total)
    q = e / total
    surprise = torch.where(q > 0, log_q, torch.zeros_like(q))
    entropy = -(q * surprise).sum(dim=1)
    if case["op"] in ("token", "linear"):
        none = torch.zeros_like(entropy)
        out = {"logprob": torch.where(counts, log_q.gather(1, token)[:, 0], none), "entropy": torch.where(counts, entropy, none)}
        if case["k"]:
            index = _order(z).topk(case["k"], dim=1).indices
            logprob = log_q.gather(1, index)
            there = counts[:, None] & (logprob > -math.inf)
            out["top_index"] = torch.where(there, index, torch.full_like(index, -1)).to(torch.int32)
            out["top_logprob"] = torch.where(there, logprob, torch.full_like(logprob, -math.inf))
        return out
    none = torch.zeros_like(state["d_logprob"])
    a = torch.where(counts, state["d_logprob"], none)[:, None] / T
    h = torch.where(counts, state["d_entropy"], none)[:, None] / T
    g = q * (-a - h * (surprise + entropy[:, None]))
    g.scatter_add_(1, token, a)
    if case["op"] == "token_grad":
        return {"dlogits": g.to(dtype)}
    out = {"dX": (g @ W.t()).to(dtype), "dW": (x.t() @ g).to(dtype)}
    if case["bias"]:
        out["dbias"] = g.sum(dim=0)
    return out


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


def work(case):
    """Each input read once, each output written once; two operations per multiply-add of the products, per logit what a
    softmax with its entropy needs (a maximum, a difference, an exponential, two sums, a product) and a gradient besides, per
    parameter a square, a sum and the step's products."""
    size = SIZE[case["dtype"]]
    if case["op"] in ("clip_step", "clip"):
        n = _parameters(case)
        if case["op"] == "clip":
            return {"bytes": 2 * size * n + 4, "flops": 3 * n}
        adam = case["kind"] == "adam"
        return {"bytes": n * (4 + (24 if adam else 8) + (2 if case["dtype"] == "bf16" else 0)) + 4, "flops": (18 if adam else 7) * n}
    rows, classes = case["rows"], case["classes"]
    nbytes = rows * 4
    if case["op"] in ("token", "linear"):
        nbytes += rows * 8 + rows * case["k"] * 8
    else:
        nbytes += rows * 8
    if case["op"].startswith("token"):
        grad = case["op"] == "token_grad"
        return {"bytes": nbytes + (2 if grad else 1) * rows * classes * size, "flops": (9 if grad else 6) * rows * classes}
    train, d_in = case["op"] == "linear_grad", case["d_in"]
    nbytes += (rows * d_in * (2 if train else 1) + d_in * classes * (2 if train else 1)) * size
    if not train:
        return {"bytes": nbytes + (classes * 4 if case["bias"] else 0), "flops": 2 * rows * d_in * classes + 6 * rows * classes}
    nbytes += classes * 8 if case["bias"] else 0
    return {"bytes": nbytes, "flops": 6 * rows * d_in * classes + 9 * rows * classes}


def _exact_clip(case, state):
    f64 = {name[:-5]: t.double() for name, t in state.items() if name.endswith("_flat")}
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in state["grads"]))
    g = f64["grads"] * (state["max_norm"] / norm if norm > state["max_norm"] else 1.0)
    out = {"norm": torch.tensor([norm], dtype=torch.float64, device="cuda")}
    if case["op"] == "clip":
        out["clipped"] = g
        return out
    w = f64["master" if case["dtype"] == "bf16" else "params"]
    g = g + L2 * w
    step = g
    if case["kind"] == "adam":
        m, v = BETA1 * f64["m"] + (1 - BETA1) * g, BETA2 * f64["v"] + (1 - BETA2) * g ** 2
        step = m / (1 - BETA1 ** STEP) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS)
        out["m_flat"], out["v_flat"] = m, v
    out["params_flat"] = w - LR * step
    if case["dtype"] == "bf16":
        out["master_flat"] = out["params_flat"]
    return out


def exact(case, seed):
    """By the definition, in 64 bits, a block of rows at a time: log q = log softmax(z / T), H = - sum q log q, the k largest
    logits in order, and dz = (a (onehot - q) - h q (log q + H)) / T for the gradients a of log q[token] and h of H."""
    state = prepare(case, seed)
    if case["op"] in ("clip_step", "clip"):
        return _exact_clip(case, state)
    rows, classes, T = case["rows"], case["classes"], case["temperature"]
    linear = case["op"].startswith("linear")
    train = case["op"].endswith("grad")
    if (6.0 if train else 2.0) * rows * classes * case.get("d_in", 1) > 1.5e13:
        return None
    ids = state["tokens"].long()
    valid = (ids >= 0) & (ids < classes)
    f64 = dict(device="cuda", dtype=torch.float64)
    out = {}
    if not train:
        out["logprob"], out["entropy"] = torch.zeros(rows, **f64), torch.zeros(rows, **f64)
        if case["k"]:
            out["top_index"] = torch.full((rows, case["k"]), -1, device="cuda", dtype=torch.int32)
            out["top_logprob"] = torch.full((rows, case["k"]), -math.inf, **f64)
    elif linear:
        out["dX"], out["dW"] = torch.zeros(rows, case["d_in"], **f64), torch.zeros(case["d_in"], classes, **f64)
        if case["bias"]:
            out["dbias"] = torch.zeros(classes, **f64)
    else:
        out["dlogits"] = torch.zeros(rows, classes, **f64)
    W = state["W"].double() if linear else None
    block = 512
    for r in range(0, rows, block):
        at = slice(r, min(rows, r + block))
        if linear:
            xb = state["x"][at].double()
            z = xb @ W
            if case["bias"]:
                z += state["bias"].double()
        else:
            z = state["logits"][at].double()
        use = valid[at]
        log_q = torch.log_softmax(z / T, dim=1)
        p = torch.exp(log_q)
        plogp = torch.special.xlogy(p, p)
        H = -plogp.sum(dim=1)
        where = ids[at].clamp(0, classes - 1)[:, None]
        if not train:
            out["logprob"][at] = torch.where(use, torch.gather(log_q, 1, where)[:, 0], out["logprob"][at])
            out["entropy"][at] = torch.where(use, H, out["entropy"][at])
            if case["k"]:
                best = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :case["k"]]
                values = torch.gather(log_q, 1, best)
                there = use[:, None] & torch.isfinite(values)
                out["top_index"][at] = torch.where(there, best.to(torch.int32), out["top_index"][at])
                out["top_logprob"][at] = torch.where(there, values, out["top_logprob"][at])
            continue
        a, h = state["d_logprob"][at].double()[:, None], state["d_entropy"][at].double()[:, None]
        dz = -a * p - h * (plogp + p * H[:, None])
        dz.scatter_add_(1, where, a)
        dz *= use.double()[:, None] / T
        if not linear:
            out["dlogits"][at] = dz
            continue
        out["dX"][at] = dz @ W.t()
        out["dW"] += xb.t() @ dz
        if case["bias"]:
            out["dbias"] += dz.sum(dim=0)
    return out

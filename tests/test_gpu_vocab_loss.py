"""Losses over a vocabulary (rad_linear_ce, rad_distill_ce, rad_linear_distill) against their definition in fp64, element by
element, with bounds counted from the roundings: h = 2^-8 (bf16) or 2^-24 (fp32) is half a step of the layer's type, u = 2^-24
that of the sums, and a sum of K terms is off by at most 8 u sqrt(K) sum|terms| (its error is a random walk; 8 standard
deviations)."""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {0: 2.0 ** -24, 1: 2.0 ** -8}


def torch_dtype(dtype):
    import torch
    return torch.bfloat16 if dtype else torch.float32


class Ctx:
    def __init__(self, stream=None):
        from paper_2007_10412_amd import binding as B
        self.ctx = B.rad_ctx_create(stream)

    def __enter__(self):
        return self.ctx

    def __exit__(self, *_):
        from paper_2007_10412_amd import binding as B
        B.rad_ctx_destroy(self.ctx)


def lists(labels=None, teacher=None, classes=0, T=1.0):
    """(index, probability, entropy, counts) in fp64; entries left out have probability 0."""
    import torch
    if labels is not None:
        idx = labels.long()[:, None]
        valid = (idx >= 0) & (idx < classes)
        return idx.clamp(0, classes - 1), valid.double(), torch.zeros(len(idx), device="cuda", dtype=torch.float64), valid[:, 0]
    index, logit = teacher
    idx = index.long()
    t = logit.double() / T
    valid = (idx >= 0) & (idx < classes) & (logit != -math.inf)
    t = torch.where(valid, t, torch.full_like(t, -math.inf))
    counts = valid.any(dim=1)
    top = torch.where(counts[:, None], t.max(dim=1, keepdim=True).values, torch.zeros_like(t[:, :1]))
    e = torch.where(valid, torch.exp(t - top), torch.zeros_like(t))
    p = e / e.sum(dim=1, keepdim=True).clamp(min=1e-300)
    ent = torch.where(p > 0, p * torch.log(p.clamp(min=1e-300)), torch.zeros_like(p)).sum(dim=1)
    return idx.clamp(0, classes - 1), p, ent, counts


def definition(z, targets, weight, T):
    """row_loss, loss, dz and the softmax part |w| T q in fp64, and the weights."""
    import torch
    idx, p, ent, counts = targets
    n = int(counts.sum())
    w = torch.full((len(z),), 1.0 / n if n else 0.0, device="cuda", dtype=torch.float64) if weight is None else weight.double()
    w = torch.where(counts, w, torch.zeros_like(w))
    log_q = torch.log_softmax(z / T, dim=1)
    at = torch.gather(log_q, 1, idx)
    row = T * T * (ent - torch.where(p > 0, p * at, torch.zeros_like(p)).sum(dim=1))
    row = torch.where(counts, row, torch.zeros_like(row))
    q = torch.where(counts[:, None], torch.exp(log_q), torch.zeros_like(log_q))
    target = torch.zeros_like(q).scatter_add_(1, idx, p)
    wt = (w * T)[:, None]
    return row, (row * w).sum(), wt * (q - target), wt.abs() * q, wt.abs() * target


def close(got, want, bound, tag):
    import torch
    got = got.double()
    assert got.shape == want.shape, tag
    assert torch.isfinite(got).all(), tag + ": not finite"
    over = (got - want).abs() - bound
    worst = int(over.argmax())
    assert float(over.max()) <= 0, "%s: element %d is %g, not %g (bound %g); %d are off" % (
        tag, worst, got.flatten()[worst], want.flatten()[worst], bound.flatten()[worst], int((over > 0).sum()))


# what 64-bit statistics of fp32 logits are off by in fp32: dz_rel of a softmax value, from an error `ez` of every logit over T
def softmax_error(ez, classes):
    return 2 * ez + 8 * U * math.sqrt(classes) + 64 * U


# A listed probability exp(t_j / T - m) / s in fp32: t / T comes from two roundings (1 / T, the product), as does m; their
# difference d, |d| <= 2 max|t| / T, from one more; these absolute errors of an exponent are relative ones of the exponential:
# (2 + 2 + 2) max|t| / T roundings.  The exponential, the division and a join of equal entries add 2 + 2 + 2, s a sum's 8 sqrt(k).
def list_error(teacher, T):
    import torch
    t = teacher[1][torch.isfinite(teacher[1])].abs()
    return U * (6 * (float(t.max()) if t.numel() else 0.0) / T + 6 + 8 * math.sqrt(teacher[1].shape[1]))


def labels_for(rows, classes, gen, ignored=0.0):
    import torch
    lab = torch.randint(0, classes, (rows,), device="cuda", generator=gen)
    if ignored:
        out = torch.rand(rows, device="cuda", generator=gen) < ignored
        other = torch.tensor([-1, -100, classes, 2 ** 31 - 1, -2 ** 31], device="cuda")[torch.arange(rows, device="cuda") % 5]
        lab = torch.where(out, other, lab)
    return lab.to(torch.int32)


def teacher_for(rows, classes, k, gen, missing=0.0, doubles=False):
    import torch
    index = torch.rand(rows, classes, device="cuda", generator=gen).argsort(dim=1)[:, :k] if classes <= 4096 else \
        (torch.randint(0, classes, (rows, 1), device="cuda", generator=gen) + torch.arange(k, device="cuda") * max(1, classes // k)) % classes
    if index.shape[1] < k or doubles:
        index = torch.randint(0, max(1, min(classes, k // 2)), (rows, k), device="cuda", generator=gen)
    logit = 2 * torch.randn(rows, k, device="cuda", generator=gen)
    if missing:
        gone = torch.rand(rows, k, device="cuda", generator=gen) < missing
        index = torch.where(gone, torch.tensor([-1, classes, -7], device="cuda")[torch.arange(k, device="cuda") % 3], index)
        index[::5] = -1                                             # empty lists
        logit = torch.where(torch.rand(rows, k, device="cuda", generator=gen) < 0.1, torch.full_like(logit, -math.inf), logit)
    return index.to(torch.int32).contiguous(), logit.contiguous()


def check_linear(ctx, dtype, rows, d_in, classes, bias=False, ignored=0.0, k=0, T=1.0, weight=None, beta=0.0, dw_dtype=None,
                 outputs=("row_loss", "loss", "dX", "dW", "dbias"), scale=3.0, bias_values=None, missing=0.0, seed=1, tag=""):
    import torch
    from paper_2007_10412_amd import binding as B
    tag = "%s dtype %d, %d x %d x %d, k %d" % (tag, dtype, rows, d_in, classes, k)
    print(tag, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(seed + rows + 3 * d_in + 7 * classes)
    td = torch_dtype(dtype)
    wd = torch_dtype(dtype if dw_dtype is None else dw_dtype)
    f32 = dict(device="cuda", dtype=torch.float32)
    x = torch.randn(rows, d_in, device="cuda", generator=gen).to(td)
    W = (torch.randn(d_in, classes, device="cuda", generator=gen) * (scale / math.sqrt(d_in))).to(td)
    b = torch.randn(classes, device="cuda", generator=gen) if bias else None
    if bias_values is not None:
        b = bias_values(b if b is not None else torch.zeros(classes, **f32))
    layer = B.make_layer(rows, d_in, classes, dtype=dtype, relu=False, has_bias=b is not None)
    dW0 = torch.randn(d_in, classes, device="cuda", generator=gen).to(wd)
    db0 = torch.randn(classes, device="cuda", generator=gen)
    out = {"row_loss": torch.full((rows,), math.nan, **f32), "loss": torch.full((1,), math.nan, **f32),
           "dX": torch.full_like(x, math.nan), "dW": dW0.clone() if beta else torch.full_like(dW0, math.nan),
           "dbias": db0.clone() if beta else torch.full((classes,), math.nan, **f32)}
    asked = {n: out[n] for n in outputs}
    if k:
        index, logit = teacher_for(rows, classes, k, gen, missing)
        teacher = B.make_teacher(index, logit, T)
        B.rad_linear_distill(ctx, layer, x, W, b, teacher, row_weight=weight, beta=beta, **asked)
        targets = lists(teacher=(index, logit), classes=classes, T=T)
        ep = list_error((index, logit), T)
    else:
        ep = 0.0
        labels = labels_for(rows, classes, gen, ignored) if ignored < 1 else torch.full((rows,), -1, device="cuda", dtype=torch.int32)
        B.rad_linear_ce(ctx, layer, x, W, b, labels, row_weight=weight, beta=beta, **asked)
        targets = lists(labels=labels, classes=classes)
    B.rad_ctx_synchronize(ctx)
    xd, Wd = x.double(), W.double()
    z = xd @ Wd
    size = xd.abs() @ Wd.abs()                                       # sum of |terms| behind a logit
    if b is not None:
        z = z + b.double()
        size = size + torch.where(torch.isfinite(b), b.double().abs(), torch.zeros_like(b, dtype=torch.float64)).clamp(max=1e3)
    row, loss, dz, soft, target = definition(z, targets, weight, T)
    ez = 8 * U * math.sqrt(d_in + 2) * float(size.max()) / T
    rel = softmax_error(ez, classes)
    h = HALF[dtype]
    w_all = (weight.double().abs() if weight is not None else torch.ones(rows, device="cuda", dtype=torch.float64) / max(1, int(targets[3].sum())))
    row_bound = T * T * (rel + 8 * U * (targets[2].abs() + (z / T).abs().max() + 30)) * torch.ones_like(row)
    if "row_loss" in asked:
        close(out["row_loss"], row, row_bound, tag + " row_loss")
        assert (out["row_loss"][~targets[3]] == 0).all(), tag
    if "loss" in asked:
        close(out["loss"], loss.reshape(1), ((row_bound + 8 * U * math.sqrt(rows) * row.abs()) * w_all).sum().reshape(1), tag + " loss")
    # dz as the products take it: the softmax's own error, then a rounding to the type, of itself and (dW: of its rows' scale)
    e = soft * rel + 2.02 * h * (soft + target) + (4 * U + ep) * target
    if "dX" in asked:
        want = dz @ Wd.t().contiguous()
        mass = dz.abs() @ Wd.abs().t().contiguous()
        close(out["dX"], want, e @ Wd.abs().t().contiguous() + 8 * U * math.sqrt(classes) * mass + h * want.abs() + 1e-37, tag + " dX")
        assert (out["dX"][~targets[3]] == 0).all(), tag
    if "dW" in asked:
        want = xd.t().contiguous() @ dz + (dW0.double() if beta else 0)
        mass = xd.abs().t().contiguous() @ dz.abs() + (dW0.double().abs() if beta else 0)
        close(out["dW"], want, xd.abs().t().contiguous() @ e + 8 * U * math.sqrt(rows + 1) * mass + HALF[1 if wd == torch.bfloat16 else 0] * want.abs() + 1e-37, tag + " dW")
    if "dbias" in asked:
        want = dz.sum(dim=0) + (db0.double() if beta else 0)
        close(out["dbias"], want, e.sum(dim=0) + 8 * U * math.sqrt(rows + 1) * (dz.abs().sum(dim=0) + (db0.double().abs() if beta else 0)) + 1e-37, tag + " dbias")
    return out


SHAPES = [(1, 1, 1), (1, 5, 3), (3, 7, 1), (5, 64, 33), (150, 300, 10), (64, 256, 1000), (130, 129, 131), (257, 520, 1003),
          (300, 512, 4096), (1000, 72, 2500), (512, 1024, 8192), (17, 1030, 20011),
          (513, 260, 25601), (700, 512, 32000), (20, 129, 30000), (2000, 264, 4104), (1025, 1000, 8200), (4096, 64, 2048)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", SHAPES)
def test_linear_ce(dtype, rows, d_in, classes):
    with Ctx() as ctx:
        check_linear(ctx, dtype, rows, d_in, classes, bias=rows % 2 == 0, ignored=0.3 if rows > 4 else 0.0)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes,k,T,missing", [(1, 5, 3, 3, 1.0, 0.0), (5, 64, 33, 1, 2.0, 0.0), (150, 300, 10, 7, 1.5, 0.4),
                                                           (257, 520, 1003, 65, 0.7, 0.3), (300, 512, 4096, 300, 4.0, 0.0),
                                                           (512, 1024, 8192, 16, 1.0, 0.2), (17, 1030, 20011, 1024, 2.0, 0.1),
                                                           (700, 520, 30001, 33, 1.3, 0.3), (1025, 256, 8200, 1000, 1.0, 0.1)])
def test_linear_distill(dtype, rows, d_in, classes, k, T, missing):
    with Ctx() as ctx:
        check_linear(ctx, dtype, rows, d_in, classes, bias=rows % 2 == 1, k=k, T=T, missing=missing)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", [(1, 256, 5000), (2, 300, 1001), (9, 1024, 32000), (33, 768, 10007), (64, 512, 4096),
                                               (100, 2048, 8000), (500, 512, 3001), (1, 520, 40003), (260, 512, 40000)])
def test_scoring(dtype, rows, d_in, classes):
    """Forward only."""
    with Ctx() as ctx:
        check_linear(ctx, dtype, rows, d_in, classes, bias=rows % 2 == 1, ignored=0.2 if rows > 8 else 0.0, outputs=("row_loss", "loss"))
        check_linear(ctx, dtype, rows, d_in, classes, k=5, T=2.0, outputs=("row_loss",))


@pytest.mark.parametrize("dtype,dw_dtype", [(0, 0), (1, 0), (1, 1)])
@pytest.mark.parametrize("rows,d_in,classes", [(70, 136, 264), (257, 129, 1003), (512, 512, 4096), (600, 200, 20005),
                                               (700, 2048, 8003)])
def test_weights_and_accumulation(dtype, dw_dtype, rows, d_in, classes):
    """Row weights of any sign, gradients added to what is there."""
    import torch
    weight = torch.randn(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(rows))
    weight[::7] = 0.0
    with Ctx() as ctx:
        check_linear(ctx, dtype, rows, d_in, classes, bias=True, ignored=0.3, weight=weight, beta=1.0, dw_dtype=dw_dtype)
        check_linear(ctx, dtype, rows, d_in, classes, k=9, T=1.5, missing=0.3, weight=weight, dw_dtype=dw_dtype)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("outputs", [("row_loss",), ("loss",), ("dX",), ("dW",), ("dbias",), ("dX", "row_loss"), ("dW", "dbias")])
def test_some_outputs(dtype, outputs):
    with Ctx() as ctx:
        check_linear(ctx, dtype, 260, 136, 1030, bias=True, ignored=0.1, outputs=outputs)
        check_linear(ctx, dtype, 600, 136, 20005, bias=True, ignored=0.1, outputs=outputs)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", [(150, 300, 10), (300, 256, 4096), (600, 256, 20000)])
def test_no_row_counts(dtype, rows, d_in, classes):
    """Every label outside the vocabulary: no loss, gradients of zeros (or what was there)."""
    with Ctx() as ctx:
        for beta in (0.0, 1.0):
            check_linear(ctx, dtype, rows, d_in, classes, bias=True, ignored=1.0, beta=beta, dw_dtype=0)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", [(20, 64, 1000), (300, 256, 4096), (512, 512, 8192), (600, 256, 20000)])
@pytest.mark.parametrize("masked", [-math.inf, -3.0e38])
def test_masked_classes(dtype, rows, d_in, classes, masked):
    """Classes that a bias of -infinity, or of the type's lowest values, takes out (whole tiles of them among these)."""
    import torch

    def values(b):
        b = b.clone()
        b[classes // 2:] = masked
        b[1:classes // 2:3] = masked
        return b
    import paper_2007_10412_amd.binding as B
    gen = torch.Generator(device="cuda").manual_seed(5)
    td = torch_dtype(dtype)
    x = torch.randn(rows, d_in, device="cuda", generator=gen).to(td)
    W = (torch.randn(d_in, classes, device="cuda", generator=gen) * (2 / math.sqrt(d_in))).to(td)
    b = values(torch.zeros(classes, device="cuda"))
    left = torch.nonzero(b == 0).flatten()
    labels = left[torch.randint(0, len(left), (rows,), device="cuda", generator=gen)].to(torch.int32)
    layer = B.make_layer(rows, d_in, classes, dtype=dtype, relu=False, has_bias=True)
    row, dX, dW = torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty_like(W)
    with Ctx() as ctx:
        B.rad_linear_ce(ctx, layer, x, W, b, labels, row_loss=row, dX=dX, dW=dW)
        B.rad_ctx_synchronize(ctx)
    xd, Wd = x.double(), W.double()[:, left].contiguous()
    where = torch.full((classes,), -1, device="cuda", dtype=torch.long)
    where[left] = torch.arange(len(left), device="cuda")
    z = xd @ Wd
    r, _, dz, soft, target = definition(z, lists(labels=where[labels.long()].to(torch.int32), classes=len(left)), None, 1.0)
    rel = softmax_error(8 * U * math.sqrt(d_in) * float((xd.abs() @ Wd.abs()).max()), classes)
    h = HALF[dtype]
    close(row, r, torch.full_like(r, rel + 8 * U * 50), "row_loss")
    e = soft * rel + 2.02 * h * (soft + target) + 4 * U * target
    want = dz @ Wd.t().contiguous()
    close(dX, want, (e + 8 * U * math.sqrt(classes) * dz.abs()) @ Wd.abs().t().contiguous() + h * want.abs() + 1e-37, "dX")
    want = xd.t().contiguous() @ dz
    close(dW[:, left], want, xd.abs().t().contiguous() @ (e + 8 * U * math.sqrt(rows) * dz.abs()) + h * want.abs() + 1e-37, "dW")
    gone = torch.ones(classes, device="cuda", dtype=torch.bool)
    gone[left] = False
    assert (dW[:, gone] == 0).all()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("offset", [-400.0, -95.0, 95.0, 400.0])
def test_logits_far_from_zero(dtype, offset):
    """Rows whose logits all lie far from zero, where exponentials of the logits themselves leave the type."""
    with Ctx() as ctx:
        for rows, d_in, classes in ((20, 64, 1000), (512, 512, 4096), (600, 256, 20001)):
            check_linear(ctx, dtype, rows, d_in, classes, bias=True, bias_values=lambda b: b + offset)


@pytest.mark.parametrize("dtype", [0, 1])
def test_peaked_rows(dtype):
    """Logits of a standard deviation of 60: one class has all of a row, and the label's loss is a hundred and more."""
    with Ctx() as ctx:
        for rows, d_in, classes in ((20, 64, 1000), (512, 512, 4096), (600, 256, 20001)):
            check_linear(ctx, dtype, rows, d_in, classes, scale=60.0, ignored=0.1)


@pytest.mark.parametrize("dtype", [0, 1])
def test_more_rows_than_a_piece(dtype):
    """Logits of over a GiB: the rows go through in pieces, and dW is the sum over them."""
    with Ctx() as ctx:
        check_linear(ctx, dtype, 600, 16, 1100003, ignored=0.2, dw_dtype=0)
        if dtype:
            check_linear(ctx, dtype, 1000, 16, 1300003, ignored=0.2, dw_dtype=0)
            check_linear(ctx, dtype, 900, 8, 1300000, k=3, dw_dtype=1)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,classes", [(5, 40), (5, 9000), (300, 1000), (600, 20000)])
def test_every_class_at_the_lowest_value(dtype, rows, classes):
    """A mask of the lowest value over all classes leaves a uniform softmax (one of -infinity leaves none: NaN)."""
    import torch
    from paper_2007_10412_amd import binding as B
    x = torch.zeros(rows, 64, device="cuda", dtype=torch_dtype(dtype))
    W = torch.zeros(64, classes, device="cuda", dtype=torch_dtype(dtype))
    labels = torch.arange(rows, device="cuda", dtype=torch.int32)
    index = torch.stack([labels, labels + 1], dim=1).clamp(max=classes - 1).contiguous()
    logit = torch.zeros(rows, 2, device="cuda")
    layer = B.make_layer(rows, 64, classes, dtype=dtype, relu=False, has_bias=True)
    row, db = torch.empty(rows, device="cuda"), torch.empty(classes, device="cuda")
    with Ctx() as ctx:
        for low, want in ((torch.finfo(torch.float32).min, math.log(classes)), (-math.inf, math.nan)):
            b = torch.full((classes,), low, device="cuda")
            B.rad_linear_ce(ctx, layer, x, W, b, labels, row_loss=row, dbias=db)
            B.rad_ctx_synchronize(ctx)
            if math.isnan(want):
                assert torch.isnan(row).all() and torch.isnan(db).all()
                continue
            assert float((row - want).abs().max()) < 1e-5 * want
            assert float((db[rows:] - 1 / classes).abs().max()) <= 2 ** -8 / classes if rows < classes else True
            z = torch.full((rows, classes), torch.finfo(torch_dtype(dtype)).min, device="cuda", dtype=torch_dtype(dtype))
            dz = torch.empty_like(z)
            B.rad_distill_ce(ctx, z, B.make_teacher(index, logit), dtype, dz, row_loss=row)
            B.rad_ctx_synchronize(ctx)
            assert float((row[:-1] - (want - math.log(2))).abs().max()) < 1e-5 * want
            assert torch.isfinite(dz.float()).all()


def test_not_a_number_stays_in_its_row():
    import torch
    from paper_2007_10412_amd import binding as B
    for dtype in (0, 1):
        x = torch.randn(300, 64, device="cuda").to(torch_dtype(dtype))
        W = torch.randn(64, 1000, device="cuda").to(torch_dtype(dtype))
        x[7, 3] = math.nan
        labels = torch.randint(0, 1000, (300,), device="cuda", dtype=torch.int32)
        row, dX = torch.empty(300, device="cuda"), torch.empty_like(x)
        with Ctx() as ctx:
            B.rad_linear_ce(ctx, B.make_layer(300, 64, 1000, dtype=dtype, relu=False), x, W, None, labels, row_loss=row, dX=dX)
            B.rad_ctx_synchronize(ctx)
        bad = torch.isnan(row)
        assert bad[7] and int(bad.sum()) == 1 and torch.isnan(dX[7]).all() and int(torch.isnan(dX).any(dim=1).sum()) == 1


# ------------------------------------------------------------------ dense logits
def check_distill(ctx, dtype, rows, classes, k, T=1.0, missing=0.0, weight=None, in_place=False, shift=0, doubles=False, scale=3.0,
                  masked=0.0, outputs=("dlogits", "row_loss", "loss")):
    import torch
    from paper_2007_10412_amd import binding as B
    tag = "distill dtype %d, %d x %d, k %d" % (dtype, rows, classes, k)
    print(tag, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + 3 * classes + k)
    td = torch_dtype(dtype)
    room = torch.empty(rows * classes + shift, device="cuda", dtype=td)
    z = room[shift:].view(rows, classes)
    z.copy_((scale * torch.randn(rows, classes, device="cuda", generator=gen)).to(td))
    index, logit = teacher_for(rows, classes, k, gen, missing, doubles)
    if masked:
        out = torch.rand(rows, classes, device="cuda", generator=gen) < masked
        out.scatter_(1, index.long().clamp(0, classes - 1), False)
        z.masked_fill_(out, -math.inf)
    zd = z.double()
    f32 = dict(device="cuda", dtype=torch.float32)
    dz = z if in_place else torch.full_like(z, math.nan)
    got = {"dlogits": dz, "row_loss": torch.full((rows,), math.nan, **f32), "loss": torch.full((1,), math.nan, **f32)}
    B.rad_distill_ce(ctx, z, B.make_teacher(index, logit, T), dtype, row_weight=weight, **{n: got[n] for n in outputs})
    B.rad_ctx_synchronize(ctx)
    targets = lists(teacher=(index, logit), classes=classes, T=T)
    row, loss, want, soft, target = definition(zd, targets, weight, T)
    rel = softmax_error(4 * U * float(zd[torch.isfinite(zd)].abs().max()) / T, classes)
    row_bound = T * T * (rel + 8 * U * (targets[2].abs() + 30 + float(zd[torch.isfinite(zd)].abs().max()) / T))
    if "row_loss" in outputs:
        close(got["row_loss"], row, row_bound * torch.ones_like(row), tag + " row_loss")
    if "loss" in outputs:
        w_all = weight.double().abs() if weight is not None else torch.ones_like(row) / max(1, int(targets[3].sum()))
        close(got["loss"], loss.reshape(1), ((row_bound + 8 * U * math.sqrt(rows) * row.abs()) * w_all).sum().reshape(1), tag + " loss")
    if "dlogits" in outputs:
        close(dz, want, soft * rel + (4 * U + list_error((index, logit), T)) * target + HALF[dtype] * want.abs() + 1e-37, tag + " dlogits")
        assert (dz[~targets[3]] == 0).all()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,classes,k", [(1, 1, 1), (1, 7, 3), (5, 1000, 64), (300, 1001, 17), (300, 9000, 1024), (256, 33333, 5),
                                            (260, 70001, 33), (257, 131072, 8), (2, 300001, 128), (300, 140001, 2), (700, 10, 10), (255, 4096, 64)])
def test_distill(dtype, rows, classes, k):
    with Ctx() as ctx:
        check_distill(ctx, dtype, rows, classes, k, T=1.0 if k % 2 else 2.0)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,classes,k", [(6, 1000, 64), (300, 1001, 17), (300, 9001, 130), (3, 50001, 1000)])
@pytest.mark.parametrize("how", ["missing", "weight", "in_place", "shifted", "shifted_in_place", "doubles", "masked", "loss", "gradient"])
def test_distill_kinds(dtype, rows, classes, k, how):
    import torch
    weight = torch.randn(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(rows)) if how == "weight" else None
    with Ctx() as ctx:
        check_distill(ctx, dtype, rows, classes, k, T=0.8, missing=0.4 if how == "missing" else 0.0, weight=weight,
                      in_place=how.endswith("in_place"), shift=3 if how.startswith("shifted") else 0, doubles=how == "doubles",
                      masked=0.5 if how == "masked" else 0.0,
                      outputs={"loss": ("loss",), "gradient": ("dlogits",)}.get(how, ("dlogits", "row_loss", "loss")))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,classes,offset,scale", [(40, 3000, 0.0, 100.0), (300, 3000, 0.0, 100.0), (2, 40000, 0.0, 50.0)])
def test_distill_peaked(dtype, rows, classes, offset, scale):
    with Ctx() as ctx:
        check_distill(ctx, dtype, rows, classes, 9, T=1.0, scale=scale)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows", [3, 300])
def test_impossible_target(dtype, rows):
    """A target whose logit is -infinity costs infinity; one whose probability rounds to zero costs nothing."""
    import torch
    from paper_2007_10412_amd import binding as B
    z = torch.randn(rows, 500, device="cuda").to(torch_dtype(dtype))
    z[:, 3] = -math.inf
    index = torch.tensor([[3, 5]], device="cuda", dtype=torch.int32).repeat(rows, 1)
    logit = torch.tensor([[0.0, 1.0]], device="cuda").repeat(rows, 1)
    logit[1, 0] = -200.0
    row, dz = torch.empty(rows, device="cuda"), torch.empty_like(z)
    with Ctx() as ctx:
        B.rad_distill_ce(ctx, z, B.make_teacher(index, logit), dtype, dz, row_loss=row)
        B.rad_ctx_synchronize(ctx)
    assert torch.isinf(row[0]) and row[0] > 0 and torch.isfinite(row[1]) and torch.isinf(row[2])
    assert torch.isfinite(dz.float()).all()


# ------------------------------------------------------------------ gradients against differences
def test_gradients_against_differences():
    """fp64 differences of the loss that the call itself returns, along random directions of x and W (fp32).  The loss L of 12
    rows is a mean of fp32 row losses: a value is off by at most 1e-5 (8 u (lse + |z|) with both below 12, and the logits'
    own 8 u sqrt(40) sum|terms|), a difference over 2 eps = 0.02 by 1e-3, and the curvature adds eps^2 / 6 times a third
    derivative of at most 8 |direction of z|^3 <= 8 x 3^3: 4e-3."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows, d, v = 12, 40, 77
    x = torch.randn(rows, d, device="cuda", generator=gen)
    W = torch.randn(d, v, device="cuda", generator=gen) / math.sqrt(d)
    labels = labels_for(rows, v, gen)
    index, logit = teacher_for(rows, v, 6, gen)
    layer = B.make_layer(rows, d, v, relu=False)
    with Ctx() as ctx:
        for kind in ("ce", "distill"):
            def call(x_, W_, **out):
                if kind == "ce":
                    B.rad_linear_ce(ctx, layer, x_, W_, None, labels, **out)
                else:
                    B.rad_linear_distill(ctx, layer, x_, W_, None, B.make_teacher(index, logit, 1.5), **out)
                B.rad_ctx_synchronize(ctx)
            dX, dW, loss = torch.empty_like(x), torch.empty_like(W), torch.empty(1, device="cuda")
            call(x, W, dX=dX, dW=dW)
            for n in range(4):
                ux = torch.randn(rows, d, device="cuda", generator=gen) / math.sqrt(d)
                uW = torch.randn(d, v, device="cuda", generator=gen) / math.sqrt(d)
                want = float((dX.double() * ux).sum() + (dW.double() * uW).sum())
                eps, ends = 0.01, []
                for sign in (1, -1):
                    call(x + sign * eps * ux, W + sign * eps * uW, loss=loss)
                    ends.append(float(loss))
                assert abs((ends[0] - ends[1]) / (2 * eps) - want) < 5e-3, (kind, n)


# ------------------------------------------------------------------ how a program uses them
def test_two_calls_agree_bit_by_bit():
    import torch
    with Ctx() as ctx:
        for dtype in (0, 1):
            for shape in ((300, 512, 4096), (600, 512, 20000)):
                a = check_linear(ctx, dtype, *shape, bias=True, k=9)
                b = check_linear(ctx, dtype, *shape, bias=True, k=9)
                assert all(torch.equal(a[n], b[n]) for n in a)


def test_other_stream():
    """The calls run on the context's stream, beside work on torch's own."""
    import torch
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with Ctx(stream) as ctx:
        with torch.cuda.stream(stream):
            check_linear(ctx, 1, 300, 512, 4096, k=5)
            check_distill(ctx, 1, 300, 4097, 5)


@pytest.mark.parametrize("dtype,rows,d_in,classes", [(0, 150, 300, 10), (1, 300, 512, 4096), (1, 5, 512, 4096), (0, 40, 256, 3000),
                                                     (1, 600, 264, 20001)])
def test_captured(dtype, rows, d_in, classes):
    """Recorded after one call of the same sizes, replayed with other inputs and eager work in between."""
    import torch
    from paper_2007_10412_amd import binding as B
    td = torch_dtype(dtype)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, d_in, device="cuda", generator=gen).to(td)
    W = (torch.randn(d_in, classes, device="cuda", generator=gen) / 8).to(td)
    labels = labels_for(rows, classes, gen, 0.2)
    index, logit = teacher_for(rows, classes, 5, gen, 0.2)
    layer = B.make_layer(rows, d_in, classes, dtype=dtype, relu=False)
    z = torch.randn(rows, classes, device="cuda", generator=gen).to(td)

    def outputs():
        return [torch.empty(1, device="cuda"), torch.empty_like(x), torch.empty_like(W), torch.empty(1, device="cuda"),
                torch.empty_like(x), torch.empty_like(W), torch.empty_like(z), torch.empty(1, device="cuda")]
    stream = torch.cuda.Stream()
    held, eager = outputs(), outputs()
    torch.cuda.synchronize()

    def calls(ctx, o):
        B.rad_linear_ce(ctx, layer, x, W, None, labels, loss=o[0], dX=o[1], dW=o[2])
        B.rad_linear_distill(ctx, layer, x, W, None, B.make_teacher(index, logit, 1.5), loss=o[3], dX=o[4], dW=o[5])
        B.rad_distill_ce(ctx, z, B.make_teacher(index, logit, 1.5), dtype, o[6], loss=o[7])
    with Ctx(stream) as ctx:
        calls(ctx, held)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            calls(ctx, held)
        for n in range(4):
            x.copy_(torch.randn(rows, d_in, device="cuda", generator=gen))
            labels.copy_(labels_for(rows, classes, gen, 0.2))
            z.copy_(torch.randn(rows, classes, device="cuda", generator=gen))
            for o in held:
                o.fill_(math.nan)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            calls(ctx, eager)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, eager)), n
            assert all(torch.isfinite(a.float()).all() for a in held)
        graph = None


def test_refusals():
    import torch
    from paper_2007_10412_amd import binding as B
    x, W = torch.randn(4, 8, device="cuda"), torch.randn(8, 16, device="cuda")
    labels = torch.zeros(4, device="cuda", dtype=torch.int32)
    index, logit = torch.zeros(4, 2, device="cuda", dtype=torch.int32), torch.zeros(4, 2, device="cuda")
    loss = torch.zeros(1, device="cuda")
    make = lambda **kw: B.make_layer(4, 8, 16, **{"relu": False, **kw})  # noqa: E731
    big = B.make_layer(4, 1 << 17, 1 << 15, relu=False)

    def refused(status, call):
        with pytest.raises(B.RadError) as e:
            call()
        assert e.value.status == status, e.value
    with Ctx() as ctx:
        def ce(status, layer=make(), x=x, W=W, bias=None, labels=labels, **kw):
            refused(status, lambda: B.rad_linear_ce(ctx, layer, x, W, bias, labels, **(kw or {"loss": loss})))
        ce(B.RAD_ERR_NULL, x=None)
        ce(B.RAD_ERR_NULL, W=None)
        ce(B.RAD_ERR_NULL, labels=None)
        ce(B.RAD_ERR_NULL, layer=make(has_bias=True))
        ce(B.RAD_ERR_NULL, bias=torch.zeros(16, device="cuda"))
        ce(B.RAD_ERR_NULL, beta=1.0)                                # no output
        ce(B.RAD_ERR_PARAM, loss=loss, beta=0.5)
        ce(B.RAD_ERR_PARAM, layer=make(relu=True))
        ce(B.RAD_ERR_PARAM, layer=make(dtype=7))
        ce(B.RAD_ERR_PARAM, dW=torch.empty(8, 16, device="cuda", dtype=torch.bfloat16))      # of an fp32 layer
        ce(B.RAD_ERR_SHAPE, layer=B.make_layer(0, 8, 16, relu=False))
        ce(B.RAD_ERR_SHAPE, layer=big)
        ce(B.RAD_ERR_SHAPE, x=torch.randn(8, 4, device="cuda").t())
        for k, T, status in ((0, 1.0, B.RAD_ERR_SHAPE), (1025, 1.0, B.RAD_ERR_SHAPE), (2, 0.0, B.RAD_ERR_PARAM),
                             (2, -1.0, B.RAD_ERR_PARAM), (2, math.inf, B.RAD_ERR_PARAM), (2, math.nan, B.RAD_ERR_PARAM)):
            t = B.make_teacher(index, logit, T)
            t.k = k
            refused(status, lambda: B.rad_linear_distill(ctx, make(), x, W, None, t, loss=loss))
            refused(status, lambda: B.rad_distill_ce(ctx, torch.randn(4, 16, device="cuda"), t, B.RAD_F32, loss=loss))
        t = B.make_teacher(index, logit)
        refused(B.RAD_ERR_NULL, lambda: B.rad_distill_ce(ctx, torch.randn(4, 16, device="cuda"), t, B.RAD_F32))
        refused(B.RAD_ERR_PARAM, lambda: B.rad_distill_ce(ctx, torch.randn(4, 16, device="cuda"), t, 5, loss=loss))
        t.index = None
        refused(B.RAD_ERR_NULL, lambda: B.rad_distill_ce(ctx, torch.randn(4, 16, device="cuda"), t, B.RAD_F32, loss=loss))
        B.rad_linear_ce(ctx, make(), x, W, None, labels, loss=loss)  # the context goes on
        B.rad_ctx_synchronize(ctx)
        assert torch.isfinite(loss).all()


@pytest.mark.parametrize("dtype", [0, 1])
def test_training_step_of_two_layers(dtype):
    """A sampled layer below, the loss over the vocabulary on top, both updated: as one step of a program."""
    import torch
    from paper_2007_10412_amd import binding as B
    from tests.gpu_util import rel_err
    rows, d0, d1, v = 256, 96, 128, 1000
    gen = torch.Generator(device="cuda").manual_seed(11)
    td = torch_dtype(dtype)
    x = torch.randn(rows, d0, device="cuda", generator=gen).to(td)
    W0 = (torch.randn(d0, d1, device="cuda", generator=gen) / math.sqrt(d0))
    W1 = (torch.randn(d1, v, device="cuda", generator=gen) / math.sqrt(d1))
    p0, p1 = W0.to(td).clone(), W1.to(td).clone()     # (updated in place)
    master = [p0.float(), p1.float()]
    labels = labels_for(rows, v, gen, 0.1)
    L0 = B.make_layer(rows, d0, d1, dtype=dtype, relu=True)
    L1 = B.make_layer(rows, d1, v, dtype=dtype, relu=False)
    h, dh = torch.empty(rows, d1, device="cuda", dtype=td), torch.empty(rows, d1, device="cuda", dtype=td)
    g0, g1, loss = torch.empty(d0, d1, device="cuda"), torch.empty(d1, v, device="cuda"), torch.empty(1, device="cuda")
    with Ctx() as ctx:
        store = B.rad_store_create(ctx, L0, B.RAD_EXACT, 1.0)
        B.rad_forward_sample(ctx, L0, B.make_sampling(B.RAD_EXACT, 1.0, 1), x, p0, None, h, store)
        B.rad_linear_ce(ctx, L1, h, p1, None, labels, loss=loss, dX=dh, dW=g1)
        B.rad_backward_dW(ctx, L0, store, dh, g0)
        B.rad_optimizer_step(ctx, B.make_optimizer(B.RAD_SGD, 0.5), 1, dtype, [p0, p1], [g0, g1], master=master if dtype else None)
        B.rad_ctx_synchronize(ctx)
        B.rad_store_destroy(store)
    hd = torch.relu(x.double() @ (W0.to(td).double())).to(td).double()
    w1 = W1.to(td).double()
    _, want, dz, _, _ = definition(hd @ w1, lists(labels=labels, classes=v), None, 1.0)
    dhd = (dz @ w1.t().contiguous()) * (h > 0)
    tol = 2e-5 if dtype == 0 else 2 ** -6      # four roundings to bf16 in a chain (h, dz, dh, and h again where it differs)
    assert abs(float(loss) - float(want)) < (1e-4 if dtype == 0 else 1e-2)
    assert rel_err(g1.cpu().numpy(), (hd.t().contiguous() @ dz).cpu().numpy()) < tol
    assert rel_err(g0.cpu().numpy(), (x.double().t().contiguous() @ dhd).cpu().numpy()) < tol
    moved = (master if dtype else [p0, p1])
    assert rel_err(moved[1].cpu().numpy(), (w1 - 0.5 * (hd.t().contiguous() @ dz)).cpu().numpy()) < tol


@pytest.mark.parametrize("rows,d_in,classes", [(463, 256, 3990), (455, 300, 30000)])
@pytest.mark.parametrize("how", ["mean", "weight", "temperature"])
def test_a_common_factor_is_not_rounded(rows, d_in, classes, how):
    """A factor of all rows (1 / n, a weight that they share, T) belongs to the fp32 ends of the gradients: rounded to bf16 into
    every dz, its error of up to 2^-9 would be that of all of dX and dW.  Seen as the scale of what comes out along what should:
    the roundings that are left are independent ones, of 2^-8 at most, over 10^5 elements and more, whose share of that scale is
    8 standard deviations of 2^-8 / sqrt(10^5) < 2^-13 at most; targets near -1 and 0.5 themselves round by less than 2^-11 of
    the whole (1 - q and 0.5 - q with q of a few thousandths)."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, d_in, device="cuda", generator=gen).to(torch.bfloat16)
    W = (torch.randn(d_in, classes, device="cuda", generator=gen) / math.sqrt(d_in)).to(torch.bfloat16)
    index = torch.stack([torch.arange(rows, device="cuda"), torch.arange(rows, device="cuda") + rows], dim=1).to(torch.int32)
    logit = torch.zeros(rows, 2, device="cuda")
    T = 0.7 if how == "temperature" else 1.0
    weight = torch.full((rows,), 0.3003, device="cuda") if how == "weight" else None
    layer = B.make_layer(rows, d_in, classes, dtype=B.RAD_BF16, relu=False)
    xd, Wd = x.double(), W.double()
    with Ctx() as ctx:
        for kind in ("ce", "distill"):
            dX, dW = torch.empty_like(x), torch.empty(d_in, classes, device="cuda")
            if kind == "ce":
                labels = index[:, 0].contiguous()
                B.rad_linear_ce(ctx, layer, x, W, None, labels, row_weight=weight, dX=dX, dW=dW)
                _, _, dz, _, _ = definition(xd @ Wd, lists(labels=labels, classes=classes), weight, 1.0)
            else:
                B.rad_linear_distill(ctx, layer, x, W, None, B.make_teacher(index, logit, T), row_weight=weight, dX=dX, dW=dW)
                _, _, dz, _, _ = definition(xd @ Wd, lists(teacher=(index, logit), classes=classes, T=T), weight, T)
            B.rad_ctx_synchronize(ctx)
            for got, want in ((dX, dz @ Wd.t().contiguous()), (dW, xd.t().contiguous() @ dz)):
                scale = float((got.double() * want).sum() / (want * want).sum())
                assert abs(scale - 1) < 2.0 ** -11 + 2.0 ** -13, (kind, how, scale)


# ------------------------------------------------------------------ what a call may meet
# small layers of few classes, tiles of 64, 128 and 256 rows, products with a split K
ROUTES = [(150, 300, 10), (40, 1024, 5000), (300, 512, 4096), (600, 256, 20000), (1100, 512, 1000)]


def run_linear(ctx, layer, x, W, labels=None, teacher=None, weight=None, shift=0):
    """All outputs, each a view `shift` elements into its memory."""
    import torch
    from paper_2007_10412_amd import binding as B

    def room(like, dtype=None):
        t = torch.full((like.numel() + shift,), math.nan, device="cuda", dtype=dtype or like.dtype)
        return t[shift:].view(like.shape)
    one = torch.empty(1, device="cuda")
    out = {"row_loss": room(x[:, 0], torch.float32), "loss": room(one), "dX": room(x), "dW": room(W), "dbias": room(W[0], torch.float32)}
    if labels is not None:
        B.rad_linear_ce(ctx, layer, x, W, None, labels, row_weight=weight, **out)
    else:
        B.rad_linear_distill(ctx, layer, x, W, None, teacher, row_weight=weight, **out)
    B.rad_ctx_synchronize(ctx)
    return out


def inputs(dtype, rows, d_in, classes, seed=3):
    import torch
    from paper_2007_10412_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, d_in, device="cuda", generator=gen).to(torch_dtype(dtype))
    W = (torch.randn(d_in, classes, device="cuda", generator=gen) * (3 / math.sqrt(d_in))).to(torch_dtype(dtype))
    return gen, x, W, B.make_layer(rows, d_in, classes, dtype=dtype, relu=False)


def same(a, b, tag):
    import torch
    for n in a:
        assert torch.equal(a[n], b[n]), "%s: %s" % (tag, n)
        assert torch.isfinite(a[n].float()).all(), "%s: %s" % (tag, n)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", ROUTES)
def test_views_at_odd_addresses(dtype, rows, d_in, classes):
    """Inputs and outputs that begin at any element give what others give, bit by bit."""
    import torch
    gen, x, W, layer = inputs(dtype, rows, d_in, classes)
    labels = labels_for(rows, classes, gen, 0.2)

    def moved(t):
        m = torch.empty(t.numel() + 3, device="cuda", dtype=t.dtype)[3:].view(t.shape)
        m.copy_(t)
        return m
    with Ctx() as ctx:
        want = run_linear(ctx, layer, x, W, labels)
        same(run_linear(ctx, layer, moved(x), moved(W), moved(labels), shift=1), want, "moved")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", ROUTES)
@pytest.mark.parametrize("k", [0, 4])
def test_rows_without_a_target_hold_anything(dtype, rows, d_in, classes, k):
    """What x and the weights hold in such rows, and what an earlier call left in the workspaces, reaches no output."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen, x, W, layer = inputs(dtype, rows, d_in, classes)
    labels = labels_for(rows, classes, gen, 0.3)
    gone = (labels < 0) | (labels >= classes)
    gone[-3:] = True
    labels[-3:] = -1
    assert gone.any() and not gone.all()
    index, logit = teacher_for(rows, classes, k or 1, gen)
    index[gone] = -1
    weight = torch.randn(rows, device="cuda", generator=gen)
    x[gone] = 0
    bad_x, bad_weight = x.clone(), weight.clone()
    bad_x[gone] = torch.tensor([math.nan, math.inf, -math.inf], device="cuda").to(x.dtype)[torch.arange(d_in, device="cuda") % 3]
    bad_weight[gone] = math.nan
    asked = dict(labels=labels) if not k else dict(teacher=B.make_teacher(index, logit, 1.5))
    with Ctx() as ctx:
        want = [run_linear(ctx, layer, x, W, weight=w, **asked) for w in (None, weight)]
        got = [run_linear(ctx, layer, bad_x, W, weight=w, **asked) for w in (None, bad_weight)]
        run_linear(ctx, layer, torch.full_like(x, math.nan), W, labels=torch.zeros_like(labels))
        got += [run_linear(ctx, layer, bad_x, W, weight=w, **asked) for w in (None, bad_weight)]
    for n, g in enumerate(got):
        same(g, want[n % 2], "call %d" % n)
        assert (g["dX"][gone] == 0).all() and (g["row_loss"][gone] == 0).all()


@pytest.mark.parametrize("dtype,dw_dtype", [(0, 0), (1, 0), (1, 1)])
@pytest.mark.parametrize("rows,d_in,classes,k", [(1, 1, 16, 1), (37, 65, 16, 16), (1000, 99, 7, 3), (256, 390, 12, 0), (5, 3001, 2, 0), (33, 64, 1, 2),
                                               (1700, 64, 10, 4), (1800, 64, 10, 4), (2, 3990, 16, 0), (2, 4000, 16, 0)])
def test_few_classes(dtype, dw_dtype, rows, d_in, classes, k):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows)
    weight = torch.randn(rows, device="cuda", generator=gen)
    with Ctx() as ctx:
        for w, beta in ((None, 0.0), (None, 1.0), (weight, 0.0), (weight, 1.0)):
            check_linear(ctx, dtype, rows, d_in, classes, bias=beta == 0.0, k=k, T=1.0 if not k else 1.7, ignored=0.3, missing=0.2,
                         weight=w, beta=beta, dw_dtype=dw_dtype)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes,k", [(1100, 64, 520, 3), (8192, 40, 130, 0), (8193, 40, 130, 2), (20000, 24, 77, 0), (17000, 16, 33, 5)])
def test_many_rows(dtype, rows, d_in, classes, k):
    """Lists of rows that one workgroup makes in one step, and in several."""
    import torch
    weight = torch.randn(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(rows))
    with Ctx() as ctx:
        for w in (None, weight):
            check_linear(ctx, dtype, rows, d_in, classes, bias=True, k=k, T=1.0 if not k else 2.0, ignored=0.3, missing=0.2, weight=w)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes,k", [(3, 2048, 1500, 0), (3, 2048, 1500, 9), (40, 1024, 5000, 7), (1, 4096, 257, 2), (70, 1500, 999, 0)])
def test_few_tiles(dtype, rows, d_in, classes, k):
    """Products whose K is split, with biases, lists and weights."""
    import torch
    weight = torch.randn(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(rows))
    with Ctx() as ctx:
        for w in (None, weight):
            check_linear(ctx, dtype, rows, d_in, classes, bias=True, k=k, T=1.0 if not k else 0.7, ignored=0.3 if rows > 8 else 0.0, weight=w)
            check_linear(ctx, dtype, rows, d_in, classes, bias=True, k=k, T=1.0 if not k else 0.7, weight=w, outputs=("row_loss", "loss"))


def test_two_contexts_at_once():
    """Calls of two contexts on two streams, with nothing between them that waits."""
    import torch
    from paper_2007_10412_amd import binding as B
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    jobs = []
    for n, (dtype, rows, d_in, classes) in enumerate(((1, 600, 256, 20000), (0, 300, 512, 4096))):
        gen, x, W, layer = inputs(dtype, rows, d_in, classes, seed=n)
        jobs.append((layer, x, W, labels_for(rows, classes, gen, 0.2), *teacher_for(rows, classes, 6, gen, 0.1)))

    def outputs():
        return [[torch.empty(1, device="cuda"), torch.empty_like(j[1]), torch.empty_like(j[2]), torch.empty(1, device="cuda"),
                 torch.empty_like(j[1]), torch.empty_like(j[2])] for j in jobs]

    def calls(ctx, j, o):
        B.rad_linear_ce(ctx, j[0], j[1], j[2], None, j[3], loss=o[0], dX=o[1], dW=o[2])
        B.rad_linear_distill(ctx, j[0], j[1], j[2], None, B.make_teacher(j[4], j[5]), loss=o[3], dX=o[4], dW=o[5])
    alone, together = outputs(), outputs()
    torch.cuda.synchronize()
    with Ctx(streams[0]) as a, Ctx(streams[1]) as b:
        for ctx, j, o in zip((a, b), jobs, alone):
            calls(ctx, j, o)
            torch.cuda.synchronize()
        for _ in range(5):
            for ctx, j, o in zip((a, b), jobs, together):
                calls(ctx, j, o)
        torch.cuda.synchronize()
    for x, y in zip(alone, together):
        assert all(torch.equal(p, q) for p, q in zip(x, y))


@pytest.mark.parametrize("dtype,rows,d_in,classes", [(1, 2500, 512, 1000), (0, 1500, 100, 700), (1, 9000, 64, 300)])
def test_captured_many_rows(dtype, rows, d_in, classes):
    test_captured(dtype, rows, d_in, classes)


def test_refused_overlaps():
    import torch
    from paper_2007_10412_amd import binding as B
    room = torch.randn(4096, device="cuda")
    kept = room.clone()
    x, W = room[:32].view(4, 8), room[32:160].view(8, 16)
    labels = torch.zeros(4, device="cuda", dtype=torch.int32)
    index, logit = torch.zeros(4, 2, device="cuda", dtype=torch.int32), torch.zeros(4, 2, device="cuda")
    z = room[1000:1064].view(4, 16)
    layer = B.make_layer(4, 8, 16, relu=False)
    teacher = B.make_teacher(index, logit)
    row = torch.zeros(4, device="cuda")
    with Ctx() as ctx:
        for out in (dict(dX=x), dict(dW=W), dict(dX=room[8:40].view(4, 8)), dict(dW=room[150:278].view(8, 16)), dict(row_loss=room[30:34]),
                    dict(loss=room[100:101]), dict(dbias=room[20:36]), dict(dX=room[200:232].view(4, 8), dW=room[231:359].view(8, 16)),
                    dict(row_loss=row, row_weight=row)):
            for call in (lambda: B.rad_linear_ce(ctx, layer, x, W, None, labels, **out),
                         lambda: B.rad_linear_distill(ctx, layer, x, W, None, teacher, **out)):
                with pytest.raises(B.RadError) as e:
                    call()
                assert e.value.status == B.RAD_ERR_PARAM, out.keys()
        with pytest.raises(B.RadError) as e:
            B.rad_linear_ce(ctx, layer, x, W, None, labels, loss=labels[2:3].view(torch.float32))
        assert e.value.status == B.RAD_ERR_PARAM
        for out in (dict(dlogits=room[1001:1065].view(4, 16)), dict(row_loss=room[1060:1064]), dict(dlogits=z, loss=room[1000:1001]),
                    dict(loss=logit[1, :1]), dict(row_loss=row, row_weight=row)):
            with pytest.raises(B.RadError) as e:
                B.rad_distill_ce(ctx, z, teacher, B.RAD_F32, **out)
            assert e.value.status == B.RAD_ERR_PARAM, out.keys()
        B.rad_ctx_synchronize(ctx)
    assert torch.equal(room, kept)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes,ignored", [(4096, 1024, 8000, 0.97), (4096, 512, 1000, 0.995), (2048, 256, 300, 0.99)])
def test_few_rows_of_many(dtype, rows, d_in, classes, ignored):
    """Products that are laid out for all rows, where the last parts of a split K have none that count."""
    with Ctx() as ctx:
        check_linear(ctx, dtype, rows, d_in, classes, ignored=ignored)
        check_linear(ctx, dtype, rows, d_in, classes, ignored=ignored, beta=1.0, dw_dtype=dtype)


def test_two_graphs_of_one_context():
    """They share its workspaces: replayed in turn, with eager calls of both sizes and other inputs in between."""
    import torch
    from paper_2007_10412_amd import binding as B
    stream = torch.cuda.Stream()
    jobs = [inputs(dtype, *shape, seed=n) for n, (dtype, *shape) in enumerate(((1, 600, 264, 20000), (0, 300, 200, 1003), (1, 40, 30, 10)))]
    jobs = [(gen, x, W, layer, labels_for(len(x), W.shape[1], gen, 0.2), *teacher_for(len(x), W.shape[1], 6, gen, 0.1)) for gen, x, W, layer in jobs]

    def outputs(j):
        return [torch.empty(1, device="cuda"), torch.empty_like(j[1]), torch.empty_like(j[2]), torch.empty(1, device="cuda"),
                torch.empty_like(j[1]), torch.empty_like(j[2])]

    def calls(ctx, j, o):
        B.rad_linear_ce(ctx, j[3], j[1], j[2], None, j[4], loss=o[0], dX=o[1], dW=o[2])
        B.rad_linear_distill(ctx, j[3], j[1], j[2], None, B.make_teacher(j[5], j[6]), loss=o[3], dX=o[4], dW=o[5])
    held, eager = [outputs(j) for j in jobs], [outputs(j) for j in jobs]
    torch.cuda.synchronize()
    with Ctx(stream) as ctx:
        for j, o in zip(jobs, eager):                               # (the workspaces grow here)
            calls(ctx, j, o)
        torch.cuda.synchronize()
        graphs = []
        for j, o in zip(jobs, held):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=stream):
                calls(ctx, j, o)
        for n in range(3):
            for j in jobs:
                j[1].copy_(torch.randn(j[1].shape, device="cuda", generator=j[0]))
                j[4].copy_(labels_for(len(j[1]), j[2].shape[1], j[0], 0.2))
            for o in held:
                for t in o:
                    t.fill_(math.nan)
            torch.cuda.synchronize()
            for g in graphs if n % 2 else graphs[::-1]:
                g.replay()
            torch.cuda.synchronize()
            for j, h, e in zip(jobs, held, eager):
                calls(ctx, j, e)
                torch.cuda.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(h, e)), n
        graphs = None


def test_logits_past_32_bits():
    """Dense logits of over 2^32 elements, in place: the first, middle and last rows."""
    import torch
    from paper_2007_10412_amd import binding as B
    rows, classes, k = 33000, 131071, 3
    gen = torch.Generator(device="cuda").manual_seed(2)
    z = torch.empty(rows, classes, device="cuda", dtype=torch.bfloat16)
    z.normal_(0, 2, generator=gen)
    some = torch.tensor([0, 1, 16384, 16385, 32767, 32768, 32769, rows - 2, rows - 1], device="cuda")
    kept = z[some].double()
    index, logit = torch.randint(0, classes, (rows, k), device="cuda", generator=gen).to(torch.int32), torch.randn(rows, k, device="cuda", generator=gen)
    row = torch.empty(rows, device="cuda")
    with Ctx() as ctx:
        B.rad_distill_ce(ctx, z, B.make_teacher(index, logit), B.RAD_BF16, z, row_loss=row)
        B.rad_ctx_synchronize(ctx)
    targets = lists(teacher=(index[some], logit[some]), classes=classes)
    want_row, _, _, _, _ = definition(kept, targets, None, 1.0)
    _, _, dz, soft, target = definition(kept, targets, torch.full((len(some),), 1 / rows, device="cuda"), 1.0)
    rel = softmax_error(4 * U * float(kept.abs().max()), classes)
    close(row[some], want_row, (rel + 8 * U * 50) * torch.ones_like(want_row), "row_loss")
    close(z[some], dz, soft * rel + (6 * U + list_error((index[some], logit[some]), 1.0)) * target + HALF[1] * dz.abs() + 1e-37, "dlogits")


def test_rows_past_32_bits():
    """x of over 2^32 bytes: rows in pieces, dW and the loss over all of them."""
    import torch
    from paper_2007_10412_amd import binding as B
    rows, d_in, classes = 1100001, 2048, 24
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.empty(rows, d_in, device="cuda", dtype=torch.bfloat16)
    x.normal_(0, 1, generator=gen)
    W = (torch.randn(d_in, classes, device="cuda", generator=gen) / math.sqrt(d_in)).to(torch.bfloat16)
    labels = labels_for(rows, classes, gen, 0.2)
    counts = (labels >= 0) & (labels < classes)
    row, loss, dX, dW = torch.empty(rows, device="cuda"), torch.empty(1, device="cuda"), torch.full_like(x, math.nan), torch.empty(d_in, classes, device="cuda")
    with Ctx() as ctx:
        B.rad_linear_ce(ctx, B.make_layer(rows, d_in, classes, dtype=1, relu=False), x, W, None, labels, row_loss=row, loss=loss, dX=dX, dW=dW)
        B.rad_ctx_synchronize(ctx)
    n, Wd, total = int(counts.sum()), W.double(), 0.0
    want_dW, bound, mass = (torch.zeros(d_in, classes, device="cuda", dtype=torch.float64) for _ in range(3))
    for r in range(0, rows, 100000):
        at = slice(r, min(rows, r + 100000))
        xd = x[at].double()
        weight = torch.full((len(xd),), 1 / n, device="cuda", dtype=torch.float64)
        want, part, dz, soft, target = definition(xd @ Wd, lists(labels=labels[at], classes=classes), weight, 1.0)
        rel = softmax_error(8 * U * math.sqrt(d_in) * float((xd.abs() @ Wd.abs()).max()), classes)
        close(row[at], want, (rel + 8 * U * 50) * torch.ones_like(want), "row_loss %d" % r)
        total += float(part)
        e = soft * rel + 2.02 * HALF[1] * (soft + target) + 4 * U * target
        want_dX = dz @ Wd.t().contiguous()
        close(dX[at], want_dX, (e + 8 * U * math.sqrt(classes) * dz.abs()) @ Wd.abs().t().contiguous() + HALF[1] * want_dX.abs() + 1e-37, "dX %d" % r)
        want_dW += xd.t().contiguous() @ dz
        bound += xd.abs().t().contiguous() @ e
        mass += xd.abs().t().contiguous() @ dz.abs()
    close(dW, want_dW, bound + 8 * U * math.sqrt(rows) * mass, "dW")
    assert abs(float(loss) - total) < (rel + 8 * U * 50 + 8 * U * math.sqrt(rows)) * max(1.0, total)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,classes,k", [(204, 3000, 20), (205, 3000, 20), (256, 500, 16), (257, 500, 2), (16, 50257, 256), (15, 50257, 257), (2, 300001, 129),
                                            (255, 140003, 3), (1, 40, 200)])
@pytest.mark.parametrize("how", ["", "missing", "doubles", "weight", "in_place", "loss", "gradient"])
def test_short_lists(dtype, rows, classes, k, how):
    """Few rows: whole ones of every size of part, and rows in parts, with lists of up to 257 entries."""
    import torch
    weight = torch.randn(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(rows)) if how == "weight" else None
    with Ctx() as ctx:
        check_distill(ctx, dtype, rows, classes, k, T=1.3, missing=0.4 if how == "missing" else 0.0, weight=weight, in_place=how == "in_place",
                      doubles=how == "doubles", outputs=("loss",) if how == "loss" else ("dlogits",) if how in ("gradient", "in_place") else
                      ("dlogits", "row_loss", "loss"))

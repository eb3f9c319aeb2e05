"""Losses over a vocabulary at the ends of what their arguments may hold, against the definition in fp64 with the bounds of
test_gpu_vocab_loss (whose helpers these tests use)."""
import math

import pytest

from tests.test_gpu_vocab_loss import (HALF, ROUTES, U, Ctx, check_distill, check_linear, close, definition, inputs, labels_for, lists,
                                       run_linear, softmax_error, teacher_for, torch_dtype)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ row weights
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", ROUTES)
@pytest.mark.parametrize("k", [0, 4])
@pytest.mark.parametrize("how", ["nan", "inf", "all_nan"])
def test_weights_that_are_not_finite(dtype, rows, d_in, classes, k, how):
    """They reach their own rows of dX, and all of dW, dbias and the loss; rows of other weights keep their gradient."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen, x, W, layer = inputs(dtype, rows, d_in, classes)
    labels = labels_for(rows, classes, gen, 0.3)
    labels[1], labels[2] = 1, -1
    counts = (labels >= 0) & (labels < classes)
    index, logit = teacher_for(rows, classes, k or 1, gen)
    index[~counts] = -1
    asked = dict(labels=labels) if not k else dict(teacher=B.make_teacher(index, logit))
    finite = torch.rand(rows, device="cuda", generator=gen) + 0.5
    bad = torch.arange(rows, device="cuda") % 17 == 1
    if how == "all_nan":
        bad = counts.clone()
    weight = torch.where(bad, torch.full_like(finite, math.inf if how == "inf" else math.nan), finite)
    with Ctx() as ctx:
        out = run_linear(ctx, layer, x, W, weight=weight, **asked)
    xd, Wd = x.double(), W.double()
    z = xd @ Wd
    targets = lists(labels=labels, classes=classes) if not k else lists(teacher=(index, logit), classes=classes)
    row, _, dz, soft, target = definition(z, targets, finite, 1.0)
    rel = softmax_error(8 * U * math.sqrt(d_in + 2) * float((xd.abs() @ Wd.abs()).max()), classes)
    ep = U * (6 * float(logit.abs().max()) + 6 + 8 * math.sqrt(logit.shape[1])) if k else 0.0
    e = soft * rel + 2.02 * HALF[dtype] * (soft + target) + (4 * U + ep) * target
    want = dz @ Wd.t().contiguous()
    bound = (e + 8 * U * math.sqrt(classes) * dz.abs()) @ Wd.abs().t().contiguous() + HALF[dtype] * want.abs() + 1e-37
    good = ~(bad & counts)
    close(out["dX"][good], want[good], bound[good], "dX")
    assert (out["dX"][~counts] == 0).all()
    close(out["row_loss"], row, (rel + 8 * U * (targets[2].abs() + z.abs().max() + 30)) * torch.ones_like(row), "row_loss")
    assert not torch.isfinite(out["dX"][bad & counts]).any()
    for n in ("loss", "dW", "dbias"):
        assert not torch.isfinite(out[n]).any(), n


@pytest.mark.parametrize("dtype,dw_dtype", [(0, 0), (1, 0), (1, 1)])
@pytest.mark.parametrize("rows,d_in,classes", ROUTES)
@pytest.mark.parametrize("scale", [1e22, 1e-15, 1e-34])
def test_weights_far_apart(dtype, dw_dtype, rows, d_in, classes, scale):
    """Weights of 10^44 times each other (down to 10^-35 of 1): none of them is lost beside the others."""
    import torch
    weight = torch.tensor([scale, 1e-22, -1.0, 0.0] if scale > 1 else [scale, -scale, 0.1 * scale], device="cuda")
    weight = weight[torch.arange(rows, device="cuda") % len(weight)].contiguous()
    with Ctx() as ctx:
        check_linear(ctx, dtype, rows, d_in, classes, bias=True, ignored=0.3, weight=weight, dw_dtype=dw_dtype)
        check_linear(ctx, dtype, rows, d_in, classes, k=5, T=2.0, weight=weight, dw_dtype=dw_dtype)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", ROUTES)
@pytest.mark.parametrize("k", [0, 4])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_rows_without_a_target_have_no_gradient_whatever_w_holds(dtype, rows, d_in, classes, k, value):
    import torch
    from paper_2007_10412_amd import binding as B
    gen, x, W, layer = inputs(dtype, rows, d_in, classes)
    labels = labels_for(rows, classes, gen, 0.3)
    labels[:2] = -1
    gone = (labels < 0) | (labels >= classes)
    index, logit = teacher_for(rows, classes, k or 1, gen)
    index[gone] = -1
    W[d_in // 2, classes // 2] = value
    asked = dict(labels=labels) if not k else dict(teacher=B.make_teacher(index, logit))
    with Ctx() as ctx:
        out = run_linear(ctx, layer, x, W, **asked)
    assert (out["dX"][gone] == 0).all() and (out["row_loss"][gone] == 0).all()


# ------------------------------------------------------------------ masks of the type's lowest value
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,classes", [(5, 40), (300, 1000), (40, 20000), (3, 140001)])
@pytest.mark.parametrize("T", [1.0, 2.0, 0.7])
def test_first_target_masked_in_both(dtype, rows, classes, T):
    """The teacher's list begins with classes that both models mask with their type's lowest value: they have no share of the
    loss, which is the others'."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(rows)
    td = torch_dtype(dtype)
    z = (3 * torch.randn(rows, classes, device="cuda", generator=gen)).to(td)
    top = float(z.abs().max())
    z[:, :3] = torch.finfo(td).min
    index = torch.cat([torch.tensor([[1, 0, 2]], device="cuda").repeat(rows, 1),
                       3 + torch.rand(rows, min(classes - 3, 4096), device="cuda", generator=gen).argsort(dim=1)[:, :6]], dim=1).to(torch.int32)
    logit = 2 * torch.randn(rows, 9, device="cuda", generator=gen)
    logit[:, :3] = torch.finfo(torch.float32).min
    row, dz = torch.empty(rows, device="cuda"), torch.empty_like(z)
    with Ctx() as ctx:
        B.rad_distill_ce(ctx, z, B.make_teacher(index, logit, T), dtype, dz, row_loss=row)
        B.rad_ctx_synchronize(ctx)
    targets = lists(teacher=(index, logit), classes=classes, T=T)
    want, _, g, soft, target = definition(z.double(), targets, None, T)
    rel = softmax_error(4 * U * top / T, classes)
    close(row, want, T * T * (rel + 8 * U * (targets[2].abs() + 30 + top / T)) * torch.ones_like(want), "row_loss")
    ep = U * (6 * float(logit[:, 3:].abs().max()) / T + 6 + 8 * 3)
    close(dz, g, soft * rel + (4 * U + ep) * target + HALF[dtype] * g.abs() + 1e-37, "dlogits")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", ROUTES)
@pytest.mark.parametrize("T", [1.0, 0.7])
def test_first_target_masked_by_a_bias(dtype, rows, d_in, classes, T):
    import torch
    from paper_2007_10412_amd import binding as B
    gen, x, W, _ = inputs(dtype, rows, d_in, classes)
    layer = B.make_layer(rows, d_in, classes, dtype=dtype, relu=False, has_bias=True)
    bias = torch.zeros(classes, device="cuda")
    bias[:2] = torch.finfo(torch.float32).min
    index = torch.tensor([[0, 5, 1, 7]], device="cuda", dtype=torch.int32).repeat(rows, 1)
    logit = torch.randn(rows, 4, device="cuda", generator=gen)
    logit[:, 0] = logit[:, 2] = torch.finfo(torch.float32).min
    row, loss = torch.empty(rows, device="cuda"), torch.empty(1, device="cuda")
    with Ctx() as ctx:
        B.rad_linear_distill(ctx, layer, x, W, bias, B.make_teacher(index, logit, T), row_loss=row, loss=loss)
        B.rad_ctx_synchronize(ctx)
    xd, Wd = x.double(), W.double()
    z = xd @ Wd
    size, top = float((xd.abs() @ Wd.abs()).max()), float(z.abs().max())
    targets = lists(teacher=(index, logit), classes=classes, T=T)
    want, total, _, _, _ = definition(z + bias.double(), targets, None, T)
    bound = T * T * (softmax_error(8 * U * math.sqrt(d_in + 2) * size / T, classes) + 8 * U * (float(targets[2].abs().max()) + top / T + 30))
    close(row, want, bound * torch.ones_like(want), "row_loss")
    assert abs(float(loss) - float(total)) <= bound + 8 * U * math.sqrt(rows) * float(want.abs().max())


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,classes", [(6, 40), (300, 1000), (3, 140001)])
@pytest.mark.parametrize("T", [0.5, 1e-6, 3.0])
def test_teacher_logits_at_the_ends_of_fp32(dtype, rows, classes, T):
    """Logits that leave fp32 when they are divided by T count as what they are: a list of the lowest value is one of equal
    entries, the highest value has all of its row."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(rows)
    z = torch.randn(rows, classes, device="cuda", generator=gen).to(torch_dtype(dtype)) * min(T, 1.0)
    f = torch.finfo(torch.float32)
    index = torch.tensor([[3, 11, 7, 2]], device="cuda", dtype=torch.int32).repeat(rows, 1)
    logit = torch.tensor([[f.min] * 4, [f.max, 0.0, 1.0, f.min], [f.min, -math.inf, f.min, 0.25 * f.min]], device="cuda")
    logit = logit[torch.arange(rows, device="cuda") % 3].contiguous()
    row, loss, dz = torch.empty(rows, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(z)
    with Ctx() as ctx:
        B.rad_distill_ce(ctx, z, B.make_teacher(index, logit, T), dtype, dz, row_loss=row, loss=loss)
        B.rad_ctx_synchronize(ctx)
    targets = lists(teacher=(index, logit), classes=classes, T=T)
    assert targets[3].all()
    want, total, g, soft, target = definition(z.double(), targets, None, T)
    # (the lists' probabilities are 1, 0, 1/4: the exponentials of 0 and -infinity, and a division)
    rel = softmax_error(4 * U * float(z.double().abs().max()) / T, classes)
    bound = T * T * (rel + 8 * U * (targets[2].abs() + 30 + float(z.double().abs().max()) / T))
    close(row, want, bound * torch.ones_like(want), "row_loss")
    close(loss.double(), total.reshape(1), (bound + 8 * U * math.sqrt(rows) * want.abs()).mean().reshape(1), "loss")
    close(dz, g, soft * rel + 8 * U * target + HALF[dtype] * g.abs() + 1e-37, "dlogits")


# ------------------------------------------------------------------ rows in pieces
def test_workspaces_of_wide_rows():
    """x of 5 GB in rows of odd width: they are copied, and gathered for dW, a piece at a time, and the context holds no more than
    its header says; the gradients are those of all rows."""
    import torch
    from paper_2007_10412_amd import binding as B
    rows, d_in, classes = 600001, 4095, 24
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.empty(rows, d_in, device="cuda", dtype=torch.bfloat16)
    x.normal_(0, 1, generator=gen)
    W = (torch.randn(d_in, classes, device="cuda", generator=gen) / math.sqrt(d_in)).to(torch.bfloat16)
    labels = labels_for(rows, classes, gen, 0.2)
    counts = (labels >= 0) & (labels < classes)
    row, dX, dW = torch.empty(rows, device="cuda"), torch.full_like(x, math.nan), torch.empty(d_in, classes, device="cuda")
    with Ctx() as ctx:
        torch.cuda.synchronize()
        before = torch.cuda.mem_get_info()[0]
        B.rad_linear_ce(ctx, B.make_layer(rows, d_in, classes, dtype=1, relu=False), x, W, None, labels, row_loss=row, dX=dX, dW=dW)
        B.rad_ctx_synchronize(ctx)
        held = before - torch.cuda.mem_get_info()[0]
    piece = 2 ** 31 // (4096 * 2)
    partial = 64 * d_in * 64 * 4                                    # K of dW in up to 64 splits
    small = piece * (64 * 2 + 8 + 16) + rows * 12 + d_in * 64 * 2
    assert held <= 2 * 2 ** 31 + small + partial + 2 ** 26, held    # (and what modules and allocation granules take)
    n, Wd = int(counts.sum()), W.double()
    want_dW, bound, mass = (torch.zeros(d_in, classes, device="cuda", dtype=torch.float64) for _ in range(3))
    for r in range(0, rows, 60000):
        at = slice(r, min(rows, r + 60000))
        xd = x[at].double()
        weight = torch.full((len(xd),), 1 / n, device="cuda", dtype=torch.float64)
        want, _, dz, soft, target = definition(xd @ Wd, lists(labels=labels[at], classes=classes), weight, 1.0)
        rel = softmax_error(8 * U * math.sqrt(d_in) * float((xd.abs() @ Wd.abs()).max()), classes)
        close(row[at], want, (rel + 8 * U * 50) * torch.ones_like(want), "row_loss %d" % r)
        e = soft * rel + 2.02 * HALF[1] * (soft + target) + 4 * U * target
        want_dX = dz @ Wd.t().contiguous()
        close(dX[at], want_dX, (e + 8 * U * math.sqrt(classes) * dz.abs()) @ Wd.abs().t().contiguous() + HALF[1] * want_dX.abs() + 1e-37, "dX %d" % r)
        xt = xd.t().contiguous()
        want_dW += xt @ dz
        bound += xt.abs() @ e
        mass += xt.abs() @ dz.abs()
    close(dW, want_dW, bound + 8 * U * math.sqrt(rows) * mass, "dW")


def test_most_rows_of_an_odd_width():
    """2^24 rows of x, whose copy to whole vectors has 2^32 of them: more than one launch has threads."""
    import torch
    from paper_2007_10412_amd import binding as B
    rows, d_in, classes = 1 << 24, 2041, 17
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("takes 76 GB of GPU memory")
    gen = torch.Generator(device="cuda").manual_seed(4)
    some = (torch.randn(4093, d_in, device="cuda", generator=gen)).to(torch.bfloat16)
    x = torch.empty(rows, d_in, device="cuda", dtype=torch.bfloat16)
    for r in range(0, rows, len(some)):
        x[r:r + len(some)] = some[:min(len(some), rows - r)]
    W = (torch.randn(d_in, classes, device="cuda", generator=gen) / math.sqrt(d_in)).to(torch.bfloat16)
    label = labels_for(len(some), classes, gen, 0.2)
    labels = label.repeat(rows // len(some) + 1)[:rows].contiguous()
    row = torch.full((rows,), math.nan, device="cuda")
    with Ctx() as ctx:
        B.rad_linear_ce(ctx, B.make_layer(rows, d_in, classes, dtype=1, relu=False), x, W, None, labels, row_loss=row)
        B.rad_ctx_synchronize(ctx)
    xd, Wd = some.double(), W.double()
    want, _, _, _, _ = definition(xd @ Wd, lists(labels=label, classes=classes), None, 1.0)
    rel = softmax_error(8 * U * math.sqrt(d_in) * float((xd.abs() @ Wd.abs()).max()), classes)
    close(row[:len(some)], want, (rel + 8 * U * 50) * torch.ones_like(want), "row_loss")
    for r in range(len(some), rows, 512 * len(some)):               # (the same rows, in other places of other pieces)
        n = min(512 * len(some), rows - r)
        assert torch.equal(row[r:r + n], row[:len(some)].repeat(512)[:n]), r


@pytest.mark.parametrize("dtype,rows,classes", [(1, 1, 32760), (1, 64, 33000), (1, 65, 33000), (1, 1, 65537), (1, 128, 66001), (1, 129, 66001), (1, 3, 131064),
                                                (0, 1, 32765), (0, 16, 33001), (0, 17, 33001), (0, 5, 65530)])
@pytest.mark.parametrize("how", ["", "missing", "in_place", "shifted", "loss"])
def test_few_long_rows(dtype, rows, classes, how):
    """Rows of one workgroup or of several, on both sides of the borders between them."""
    with Ctx() as ctx:
        check_distill(ctx, dtype, rows, classes, 9, T=1.3, missing=0.4 if how == "missing" else 0.0, in_place=how == "in_place",
                      shift=3 if how == "shifted" else 0, outputs=("row_loss", "loss") if how == "loss" else ("dlogits", "row_loss", "loss"))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes,k", [(150, 300, 10, 1024), (5, 64, 1, 130), (300, 512, 1000, 1024), (64, 128, 300, 129), (7, 64, 2100, 64)])
def test_lists_that_repeat_themselves(dtype, rows, d_in, classes, k):
    """Longer than there are classes, or from half of them: every class of a list comes several times."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen, x, W, layer = inputs(dtype, rows, d_in, classes)
    index, logit = teacher_for(rows, classes, k, gen, missing=0.2, doubles=True)
    row, dX, dW, dz = torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty_like(W), torch.empty(rows, classes, device="cuda")
    z32 = (x.float() @ W.float()).contiguous()
    dense = torch.empty(rows, device="cuda")
    with Ctx() as ctx:
        B.rad_linear_distill(ctx, layer, x, W, None, B.make_teacher(index, logit, 1.5), row_loss=row, dX=dX, dW=dW)
        B.rad_distill_ce(ctx, z32, B.make_teacher(index, logit, 1.5), B.RAD_F32, dz, row_loss=dense)
        B.rad_ctx_synchronize(ctx)
    xd, Wd = x.double(), W.double()
    z = xd @ Wd
    targets = lists(teacher=(index, logit), classes=classes, T=1.5)
    want, _, g, soft, target = definition(z, targets, None, 1.5)
    rel = softmax_error(8 * U * math.sqrt(d_in + 2) * float((xd.abs() @ Wd.abs()).max()) / 1.5, classes)
    ep = U * (6 * float(logit[torch.isfinite(logit)].abs().max()) / 1.5 + 6 + 8 * math.sqrt(k))
    bound = 1.5 ** 2 * (rel + ep * (z.abs().max() + 30) + 8 * U * (targets[2].abs() + z.abs().max() / 1.5 + 30)) * torch.ones_like(want)
    close(row, want, bound, "row_loss")
    e = soft * rel + 2.02 * HALF[dtype] * (soft + target) + (4 * U + ep) * target
    want_dX = g @ Wd.t().contiguous()
    close(dX, want_dX, (e + 8 * U * math.sqrt(classes) * g.abs()) @ Wd.abs().t().contiguous() + HALF[dtype] * want_dX.abs() + 1e-37, "dX")
    want_dW = xd.t().contiguous() @ g
    close(dW, want_dW, xd.abs().t().contiguous() @ (e + 8 * U * math.sqrt(rows) * g.abs()) + HALF[dtype] * want_dW.abs() + 1e-37, "dW")
    # (dense logits: as z32 has them)
    want, _, g, soft, target = definition(z32.double(), targets, None, 1.5)
    rel = softmax_error(4 * U * float(z32.abs().max()) / 1.5, classes)
    close(dense, want, bound, "dense row_loss")
    close(dz, g, soft * rel + (4 * U + ep) * target + U * g.abs() + 1e-37, "dlogits")

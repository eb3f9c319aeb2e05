"""What the Python calls of the losses over a vocabulary refuse before the library sees a pointer: tensors of another size, type or
layout than the layer says."""
import math

import pytest
import torch

from paper_2007_10412_amd import binding as B

F, H, I = torch.float32, torch.bfloat16, torch.int32


def refused(call, status=None):
    with pytest.raises(B.RadError) as e:
        call()
    assert e.value.status == (B.RAD_ERR_SHAPE if status is None else status), e.value


@pytest.mark.parametrize("index,logit", [
    (torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 2)), (torch.zeros(4, 2, dtype=I), torch.zeros(4, 2, dtype=torch.float64)),
    (torch.zeros(4, 2, dtype=I), torch.zeros(4, 3)), (torch.zeros(4, 2, dtype=I), torch.zeros(2, 4)), (torch.zeros(8, dtype=I), torch.zeros(8)),
    (torch.zeros(2, 4, dtype=I).t(), torch.zeros(4, 2)), (torch.zeros(4, 2, dtype=I), torch.zeros(4, 4)[:, ::2])])
def test_lists(index, logit):
    refused(lambda: B.make_teacher(index, logit))


def test_a_teacher_holds_its_lists():
    t = B.make_teacher(torch.zeros(4, 2, dtype=I), torch.zeros(4, 2), 2.0)
    assert t.k == 2 and t.temperature == 2.0 and t.index == t.lists[0].data_ptr() and t.logit == t.lists[1].data_ptr()


def bad(shape, dtype):
    """tensors that are not contiguous ones of `shape` and `dtype`"""
    n = math.prod(shape)
    other = H if dtype == F else F
    some = [torch.zeros(n + 1, dtype=dtype), torch.zeros(n - 1, dtype=dtype), torch.zeros(shape, dtype=other)]
    return some + ([torch.zeros(2 * n, dtype=dtype)[::2]] if n > 1 else [])


@pytest.mark.parametrize("kind,td", [(B.RAD_F32, F), (B.RAD_BF16, H)])
def test_linear(kind, td):
    layer = B.make_layer(4, 8, 16, dtype=kind, relu=False, has_bias=True)
    given = dict(x=((4, 8), td), W=((8, 16), td), bias=((16,), F), row_weight=((4,), F), row_loss=((4,), F), loss=((1,), F),
                 dX=((4, 8), td), dW=((8, 16), F), dbias=((16,), F))
    labels, teacher = torch.zeros(4, dtype=I), B.make_teacher(torch.zeros(4, 2, dtype=I), torch.zeros(4, 2))
    good = {n: torch.zeros(s, dtype=t) for n, (s, t) in given.items()}
    for name, (shape, dtype) in given.items():
        for t in bad(shape, dtype):
            if name == "dW" and t.shape == shape:       # fp32 or the layer's type
                continue
            refused(lambda: B.rad_linear_ce(None, layer, labels=labels, **{**good, name: t}))
            refused(lambda: B.rad_linear_distill(None, layer, teacher=teacher, **{**good, name: t}))
    refused(lambda: B.rad_linear_ce(None, layer, labels=labels, **{**good, "dW": torch.zeros(8, 16, dtype=torch.float16)}), B.RAD_ERR_PARAM)
    for t in (torch.zeros(4, dtype=torch.int64), torch.zeros(5, dtype=I), torch.zeros(8, dtype=I)[::2]):
        refused(lambda: B.rad_linear_ce(None, layer, labels=t, **good))
    few = B.make_teacher(torch.zeros(3, 2, dtype=I), torch.zeros(3, 2))
    refused(lambda: B.rad_linear_distill(None, layer, teacher=few, **good))


@pytest.mark.parametrize("kind,td", [(B.RAD_F32, F), (B.RAD_BF16, H)])
def test_distill(kind, td):
    teacher = B.make_teacher(torch.zeros(4, 2, dtype=I), torch.zeros(4, 2))
    given = dict(row_weight=((4,), F), row_loss=((4,), F), loss=((1,), F), dlogits=((4, 16), td))
    good = {n: torch.zeros(s, dtype=t) for n, (s, t) in given.items()}
    z = torch.zeros(4, 16, dtype=td)
    for name, (shape, dtype) in given.items():
        for t in bad(shape, dtype):
            refused(lambda: B.rad_distill_ce(None, z, teacher, kind, **{**good, name: t}))
    for t in (torch.zeros(4, 16, dtype=H if td == F else F), torch.zeros(16, 4, dtype=td).t(), torch.zeros(5, 16, dtype=td)):
        refused(lambda: B.rad_distill_ce(None, t, teacher, kind, **good))


@pytest.mark.parametrize("kind,td", [(B.RAD_F32, F), (B.RAD_BF16, H)])
def test_tensors_in_host_memory(kind, td):
    """Labels and lists come from data loaders: a call on host tensors of the right sizes is refused, not handed to a kernel."""
    layer = B.make_layer(4, 8, 16, dtype=kind, relu=False, has_bias=True)
    x, W, bias, loss = torch.zeros(4, 8, dtype=td), torch.zeros(8, 16, dtype=td), torch.zeros(16), torch.zeros(1)
    teacher = B.make_teacher(torch.zeros(4, 2, dtype=I), torch.zeros(4, 2))
    for call in (lambda: B.rad_linear_ce(None, layer, x, W, bias, torch.zeros(4, dtype=I), loss=loss),
                 lambda: B.rad_linear_distill(None, layer, x, W, bias, teacher, loss=loss),
                 lambda: B.rad_distill_ce(None, torch.zeros(4, 16, dtype=td), teacher, kind, loss=loss)):
        with pytest.raises(B.RadError, match="not on the context's GPU") as e:
            call()
        assert e.value.status == B.RAD_ERR_PARAM


class Placed:
    """What the checks read of a tensor that lies on GPU `at` (-1: in host memory)."""

    def __init__(self, t, at):
        self.t, self.at, self.device = t, at, "cuda:%d" % at if at >= 0 else "cpu"

    def get_device(self):
        return self.at

    def __getattr__(self, name):
        return getattr(self.t, name)

    def __len__(self):
        return len(self.t)


@pytest.mark.parametrize("known", [True, False])
def test_every_tensor_is_on_the_context_s_gpu(known, monkeypatch):
    """Each argument in turn in host memory or on a second GPU; the call itself is taken out, and seen only where all are right."""
    given = dict(x=(4, 8), W=(8, 16), bias=(16,), row_weight=(4,), row_loss=(4,), loss=(1,), dX=(4, 8), dW=(8, 16), dbias=(16,))
    layer, reached = B.make_layer(4, 8, 16, relu=False, has_bias=True), []

    class Library:
        def __getattr__(self, name):
            return lambda *_: reached.append(name) or B.RAD_OK
    monkeypatch.setattr(B, "lib", Library)
    ctx = B.P()
    if known:
        ctx.device = 1

    def arguments(other=None, at=1):
        place = lambda name, t: Placed(t, at if name == other else 1)  # noqa: E731
        teacher = B.rad_teacher(2, 1.0, None, None)
        teacher.lists = place("index", torch.zeros(4, 2, dtype=I)), place("logit", torch.zeros(4, 2))
        tensors = {n: place(n, torch.zeros(s)) for n, s in given.items()}
        return tensors, place("labels", torch.zeros(4, dtype=I)), teacher, place("logits", torch.zeros(4, 16)), place("dlogits", torch.zeros(4, 16))

    def calls(other=None, at=1):
        t, labels, teacher, z, dz = arguments(other, at)
        dense = {n: t[n] for n in ("row_weight", "row_loss", "loss")}
        return [("rad_linear_ce", set(given) | {"labels"}, lambda: B.rad_linear_ce(ctx, layer, labels=labels, **t)),
                ("rad_linear_distill", set(given) | {"index", "logit"}, lambda: B.rad_linear_distill(ctx, layer, teacher=teacher, **t)),
                ("rad_distill_ce", {"logits", "dlogits", "index", "logit", *dense}, lambda: B.rad_distill_ce(ctx, z, teacher, B.RAD_F32, dz, **dense))]
    for name, _, call in calls():
        call()
    assert reached == ["rad_linear_ce", "rad_linear_distill", "rad_distill_ce"]
    for other in list(given) + ["labels", "index", "logit", "logits", "dlogits"]:
        for at in (-1, 0):
            for name, takes, call in calls(other, at):
                if other in takes:
                    with pytest.raises(B.RadError) as e:
                        call()
                    assert e.value.status == B.RAD_ERR_PARAM, (name, other, at)
    assert len(reached) == 3


def test_lists_of_another_length_than_the_teacher_says():
    """k is a field that a program can set: more than the tensors have would be read past their ends."""
    layer = B.make_layer(4, 8, 16, relu=False)
    for k in (1, 3, 1024):
        teacher = B.make_teacher(torch.zeros(4, 2, dtype=I), torch.zeros(4, 2))
        teacher.k = k
        refused(lambda: B.rad_linear_distill(None, layer, torch.zeros(4, 8), torch.zeros(8, 16), None, teacher, loss=torch.zeros(1)))
        refused(lambda: B.rad_distill_ce(None, torch.zeros(4, 16), teacher, B.RAD_F32, loss=torch.zeros(1)))

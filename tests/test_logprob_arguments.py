"""What the Python calls of the log probabilities refuse before the library sees a pointer: tensors of another size, type, layout or place."""
import math

import pytest
import torch

from paper_2007_10412_amd import binding as B

F, H, I = torch.float32, torch.bfloat16, torch.int32


def refused(call, status=None):
    with pytest.raises(B.RadError) as e:
        call()
    assert e.value.status == (B.RAD_ERR_SHAPE if status is None else status), e.value


def bad(shape, dtype):
    """tensors that are not contiguous ones of `shape` and `dtype`"""
    n = math.prod(shape)
    some = [torch.zeros(n + 1, dtype=dtype), torch.zeros(n - 1, dtype=dtype), torch.zeros(shape, dtype=torch.float64)]
    return some + ([torch.zeros(2 * n, dtype=dtype)[::2]] if n > 1 else [])


LIST = dict(top_index=torch.zeros(4, 3, dtype=I), top_logprob=torch.zeros(4, 3))
SCORES = dict(tokens=((4,), I), logprob=((4,), F), entropy=((4,), F))
GRADS = dict(tokens=((4,), I), d_logprob=((4,), F), d_entropy=((4,), F))


def each(given, call):
    good = {n: torch.zeros(s, dtype=t) for n, (s, t) in given.items()}
    for name, (shape, dtype) in given.items():
        for t in bad(shape, dtype):
            if name == "dW" and t.dtype == torch.float64:
                refused(lambda: call(**{**good, name: t}), B.RAD_ERR_PARAM)
            else:
                refused(lambda: call(**{**good, name: t}))
    with pytest.raises(B.RadError, match="not on the context's GPU"):
        call(**good)


@pytest.mark.parametrize("kind,td", [(B.RAD_F32, F), (B.RAD_BF16, H)])
def test_sizes_types_layouts(kind, td):
    z = torch.zeros(4, 16, dtype=td)
    each(SCORES, lambda **k: B.rad_token_logprobs(None, z, kind, **k, **LIST))
    each({**GRADS, "dlogits": ((4, 16), td)}, lambda **k: B.rad_token_logprobs_grad(None, z, kind, **k))
    layer = B.make_layer(4, 8, 16, dtype=kind, relu=False, has_bias=True)
    inputs = dict(x=((4, 8), td), W=((8, 16), td), bias=((16,), F))
    each({**inputs, **SCORES}, lambda **k: B.rad_linear_logprobs(None, layer, **k, **LIST))
    each({**inputs, **GRADS, "dX": ((4, 8), td), "dW": ((8, 16), F), "dbias": ((16,), F)}, lambda **k: B.rad_linear_logprobs_grad(None, layer, **k))
    for other in (torch.zeros(16, 4, dtype=td).t(), torch.zeros(4, 16, dtype=H if td == F else F)):
        refused(lambda: B.rad_token_logprobs(None, other, kind, entropy=torch.zeros(4)))
        refused(lambda: B.rad_token_logprobs_grad(None, other, kind, torch.zeros(4, 16, dtype=td), d_entropy=torch.zeros(4)))


@pytest.mark.parametrize("index,logprob,status", [
    (torch.zeros(4, 3, dtype=I), None, B.RAD_ERR_NULL), (None, torch.zeros(4, 3), B.RAD_ERR_NULL),
    (torch.zeros(4, 3, dtype=I), torch.zeros(4, 2), None), (torch.zeros(3, 4, dtype=I), torch.zeros(3, 4), None),
    (torch.zeros(12, dtype=I), torch.zeros(12), None), (torch.zeros(4, 3, dtype=torch.int64), torch.zeros(4, 3), None),
    (torch.zeros(4, 3, dtype=I), torch.zeros(4, 3, dtype=H), None), (torch.zeros(4, 6, dtype=I)[:, ::2], torch.zeros(4, 3), None),
    (torch.zeros(4, 3, dtype=I), torch.zeros(3, 4).t(), None)])
def test_lists(index, logprob, status):
    layer = B.make_layer(4, 8, 16, relu=False)
    refused(lambda: B.rad_token_logprobs(None, torch.zeros(4, 16), B.RAD_F32, top_index=index, top_logprob=logprob), status)
    refused(lambda: B.rad_linear_logprobs(None, layer, torch.zeros(4, 8), torch.zeros(8, 16), None, top_index=index, top_logprob=logprob), status)

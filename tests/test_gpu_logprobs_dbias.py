"""The bias gradient of rad_linear_logprobs_grad in bf16: an fp32 sum of dz as it is ahead of its rounding to the layer's type.

Bound, element by element: of tests/test_gpu_logprobs.py's, all but the rounding of dz.  A logit that is not its row's token is a code, off by half of
128 / 65535 of a power of two, which moves q by 2^(64 / 65535) - 1 = 0.1734 h of itself (h = 2^-8) and log q by 0.1733 h, so dz by 0.175 h of its
parts q (|a| + |h| (d + S + 1)) / T; 0.18 h leaves room for the codes' own arithmetic (fp32 values of up to 128 and 65535, 2^-24 of which are less
than 2 % of half a step).  Sums over n rows: 8 u sqrt(n + 1) of the sum of sizes."""
import math

import pytest

from tests.test_gpu_logprobs import HALF, U, Ctx, close, gen_for, layer_inputs, layer_row, tokens_for

pytestmark = pytest.mark.gpu


def check(ctx, rows, d_in, classes, bias=True, ignored=0.0, T=1.0, beta=0.0, kinds="ah", others=("dX", "dW"), no_tokens=False, sizes=None):
    import torch
    from paper_2007_10412_amd import binding as B
    tag = "dbias %d x %d x %d %s" % (rows, d_in, classes, kinds)
    print(tag, flush=True)
    gen = gen_for(rows, d_in, classes, 31)
    x, W, b = layer_inputs(1, rows, d_in, classes, bias, gen)
    tokens = None if no_tokens else tokens_for(rows, classes, gen, ignored)
    a = torch.randn(rows, device="cuda", generator=gen) if "a" in kinds else None
    h = torch.randn(rows, device="cuda", generator=gen) if "h" in kinds else None
    if sizes is not None:
        a, h = (None if t is None else t * sizes(rows) for t in (a, h))
    before = torch.randn(classes, device="cuda", generator=gen)
    dbias = before.clone() if beta else torch.full((classes,), math.nan, device="cuda")
    out = {n: torch.empty_like(t) for n, t in (("dX", x), ("dW", W)) if n in others}
    layer = B.make_layer(rows, d_in, classes, dtype=1, relu=False, has_bias=bias)
    B.rad_linear_logprobs_grad(ctx, layer, x, W, b, tokens=tokens, temperature=T, d_logprob=a, d_entropy=h, beta=beta, dbias=dbias,
                               **{n: t.zero_() for n, t in out.items()})
    B.rad_ctx_synchronize(ctx)
    want, bound = torch.zeros(classes, device="cuda", dtype=torch.float64), torch.zeros(classes, device="cuda", dtype=torch.float64)
    mass = torch.zeros_like(want)
    for r0 in range(0, rows, 1024):
        at = slice(r0, min(rows, r0 + 1024))
        t = None if tokens is None else tokens[at]
        counts = torch.ones(len(x[at]), dtype=torch.bool, device="cuda") if t is None else (t >= 0) & (t < classes)
        part = [None if v is None else v[at] for v in (a, h)]
        row = layer_row(x[at], W, b, T)
        dz, e, parts = row.grad(t if a is not None else None, counts, *part)
        if a is not None:                               # (what is left are the parts of all but the tokens' own terms)
            own = torch.where(counts, part[0].double().abs(), torch.zeros_like(part[0], dtype=torch.float64))[:, None] / T
            parts = parts - torch.zeros_like(parts).scatter_(1, t.long().clamp(0, classes - 1)[:, None], own)
        want += dz.sum(dim=0)
        bound += (e + 0.18 * HALF[1] * parts).sum(dim=0)
        mass += dz.abs().sum(dim=0)
    if beta:
        want += before.double()
        mass += before.double().abs()
    close(dbias, want, bound + 8 * U * math.sqrt(rows + 1) * mass + 1e-37, tag)


@pytest.mark.parametrize("rows,d_in,classes", [(1, 64, 500), (1, 2048, 50257), (3, 40, 10), (15, 64, 1003), (16, 64, 1000), (17, 64, 130), (150, 300, 10), (257, 129, 1003),
                                               (300, 512, 4096), (64, 256, 20000), (600, 512, 20005), (1025, 136, 8200), (2050, 64, 2048),
                                               (40, 1030, 33003)])
def test_bias_gradient_is_a_sum_of_unrounded_values(rows, d_in, classes):
    with Ctx() as ctx:
        check(ctx, rows, d_in, classes, ignored=0.3 if rows > 4 else 0.0)
        check(ctx, rows, d_in, classes, kinds="a", T=0.7, beta=1.0, others=())
        check(ctx, rows, d_in, classes, kinds="h", T=1.5, no_tokens=True, others=("dW",), bias=False)
        check(ctx, rows, d_in, classes, kinds="h", beta=1.0, ignored=0.5, others=("dX",))


def test_of_rows_that_differ_in_size():
    """Gradients of a row over twelve powers of ten."""
    import torch
    with Ctx() as ctx:
        check(ctx, 700, 128, 5001, sizes=lambda n: 10.0 ** -(torch.arange(n, device="cuda") % 12).float())


def test_of_several_pieces():
    with Ctx() as ctx:
        check(ctx, 8300, 32, 131000, ignored=0.2, others=())


def test_of_no_rows():
    import torch
    from paper_2007_10412_amd import binding as B
    with Ctx() as ctx:
        for beta in (0.0, 1.0):
            x, W, b = layer_inputs(1, 40, 64, 1003, True, gen_for(1))
            dbias = torch.full((1003,), 7.0, device="cuda")
            B.rad_linear_logprobs_grad(ctx, B.make_layer(40, 64, 1003, dtype=1, relu=False, has_bias=True), x, W, b,
                                       tokens=torch.full((40,), -1, device="cuda", dtype=torch.int32), d_logprob=torch.randn(40, device="cuda"), dbias=dbias, beta=beta)
            B.rad_ctx_synchronize(ctx)
            assert (dbias == 7.0 * beta).all()

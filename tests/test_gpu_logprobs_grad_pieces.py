"""rad_linear_logprobs_grad of more rows than a piece takes, and of more than the list of rows that the tiles make themselves, against the definition in fp64
with the bounds of tests/test_gpu_logprobs.py."""
import math

import pytest

from tests.test_gpu_logprobs import HALF, U, Ctx, check_linear_grad, close, gen_for, layer_inputs, layer_row, tokens_for, torch_dtype

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dw_dtype,beta", [(0, 0, 0.0), (0, 0, 1.0), (1, 0, 0.0), (1, 0, 1.0), (1, 1, 0.0), (1, 1, 1.0)])
@pytest.mark.parametrize("first,second", [(1e4, 1e-3), (1e-20, 1e3), (1.0, 1.0)])
def test_gradients_of_several_pieces(dtype, dw_dtype, beta, first, second):
    """Two pieces whose rows' gradients differ in size, so that each has a factor of its own; some rows of either do not count."""
    import torch
    from paper_2007_10412_amd import binding as B
    d_in, classes = 32, 131000
    piece = (2 << 30) // (131008 * (2 if dtype else 4)) // 256 * 256
    rows = piece + 104
    print("pieces", dtype, dw_dtype, beta, first, second, rows, flush=True)
    gen = gen_for(rows, dtype)
    x, W, b = layer_inputs(dtype, rows, d_in, classes, True, gen)
    tokens = tokens_for(rows, classes, gen, 0.2)
    size = torch.where(torch.arange(rows, device="cuda") < piece, first, second).float()
    a, h = torch.randn(rows, device="cuda", generator=gen) * size, torch.randn(rows, device="cuda", generator=gen) * size
    wd = torch_dtype(dw_dtype)
    dW0 = torch.randn(d_in, classes, device="cuda", generator=gen).to(wd)
    db0 = torch.randn(classes, device="cuda", generator=gen)
    dX, dW, db = torch.full_like(x, math.nan), dW0.clone() if beta else torch.full_like(dW0, math.nan), db0.clone() if beta else torch.full_like(db0, math.nan)
    with Ctx() as ctx:
        B.rad_linear_logprobs_grad(ctx, B.make_layer(rows, d_in, classes, dtype=dtype, relu=False, has_bias=True), x, W, b, tokens=tokens, temperature=1.5,
                                   d_logprob=a, d_entropy=h, dX=dX, dW=dW, dbias=db, beta=beta)
        B.rad_ctx_synchronize(ctx)
    # columns: every 400th, and the tokens of the last piece
    cols = torch.cat([torch.arange(0, classes, 400, device="cuda"), tokens[piece:].long().clamp(0, classes - 1)])
    Wt = W.double().t().contiguous()
    gw, gb, ew, eb, mw, mb = (torch.zeros((d_in, len(cols)) if i % 2 == 0 else (len(cols),), device="cuda", dtype=torch.float64) for i in range(6))
    for r0 in range(0, rows, 512):
        at = slice(r0, min(rows, r0 + 512))
        counts = (tokens[at] >= 0) & (tokens[at] < classes)
        dz, e, parts = layer_row(x[at], W, b, 1.5).grad(tokens[at], counts, a[at], h[at])
        e = e + 2.02 * HALF[dtype] * parts
        xt = x[at].double().t().contiguous()
        gw += xt @ dz[:, cols]; ew += xt.abs() @ e[:, cols]; mw += xt.abs() @ dz[:, cols].abs()
        gb += dz[:, cols].sum(dim=0); eb += e[:, cols].sum(dim=0); mb += dz[:, cols].abs().sum(dim=0)
        if r0 % 2048 == 0 or r0 + 1024 >= piece:
            want, mass = dz @ Wt, dz.abs() @ Wt.abs()
            close(dX[at], want, e @ Wt.abs() + 8 * U * math.sqrt(classes) * mass + HALF[dtype] * want.abs() + 1e-37, "dX from row %d" % r0)
            assert (dX[at][~counts] == 0).all()
    if beta:
        gw += dW0[:, cols].double(); mw += dW0[:, cols].double().abs()
        gb += db0[cols].double(); mb += db0[cols].double().abs()
    n = 8 * U * math.sqrt(rows + 1)
    close(dW[:, cols], gw, ew + n * mw + HALF[dw_dtype] * gw.abs() + 1e-37, "dW")
    close(db[cols], gb, eb + n * mb + 1e-37, "dbias")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", [(8193, 40, 300), (20000, 40, 500)])
def test_gradients_of_many_rows(dtype, rows, d_in, classes):
    with Ctx() as ctx:
        check_linear_grad(ctx, dtype, rows, d_in, classes, bias=True, ignored=0.3)
        check_linear_grad(ctx, dtype, rows, d_in, classes, kinds="h", ignored=0.6, beta=1.0, dw_dtype=0)
        check_linear_grad(ctx, dtype, rows, d_in, classes, bias=True, kinds="a", T=0.7)
        check_linear_grad(ctx, dtype, rows, d_in, classes, kinds="h", no_tokens=True, T=2.0)

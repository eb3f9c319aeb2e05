"""rad_optimizer_step over tensors that take more than one launch's grid."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_tensor_of_more_than_a_launch():
    """2^33 + 1003 elements and a small tensor behind them: every element is stepped once."""
    import torch
    from paper_2007_10412_amd import binding as B
    ctx = B.rad_ctx_create()
    n = 2 ** 33 + 1003
    w, g = torch.full((n,), 1.0, device="cuda"), torch.full((n,), 2.0, device="cuda")
    w2, g2 = torch.full((77,), 3.0, device="cuda"), torch.full((77,), 4.0, device="cuda")
    g[2 ** 33 - 2:2 ** 33 + 2] = torch.tensor([4.0, 6.0, 8.0, 10.0], device="cuda")
    B.rad_optimizer_step(ctx, B.make_optimizer(B.RAD_SGD, 0.25), 1, B.RAD_F32, [w, w2], [g, g2])
    B.rad_ctx_synchronize(ctx)
    assert w[2 ** 33 - 2:2 ** 33 + 2].tolist() == [0.0, -0.5, -1.0, -1.5]
    w[2 ** 33 - 2:2 ** 33 + 2] = 0.5
    assert float(w.min()) == 0.5 and float(w.max()) == 0.5 and (w2 == 2.0).all()
    B.rad_ctx_destroy(ctx)
    del w, g
    torch.cuda.empty_cache()                             # (64 GiB)

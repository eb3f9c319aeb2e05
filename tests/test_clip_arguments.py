"""What the Python calls of the gradient norm, clipping and the scaled step refuse before the library sees a pointer."""
import pytest
import torch

from paper_2007_10412_amd import binding as B

F, H = torch.float32, torch.bfloat16


def refused(call, status):
    with pytest.raises(B.RadError) as e:
        call()
    assert e.value.status == status, e.value


def test_gradients():
    good = [torch.zeros(4, 4), torch.zeros(3, dtype=H)]
    one = torch.zeros(1)
    refused(lambda: B.rad_gradient_norm(None, [torch.zeros(4, dtype=torch.float64)], norm=one), B.RAD_ERR_PARAM)
    refused(lambda: B.rad_gradient_norm(None, [torch.zeros(4, dtype=torch.float16)], norm=one), B.RAD_ERR_PARAM)
    refused(lambda: B.rad_gradient_norm(None, [torch.zeros(4, 4).t()[:, :2]], norm=one), B.RAD_ERR_SHAPE)
    for bad in (torch.zeros(2), torch.zeros(1, dtype=H), torch.zeros(1, dtype=torch.float64)):
        refused(lambda: B.rad_gradient_norm(None, good, norm=bad), B.RAD_ERR_SHAPE)
        refused(lambda: B.rad_gradient_norm(None, good, scale=bad), B.RAD_ERR_SHAPE)
        refused(lambda: B.rad_clip_gradients(None, good, 1.0, norm=bad), B.RAD_ERR_SHAPE)
    for clipped in ([good[0]], [good[0], torch.zeros(3)], [good[0], torch.zeros(4, dtype=H)], [torch.zeros(4, 8)[:, ::2], good[1]]):
        refused(lambda: B.rad_clip_gradients(None, good, 1.0, clipped=clipped), B.RAD_ERR_SHAPE)
    refused(lambda: B.rad_gradient_norm(None, good, norm=one), B.RAD_ERR_PARAM)          # host memory
    refused(lambda: B.rad_clip_gradients(None, good, 1.0), B.RAD_ERR_PARAM)


@pytest.mark.parametrize("kind,td", [(B.RAD_F32, F), (B.RAD_BF16, H)])
def test_scaled_step(kind, td):
    opt = B.make_optimizer(B.RAD_ADAM, 1e-3)
    good = dict(params=[torch.zeros(4, dtype=td)], grads=[torch.zeros(4)], scale=torch.zeros(1), m=[torch.zeros(4)], v=[torch.zeros(4)],
                master=[torch.zeros(4)] if kind == B.RAD_BF16 else None)
    for name in ("params", "grads", "m", "v", "master"):
        if good[name] is None:
            continue
        t = good[name][0]
        wrong = [torch.zeros(4, dtype=H if t.dtype == F else F)], [torch.zeros(8, dtype=t.dtype)[::2]], [t, t], []
        for bad in wrong + (() if name == "params" else ([torch.zeros(5, dtype=t.dtype)],)):
            if name == "params" and bad == []:
                continue
            refused(lambda: B.rad_optimizer_step_scaled(None, opt, 1, kind, **{**good, name: bad}), B.RAD_ERR_SHAPE)
    refused(lambda: B.rad_optimizer_step_scaled(None, opt, 1, kind, **{**good, "scale": torch.zeros(2)}), B.RAD_ERR_SHAPE)
    refused(lambda: B.rad_optimizer_step_scaled(None, opt, 1, kind, **good), B.RAD_ERR_PARAM)    # host memory

"""Gradients whose finite norm is so many times max_norm that the scale, max_norm / norm, is a subnormal fp32 number or below all of them.

Bounds, u = 2^-24: a scale is the quotient rounded once, to a multiple of 2^-149 where it is subnormal (off by 2^-150 then), and 2^-149 at
least, so off by 2^-149; a step's gradient is the product of that scale and g, rounded as fp32 does.  A clipped element takes the quotient
itself, in two factors: 2 u (one rounding of a factor, one of the product), half a step of the type (bf16 2^-8), and at the lower end of the
numbers some last places: the first factor's product is rounded where it is subnormal, 2^-150 times a second factor of 4 at most (max_norm is below
2^2 where the quotient is below 2^-126, and the second factor is at most twice that), 2^-147 in all with the product's own, and half a step of bf16's
subnormals, 2^-134."""
import math

import pytest

from tests.test_gpu_clip import U, Ctx, call_norm, mixed, norm_of, tensors

pytestmark = pytest.mark.gpu

# (size of the gradients, max_norm): quotients from the smallest normal number's neighbourhood down to none that even fp64 holds
CASES = [(1e35, 1.0), (1e35, 1e-2), (1e35, 1e-6), (1e35, 1e-9), (1e35, 1e-12), (1e35, 1e-200), (1e35, 1e-310), (1.0, 1e-37), (1.0, 1e-40),
         (1.0, 1e-44), (1.0, 1e-46), (1.0, 1e-300), (1e-20, 1e-60), (1e-36, 1e-80), (1e33, 3.0)]
SIZES = [1, 1030, 4096 * 3 + 2, 0, 4096]


def gradients(size, how, seed, offset=0, sizes=SIZES):
    return [(t.double() * size).to(t.dtype) if offset == 0 else t.mul_(size) for t in tensors(sizes, mixed(len(sizes), how), seed, offset)]


@pytest.mark.parametrize("size,max_norm", CASES)
def test_scale_of_a_finite_norm_is_not_zero(size, max_norm):
    with Ctx() as ctx:
        grads = gradients(size, "f32", 3)
        want = norm_of(grads)
        norm, scale = call_norm(ctx, grads, max_norm)
        q = min(1.0, max_norm / want)
        print(size, max_norm, norm, scale, flush=True)
        assert abs(norm - want) <= 2 * U * want and scale > 0.0
        assert abs(scale - q) <= 2 * U * q + 2.0 ** -149


@pytest.mark.parametrize("size,max_norm", CASES)
@pytest.mark.parametrize("how", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("offset,place", [(0, "in place"), (0, "apart"), (1, "apart")])
def test_clipped_to_a_small_norm(size, max_norm, how, offset, place):
    import torch
    from paper_2007_10412_amd import binding as B
    with Ctx() as ctx:
        grads = gradients(size, how, 9, offset)
        before = [g.double() for g in grads]
        want = norm_of(grads)
        out = grads if place == "in place" else [torch.full_like(g, math.nan) for g in grads]
        norm = torch.zeros(1, device="cuda")
        B.rad_clip_gradients(ctx, grads, max_norm, clipped=None if place == "in place" else out, norm=norm)
        B.rad_ctx_synchronize(ctx)
        assert abs(float(norm) - want) <= 2 * U * want
        f = min(1.0, max_norm / want)
        for o, b in zip(out, before):
            half, last = (2.0 ** -8, 2.0 ** -134) if o.dtype == torch.bfloat16 else (U, 0.0)
            assert ((o.double() - f * b).abs() <= (half + 2.02 * U) * f * b.abs() + 2.0 ** -147 + last).all()


@pytest.mark.parametrize("how,n", [("f32", 68_000_001), ("bf16", 136_000_001)])
def test_clipped_to_a_small_norm_past_the_caches(how, n):
    import torch
    from paper_2007_10412_amd import binding as B
    with Ctx() as ctx:
        grads = gradients(1e33, how, 6, sizes=[n])
        want, before = norm_of(grads), grads[0][:100000].double()
        B.rad_clip_gradients(ctx, grads, 1e-6)
        B.rad_ctx_synchronize(ctx)
        f, half = 1e-6 / want, 2.0 ** -8 if how == "bf16" else U
        assert f < 2.0 ** -126 and torch.isfinite(grads[0]).all()
        assert ((grads[0][:100000].double() - f * before).abs() <= (half + 2.02 * U) * f * before.abs() + 2.0 ** -147 + (2.0 ** -134 if how == "bf16" else 0.0)).all()
        assert abs(norm_of(grads) - 1e-6) <= 1e-6 * 2.0 ** -7


@pytest.mark.parametrize("size,max_norm", [(1e35, 1e-6), (1e35, 1e-12), (1.0, 1e-46)])
@pytest.mark.parametrize("kind", [0, 1])
def test_step_after_a_small_scale_is_taken(size, max_norm, kind):
    """Its moments decay and its l2 term moves the parameters: bit by bit the step of the gradients times the scale, formed on the CPU."""
    import torch
    from paper_2007_10412_amd import binding as B
    sizes = [5000, 7]
    f32 = [torch.float32] * 2
    with Ctx() as ctx:
        grads = gradients(size, "f32", 21, sizes=sizes)
        norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        opt = B.make_optimizer(kind, 1e-2, 1e-3, 0.9, 0.99, 1e-7)

        def state():
            return tensors(sizes, f32, 22), dict(m=tensors(sizes, f32, 23), v=[t.abs() for t in tensors(sizes, f32, 24)]) if kind else {}
        (wa, a), (wb, b) = state(), state()
        B.rad_gradient_norm(ctx, grads, max_norm, norm=norm, scale=scale)
        B.rad_optimizer_step_scaled(ctx, opt, 3, B.RAD_F32, wa, grads, scale, **a)
        B.rad_ctx_synchronize(ctx)
        scaled = [(g.cpu().double() * float(scale)).float().cuda() for g in grads]
        B.rad_optimizer_step(ctx, opt, 3, B.RAD_F32, wb, scaled, **b)
        B.rad_ctx_synchronize(ctx)
        start = state()
        assert not torch.equal(wa[0], start[0][0])
        for x, y in zip(wa + sum(a.values(), []), wb + sum(b.values(), [])):
            assert torch.equal(x, y)

"""rad_gradient_norm, rad_clip_gradients and rad_optimizer_step_scaled against their definitions in fp64.

Bounds.  Squares and sums are fp64, so a norm is its fp64 value rounded to fp32 (half a step, 2^-24 relative; 2^-23 leaves room
for the sum's own 2^-50).  A scale is max_norm / norm in fp64, rounded once; a clipped element is a product of that and the
gradient, rounded to fp32 and then to the type: 2 x 2^-24 and half a step of the type (2^-8 bf16; in fp32 the product's rounding is the
only one)."""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SIZES = [1, 3, 257, 4096 * 33 + 2, 0, 1024, 4096, 8191]


class Ctx:
    def __init__(self, stream=None):
        from paper_2007_10412_amd import binding as B
        self.ctx = B.rad_ctx_create(stream)

    def __enter__(self):
        return self.ctx

    def __exit__(self, *_):
        from paper_2007_10412_amd import binding as B
        B.rad_ctx_destroy(self.ctx)


def tensors(sizes, kinds, seed, offset=0, scale=1.0):
    """gradients of sizes over three powers of ten, each `offset` elements behind a 16-byte boundary"""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, (n, k) in enumerate(zip(sizes, kinds)):
        t = torch.empty(n + offset, device="cuda", dtype=k)[offset:]
        t.copy_(torch.randn(n, device="cuda", generator=gen) * scale * 10.0 ** -(i % 4))
        out.append(t)
    return out


def mixed(n, how):
    import torch
    return [{"f32": torch.float32, "bf16": torch.bfloat16}.get(how) or (torch.bfloat16 if i % 3 == 1 else torch.float32) for i in range(n)]


def norm_of(grads):
    return math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))


def call_norm(ctx, grads, max_norm=math.inf):
    import torch
    from paper_2007_10412_amd import binding as B
    norm, scale = torch.full((1,), math.nan, device="cuda"), torch.full((1,), math.nan, device="cuda")
    B.rad_gradient_norm(ctx, grads, max_norm, norm=norm, scale=scale)
    B.rad_ctx_synchronize(ctx)
    return float(norm), float(scale)


@pytest.mark.parametrize("how", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", [[1], [7], [0, 0], [], SIZES, [4096 * 2049 + 5, 11], [129] * 300, [5] * 128 + [4099]])
def test_norm(sizes, how):
    print("norm", how, sizes[:8], len(sizes), flush=True)
    with Ctx() as ctx:
        for offset in (0, 1):
            grads = tensors(sizes, mixed(len(sizes), how), 3 + len(sizes), offset)
            want = norm_of(grads)
            got, scale = call_norm(ctx, grads)
            assert abs(got - want) <= 2 * U * want and scale == 1.0, (got, want)
            if want > 0:
                for part in (0.25, 0.999, 1.001, 100.0):
                    got, scale = call_norm(ctx, grads, part * want)
                    to = min(1.0, part)
                    assert abs(scale - to) <= 2 * U * to, (scale, to)


@pytest.mark.parametrize("size", [1e-30, 1e-22, 1e18, 2e30])
def test_norms_at_the_ends_of_fp32(size):
    """Squares that fp32 cannot hold."""
    import torch
    with Ctx() as ctx:
        grads = [t * size for t in tensors([1000, 40000], [torch.float32] * 2, 5)]
        want = norm_of(grads)
        got, scale = call_norm(ctx, grads, want * 0.5)
        assert abs(got - want) <= 2 * U * want and abs(scale - 0.5) <= 2 * U
        big = [torch.full((64,), 3e38, device="cuda")]
        assert call_norm(ctx, big) == (math.inf, 0.0)          # (2.4e39)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("how", ["f32", "bf16"])
def test_not_finite(value, how):
    """One such element makes a norm that is not finite and a scale of 0; gradients stay as they are, a step is skipped."""
    import torch
    from paper_2007_10412_amd import binding as B
    kinds = mixed(3, how)
    with Ctx() as ctx:
        grads = tensors([100, 5000, 9], kinds, 6)
        grads[1][4999] = value
        before = [g.clone() for g in grads]
        got, scale = call_norm(ctx, grads, 1.0)
        assert not math.isfinite(got) and scale == 0.0
        other = [torch.zeros_like(g) for g in grads]
        B.rad_clip_gradients(ctx, grads, 1.0, clipped=other)
        B.rad_clip_gradients(ctx, grads, 1.0)
        B.rad_ctx_synchronize(ctx)
        for g, o, b in zip(grads, other, before):
            assert torch.equal(g.view(torch.uint8), b.view(torch.uint8)) and torch.equal(o.view(torch.uint8), b.view(torch.uint8))
        if how == "f32":
            w, m, v = ([torch.rand_like(g) for g in grads] for _ in range(3))
            kept = [t.clone() for t in w + m + v]
            B.rad_optimizer_step_scaled(ctx, B.make_optimizer(B.RAD_ADAM, 1e-2), 1, B.RAD_F32, w, grads, torch.zeros(1, device="cuda"), m, v)
            B.rad_ctx_synchronize(ctx)
            assert all(torch.equal(a, b) for a, b in zip(w + m + v, kept))


@pytest.mark.parametrize("how", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("part", [0.01, 0.7, 2.0])
@pytest.mark.parametrize("place", ["in place", "apart", "both"])
def test_clip(how, offset, part, place):
    import torch
    from paper_2007_10412_amd import binding as B
    print("clip", how, offset, part, place, flush=True)
    sizes = SIZES + [33] * 100
    kinds = mixed(len(sizes), how)
    with Ctx() as ctx:
        grads = tensors(sizes, kinds, 9, offset)
        before = [g.double() for g in grads]
        want = norm_of(grads)
        to = [g if place == "in place" or (place == "both" and i % 2) else torch.full_like(g, math.nan) for i, g in enumerate(grads)]
        norm = torch.zeros(1, device="cuda")
        B.rad_clip_gradients(ctx, grads, part * want, clipped=None if place == "in place" else to, norm=norm)
        B.rad_ctx_synchronize(ctx)
        assert abs(float(norm) - want) <= 2 * U * want
        factor = min(1.0, part)
        for g, t, b, k in zip(grads, to, before, kinds):
            half = 2.0 ** -8 if k == torch.bfloat16 else U
            assert ((t.double() - factor * b).abs() <= (half + 2.02 * U) * factor * b.abs() + 1e-40).all()
            if t is not g:
                assert torch.equal(g.double(), b)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("offset", [0, 1])
def test_scaled_step_is_the_step_of_scaled_gradients(dtype, kind, offset):
    """Bit by bit the step that rad_optimizer_step makes of the gradients times the scale; more tensors than one launch takes."""
    import torch
    from paper_2007_10412_amd import binding as B
    sizes = SIZES + [65, 1030] * 40
    f32 = [torch.float32] * len(sizes)
    with Ctx() as ctx:
        grads = tensors(sizes, f32, 21, offset)
        scale = torch.tensor([0.3125], device="cuda")
        scaled = [(g * scale) for g in grads]
        opt = B.make_optimizer(kind, 1e-2, 1e-3, 0.9, 0.99, 1e-7)

        def state():
            w = tensors(sizes, f32, 22, offset)
            extra = dict(m=tensors(sizes, f32, 23, offset), v=[t.abs() for t in tensors(sizes, f32, 24, offset)]) if kind == 1 else {}
            if dtype == B.RAD_BF16:
                return [t.to(torch.bfloat16) for t in w], dict(extra, master=w)
            return w, extra
        (pa, a), (pb, b) = state(), state()
        B.rad_optimizer_step_scaled(ctx, opt, 3, dtype, pa, grads, scale, **a)
        for i in range(len(sizes)):                              # one at a time
            B.rad_optimizer_step(ctx, opt, 3, dtype, pb[i:i + 1], scaled[i:i + 1], **{n: t[i:i + 1] for n, t in b.items()})
        B.rad_ctx_synchronize(ctx)
        for x, y in zip(pa + sum(a.values(), []), pb + sum(b.values(), [])):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("scaled", [False, True])
def test_steps_that_the_caches_cannot_hold(dtype, kind, scaled):
    """One step of 46 million elements (552 MB of SGD, 1288 of Adam) has the bits of steps of its pieces."""
    import torch
    from paper_2007_10412_amd import binding as B
    n, piece = 46_000_003, 4096 * 700
    gen = torch.Generator(device="cuda").manual_seed(5)
    g, w, m = (torch.randn(n, device="cuda", generator=gen) for _ in range(3))
    v, scale = torch.rand(n, device="cuda", generator=gen), torch.full((1,), 0.3, device="cuda")
    opt = B.make_optimizer(B.RAD_ADAM if kind else B.RAD_SGD, 1e-2, 1e-4)
    with Ctx() as ctx:
        def state():
            return {"master": w.clone(), "m": m.clone(), "v": v.clone(), "params": w.to(torch.bfloat16) if dtype else None}

        def step(s, lo, hi):
            part = {k: None if t is None else [t[lo:hi]] for k, t in s.items()}
            master = part.pop("master")
            params = part.pop("params") if dtype else master
            args = (ctx, opt, 3, dtype, params, [g[lo:hi]]) + ((scale,) if scaled else ())
            part.pop("params", None)
            if not kind:
                part = {"m": None, "v": None}
            (B.rad_optimizer_step_scaled if scaled else B.rad_optimizer_step)(*args, **part, master=master if dtype else None)
        whole, pieces = state(), state()
        step(whole, 0, n)
        for lo in range(0, n, piece):
            step(pieces, lo, min(n, lo + piece))
        B.rad_ctx_synchronize(ctx)
        for k in whole:
            assert whole[k] is None or torch.equal(whole[k], pieces[k]), k
        assert not torch.equal(whole["master"], w)


@pytest.mark.parametrize("how,n", [("f32", 68_000_001), ("bf16", 136_000_001)])
@pytest.mark.parametrize("place", ["in place", "apart"])
def test_clipping_what_the_caches_cannot_hold(how, n, place):
    """Bits: a product rounded to fp32 and that to the type."""
    import torch
    from paper_2007_10412_amd import binding as B
    grads = tensors([n], mixed(1, how), 6)
    norm, scale = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    with Ctx() as ctx:
        B.rad_gradient_norm(ctx, grads, 100.0, norm=norm, scale=scale)
        B.rad_ctx_synchronize(ctx)
        want = (grads[0].float() * scale).to(grads[0].dtype)
        out = None if place == "in place" else [torch.zeros_like(grads[0])]
        B.rad_clip_gradients(ctx, grads, 100.0, clipped=out)
        B.rad_ctx_synchronize(ctx)
        assert 0 < float(scale) < 1 and torch.equal((out or grads)[0], want)


def test_tensors_that_share_memory_are_stepped_in_order():
    """A tensor that comes twice gets two steps, also when it is the second half of another."""
    import torch
    from paper_2007_10412_amd import binding as B
    with Ctx() as ctx:
        opt = B.make_optimizer(B.RAD_SGD, 0.5)
        w = torch.zeros(20000, device="cuda")
        g = torch.ones(20000, device="cuda")
        B.rad_optimizer_step(ctx, opt, 1, B.RAD_F32, [w, w, w[10000:]], [g, g, g[10000:]])
        B.rad_ctx_synchronize(ctx)
        assert (w[:10000] == -1.0).all() and (w[10000:] == -1.5).all()
        # a gradient that an earlier step writes
        a, b = torch.zeros(5000, device="cuda"), torch.zeros(5000, device="cuda")
        B.rad_optimizer_step_scaled(ctx, opt, 1, B.RAD_F32, [a, b], [g[:5000], a], torch.ones(1, device="cuda"))
        B.rad_ctx_synchronize(ctx)
        assert (a == -0.5).all() and (b == 0.25).all()


def test_clipped_training_step():
    """Whole iterations (rad_train_step, rad_gradient_norm, rad_optimizer_step_scaled): the parameters against the update in fp64 of the
    gradients that the step left, clipped by their norm."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(4)
    dims, batch = (784, 300, 10), 150
    with Ctx() as ctx:
        model = B.rad_model_create_mlp(ctx, B.RAD_F32, batch, list(dims), True, B.RAD_FIXEDK_PER_EXAMPLE, 0.1)
        params = []
        for i, o in zip(dims, dims[1:]):
            params += [torch.randn(i, o, device="cuda", generator=gen) / math.sqrt(i), torch.zeros(o, device="cuda")]
        grads = [torch.zeros_like(p) for p in params]
        x = torch.randn(batch, 784, device="cuda", generator=gen)
        labels = torch.randint(0, 10, (batch,), device="cuda", generator=gen).to(torch.int32)
        norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        opt = B.make_optimizer(B.RAD_SGD, 0.1)
        for step in range(3):
            B.rad_train_step(ctx, model, B.make_sampling(B.RAD_FIXEDK_PER_EXAMPLE, 0.1, step, 0, 0), x, labels, params, grads, want_loss=False)
            before = [p.double() for p in params]
            B.rad_gradient_norm(ctx, grads, 0.25, norm=norm, scale=scale)
            B.rad_optimizer_step_scaled(ctx, opt, step + 1, B.RAD_F32, params, grads, scale)
            B.rad_ctx_synchronize(ctx)
            want = norm_of(grads)
            assert want > 0.25 and abs(float(norm) - want) <= 2 * U * want
            f = 0.25 / want
            for p, b, g in zip(params, before, grads):
                move = 0.1 * f * g.double()
                # roundings: of the scale (1), the product (1), lr (1), the step's product (1), and of the difference
                assert ((p.double() - (b - move)).abs() <= 4.1 * U * move.abs() + U * (b - move).abs() + 1e-40).all()
        B.rad_model_destroy(model)


def test_captured_and_other_stream():
    """Norm, clip and step in a graph on a stream of its own, replayed with other gradients and eager calls between the replays."""
    import torch
    from paper_2007_10412_amd import binding as B
    stream = torch.cuda.Stream()
    sizes = [300, 4096 * 40 + 3, 17]
    f32 = [torch.float32] * 3
    with Ctx(stream) as ctx, Ctx() as plain:
        grads = tensors(sizes, f32, 31)
        w, m, v = tensors(sizes, f32, 32), [torch.zeros(n, device="cuda") for n in sizes], [torch.zeros(n, device="cuda") for n in sizes]
        out = [torch.zeros(n, device="cuda") for n in sizes]
        norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        opt = B.make_optimizer(B.RAD_ADAM, 1e-2)
        torch.cuda.synchronize()

        def calls(c, w, m, v, out, norm, scale):
            B.rad_clip_gradients(c, grads, 0.5, clipped=out)
            B.rad_gradient_norm(c, grads, 0.5, norm=norm, scale=scale)
            B.rad_optimizer_step_scaled(c, opt, 2, B.RAD_F32, w, grads, scale, m, v)
        with torch.cuda.stream(stream):
            calls(ctx, *[[t.clone() for t in q] for q in (w, m, v, out)], norm.clone(), scale.clone())
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                calls(ctx, w, m, v, out, norm, scale)
        mine = [[t.clone() for t in q] for q in (w, m, v, out)]
        n2, s2 = norm.clone(), scale.clone()
        for r in range(4):
            for g in grads:
                g.copy_(torch.randn_like(g) * (0.001 if r == 2 else 1.0))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            calls(plain, *mine, n2, s2)
            B.rad_ctx_synchronize(plain)
            assert float(norm) == float(n2) and float(scale) == float(s2) and (float(scale) == 1.0) == (r == 2)
            for a, b in zip((w, m, v, out), mine):
                assert all(torch.equal(x, y) for x, y in zip(a, b)), r
        del graph


def test_first_norm_is_not_recorded():
    import torch
    from paper_2007_10412_amd import binding as B
    stream = torch.cuda.Stream()
    g, n = torch.full((1000,), 2.0, device="cuda"), torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    with Ctx(stream) as ctx:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            torch.zeros(1, device="cuda").add_(1)
            for call in (lambda: B.rad_gradient_norm(ctx, [g], 1.0, norm=n), lambda: B.rad_clip_gradients(ctx, [g], 1.0)):
                with pytest.raises(B.RadError, match="recorded"):
                    call()
        B.rad_gradient_norm(ctx, [g], 1.0, norm=n)
        B.rad_ctx_synchronize(ctx)
        assert abs(float(n) - math.sqrt(4000.0)) <= 2 * U * math.sqrt(4000.0)


def test_refusals():
    import torch
    from paper_2007_10412_amd import binding as B
    with Ctx() as ctx:
        g, h = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
        n = torch.zeros(1, device="cuda")
        for call, status in (
                (lambda: B.rad_gradient_norm(ctx, [g], 0.0, norm=n), B.RAD_ERR_PARAM),
                (lambda: B.rad_gradient_norm(ctx, [g], -1.0, norm=n), B.RAD_ERR_PARAM),
                (lambda: B.rad_gradient_norm(ctx, [g], math.nan, norm=n), B.RAD_ERR_PARAM),
                (lambda: B.rad_gradient_norm(ctx, [g], 1.0), B.RAD_ERR_NULL),
                (lambda: B.rad_gradient_norm(ctx, [g], 1.0, norm=n, scale=n), B.RAD_ERR_PARAM),
                (lambda: B.rad_gradient_norm(ctx, [g], 1.0, norm=g[3:4]), B.RAD_ERR_PARAM),
                (lambda: B.rad_clip_gradients(ctx, [g, g], 1.0), B.RAD_ERR_PARAM),
                (lambda: B.rad_clip_gradients(ctx, [g], 1.0, norm=g[:1]), B.RAD_ERR_PARAM),
                (lambda: B.rad_clip_gradients(ctx, [g, h], 1.0, clipped=[h, g]), B.RAD_ERR_PARAM),
                (lambda: B.rad_clip_gradients(ctx, [g[:60]], 1.0, clipped=[g[4:]]), B.RAD_ERR_PARAM),
                (lambda: B.rad_optimizer_step_scaled(ctx, B.make_optimizer(B.RAD_SGD, 1e-2), 1, 0, [g], [h], g[63:]), B.RAD_ERR_PARAM),
                (lambda: B.rad_optimizer_step_scaled(ctx, B.make_optimizer(B.RAD_SGD, 1e-2), 1, 7, [g], [h], n), B.RAD_ERR_PARAM)):
            with pytest.raises(B.RadError) as e:
                call()
            assert e.value.status == status, e.value
        B.rad_ctx_synchronize(ctx)
        assert (g == 1).all() and (h == 1).all() and float(n) == 0.0

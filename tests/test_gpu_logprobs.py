"""rad_token_logprobs, rad_linear_logprobs and their gradients against their definitions in fp64, element by element.

Bounds are counted from the roundings, u = 2^-24 the half step of fp32 and h that of the layer's type (2^-8 bf16).  With d_v = (m - z_v) / T
and S = sum q d:
  an exponential's argument has two roundings of d (2 u d relative to the exponential) and the exponential itself two units (4 u); a sum
  of n of them is off by 8 u sqrt(n) (eight standard deviations of a random walk), so s, and ln s absolutely, by
  R = (8 sqrt(n) + 64) u beside 4 u S;
  log q = -d - ln s: R + 4 u (d + ln n + S + 1);
  H = ln s - ln 2 u' / s, u' = sum e l: R (1 + S + ln n) + 4 u sum q d^2 + 4 u (S + ln n + 1);
  dz = q (-a - h (log q + H)) / T: with M = q (|a| + |h| (d + S + 1)) / T the size of its parts, M (2 R + 8 u (d + S)) + q |h| / T times
  H's bound, 8 u |a| / T at the token, and the rounding to the type.  The hardware's exponential is 0 below 2^-126, and s is at least 1, so q may
  be off by 2^-126 besides, and dz by as much of (|a| + |h| (d + S + 1)) / T.
Logits of a layer are off by E = 8 u sqrt(d_in + 2) max sum |x| |W| each before T: 2 E / T in log q, 2 E / T (1 + S + ln n) in H (its derivative
is q (log q + H)); in bf16 training a logit is a code, off by half a step of 2^-9 of a power of two (0.18 h), and dz is rounded to the
type: 2.02 h M."""
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


def gen_for(*numbers):
    import torch
    return torch.Generator(device="cuda").manual_seed(sum(n * 7 ** i for i, n in enumerate(numbers)))


class Row:
    """What the definition says of rows of fp64 logits, and the bounds' parts."""

    def __init__(self, z, T, e_logit=0.0):
        import torch
        n = z.shape[1]
        self.z, self.T, self.e = z, T, e_logit / T
        self.log_q = torch.log_softmax(z / T, dim=1)
        self.q = torch.exp(self.log_q)
        zero = torch.zeros_like(self.q)
        self.s_log = torch.where(self.q > 0, self.log_q, zero)          # (q log q is 0 where q is)
        self.H = -(self.q * self.s_log).sum(dim=1)
        top = z.max(dim=1, keepdim=True).values
        self.d = torch.where(self.q > 0, (top - z) / T, zero)
        self.S = (self.q * self.d).sum(dim=1)
        self.D2 = (self.q * self.d ** 2).sum(dim=1)
        self.ln = math.log(n) + 1.0
        self.R = (8 * math.sqrt(n) + 64) * U
        self.bound_H = self.R * (self.S + self.ln) + 4 * U * (self.D2 + self.S + self.ln) + 2 * self.e * (self.S + self.ln)

    def bound_log_q(self, d, S):
        return self.R + 2 * self.e + 4 * U * (d.abs() + S + self.ln)

    def grad(self, token, counts, a, h):
        """dz, and its bound ahead of the last rounding, and the size of its parts"""
        import torch
        zero = torch.zeros(len(self.z), device="cuda", dtype=torch.float64)
        a = zero if a is None else torch.where(counts, a.double(), zero)
        h = zero if h is None else torch.where(counts, h.double(), zero)
        a, h = a[:, None] / self.T, h[:, None] / self.T
        dz = self.q * (-a - h * (self.s_log + self.H[:, None]))
        at = torch.zeros_like(dz)
        if token is not None:
            at.scatter_(1, token.long().clamp(0, dz.shape[1] - 1)[:, None], a.expand(-1, 1))
        size = a.abs() + h.abs() * (self.d + self.S[:, None] + 1)
        parts = self.q * size
        e = 2.0 ** -126 * size + parts * (2 * self.R + 2 * self.e + 8 * U * (self.d + self.S[:, None])) + self.q * h.abs() * (self.bound_H[:, None] + self.e) + 8 * U * at.abs()
        return dz + at, e, parts + at.abs()


def close(got, want, bound, tag):
    import torch
    got = got.double()
    assert got.shape == want.shape, tag
    want = torch.where(want.float().isinf(), want.float().double(), want)           # (what fp32 cannot hold is an infinity)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    assert (torch.isfinite(got) | same).all(), tag + ": not finite"
    over = torch.where(same, torch.zeros_like(want), (got - want).abs() - bound)
    if over.numel() == 0:
        return
    worst = int(over.argmax())
    assert float(over.max()) <= 0, "%s: element %d is %.9g, not %.9g (bound %.3g); %d are off" % (
        tag, worst, got.flatten()[worst], want.flatten()[worst], (bound + 0 * want).flatten()[worst], int((over > 0).sum()))


def likeliest(z, k):
    """The k largest of rows, in order, ties to the lowest place: indexes, -1 where nothing above -infinity is left."""
    import torch
    z = torch.where(torch.isnan(z), torch.full_like(z, -math.inf), z)
    order = torch.sort(z, dim=1, descending=True, stable=True)
    index = torch.where(order.values == -math.inf, torch.full_like(order.indices, -1), order.indices)[:, :k]
    if index.shape[1] < k:
        index = torch.cat([index, torch.full((len(z), k - index.shape[1]), -1, device="cuda")], dim=1)
    return index


def outputs(rows, k, names=("logprob", "entropy", "top")):
    import torch
    out = {}
    for n in ("logprob", "entropy"):
        if n in names:
            out[n] = torch.full((rows,), 77.0, device="cuda")
    if "top" in names and k:
        out["top_index"] = torch.full((rows, k), 77, device="cuda", dtype=torch.int32)
        out["top_logprob"] = torch.full((rows, k), 77.0, device="cuda")
    return out


def check_answer(out, row, tokens, k, tag, index=None):
    """Outputs against the definition; index: what the lists' indexes are to be (None: by row.z)."""
    import torch
    n, classes = row.z.shape
    counts = torch.ones(n, dtype=torch.bool, device="cuda") if tokens is None else (tokens >= 0) & (tokens < classes)
    zero = torch.zeros(n, device="cuda", dtype=torch.float64)
    if "logprob" in out:
        at = tokens.long().clamp(0, classes - 1)[:, None]
        want = torch.where(counts, row.log_q.gather(1, at)[:, 0], zero)
        d = torch.where(torch.isfinite(want), want, zero)
        close(out["logprob"], want, torch.where(counts, row.bound_log_q(d, row.S), zero), tag + " logprob")
    if "entropy" in out:
        close(out["entropy"], torch.where(counts, row.H, zero), torch.where(counts, row.bound_H, zero), tag + " entropy")
    if "top_index" in out:
        got = out["top_index"].long()
        want = likeliest(row.z, k) if index is None else index
        want = torch.where(counts[:, None], want, torch.full_like(want, -1))
        assert torch.equal(got, want), "%s: %d places of the lists differ, first %s" % (tag, int((got != want).sum()), (got != want).nonzero()[0].tolist())
        lp = torch.where(want >= 0, row.log_q.gather(1, want.clamp(min=0)), torch.full(want.shape, -math.inf, device="cuda", dtype=torch.float64))
        d = torch.where(torch.isfinite(lp), lp, torch.zeros_like(lp))
        close(out["top_logprob"], lp, row.bound_log_q(d, row.S[:, None]), tag + " top_logprob")


def tokens_for(rows, classes, gen, ignored=0.0):
    import torch
    t = torch.randint(0, classes, (rows,), device="cuda", generator=gen)
    if ignored:
        out = torch.rand(rows, device="cuda", generator=gen) < ignored
        other = torch.tensor([-1, -100, classes, 2 ** 31 - 1, -2 ** 31], device="cuda")[torch.arange(rows, device="cuda") % 5]
        t = torch.where(out, other, t)
    return t.to(torch.int32)


def call_dense(ctx, dtype, z, k, T=1.0, tokens=None, names=("logprob", "entropy", "top")):
    from paper_2007_10412_amd import binding as B
    out = outputs(len(z), k, [n for n in names if n != "logprob" or tokens is not None])
    B.rad_token_logprobs(ctx, z, dtype, tokens=tokens, temperature=T, **out)
    B.rad_ctx_synchronize(ctx)
    return out


# (every size of row that a workgroup keeps, and rows in parts; widths that are no whole vectors)
WIDTHS = [1, 2, 7, 9, 64, 255, 1000, 2047, 2048, 2049, 4100, 8191, 8200, 16390, 33001, 52900, 53100, 65536, 65600, 105900, 131071, 131080, 150001]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows", [1, 3, 70])
@pytest.mark.parametrize("classes", WIDTHS)
def test_dense(dtype, rows, classes):
    import torch
    gen = gen_for(rows, classes, dtype)
    z = (3 * torch.randn(rows, classes, device="cuda", generator=gen)).to(torch_dtype(dtype))
    tokens = tokens_for(rows, classes, gen, 0.3 if rows > 3 else 0.0)
    with Ctx() as ctx:
        for k, T in ((0, 1.0), (1, 0.7), (5, 1.0), (20, 2.0), (64, 1.0), (200, 1.0), (256, 3.0)):
            tag = "dense dtype %d %d x %d k %d" % (dtype, rows, classes, k)
            print(tag, flush=True)
            check_answer(call_dense(ctx, dtype, z, k, T, tokens), Row(z.double(), T), tokens, k, tag)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("names", [("logprob",), ("entropy",), ("top",), ("entropy", "top"), ("logprob", "top")])
@pytest.mark.parametrize("rows,classes", [(5, 1003), (2, 140001), (9, 40000)])
def test_some_outputs(dtype, names, rows, classes):
    import torch
    gen = gen_for(rows, classes)
    z = (3 * torch.randn(rows, classes, device="cuda", generator=gen)).to(torch_dtype(dtype))
    tokens = tokens_for(rows, classes, gen, 0.3) if "logprob" in names else None
    with Ctx() as ctx:
        check_answer(call_dense(ctx, dtype, z, 7, 1.5, tokens, names), Row(z.double(), 1.5), tokens, 7, str(names))


def odd_rows(classes, dtype, gen):
    """Rows that a list is hard to find in: (name, values)"""
    import torch
    r = 3 * torch.randn(classes, device="cuda", generator=gen)
    at = torch.arange(classes, device="cuda")
    lowest = torch.finfo(torch_dtype(dtype)).min
    few = torch.full((classes,), -math.inf, device="cuda")
    few[classes // 3::classes // 3 + 1] = 1.5
    zeros = torch.zeros(classes, device="cuda")
    zeros[::2] = -0.0
    block = r.clone()
    block[classes // 4:] = -math.inf
    spread = torch.where(at % 50 == 7, r, torch.full_like(r, -1e30))
    return [("equal", torch.full((classes,), 2.5, device="cuda")), ("zeros of both signs", zeros), ("two values", (at % 3 == 0).float()),
            ("ascending", at / classes * 20), ("descending", -at / classes * 20), ("steps", (at // 97).float() / 40), ("few", few),
            ("half -inf", torch.where(at % 2 == 0, r, torch.full_like(r, -math.inf))), ("block", block),
            ("lowest", torch.where(at % 3 == 0, r, torch.full_like(r, lowest))), ("all lowest", torch.full((classes,), lowest, device="cuda")),
            ("far", spread), ("peak", torch.where(at == classes // 2, torch.full_like(r, 90.0), r)), ("large", r * 1e4), ("negative", r - 1e3),
            ("last ones", torch.where(at >= classes - 9, r + 40, r)), ("nothing", torch.full((classes,), -math.inf, device="cuda")),
            ("nan", torch.where(at == classes // 5, torch.full_like(r, math.nan), r)), ("inf", torch.where(at == classes // 5, torch.full_like(r, math.inf), r)),
            ("only nan", torch.full((classes,), math.nan, device="cuda")), ("random", r)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("classes", [300, 1000, 2040, 5001, 20000, 50257, 140000])
def test_odd_rows(dtype, classes):
    """Ties, masks, infinities and NaN; each in a row of its own, so that none leaves its row."""
    import torch
    rows = odd_rows(classes, dtype, gen_for(classes))
    z = torch.stack([v for _, v in rows]).to(torch_dtype(dtype))
    tokens = torch.full((len(z),), classes // 3, device="cuda", dtype=torch.int32)
    with Ctx() as ctx:
        for k in (1, 20, 129, 256):
            out = call_dense(ctx, dtype, z, k, 1.0, tokens)
            for i, (name, _) in enumerate(rows):
                tag = "%s, dtype %d, %d classes, k %d" % (name, dtype, classes, k)
                zi = z[i:i + 1].double()
                one = {n: t[i:i + 1] for n, t in out.items()}
                if name in ("nothing", "nan", "inf", "only nan"):
                    assert torch.isnan(one["logprob"]).all() and torch.isnan(one["entropy"]).all(), tag
                    want = likeliest(zi, k)
                    assert torch.equal(one["top_index"].long(), want), tag
                    assert torch.isnan(one["top_logprob"][want >= 0]).all() and (one["top_logprob"][want < 0] == -math.inf).all(), tag
                    continue
                check_answer(one, Row(zi, 1.0), tokens[i:i + 1], k, tag)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T", [1.0, 0.01])
@pytest.mark.parametrize("rows,classes", [(9, 700), (4, 5001), (90, 50257), (2, 140000)])
def test_rows_far_from_zero(dtype, T, rows, classes):
    """Offsets that an exponential's argument cannot carry along, up to the type's last values; and rows in which they meet."""
    import torch
    gen = gen_for(rows, classes, 9)
    r = 3 * torch.randn(rows, classes, device="cuda", generator=gen)
    tokens = tokens_for(rows, classes, gen)
    with Ctx() as ctx:
        for offset in (1e3, -1e3, 3e5, -3e5, 2e7, -2e7, 1e9, -1e9, 1e20, -1e20, 3e38, -3e38):
            # (a few multiples of the offset's last place apart: distinct values, a type's resolution there being what it is)
            step = abs(offset) * 2.0 ** (-7 if dtype else -22)
            z = (offset + torch.round(r) * (step if abs(offset) > 1e6 else 1.0)).clamp(-3.38e38, 3.38e38).to(torch_dtype(dtype))
            check_answer(call_dense(ctx, dtype, z, 12, T, tokens), Row(z.double(), float(torch.tensor(T, dtype=torch.float32))), tokens, 12, "offset %g T %g %d x %d" % (offset, T, rows, classes))
        z = torch.where(torch.arange(classes, device="cuda") % 11 == 3, r, -1e9 * r.abs()).to(torch_dtype(dtype))
        check_answer(call_dense(ctx, dtype, z, 12, T, tokens), Row(z.double(), float(torch.tensor(T, dtype=torch.float32))), tokens, 12, "mixed")


@pytest.mark.parametrize("dtype", [0, 1])
def test_ties_go_to_the_lowest_class(dtype):
    """Values of few different ones, so that most places of every list are ties; in rows of every kind."""
    import torch
    with Ctx() as ctx:
        for rows, classes in ((40, 500), (8, 9000), (70, 33000), (3, 100003), (1, 300000)):
            gen = gen_for(rows, classes, 5)
            z = (torch.randint(0, 60, (rows, classes), device="cuda", generator=gen).float() ** 2 / 256).to(torch_dtype(dtype))
            for k in (3, 100, 256):
                check_answer(call_dense(ctx, dtype, z, k), Row(z.double(), 1.0), None, k, "ties %d x %d k %d" % (rows, classes, k))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T", [1e-6, 0.01, 50.0, 1e6])
def test_temperatures(dtype, T):
    import torch
    gen = gen_for(3, dtype)
    z = torch.randn(6, 5000, device="cuda", generator=gen).to(torch_dtype(dtype))
    tokens = z.float().argmax(dim=1).to(torch.int32)
    with Ctx() as ctx:
        out = call_dense(ctx, dtype, z, 9, T, tokens)
        row = Row(z.double(), float(torch.tensor(T, dtype=torch.float32)))    # (the library's T is fp32)
        check_answer({n: t for n, t in out.items() if n != "top_logprob" and n != "top_index"}, row, tokens, 9, "T %g" % T)
        assert torch.equal(out["top_index"].long(), likeliest(z.double(), 9))


@pytest.mark.parametrize("dtype", [0, 1])
def test_many_short_rows(dtype):
    """More rows than 65535, and a column of a larger tensor's rows at an odd address."""
    import torch
    gen = gen_for(9, dtype)
    z = torch.randn(70001 * 5 + 1, device="cuda", generator=gen).to(torch_dtype(dtype))[1:].view(70001, 5)
    tokens = tokens_for(70001, 5, gen, 0.2)
    with Ctx() as ctx:
        check_answer(call_dense(ctx, dtype, z, 3, 1.0, tokens), Row(z.double(), 1.0), tokens, 3, "short rows")


@pytest.mark.parametrize("dtype", [0, 1])
def test_widest_rows(dtype):
    """As many classes as a call may have, forward and backward."""
    import torch
    gen = gen_for(10, dtype)
    z = (3 * torch.randn(1, 2 ** 24, device="cuda", generator=gen)).to(torch_dtype(dtype))
    tokens, a, h = tokens_for(1, 2 ** 24, gen), torch.randn(1, device="cuda", generator=gen), torch.randn(1, device="cuda", generator=gen)
    with Ctx() as ctx:
        check_answer(call_dense(ctx, dtype, z, 256, 1.0, tokens), Row(z.double(), 1.0), tokens, 256, "2^24 classes")
        check_dense_grad(ctx, dtype, z, tokens, a, h, tag="2^24 classes")


@pytest.mark.parametrize("dtype,rows,classes", [(1, 1030, 2 ** 21 + 8), (1, 90000, 1001), (0, 45000, 1000), (1, 22000, 4100), (1, 6000, 16001),
                                                (0, 1400, 32000), (0, 1300, 50257), (1, 1300, 100000)])
def test_large_logits(dtype, rows, classes):
    """More than the caches hold (180 MB to 4.3 GB, the first beyond offsets of 32 bits): the first rows, some between and the last."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen = gen_for(12, rows)
    z = torch.randn(rows, classes, device="cuda", generator=gen, dtype=torch_dtype(dtype))
    tokens = tokens_for(rows, classes, gen)
    a, h = torch.randn(rows, device="cuda", generator=gen), torch.randn(rows, device="cuda", generator=gen)
    at = torch.tensor([0, 1, rows // 3, rows - 2, rows - 1], device="cuda")
    row = Row(z[at].double(), 1.0)
    with Ctx() as ctx:
        out = call_dense(ctx, dtype, z, 5, 1.0, tokens)
        check_answer({n: t[at] for n, t in out.items()}, row, tokens[at], 5, "far rows")
        dz = torch.full_like(z, 77.0)
        B.rad_token_logprobs_grad(ctx, z, dtype, dz, tokens=tokens, d_logprob=a, d_entropy=h)
        B.rad_ctx_synchronize(ctx)
        want, e, _ = row.grad(tokens[at], torch.ones(5, dtype=torch.bool, device="cuda"), a[at], h[at])
        close(dz[at], want, e + HALF[dtype] * want.abs() * 1.01 + 1e-38 * 2 ** (8 if dtype else 0), "far rows' gradients")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,classes", [(1100, 2050), (1100, 4999), (1100, 9001), (1100, 19001), (4100, 9003), (4100, 17001)])
def test_many_rows(dtype, rows, classes):
    """Rows that a wave or two have to themselves: as they come, with masks, and with so few values that lists end within ties."""
    import torch
    gen = gen_for(14, dtype, rows, classes)
    z = (3 * torch.randn(rows, classes, device="cuda", generator=gen)).to(torch_dtype(dtype))
    z[::5] = z[::5].round()
    z[1::7, 3:] = -math.inf
    z[2::7] = 0.5
    z[3::7] = torch.where(torch.rand(z[3::7].shape, device="cuda", generator=gen) < 0.5, -math.inf, z[3::7].float()).to(z.dtype)
    tokens = tokens_for(rows, classes, gen, 0.2)
    row = Row(z.double(), 1.3)
    with Ctx() as ctx:
        for k in (32, 5, 1, 0):
            check_answer(call_dense(ctx, dtype, z, k, 1.3, tokens), row, tokens, k, "k %d" % k)


# ------------------------------------------------------------------ gradients of dense logits
def check_dense_grad(ctx, dtype, z, tokens, a, h, T=1.0, in_place=False, tag=""):
    import torch
    from paper_2007_10412_amd import binding as B
    rows, classes = z.shape
    zd = z.double()
    to = z.clone() if in_place else torch.full_like(z, 77.0)
    if in_place and z.data_ptr() % 16:                     # (at the same odd address)
        flat = torch.empty(z.numel() + 8, device="cuda", dtype=z.dtype)
        off = (z.data_ptr() % 16) // z.element_size()
        to = flat[off:off + z.numel()].view(rows, classes)
        to.copy_(z)
    B.rad_token_logprobs_grad(ctx, to if in_place else z, dtype, to, tokens=tokens, temperature=T, d_logprob=a, d_entropy=h)
    B.rad_ctx_synchronize(ctx)
    counts = torch.ones(rows, dtype=torch.bool, device="cuda") if tokens is None else (tokens >= 0) & (tokens < classes)
    want, e, _ = Row(zd, T).grad(tokens if a is not None else None, counts, a, h)
    close(to, want, e + HALF[dtype] * want.abs() * 1.01 + 1e-38 * 2 ** (8 if dtype else 0), "%s dtype %d %d x %d" % (tag, dtype, rows, classes))
    assert (to[~counts] == 0).all()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows", [1, 3, 70])
@pytest.mark.parametrize("classes", WIDTHS)
def test_dense_grad(dtype, rows, classes):
    import torch
    gen = gen_for(rows, classes, dtype, 2)
    z = (3 * torch.randn(rows, classes, device="cuda", generator=gen)).to(torch_dtype(dtype))
    tokens = tokens_for(rows, classes, gen, 0.3 if rows > 3 else 0.0)
    a, h = torch.randn(rows, device="cuda", generator=gen), torch.randn(rows, device="cuda", generator=gen)
    with Ctx() as ctx:
        print("dense grad", dtype, rows, classes, flush=True)
        check_dense_grad(ctx, dtype, z, tokens, a, h)
        check_dense_grad(ctx, dtype, z, tokens, a, None, T=0.7, in_place=True, tag="in place")
        check_dense_grad(ctx, dtype, z, None, None, h, T=2.0, tag="entropy")
        check_dense_grad(ctx, dtype, z, tokens, None, h, T=2.0, tag="entropy of some rows")


@pytest.mark.parametrize("dtype", [0, 1])
def test_grad_of_many_short_rows(dtype):
    import torch
    gen = gen_for(11, dtype)
    z = torch.randn(70001 * 5 + 1, device="cuda", generator=gen).to(torch_dtype(dtype))[1:].view(70001, 5)
    tokens = tokens_for(70001, 5, gen, 0.2)
    a, h = torch.randn(70001, device="cuda", generator=gen), torch.randn(70001, device="cuda", generator=gen)
    with Ctx() as ctx:
        check_dense_grad(ctx, dtype, z, tokens, a, h, tag="short rows")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("classes", [1000, 50257, 140000])
def test_masked_grad(dtype, classes):
    """-infinity and a type's lowest values have no gradient; a row that does not count has zeros whatever it and its weights hold; a NaN stays
    in its row."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen = gen_for(classes, dtype)
    td = torch_dtype(dtype)
    z = 3 * torch.randn(8, classes, device="cuda", generator=gen)
    tokens = torch.full((8,), 4, device="cuda", dtype=torch.int32)
    z[0, 5:] = -math.inf
    z[1, 5::2] = torch.finfo(td).min
    z[2, classes // 2:] = -1e30
    tokens[3] = -1
    z[3] = math.nan
    tokens[4] = classes
    z[5, 17] = math.nan
    z[6, :] = torch.finfo(td).min
    a, h = torch.randn(8, device="cuda", generator=gen), torch.randn(8, device="cuda", generator=gen)
    a[3], h[3], a[4], h[4] = math.nan, math.inf, math.inf, math.nan
    z = z.to(td)
    with Ctx() as ctx:
        for i in (0, 1, 2, 6, 7):
            check_dense_grad(ctx, dtype, z[i:i + 1].contiguous(), tokens[i:i + 1], a[i:i + 1], h[i:i + 1], tag="masked row %d" % i)
        out = torch.full_like(z, 7.0)
        B.rad_token_logprobs_grad(ctx, z, dtype, out, tokens=tokens, d_logprob=a, d_entropy=h)
        B.rad_ctx_synchronize(ctx)
        assert (out[3:5] == 0).all() and torch.isnan(out[5]).all()
        assert (out[0, 5:] == 0).all() and (out[1, 5::2] == 0).all() and (out[2, classes // 2:] == 0).all()
        rest = torch.tensor([0, 1, 2, 6, 7], device="cuda")
        assert torch.isfinite(out[rest]).all()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T", [1.0, 0.01])
@pytest.mark.parametrize("rows,classes", [(9, 700), (4, 5001), (90, 50257), (2, 140000)])
def test_grad_of_rows_far_from_zero(dtype, T, rows, classes):
    import torch
    gen = gen_for(rows, classes, 10)
    r = 3 * torch.randn(rows, classes, device="cuda", generator=gen)
    tokens = tokens_for(rows, classes, gen, 0.2)
    a, h = torch.randn(rows, device="cuda", generator=gen), torch.randn(rows, device="cuda", generator=gen)
    T32 = float(torch.tensor(T, dtype=torch.float32))
    with Ctx() as ctx:
        for offset in (1e3, -3e5, 2e7, -2e7, 1e9, -1e20, 3e38, -3e38):
            step = abs(offset) * 2.0 ** (-7 if dtype else -22)
            z = (offset + torch.round(r) * (step if abs(offset) > 1e6 else 1.0)).clamp(-3.38e38, 3.38e38).to(torch_dtype(dtype))
            check_dense_grad(ctx, dtype, z, tokens, a, h, T=T32, in_place=offset < 0, tag="offset %g T %g" % (offset, T))


@pytest.mark.parametrize("dtype", [0])
def test_gradients_against_differences(dtype):
    """Central differences of the library's own outputs: of f = sum a log q[token] + h H along random directions.  With logits of size 1 and a
    step of 2^-4, the third derivatives of log q and H are of the order of 1, so the differences' error is 2^-8 / 6 times the
    directions' cubes (|v|_inf = 1) beside fp32's 2^-20 / 2^-4; a bound of 0.02 on each of 20 covers both."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen = gen_for(77)
    rows, classes = 4, 11
    z = torch.randn(rows, classes, device="cuda", generator=gen)
    tokens = tokens_for(rows, classes, gen)
    a, h = torch.randn(rows, device="cuda", generator=gen), torch.randn(rows, device="cuda", generator=gen)

    def f(zz):
        out = call_dense(ctx, 0, zz.contiguous(), 0, 1.3, tokens)
        return float((a.double() * out["logprob"].double() + h.double() * out["entropy"].double()).sum())
    with Ctx() as ctx:
        dz = torch.empty_like(z)
        B.rad_token_logprobs_grad(ctx, z, 0, dz, tokens=tokens, temperature=1.3, d_logprob=a, d_entropy=h)
        B.rad_ctx_synchronize(ctx)
        for i in range(20):
            v = torch.randint(0, 2, z.shape, device="cuda", generator=gen).float() * 2 - 1
            v *= (torch.rand(z.shape, device="cuda", generator=gen) < 0.2)
            s = 2.0 ** -4
            assert abs((f(z + s * v) - f(z - s * v)) / (2 * s) - float((dz.double() * v.double()).sum())) < 0.02, i


# ------------------------------------------------------------------ with the layer in it
def layer_inputs(dtype, rows, d_in, classes, bias, gen, grid=False, scale=3.0):
    import torch
    td = torch_dtype(dtype)
    if grid:        # sums of products that are exact in fp32: |x| <= 64 and |W| <= 128 steps, sums of 4096 of them far below 2^24 steps
        step = 2.0 ** round(math.log2(scale / math.sqrt(d_in))) / 32
        x = ((torch.randn(rows, d_in, device="cuda", generator=gen) * 16).round().clamp(-64, 64) / 16).to(td)
        W = ((torch.randn(d_in, classes, device="cuda", generator=gen) * 32).round().clamp(-128, 128) * step).to(td)
        b = (torch.randn(classes, device="cuda", generator=gen) * 16).round() / 16 if bias else None
    else:
        x = torch.randn(rows, d_in, device="cuda", generator=gen).to(td)
        W = (torch.randn(d_in, classes, device="cuda", generator=gen) * (scale / math.sqrt(d_in))).to(td)
        b = torch.randn(classes, device="cuda", generator=gen) if bias else None
    return x, W, b


def layer_row(x, W, b, T):
    """the definition of a layer's logits"""
    xd, Wd = x.double(), W.double()
    z, size = xd @ Wd, xd.abs() @ Wd.abs()
    if b is not None:
        z = z + b.double()
        size = size + b.double().abs().clamp(max=1e3)
    return Row(z, T, 8 * U * math.sqrt(x.shape[1] + 2) * float(size.max()))


def check_linear(ctx, dtype, rows, d_in, classes, k, bias=False, ignored=0.0, T=1.0, grid=True, no_tokens=False, names=("logprob", "entropy", "top"), values=None):
    import torch
    from paper_2007_10412_amd import binding as B
    tag = "linear dtype %d %d x %d x %d k %d %s" % (dtype, rows, d_in, classes, k, "grid" if grid else "")
    print(tag, flush=True)
    gen = gen_for(rows, d_in, classes, k)
    x, W, b = layer_inputs(dtype, rows, d_in, classes, bias, gen, grid)
    if values is not None:
        b = values(b)
    tokens = None if no_tokens else tokens_for(rows, classes, gen, ignored)
    out = outputs(rows, k, [n for n in names if n != "logprob" or tokens is not None])
    layer = B.make_layer(rows, d_in, classes, dtype=dtype, relu=False, has_bias=b is not None)
    B.rad_linear_logprobs(ctx, layer, x, W, b, tokens=tokens, temperature=T, **out)
    B.rad_ctx_synchronize(ctx)
    row = layer_row(x, W, b, T)
    if grid or "top_index" not in out:
        check_answer(out, row, tokens, k, tag)
        return
    # logits in fp32 may change places within twice their error: each listed one is as large as the one due there, and none comes twice
    got = out["top_index"].long()
    counts = torch.ones(rows, dtype=torch.bool, device="cuda") if tokens is None else (tokens >= 0) & (tokens < classes)
    due = row.z.gather(1, likeliest(row.z, k).clamp(min=0))
    there = row.z.gather(1, got.clamp(min=0))
    assert ((due - there).abs() <= 2 * row.e * T)[counts].all(), tag
    assert (got[counts].sort(dim=1).values.diff(dim=1) > 0).all() and (got[~counts] == -1).all(), tag
    check_answer(out, row, tokens, k, tag, index=got)


SHAPES = [(1, 1, 1), (1, 5, 3), (3, 7, 1), (5, 64, 33), (150, 300, 10), (64, 256, 1000), (130, 129, 131), (257, 520, 1003),
          (300, 512, 4096), (1000, 72, 2500), (512, 1024, 8192), (17, 1030, 20011), (513, 260, 25601), (700, 512, 32000),
          (20, 129, 30000), (1025, 1000, 8200), (1, 2048, 50257), (2, 300, 128000), (190, 1000, 28003), (381, 1000, 25009)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", SHAPES)
def test_linear(dtype, rows, d_in, classes):
    with Ctx() as ctx:
        check_linear(ctx, dtype, rows, d_in, classes, 20, bias=rows % 2 == 0, ignored=0.3 if rows > 4 else 0.0)
        check_linear(ctx, dtype, rows, d_in, classes, 1, bias=rows % 2 == 1, T=0.7, no_tokens=True)
        check_linear(ctx, dtype, rows, d_in, classes, 256, T=2.0)
        check_linear(ctx, dtype, rows, d_in, classes, 0, bias=True, grid=False, T=1.5)
        check_linear(ctx, dtype, rows, d_in, classes, min(5, classes), grid=False, names=("top", "logprob"))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8])
@pytest.mark.parametrize("d_in,classes", [(1, 64), (31, 65), (32, 127), (33, 128), (100, 129), (512, 1000), (700, 4099), (2049, 20011), (1030, 16384),
                                          (5000, 4097), (2048, 33000)])
def test_linear_few_rows(dtype, rows, d_in, classes):
    with Ctx() as ctx:
        check_linear(ctx, dtype, rows, d_in, classes, 5, bias=rows % 2 == 0, ignored=0.4 if rows > 1 else 0.0)
        check_linear(ctx, dtype, rows, d_in, classes, min(64, classes), bias=True, T=0.7, no_tokens=True)
        check_linear(ctx, dtype, rows, d_in, classes, 0, grid=False, T=1.5)


@pytest.mark.parametrize("dtype,rows,d_in,classes", [(1, 4, 4096, 1000), (0, 8, 8192, 2048), (1, 3, 8192, 4096), (0, 8, 4096, 8192), (1, 4, 4096, 65536), (1, 1, 4096, 16384), (0, 3, 2048, 16000)])
def test_linear_few_rows_of_large_layers(dtype, rows, d_in, classes):
    with Ctx() as ctx:
        check_linear(ctx, dtype, rows, d_in, classes, 20, bias=True, ignored=0.3 if rows > 1 else 0.0)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("masked", [-math.inf, -3.0e38])
@pytest.mark.parametrize("rows,d_in,classes", [(3, 64, 1000), (300, 256, 4096), (600, 256, 20000)])
def test_linear_masked_classes(dtype, masked, rows, d_in, classes):
    """Classes that a bias takes out, whole tiles of them among these, and all but a few."""
    import torch

    def half(b):
        b = b.clone()
        b[classes // 2:] = masked
        b[1:classes // 2:3] = masked
        return b

    def few(b):
        b = torch.full_like(b, masked)
        b[classes // 3], b[classes // 2] = 0.0, 0.0
        return b
    with Ctx() as ctx:
        for values in (half, few):
            if values is few and masked > -math.inf:      # (the lowest values come in the order of their fp32 sums)
                check_linear(ctx, dtype, rows, d_in, classes, 2, bias=True, values=values, no_tokens=True)
                continue
            check_linear(ctx, dtype, rows, d_in, classes, 40, bias=True, values=values, no_tokens=masked == -math.inf,
                         names=("entropy", "top") if masked == -math.inf else ("entropy",))


@pytest.mark.parametrize("dtype", [0, 1])
def test_linear_equal_logits(dtype):
    """A head that begins as zeros: every list is the first classes."""
    import torch
    from paper_2007_10412_amd import binding as B
    with Ctx() as ctx:
        for rows, classes in ((1, 5000), (300, 32000), (70, 1000)):
            x = torch.randn(rows, 64, device="cuda").to(torch_dtype(dtype))
            W = torch.zeros(64, classes, device="cuda").to(torch_dtype(dtype))
            out = outputs(rows, 50, ("entropy", "top"))
            B.rad_linear_logprobs(ctx, B.make_layer(rows, 64, classes, dtype=dtype, relu=False), x, W, None, **out)
            B.rad_ctx_synchronize(ctx)
            assert torch.equal(out["top_index"].long(), torch.arange(50, device="cuda").expand(rows, 50))
            assert (out["top_logprob"] + math.log(classes)).abs().max() < 1e-5 and (out["entropy"] - math.log(classes)).abs().max() < 1e-5


def check_linear_grad(ctx, dtype, rows, d_in, classes, bias=False, ignored=0.0, T=1.0, beta=0.0, dw_dtype=None, kinds="ah", outputs=("dX", "dW", "dbias"),
                      no_tokens=False, scale=3.0):
    import torch
    from paper_2007_10412_amd import binding as B
    tag = "linear grad dtype %d %d x %d x %d" % (dtype, rows, d_in, classes)
    print(tag, flush=True)
    gen = gen_for(rows, d_in, classes, 3)
    wd = torch_dtype(dtype if dw_dtype is None else dw_dtype)
    x, W, b = layer_inputs(dtype, rows, d_in, classes, bias, gen, scale=scale)
    tokens = None if no_tokens else tokens_for(rows, classes, gen, ignored) if ignored < 1 else torch.full((rows,), -1, device="cuda", dtype=torch.int32)
    a = torch.randn(rows, device="cuda", generator=gen) if "a" in kinds else None
    h = torch.randn(rows, device="cuda", generator=gen) if "h" in kinds else None
    layer = B.make_layer(rows, d_in, classes, dtype=dtype, relu=False, has_bias=b is not None)
    dW0 = torch.randn(d_in, classes, device="cuda", generator=gen).to(wd)
    db0 = torch.randn(classes, device="cuda", generator=gen)
    out = {"dX": torch.full_like(x, math.nan), "dW": dW0.clone() if beta else torch.full_like(dW0, math.nan),
           "dbias": db0.clone() if beta else torch.full((classes,), math.nan, device="cuda")}
    asked = {n: out[n] for n in outputs}
    B.rad_linear_logprobs_grad(ctx, layer, x, W, b, tokens=tokens, temperature=T, d_logprob=a, d_entropy=h, beta=beta, **asked)
    B.rad_ctx_synchronize(ctx)
    counts = torch.ones(rows, dtype=torch.bool, device="cuda") if tokens is None else (tokens >= 0) & (tokens < classes)
    dz, e, parts = layer_row(x, W, b, T).grad(tokens if a is not None else None, counts, a, h)
    xd, Wd = x.double(), W.double()
    e = e + 2.02 * HALF[dtype] * parts
    if "dX" in asked:
        want = dz @ Wd.t().contiguous()
        mass = dz.abs() @ Wd.abs().t().contiguous()
        close(out["dX"], want, e @ Wd.abs().t().contiguous() + 8 * U * math.sqrt(classes) * mass + HALF[dtype] * want.abs() + 1e-37, tag + " dX")
        assert (out["dX"][~counts] == 0).all(), tag
    if "dW" in asked:
        want = xd.t().contiguous() @ dz + (dW0.double() if beta else 0)
        mass = xd.abs().t().contiguous() @ dz.abs() + (dW0.double().abs() if beta else 0)
        close(out["dW"], want, xd.abs().t().contiguous() @ e + 8 * U * math.sqrt(rows + 1) * mass + HALF[1 if wd == torch.bfloat16 else 0] * want.abs() + 1e-37, tag + " dW")
    if "dbias" in asked:
        want = dz.sum(dim=0) + (db0.double() if beta else 0)
        close(out["dbias"], want, e.sum(dim=0) + 8 * U * math.sqrt(rows + 1) * (dz.abs().sum(dim=0) + (db0.double().abs() if beta else 0)) + 1e-37, tag + " dbias")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", SHAPES)
def test_linear_grad(dtype, rows, d_in, classes):
    with Ctx() as ctx:
        check_linear_grad(ctx, dtype, rows, d_in, classes, bias=rows % 2 == 0, ignored=0.3 if rows > 4 else 0.0)
        check_linear_grad(ctx, dtype, rows, d_in, classes, kinds="h", no_tokens=True, T=1.5)


def test_linear_gradients_against_differences():
    """As for dense logits, in directions of x, W and the bias of +-1 in a fifth of their elements: logits move by |dz| <= 3 times the step of 2^-6
    (8 inputs of size 1/2, weights of size 1/2), so 4 rows of third derivatives of the order of 2 leave 4 x 2 x 27 x 2^-12 / 6 = 0.009 at most beside
    rounding's 2^-19 / 2^-6; a bound of 0.03 covers both."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen = gen_for(78)
    rows, d_in, classes = 4, 8, 11
    x, W = torch.randn(rows, d_in, device="cuda", generator=gen) / 2, torch.randn(d_in, classes, device="cuda", generator=gen) / 2
    b = torch.randn(classes, device="cuda", generator=gen) / 2
    tokens = tokens_for(rows, classes, gen)
    a, h = torch.randn(rows, device="cuda", generator=gen), torch.randn(rows, device="cuda", generator=gen)
    layer = B.make_layer(rows, d_in, classes, dtype=0, relu=False, has_bias=True)
    with Ctx() as ctx:
        def f(*at):
            out = outputs(rows, 0)
            B.rad_linear_logprobs(ctx, layer, *at, tokens=tokens, temperature=1.3, **out)
            B.rad_ctx_synchronize(ctx)
            return float((a.double() * out["logprob"].double() + h.double() * out["entropy"].double()).sum())
        dX, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty_like(b)
        B.rad_linear_logprobs_grad(ctx, layer, x, W, b, tokens=tokens, temperature=1.3, d_logprob=a, d_entropy=h, dX=dX, dW=dW, dbias=db)
        B.rad_ctx_synchronize(ctx)
        for i in range(30):
            which = i % 3
            t, g = ((x, dX), (W, dW), (b, db))[which]
            v = torch.randint(0, 2, t.shape, device="cuda", generator=gen).float() * 2 - 1
            v *= (torch.rand(t.shape, device="cuda", generator=gen) < 0.2)
            s = 2.0 ** -6
            up, down = ([u + e * s * v if j == which else u for j, u in enumerate((x, W, b))] for e in (1.0, -1.0))
            assert abs((f(*up) - f(*down)) / (2 * s) - float((g.double() * v.double()).sum())) < 0.03, (i, which)


@pytest.mark.parametrize("dtype,dw_dtype", [(0, 0), (1, 0), (1, 1)])
@pytest.mark.parametrize("rows,d_in,classes", [(70, 136, 264), (257, 129, 1003), (512, 512, 4096), (600, 200, 20005)])
def test_linear_grad_accumulation(dtype, dw_dtype, rows, d_in, classes):
    with Ctx() as ctx:
        check_linear_grad(ctx, dtype, rows, d_in, classes, bias=True, ignored=0.3, beta=1.0, dw_dtype=dw_dtype, T=0.7)
        check_linear_grad(ctx, dtype, rows, d_in, classes, bias=True, kinds="a", dw_dtype=dw_dtype)
        check_linear_grad(ctx, dtype, rows, d_in, classes, bias=True, kinds="h", ignored=0.4, dw_dtype=dw_dtype)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("names", [("dX",), ("dW",), ("dbias",), ("dW", "dbias")])
def test_linear_grad_some_outputs(dtype, names):
    with Ctx() as ctx:
        check_linear_grad(ctx, dtype, 260, 136, 1030, bias=True, ignored=0.1, outputs=names)
        check_linear_grad(ctx, dtype, 600, 136, 20005, bias=True, ignored=0.1, outputs=names)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", [(150, 300, 10), (300, 256, 4096), (600, 256, 20000)])
def test_linear_no_row_counts(dtype, rows, d_in, classes):
    import torch
    from paper_2007_10412_amd import binding as B
    with Ctx() as ctx:
        for beta in (0.0, 1.0):
            check_linear_grad(ctx, dtype, rows, d_in, classes, bias=True, ignored=1.0, beta=beta, dw_dtype=0)
        x, W, _ = layer_inputs(dtype, rows, d_in, classes, False, gen_for(1))
        out = outputs(rows, 4)
        B.rad_linear_logprobs(ctx, B.make_layer(rows, d_in, classes, dtype=dtype, relu=False), x, W, None,
                              tokens=torch.full((rows,), classes, device="cuda", dtype=torch.int32), **out)
        B.rad_ctx_synchronize(ctx)
        assert (out["logprob"] == 0).all() and (out["entropy"] == 0).all() and (out["top_index"] == -1).all() and (out["top_logprob"] == -math.inf).all()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", [(40, 64, 200), (300, 256, 4096), (600, 256, 20000)])
def test_linear_rows_that_do_not_count_hold_anything(dtype, rows, d_in, classes):
    """NaN in a row's x and gradients where its token says that it does not count; a NaN or an infinity in a counting row's gradients stays in its row
    of dX."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen = gen_for(rows, classes)
    x, W, _ = layer_inputs(dtype, rows, d_in, classes, False, gen)
    tokens = tokens_for(rows, classes, gen)
    a, h = torch.randn(rows, device="cuda", generator=gen), torch.randn(rows, device="cuda", generator=gen)
    layer = B.make_layer(rows, d_in, classes, dtype=dtype, relu=False)
    tokens[3::7] = -1
    with Ctx() as ctx:
        def grads(x, a, h):
            dX, dW = torch.empty_like(x), torch.empty(d_in, classes, device="cuda")
            B.rad_linear_logprobs_grad(ctx, layer, x, W, None, tokens=tokens, d_logprob=a, d_entropy=h, dX=dX, dW=dW)
            B.rad_ctx_synchronize(ctx)
            return dX, dW
        dX, dW = grads(x, a, h)
        x2, a2, h2 = x.clone(), a.clone(), h.clone()
        x2[3::7], a2[3::7], h2[3::7] = math.nan, math.inf, math.nan
        dX2, dW2 = grads(x2, a2, h2)
        assert torch.equal(dX, dX2) and torch.equal(dW, dW2)
        assert (dX[3::7] == 0).all() and torch.isfinite(dX).all()
        for value in (math.nan, math.inf):
            a2 = a.clone()
            a2[5] = value
            dX2, _ = grads(x, a2, h)
            assert torch.isfinite(dX2[:5]).all() and torch.isfinite(dX2[6:]).all() and not torch.isfinite(dX2[5]).any()
            # the other rows are within the bounds of the definition (a difference of two results may have both results' errors:
            # 4 h max|dX|, as it stood here, is less than what two sums over 200 classes may differ by)
            others = torch.arange(rows, device="cuda") != 5
            dz, e, parts = layer_row(torch.where(torch.isnan(x), torch.zeros_like(x), x), W, None, 1.0).grad(tokens, tokens >= 0, a, h)
            Wt = W.double().t().contiguous()
            want, bound = dz @ Wt, (e + 2.02 * HALF[dtype] * parts) @ Wt.abs() + 8 * U * math.sqrt(classes) * (dz.abs() @ Wt.abs())
            close(dX2[others], want[others], (bound + HALF[dtype] * want.abs() + 1e-37)[others], "dX beside a row of %s" % value)


@pytest.mark.parametrize("dtype", [0, 1])
def test_pieces(dtype):
    """More logits than a piece takes: results are those of the rows alone."""
    import torch
    from paper_2007_10412_amd import binding as B
    rows, d_in, classes = (4200, 32, 131000) if dtype else (4200, 32, 131000)
    gen = gen_for(8, dtype)
    x, W, _ = layer_inputs(dtype, rows, d_in, classes, False, gen, grid=True)
    tokens = tokens_for(rows, classes, gen, 0.2)
    with Ctx() as ctx:
        out = outputs(rows, 6)
        B.rad_linear_logprobs(ctx, B.make_layer(rows, d_in, classes, dtype=dtype, relu=False), x, W, None, tokens=tokens, temperature=1.5, **out)
        B.rad_ctx_synchronize(ctx)
        for r0 in (0, 4000, 4100):
            at = slice(r0, r0 + 100)
            row = layer_row(x[at], W, None, 1.5)
            check_answer({n: t[at] for n, t in out.items()}, row, tokens[at], 6, "rows from %d" % r0)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d_in,classes", [(40, 136, 1000), (300, 129, 4099), (3, 520, 20003)])
def test_views_at_odd_addresses(dtype, rows, d_in, classes):
    import torch
    from paper_2007_10412_amd import binding as B
    gen = gen_for(rows, d_in)
    x, W, b = layer_inputs(dtype, rows, d_in, classes, True, gen, grid=True)

    def moved(t, fill=None):
        flat = torch.zeros(t.numel() + 3, device="cuda", dtype=t.dtype)
        v = flat[1:1 + t.numel()].view(t.shape)
        v.copy_(t)
        return v
    tokens = tokens_for(rows, classes, gen, 0.2)
    a, h = torch.randn(rows, device="cuda", generator=gen), torch.randn(rows, device="cuda", generator=gen)
    layer = B.make_layer(rows, d_in, classes, dtype=dtype, relu=False, has_bias=True)
    with Ctx() as ctx:
        results = []
        for f in (lambda t: t, moved):
            out = {n: f(t) for n, t in outputs(rows, 9).items()}
            B.rad_linear_logprobs(ctx, layer, f(x), f(W), f(b), tokens=f(tokens), **out)
            g = {"dX": f(torch.zeros_like(x)), "dW": f(torch.zeros_like(W)), "dbias": f(torch.zeros_like(b))}
            B.rad_linear_logprobs_grad(ctx, layer, f(x), f(W), f(b), tokens=f(tokens), d_logprob=f(a), d_entropy=f(h), **g)
            B.rad_ctx_synchronize(ctx)
            results.append({**out, **g})
        for n in results[0]:
            assert torch.equal(results[0][n], results[1][n]), n


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", [0, 1])
def test_lists_are_a_teachers(dtype):
    """The lists of rad_linear_logprobs as a teacher: the loss of rad_linear_distill against the same lists formed in fp64; rows that do not count
    have empty lists and learn nothing."""
    import torch
    from paper_2007_10412_amd import binding as B
    rows, d_in, classes, k = 120, 128, 3001, 32
    gen = gen_for(6, dtype)
    x, W, _ = layer_inputs(dtype, rows, d_in, classes, False, gen, grid=True)
    _, student, _ = layer_inputs(dtype, rows, d_in, classes, False, gen, grid=True)
    tokens = tokens_for(rows, classes, gen, 0.3)
    layer = B.make_layer(rows, d_in, classes, dtype=dtype, relu=False)
    with Ctx() as ctx:
        out = outputs(rows, k, ("top",))
        B.rad_linear_logprobs(ctx, layer, x, W, None, tokens=tokens, **out)
        loss = torch.zeros(rows, device="cuda")
        dX = torch.full_like(x, math.nan)
        B.rad_linear_distill(ctx, layer, x, student, None, B.make_teacher(out["top_index"], out["top_logprob"], 1.0), row_loss=loss, dX=dX)
        B.rad_ctx_synchronize(ctx)
        counts = (tokens >= 0) & (tokens < classes)
        z = x.double() @ W.double()
        best = likeliest(z, k)
        log_p = torch.log_softmax(z.gather(1, best), dim=1)
        log_q = torch.log_softmax(x.double() @ student.double(), dim=1).gather(1, best)
        want = torch.where(counts, (torch.exp(log_p) * (log_p - log_q)).sum(dim=1), torch.zeros(rows, device="cuda", dtype=torch.float64))
        assert ((loss.double() - want).abs() <= 2e-4).all()            # (fp32: logits of size 10 in sums of 3001: 1e-5; ten times that)
        assert (dX[~counts] == 0).all() and torch.isfinite(dX).all()


@pytest.mark.parametrize("dtype", [0, 1])
def test_scored_clipped_step(dtype):
    """A last layer's step by an objective of its own answers: log probabilities, the objective's gradient from them, the layer's, their norm, the clipped
    step; against the same in fp64."""
    import torch
    from paper_2007_10412_amd import binding as B
    rows, d_in, classes = 200, 96, 2000
    gen = gen_for(15, dtype)
    x, W, _ = layer_inputs(dtype, rows, d_in, classes, False, gen)
    tokens = tokens_for(rows, classes, gen, 0.25)
    old = torch.randn(rows, device="cuda", generator=gen) * 0.3 - 12.0
    advantage = torch.randn(rows, device="cuda", generator=gen)
    layer = B.make_layer(rows, d_in, classes, dtype=dtype, relu=False)
    counts = (tokens >= 0) & (tokens < classes)
    with Ctx() as ctx:
        out = outputs(rows, 0, ("logprob", "entropy"))
        B.rad_linear_logprobs(ctx, layer, x, W, None, tokens=tokens, **out)
        a = -advantage * torch.exp((out["logprob"] - old).clamp(max=3.0)) / rows
        h = torch.full((rows,), -0.01 / rows, device="cuda")
        dW = torch.empty(d_in, classes, device="cuda")
        B.rad_linear_logprobs_grad(ctx, layer, x, W, None, tokens=tokens, d_logprob=a, d_entropy=h, dW=dW)
        norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        master = W.float().clone()                         # (W stays for the definition)
        before = master.double()
        B.rad_gradient_norm(ctx, [dW], 1e-3, norm=norm, scale=scale)
        opt = B.make_optimizer(B.RAD_SGD, 0.5)
        if dtype:
            B.rad_optimizer_step_scaled(ctx, opt, 1, dtype, [W.clone()], [dW], scale, master=[master])
        else:
            B.rad_optimizer_step_scaled(ctx, opt, 1, dtype, [master], [dW], scale)
        B.rad_ctx_synchronize(ctx)
        row = layer_row(x, W, None, 1.0)
        check_answer(out, row, tokens, 0, "scored")
        dz, _, _ = row.grad(tokens, counts, a, h)
        g = x.double().t() @ dz
        f = min(1.0, 1e-3 / float(g.norm()))
        off = float(((before - master.double()) - 0.5 * f * g).norm()) / (0.5 * f * float(g.norm()))
        # (a move is a difference of fp32 weights of size 0.3: half a step of them over its own size, beside dz's rounding to the type)
        step = float((before.abs() * U).norm()) / (0.5 * f * float(g.norm()))
        assert f < 1 and off <= 2.02 * HALF[dtype] + 1e-5 + step, (off, step)


def test_two_calls_agree_bit_by_bit():
    import torch
    from paper_2007_10412_amd import binding as B
    with Ctx() as ctx:
        for dtype in (0, 1):
            gen = gen_for(44, dtype)
            z = torch.randint(0, 50, (70, 60001), device="cuda", generator=gen).to(torch_dtype(dtype))
            x, W, b = layer_inputs(dtype, 200, 300, 9000, True, gen)
            layer = B.make_layer(200, 300, 9000, dtype=dtype, relu=False, has_bias=True)
            t1, t2 = tokens_for(70, 60001, gen), tokens_for(200, 9000, gen, 0.2)
            a, h = torch.randn(200, device="cuda", generator=gen), torch.randn(200, device="cuda", generator=gen)
            first = None
            for _ in range(3):
                one, two = call_dense(ctx, dtype, z, 29, 1.0, t1), outputs(200, 31)
                B.rad_linear_logprobs(ctx, layer, x, W, b, tokens=t2, **two)
                g = {"dX": torch.empty_like(x), "dW": torch.empty_like(W), "dbias": torch.empty_like(b)}
                B.rad_linear_logprobs_grad(ctx, layer, x, W, b, tokens=t2, d_logprob=a, d_entropy=h, **g)
                B.rad_ctx_synchronize(ctx)
                all_of = list(one.values()) + list(two.values()) + list(g.values())
                first = first or all_of
                assert all(torch.equal(p, q) for p, q in zip(first, all_of))


@pytest.mark.parametrize("dtype", [0, 1])
def test_captured(dtype):
    """All four in one graph, on a stream of its own, replayed with other inputs and eager calls of another context between the replays; and a second graph
    of the context."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen = gen_for(21, dtype)
    stream = torch.cuda.Stream()
    rows, d_in, classes = 130, 200, 9001
    x, W, b = layer_inputs(dtype, rows, d_in, classes, True, gen)
    z = (3 * torch.randn(3, 140000, device="cuda", generator=gen)).to(torch_dtype(dtype))
    tz, tokens = tokens_for(3, 140000, gen), tokens_for(rows, classes, gen, 0.2)
    a, h = torch.randn(rows, device="cuda", generator=gen), torch.randn(rows, device="cuda", generator=gen)
    layer = B.make_layer(rows, d_in, classes, dtype=dtype, relu=False, has_bias=True)

    def fresh():
        return {"dense": outputs(3, 30), "linear": outputs(rows, 12), "dz": {"dlogits": torch.zeros_like(z)},
                "grads": {"dX": torch.zeros_like(x), "dW": torch.zeros_like(W), "dbias": torch.zeros_like(b)}}

    def calls(c, o):
        B.rad_token_logprobs(c, z, dtype, tokens=tz, **o["dense"])
        B.rad_linear_logprobs(c, layer, x, W, b, tokens=tokens, **o["linear"])
        B.rad_token_logprobs_grad(c, z, dtype, tokens=tz, d_logprob=a[:3], d_entropy=h[:3], **o["dz"])
        B.rad_linear_logprobs_grad(c, layer, x, W, b, tokens=tokens, d_logprob=a, d_entropy=h, **o["grads"])
    with Ctx(stream) as ctx, Ctx() as plain:
        got, second, want = fresh(), fresh(), fresh()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            calls(ctx, got)
            stream.synchronize()
            graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                calls(ctx, got)
            with torch.cuda.graph(other, stream=stream):
                calls(ctx, second)
        for r in range(4):
            x.copy_(torch.randn(x.shape, device="cuda", generator=gen))
            z.copy_(3 * torch.randn(z.shape, device="cuda", generator=gen))
            tokens.copy_(tokens_for(rows, classes, gen, 0.4))
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                graph.replay()
                other.replay()
            calls(plain, want)
            torch.cuda.synchronize()
            for name in want:
                for n in want[name]:
                    assert torch.equal(got[name][n], want[name][n]) and torch.equal(second[name][n], want[name][n]), (r, name, n)
        del graph, other


def test_first_call_is_not_recorded():
    """Rows in parts count their workgroups in memory that a context clears once: not within a graph."""
    import torch
    from paper_2007_10412_amd import binding as B
    gen = gen_for(22)
    stream = torch.cuda.Stream()
    z = torch.randn(2, 140000, device="cuda", generator=gen)
    out, want = outputs(2, 5, ("entropy", "top")), None
    torch.cuda.synchronize()
    with Ctx(stream) as ctx:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            torch.zeros(1, device="cuda").add_(1)
            with pytest.raises(B.RadError, match="recorded"):
                B.rad_token_logprobs(ctx, z, 0, **out)
        B.rad_token_logprobs(ctx, z, 0, **out)
        B.rad_ctx_synchronize(ctx)
        check_answer(out, Row(z.double(), 1.0), None, 5, "after a refusal")
        with torch.cuda.graph(graph.__class__(), stream=stream):
            B.rad_token_logprobs(ctx, z, 0, **out)


def test_two_contexts_at_once():
    """Calls of two contexts, on two streams, with nothing between them."""
    import torch
    from paper_2007_10412_amd import binding as B
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    with Ctx(s1) as c1, Ctx(s2) as c2, Ctx() as plain:
        work = []
        for i, c in enumerate((c1, c2)):
            gen = gen_for(31 + i)
            x, W, _ = layer_inputs(1, 300, 256, 8000, False, gen, grid=True)
            z = (3 * torch.randn(2, 140000, device="cuda", generator=gen)).to(torch.bfloat16)
            work.append((c, x, W, z, outputs(300, 9, ("entropy", "top")), outputs(2, 30, ("entropy", "top"))))
        layer = B.make_layer(300, 256, 8000, dtype=1, relu=False)
        torch.cuda.synchronize()
        for _ in range(20):
            for c, x, W, z, one, two in work:
                B.rad_linear_logprobs(c, layer, x, W, None, **one)
                B.rad_token_logprobs(c, z, 1, **two)
        torch.cuda.synchronize()
        for _, x, W, z, one, two in work:
            w1, w2 = outputs(300, 9, ("entropy", "top")), outputs(2, 30, ("entropy", "top"))
            B.rad_linear_logprobs(plain, layer, x, W, None, **w1)
            B.rad_token_logprobs(plain, z, 1, **w2)
            torch.cuda.synchronize()
            assert all(torch.equal(one[n], w1[n]) for n in w1) and all(torch.equal(two[n], w2[n]) for n in w2)


def test_refusals():
    import torch
    from paper_2007_10412_amd import binding as B
    z = torch.randn(4, 64, device="cuda")
    t = torch.zeros(4, device="cuda", dtype=torch.int32)
    lp, h = torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda")
    x, W = torch.randn(4, 32, device="cuda"), torch.randn(32, 64, device="cuda")
    layer = B.make_layer(4, 32, 64, relu=False)
    big = lambda k: dict(top_index=torch.zeros(4, k, device="cuda", dtype=torch.int32), top_logprob=torch.zeros(4, k, device="cuda"))  # noqa: E731
    with Ctx() as ctx:
        bad = [(lambda: B.rad_token_logprobs(ctx, z, 0), B.RAD_ERR_NULL), (lambda: B.rad_token_logprobs(ctx, z, 0, logprob=lp), B.RAD_ERR_NULL),
               (lambda: B.rad_token_logprobs(ctx, z, 0, **big(257)), B.RAD_ERR_SHAPE), (lambda: B.rad_token_logprobs(ctx, z, 5, entropy=h), B.RAD_ERR_PARAM),
               (lambda: B.rad_token_logprobs(ctx, z, 0, tokens=t, logprob=lp, entropy=lp), B.RAD_ERR_PARAM),
               (lambda: B.rad_token_logprobs(ctx, z, 0, entropy=z.view(-1)[:4]), B.RAD_ERR_PARAM),
               (lambda: B.rad_token_logprobs_grad(ctx, z, 0, torch.zeros_like(z), tokens=t), B.RAD_ERR_NULL),
               (lambda: B.rad_token_logprobs_grad(ctx, z, 0, torch.zeros_like(z), d_logprob=lp), B.RAD_ERR_NULL),
               (lambda: B.rad_token_logprobs_grad(ctx, z.view(-1)[64:].view(3, 64), 0, z.view(-1)[:192].view(3, 64), d_entropy=h[:3]), B.RAD_ERR_PARAM),
               (lambda: B.rad_token_logprobs_grad(ctx, z, 0, z, d_entropy=z.view(-1)[:4]), B.RAD_ERR_PARAM),
               (lambda: B.rad_linear_logprobs(ctx, layer, x, W, None), B.RAD_ERR_NULL),
               (lambda: B.rad_linear_logprobs(ctx, B.make_layer(4, 32, 64), x, W, None, entropy=h), B.RAD_ERR_PARAM),
               (lambda: B.rad_linear_logprobs(ctx, B.make_layer(4, 32, 64, relu=False, has_bias=True), x, W, None, entropy=h), B.RAD_ERR_NULL),
               (lambda: B.rad_linear_logprobs(ctx, layer, None, W, None, entropy=h), B.RAD_ERR_NULL),
               (lambda: B.rad_linear_logprobs(ctx, layer, x, W, None, entropy=x.view(-1)[:4]), B.RAD_ERR_PARAM),
               (lambda: B.rad_linear_logprobs_grad(ctx, layer, x, W, None, tokens=t, d_logprob=lp), B.RAD_ERR_NULL),
               (lambda: B.rad_linear_logprobs_grad(ctx, layer, x, W, None, tokens=t, d_logprob=lp, dX=x), B.RAD_ERR_PARAM),
               (lambda: B.rad_linear_logprobs_grad(ctx, layer, x, W, None, tokens=t, d_logprob=lp, dX=torch.zeros_like(x), beta=0.5), B.RAD_ERR_PARAM)]
        for T in (0.0, -1.0, math.nan, math.inf, 1e7):
            bad += [(lambda T=T: B.rad_token_logprobs(ctx, z, 0, temperature=T, entropy=h), B.RAD_ERR_PARAM),
                    (lambda T=T: B.rad_token_logprobs_grad(ctx, z, 0, torch.zeros_like(z), temperature=T, d_entropy=h), B.RAD_ERR_PARAM),
                    (lambda T=T: B.rad_linear_logprobs(ctx, layer, x, W, None, temperature=T, entropy=h), B.RAD_ERR_PARAM),
                    (lambda T=T: B.rad_linear_logprobs_grad(ctx, layer, x, W, None, temperature=T, d_entropy=h, dX=torch.zeros_like(x)), B.RAD_ERR_PARAM)]
        for i, (call, status) in enumerate(bad):
            with pytest.raises(B.RadError) as e:
                call()
            assert e.value.status == status, (i, e.value)
        B.rad_ctx_synchronize(ctx)
        assert (lp == 0).all() and (h == 0).all()

"""rad_token_logprobs of rows whose largest logit lies just below the lowest base that a row's sums are taken from (-2^24 T ln 2, where a
logit's exponent in powers of two reaches 2^24): log probabilities, entropies and lists, of which those of one class take no search,
against the definition in fp64."""
import math

import numpy as np
import pytest

from tests.test_gpu_logprobs import Ctx, Row, call_dense, check_answer, gen_for, torch_dtype

pytestmark = pytest.mark.gpu


def lowest_base(T):
    """-2^24 / (log2(e) / T), each operation rounded to fp32"""
    return -np.float32(2.0 ** 24) / (np.float32(1.44269504088896340736) / np.float32(T))


def step_below(z, dtype):
    """the next value of the type below z < 0"""
    bits = np.float32(z).view(np.uint32)
    if dtype == 0:
        return (bits + np.uint32(1)).view(np.float32)
    return ((bits & np.uint32(0xFFFF0000)) + np.uint32(0x10000)).view(np.float32)


def bf16_temperature(z):
    """T whose lowest base is the first above z by a tenth to three times T"""
    T = np.float32(-z / (2.0 ** 24 * math.log(2.0)))
    for _ in range(64):
        if 0.1 < (float(lowest_base(T)) - z) / float(T) < 3.0:
            return float(T)
        T = np.nextafter(T, np.float32(0))
    raise AssertionError("no such temperature")


def rows_below(dtype, rows, classes, T, gen):
    """logits of one to five steps below the lowest base (bf16, whose steps are far longer: of one), the rest of them far below"""
    import torch
    levels = [lowest_base(T)]
    if dtype:
        levels = [None, np.float32(-2.0 ** 23)]
    else:
        for _ in range(5):
            levels.append(step_below(levels[-1], dtype))
    values = torch.tensor([float(v) for v in levels[1:]], device="cuda")
    z = values[torch.randint(0, len(values), (rows, classes), device="cuda", generator=gen)]
    gone = torch.rand(rows, classes, device="cuda", generator=gen) < 0.3
    return torch.where(gone, torch.full_like(z, float(levels[-1]) * 4), z).to(torch_dtype(dtype))


@pytest.mark.parametrize("dtype,T", [(0, 1.0), (0, 0.01), (0, 1e-6), (0, 30.0), (1, None)])
@pytest.mark.parametrize("k", [1, 2, 30])
@pytest.mark.parametrize("rows,classes", [(3, 40), (9, 700), (4, 5001), (1100, 2050), (4, 33000), (90, 70000), (1, 140000), (2, 300000)])
def test_rows_just_below_the_lowest_base(dtype, T, k, rows, classes):
    if dtype:
        T = bf16_temperature(-2.0 ** 23)
    gen = gen_for(rows, classes, k)
    z = rows_below(dtype, rows, classes, T, gen)
    assert float(z.float().max()) < float(lowest_base(T)) and float(z.float().max()) > float(lowest_base(T)) - 3.1 * T
    tokens = z.float().argmax(dim=1).int()
    T32 = float(np.float32(T))
    print("floor", dtype, T, k, rows, classes, flush=True)
    with Ctx() as ctx:
        check_answer(call_dense(ctx, dtype, z, k, T, tokens), Row(z.double(), T32), tokens, k, "T %g k %d %d x %d" % (T, k, rows, classes))


@pytest.mark.parametrize("k", [1, 2])
def test_rows_of_equal_logits_below_the_lowest_base(k):
    """The first class of a row of equal logits, as far from the base as a row may be whose sum from there is more than a half."""
    import torch
    with Ctx() as ctx:
        for classes in (1000, 100000):
            for steps in range(0, 12):
                value = lowest_base(1.0)
                for _ in range(steps):
                    value = step_below(value, 0)
                z = torch.full((2, classes), float(value), device="cuda")
                check_answer(call_dense(ctx, 0, z, k), Row(z.double(), 1.0), None, k, "%d steps below, %d classes" % (steps, classes))

"""The caller-owned paged cache in 4 bits on the GPU where its number formats end."""
import random

import pytest
import torch

from test_gpu_paged4 import check, ints, run
from util_paged import queries
from util_paged4 import Cache4, attention, values

pytestmark = pytest.mark.gpu
KINDS = [(torch.bfloat16, 1), (torch.float32, 1), (torch.bfloat16, 40), (torch.float32, 40)]      # (bf16, 40): the chunk kernel


def judge(c, q, cu, lens, scale, window=0):
    out, st = run(c, q, cu, max(b - a for a, b in zip(cu, cu[1:])), scale=scale, window=window)
    assert st == 0
    want, bound = attention(c.k, c.v, q, cu, lens, c.table, scale, window)
    got = out.double().cpu()
    assert torch.isfinite(got).all() and ((got - want).abs() <= bound).all(), ((got - want).abs() / bound).max().item()


@pytest.mark.parametrize("dtype,new", KINDS)
@pytest.mark.parametrize("window", [0, 50])
def test_a_scale_too_small_for_the_shift(dtype, new, window):
    """scale 2^shift is below fp32's smallest number: every visible entry weighs the same, masked ones nothing."""
    H, g, d = 2, 4, 64
    lens = [100, 333]
    c = Cache4(lens, H, d, seed=30)
    c.arrays[2] = ints([-64, -64])
    c.k = values(*c.arrays[:3])
    q, cu = queries([new, new], H * g, d, dtype, seed=30)
    judge(c, q, cu, lens, 1e-30, window)


@pytest.mark.parametrize("dtype,new", KINDS)
def test_a_scale_too_large_for_the_shift(dtype, new):
    """scale 2^shift times the queries' own power of two is above fp32's largest number, and every key is zero."""
    H, g, d = 2, 4, 64
    lens = [100, 333]
    c = Cache4(lens, H, d, seed=31)
    c.arrays[0].zero_()
    c.arrays[2] = ints([64, 64])
    c.k = torch.zeros_like(c.k)
    q, cu = queries([new, new], H * g, d, dtype, seed=31)
    judge(c, q * 2.0 ** 67, cu, lens, 100.0)


# ---------------------------------------------------------------- many requests

@pytest.mark.parametrize("requests", [33, 480, 481, 1100])
def test_chunks_of_more_requests_than_the_table_has_groups(requests):
    """The chunk kernel has more warps than the table of requests has sums: chunks, single tokens and idle requests from one to three a group."""
    rng = random.Random(requests)
    lens = [rng.choice([1, 40, 64, 70, 129]) for _ in range(requests)]
    new = [min(n, rng.choice([0, 1, 1, 33, 64])) for n in lens]
    lens[-1], new[-1] = 200, 100
    check(lens, new, 1, 2, 64, torch.bfloat16, seed=36)

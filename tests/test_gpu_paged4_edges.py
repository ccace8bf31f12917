"""The caller-owned paged cache in 4 bits on the GPU where its number formats end."""
import math
import random

import pytest
import torch

from paper_2605_09649_b200 import binding
from test_gpu_paged4 import DEV, check, empty_cache, hard_values, ints, run
from util_paged import PAGE, queries
from util_paged4 import Cache4, attention, quantise, values

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


# ---------------------------------------------------------------- small weights

def far_below(c, log2_weight):
    """Keys and values of a cache of one head: the first entry outweighs every other by 2^-log2_weight and has the value 0, the others' is 1."""
    kc, ks, _, vc, vs, _ = c.arrays
    kc.zero_(), vc.fill_(0x22), ks.fill_(56), vs.fill_(56)    # code 2: 1; byte 56: 1
    first = int(c.table[0, 0])
    kc[first, 0, 0, 0], vc[first, 0, 0] = 7, 0                # channel 0: 6
    c.k, c.v = values(*c.arrays[:3]), values(*c.arrays[3:])
    return log2_weight * math.log(2.0) / 6


@pytest.mark.parametrize("dtype,new,bits,tail", [(torch.bfloat16, 1, 30.41, 32), (torch.float32, 1, 30.41, 32), (torch.bfloat16, 40, 27.41, 29), (torch.bfloat16, 40, 20.0, 29),
                                                 (torch.bfloat16, 40, 24.3, 29), (torch.bfloat16, 40, 28.6, 29), (torch.bfloat16, 1, 24.3, 32)])
def test_weights_that_fp16_rounds_coarsely(dtype, new, bits, tail):
    """Many entries whose weights are 2^-20 to 2^-31 of the largest, halfway between two fp16 numbers among them.  Each is off by 2^-tail of the
    largest at most: weights are 2^7 times their value, in the chunk kernel 2^4, and fp16's last step is 2^-24, half of it an error."""
    H, g, d, n = 1, 4, 64, 256 if new > 1 else 1000           # (so few that no second worker shares the request, with a reference of its own)
    c = Cache4([n], H, d, seed=32, shift=0)
    scale = far_below(c, bits)
    q = torch.zeros(new, H * g, d, dtype=dtype, device=DEV)
    q[:, :, 0] = 1.0
    cu = [0, new]
    out, st = run(c, q, cu, new, scale=scale)
    assert st == 0
    want, bound = attention(c.k, c.v, q, cu, [n], c.table, scale)
    bound = bound + n * (2.0 ** -tail - 2.0 ** -32)           # (every value is 1; `attention` counts 2^-32 for each entry)
    assert (want > 0).all() and ((out.double().cpu() - want).abs() <= bound).all(), ((out.double().cpu() - want).abs() / bound).max().item()


# ---------------------------------------------------------------- codes to the bit

@pytest.mark.parametrize("H,d,dtype", [(8, 128, torch.bfloat16), (2, 64, torch.float32), (3, 32, torch.bfloat16), (1, 256, torch.float32)])
@pytest.mark.parametrize("shift", [0, -3, 40])
def test_append_gives_the_defined_bytes(H, d, dtype, shift):
    """Bytes, not values: a code has the sign of its channel also where it is 0, whether the channel is small, a negative zero, or its block's
    scale is 0.  (Blocks with a NaN have a NaN scale; their codes say nothing.)"""
    T, n_pages = 100, 2
    arrays, cache = empty_cache(n_pages, H, d, [shift] * H)
    x = hard_values(T, H, d, dtype, seed=5)
    x[3, :, ::5] *= -0.0
    x[4] = -2.0 ** -100
    x[5] = -0.0
    binding.paged4_append(cache, x.to(DEV), x.to(DEV), ints(range(T)))
    codes, scale = quantise(x, torch.tensor([shift] * H))
    want = (codes & 7) + 8 * torch.signbit(x).long()
    real = (scale != 127).repeat_interleave(16, -1)
    for kv in range(2):
        got, got_s = (a.cpu().transpose(1, 2).reshape(n_pages * PAGE, H, -1)[:T].long() for a in arrays[2 * kv:2 * kv + 2])
        got = torch.stack((got & 15, got >> 4), -1).flatten(-2)
        assert torch.equal(got_s, scale)
        assert torch.equal(got[real], want[real])
    assert ((scale == 0).repeat_interleave(16, -1) & (want == 8)).any() and ((scale > 0).repeat_interleave(16, -1) & (want == 8)).any()


# ---------------------------------------------------------------- head sizes of fp32 queries

@pytest.mark.parametrize("H,g,d", [(2, 4, 32), (1, 3, 96), (2, 2, 128), (1, 2, 160), (1, 4, 256)])
def test_fp32_head_sizes(H, g, d):
    check([1, 31, 64, 65, 200, 1500], [1] * 6, H, g, d, torch.float32, seed=33)
    check([5, 40, 0, 64, 700, 130], [5, 3, 0, 0, 6, 1], H, g, d, torch.float32, seed=34)
    check([130, 300, 90], [130, 77, 1], H, g, d, torch.float32, window=40, seed=35)


# ---------------------------------------------------------------- many requests

@pytest.mark.parametrize("requests", [33, 480, 481, 1100])
def test_chunks_of_more_requests_than_the_table_has_groups(requests):
    """The chunk kernel has more warps than the table of requests has sums: chunks, single tokens and idle requests from one to three a group."""
    rng = random.Random(requests)
    lens = [rng.choice([1, 40, 64, 70, 129]) for _ in range(requests)]
    new = [min(n, rng.choice([0, 1, 1, 33, 64])) for n in lens]
    lens[-1], new[-1] = 200, 100
    check(lens, new, 1, 2, 64, torch.bfloat16, seed=36)

"""The caller-owned paged cache in 4 bits on the GPU: append, read and attention, each against a plain 64-bit statement
(tests/util_paged4.py)."""
import math
import random

import pytest
import torch

from paper_2605_09649_b200 import binding
from util_paged import PAGE, pages, queries
from util_paged4 import E4M3, LEVELS, Cache4, attention, pack, quantise, values

pytestmark = pytest.mark.gpu
DEV = "cuda"
I32 = torch.int32


def ints(x):
    return torch.tensor(x, dtype=I32, device=DEV)


def status_word():
    return torch.zeros(1, dtype=I32, device=DEV)


def empty_cache(n_pages, H, d, shift=None):
    """Arrays full of a pattern that no append writes by chance, and the cache over them."""
    arrays = []
    for x in range(2):
        arrays += [torch.full((n_pages, H, PAGE, d // 2), 0xA5, dtype=torch.uint8, device=DEV), torch.full((n_pages, H, PAGE, d // 16), 0x7B, dtype=torch.uint8, device=DEV)]
    sh = None if shift is None else ints(shift)
    return arrays, binding.Paged4Cache(*arrays, sh, sh)


def hard_values(T, H, d, dtype, seed):
    """Normal values, and rows of what can go wrong: halfway points of every scale, zeros, tiny and huge values, infinities, NaN."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(T, H, d, generator=gen).double() * torch.exp2(torch.randn(T, H, 1, generator=gen) * 2)
    blocks = x.view(-1, 16)
    mids = (LEVELS[1:] + LEVELS[:-1]) / 2
    for i in range(min(120, blocks.shape[0])):
        s = E4M3[1 + i]                                       # a block whose scale is s exactly, its values on halfway points
        blocks[i, 0] = 6 * s
        blocks[i, 1:8] = mids * s
        blocks[i, 8:15] = -mids * s
        blocks[i, 15] = 0
    special = [0.0, 2.0 ** -30, 2.0 ** -12, 3000.0, 1e30, -1e38, math.inf, -math.inf, math.nan]
    for i, v in enumerate(special):
        if 130 + i < blocks.shape[0]:
            blocks[130 + i] = torch.randn(16, generator=gen).double() if i > 2 else 0.0
            blocks[130 + i, (5 * i) % 16] = v
    # of the fp32 neighbours of halfway points: one above, one below
    for i in range(min(60, max(0, blocks.shape[0] - 150))):
        s = E4M3[30 + i]
        blocks[150 + i, 0] = 6 * s
        m = (mids * s).float()
        blocks[150 + i, 1:8] = torch.nextafter(m, torch.tensor(math.inf)).double()
        blocks[150 + i, 8:15] = -torch.nextafter(m, torch.tensor(0.0)).double()
    return x.to(dtype)


@pytest.mark.parametrize("H,d,dtype", [(8, 128, torch.bfloat16), (2, 64, torch.float32), (3, 32, torch.bfloat16), (1, 256, torch.float32), (5, 96, torch.bfloat16), (4, 224, torch.float32)])
@pytest.mark.parametrize("strided,shifted", [(False, False), (True, True)])
def test_append_equals_the_definition(H, d, dtype, strided, shifted):
    T, n_pages = 137, 4
    shift = [(-3, 5, 0, 2, -7, 1, 4, -1)[h] for h in range(H)] if shifted else [0] * H
    arrays, cache = empty_cache(n_pages, H, d, shift if shifted else None)
    x = [hard_values(T, H, d, dtype, seed) for seed in (1, 2)]
    rng = random.Random(H)
    slots = rng.sample(range(n_pages * PAGE), T)
    for i in (0, 60, T - 1):
        slots[i] = -1
    if strided:
        wide = torch.zeros(T, 2, H + 1, d, dtype=dtype)
        wide[:, 0, :H], wide[:, 1, :H] = x
        wide = wide.to(DEV)
        k, v = wide[:, 0, :H], wide[:, 1, :H]
    else:
        k, v = (t.to(DEV) for t in x)
    st = status_word()
    binding.paged4_append(cache, k, v, ints(slots), status=st)
    back = binding.paged4_read(cache, ints(slots), dtype=torch.float32, status=st)
    assert st.item() == 0
    used = torch.zeros(n_pages * PAGE, dtype=torch.bool)
    for kv in range(2):
        codes, scale = quantise(x[kv], torch.tensor(shift))
        got_c, got_s = (a.cpu().transpose(1, 2).reshape(n_pages * PAGE, H, -1) for a in arrays[2 * kv:2 * kv + 2])
        want = values(pack(codes)[:, :, None], scale.to(torch.uint8)[:, :, None], torch.tensor(shift))[:, :, 0]
        for t, s in enumerate(slots):
            if s < 0:
                assert (back[kv][t] == 0).all()
                continue
            used[s] = True
            assert torch.equal(got_s[s].long(), scale[t]), (kv, t)
            have = values(got_c[s][:, None], got_s[s][:, None], torch.tensor(shift))[:, 0]
            assert torch.equal(torch.nan_to_num(have, nan=7e9), torch.nan_to_num(want[t], nan=7e9)), (kv, t)
            assert torch.equal(torch.nan_to_num(back[kv][t].double().cpu(), nan=7e9), torch.nan_to_num(want[t], nan=7e9))
        assert (got_c[~used] == 0xA5).all() and (got_s[~used] == 0x7B).all()


def test_read_gives_every_code_and_scale():
    """All 256 bytes of codes under all 256 bytes of scales, in both types; slots given twice and slots that do not exist."""
    n_pages, d = 16, 32
    codes = (torch.arange(n_pages * PAGE * 16) % 256).to(torch.uint8).view(n_pages, 1, PAGE, 16)
    scale = torch.arange(n_pages * PAGE).repeat_interleave(2).view(n_pages, 1, PAGE, 2).div(4, rounding_mode="floor").to(torch.uint8)
    shift = torch.tensor([3])
    cache = binding.Paged4Cache(codes.to(DEV), scale.to(DEV), codes.to(DEV), scale.to(DEV).view(torch.float8_e4m3fn), ints([3]), None)
    slots = list(range(n_pages * PAGE)) + [5, 5, -1, n_pages * PAGE, -2]
    for dtype in (torch.float32, torch.bfloat16):
        st = status_word()
        k, v = binding.paged4_read(cache, ints(slots), dtype=dtype, status=st)
        assert st.item() == binding.E_ARG
        for got, sh in ((k, shift), (v, shift * 0)):
            want = values(codes, scale, sh)[:, 0].reshape(-1, d)
            want = torch.cat((want, want[5:6], want[5:6], torch.zeros(3, d, dtype=torch.float64)))
            assert torch.equal(torch.nan_to_num(got[:, 0].double().cpu(), nan=7e9), torch.nan_to_num(want, nan=7e9))


def test_append_slots_out_of_range_are_skipped():
    arrays, cache = empty_cache(2, 2, 64)
    x = torch.ones(3, 2, 64, device=DEV)
    st = status_word()
    binding.paged4_append(cache, x, x, ints([128, -5, 7]), status=st)
    assert st.item() == binding.E_ARG
    for a in arrays[::2]:
        a = a.transpose(1, 2).reshape(128, -1)
        assert (a[7] != 0xA5).all() and (a[:7] == 0xA5).all() and (a[8:] == 0xA5).all()


# ---------------------------------------------------------------- attention

def run(c, q, cu, new_max, **kw):
    st = status_word()
    out = torch.full(q.shape, 777.0, dtype=q.dtype, device=DEV)
    binding.paged4_attention(c.cache(), q, ints(cu), c.lens, c.table, new_max, out=out, status=st, **kw)
    return out, st.item()


def check(lens, new, H, g, d, dtype, window=0, seed=0, shift=3, pad=2, stride=0, spread=1.0, scale=None, max_new=None, qscale=1.0):
    c = Cache4(lens, H, d, seed=seed, shift=shift, spread=spread)
    q, cu = queries(new, H * g, d, dtype, seed=seed, pad=pad, stride=stride)
    q = q * qscale
    if stride:
        wide = torch.full((q.shape[0], stride), math.nan, dtype=dtype, device=DEV)
        wide[:, :H * g * d] = q.flatten(1)
        q = wide[:, :H * g * d].unflatten(1, (H * g, d))
    # (shifts make logits of either size: the scale brings them back to ordinary ones for the larger keys)
    scale = d ** -0.5 if scale is None else scale
    out, st = run(c, q, cu, max(new) if max_new is None else max_new, window=window, scale=scale)
    assert st == 0
    want, bound = attention(c.k, c.v, q[:cu[-1]], cu, lens, c.table, scale, window)
    got = out[:cu[-1]].double().cpu()
    assert torch.isfinite(got).all()
    worst = ((got - want).abs() / bound[...]).max().item() if got.numel() else 0.0
    assert worst <= 1.0, worst
    assert (out[cu[-1]:] == 777).all()


SHAPES = [(2, 4, 128, torch.bfloat16), (1, 8, 64, torch.bfloat16), (2, 3, 96, torch.bfloat16), (1, 2, 256, torch.bfloat16), (2, 1, 32, torch.bfloat16), (1, 7, 160, torch.bfloat16),
          (2, 2, 64, torch.float32), (1, 4, 128, torch.float32), (1, 3, 224, torch.float32)]


@pytest.mark.parametrize("H,g,d,dtype", SHAPES)
def test_single_tokens(H, g, d, dtype):
    check([1, 31, 32, 33, 63, 64, 65, 200, 1500], [1] * 9, H, g, d, dtype)


@pytest.mark.parametrize("H,g,d,dtype", SHAPES)
def test_drafts_and_idle_requests(H, g, d, dtype):
    check([5, 40, 0, 64, 700, 130], [5, 3, 0, 0, 6, 1], H, g, d, dtype, seed=1)


@pytest.mark.parametrize("H,g,d,dtype", SHAPES)
@pytest.mark.parametrize("window", [0, 1, 40, 300])
def test_chunks_and_windows(H, g, d, dtype, window):
    check([130, 300, 90], [130, 77, 1], H, g, d, dtype, window=window, seed=2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_one_long_request_is_shared_by_many_workers(dtype):
    check([20000], [1], 2, 4, 128, dtype, seed=3)
    check([9000, 64], [3, 1], 1, 16, 64, dtype, seed=4)


@pytest.mark.parametrize("g", [1, 5, 9, 16, 17, 40, 128])
def test_query_heads_per_kv_head(g):
    check([70, 513], [1, 2], 2, g, 64, torch.bfloat16, seed=5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strided_queries_and_wrong_max_new(dtype):
    check([100, 260], [3, 20], 2, 2, 64, dtype, stride=2 * 2 * 64 + 16, seed=6, max_new=1)
    check([100, 260], [3, 20], 2, 2, 64, dtype, seed=6, max_new=0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", [1, 70])
def test_peaked_and_tiny_queries(dtype, new):
    """Logits of hundreds, where the running maximum leaps; queries whose values differ by 2^40 in size from those of other cases."""
    check([900, 500], [new, 1], 1, 4, 128, dtype, seed=7, spread=4.0, scale=1.0)
    for size in (2.0 ** 40, 2.0 ** -40):
        check([300], [new], 1, 4, 64, dtype, seed=8, qscale=size, scale=0.125 / size)


@pytest.mark.parametrize("new", [1, 70])
def test_tokens_that_see_nothing_and_bad_batches(new):
    """Requests shorter than their new tokens (early tokens see nothing: zeros), a bad length and a bad page beside good requests."""
    H, g, d = 2, 4, 64
    c = Cache4([200, 300, 100], H, d, seed=9)
    q, cu = queries([new] * 3, H * g, d, torch.bfloat16, seed=9)
    want, bound = attention(c.k, c.v, q, cu, [200, 300, 100], c.table, d ** -0.5)
    c.lens[1] = 1 << 24                                       # out of range: skipped
    c.table[2, 0] = -7                                        # no such page: its entries count as masked
    out, st = run(c, q, cu, new)
    assert st == binding.E_ARG
    got = out.double().cpu()
    assert ((got - want).abs() <= bound)[cu[0]:cu[1]].all()
    assert (out[cu[1]:cu[2]] == 777).all()
    k, v = c.k.clone(), c.v.clone()
    table = c.table.cpu()
    table[2, 0] = table[2, 1]
    only = torch.arange(100)
    phys = int(table[2, 1])
    qq = q[cu[2]:cu[3]].double().cpu().unflatten(1, (H, g))
    for j in range(new):
        pos = 100 - new + j
        n = max(0, pos + 1 - 64)
        for h in range(H):
            if n == 0:
                assert (got[cu[2] + j, h * g:(h + 1) * g] == 0).all()
                continue
            w = torch.softmax(qq[j, h] @ k[phys, h, :n].T * d ** -0.5, -1)
            assert ((got[cu[2] + j, h * g:(h + 1) * g] - w @ v[phys, h, :n]).abs() < 0.02).all()
    c = Cache4([3], H, d, seed=10)
    q, cu = queries([5], H * g, d, torch.bfloat16, seed=10)
    out, st = run(c, q, cu, 5)
    assert st == 0 and (out[:2] == 0).all() and (out[2:] != 0).any()


def test_nan_scale_of_an_entry_stays_in_its_request():
    H, g, d = 1, 4, 128
    c = Cache4([100, 100], H, d, seed=11)
    c.arrays[1][int(c.table[0, 0]), 0, 3, 2] = 127
    q, cu = queries([1, 1], H * g, d, torch.bfloat16, seed=11)
    out, st = run(c, q, cu, 1)
    assert st == 0 and torch.isnan(out[0]).any() and torch.isfinite(out[1]).all()
    want, bound = attention(c.k, c.v, q, cu, [100, 100], c.table, d ** -0.5)
    assert ((out[1].double().cpu() - want[1]).abs() <= bound[1]).all()


def test_streams_graphs_and_workspaces():
    """Two captured calls with workspaces of their own, replayed on two streams at once, lengths changed in place between replays."""
    H, g, d = 2, 4, 128
    caches = [Cache4([2000, 700], H, d, seed=20 + i) for i in range(2)]
    q, cu = queries([1, 1], H * g, d, torch.bfloat16, seed=20)
    cut, outs, graphs, works = ints(cu), [], [], []
    for c in caches:
        out = torch.zeros_like(q)
        ws = torch.empty(binding.paged4_workspace_bytes(H * g, H, d), dtype=torch.uint8, device=DEV)
        c4 = c.cache()
        binding.paged4_attention(c4, q, cut, c.lens, c.table, 1, out=out, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.paged4_attention(c4, q, cut, c.lens, c.table, 1, out=out, workspace=ws)
        outs.append(out), graphs.append(graph), works.append((ws, c4))
    streams = [torch.cuda.Stream() for _ in caches]
    for lens in ([2000, 700], [1999, 65], [64, 1]):
        for c in caches:
            c.lens.copy_(ints(lens))
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                for _ in range(5):
                    graph.replay()
        torch.cuda.synchronize()
        for c, out in zip(caches, outs):
            want, bound = attention(c.k, c.v, q, cu, lens, c.table, d ** -0.5)
            assert ((out.double().cpu() - want).abs() <= bound).all()


@pytest.mark.parametrize("d", [64, 128])
def test_chunks_of_many_requests(d):
    """More requests than one warp lays out, long and short chunks and single tokens among them."""
    rng = random.Random(d)
    lens = [rng.choice([1, 64, 100, 300, 513]) for _ in range(70)]
    new = [min(n, rng.choice([0, 1, 1, 40, 130, 257])) for n in lens]
    check(lens, new, 1, 4, d, torch.bfloat16, seed=12)


def test_a_chunk_over_a_long_request():
    check([4200, 3], [300, 1], 1, 8, 128, torch.bfloat16, seed=13)
    check([4200], [300], 2, 2, 96, torch.bfloat16, seed=14, window=1000)


def test_chunk_rows_that_leap_late():
    """A few late entries outweigh all before by far more than fp16 holds: their stretch is computed again, maxima first."""
    H, g, d = 1, 2, 128
    c = Cache4([1200], H, d, seed=15)
    q, cu = queries([200], H * g, d, torch.bfloat16, seed=15)
    kc, ks = c.arrays[0], c.arrays[1]
    for e in (700, 1010, 1150):                               # these entries' keys become 64 times as large
        page = int(c.table[0, e // PAGE])
        ks[page, 0, e % PAGE] = torch.clamp(ks[page, 0, e % PAGE].int() + 48, max=126).to(torch.uint8)
        c.k[page, 0, e % PAGE] = values(kc[page, :, e % PAGE, None], ks[page, :, e % PAGE, None], c.arrays[2])[0, 0]
    out, st = run(c, q, cu, 200)
    assert st == 0
    want, bound = attention(c.k, c.v, q, cu, [1200], c.table, d ** -0.5)
    assert ((out.double().cpu() - want).abs() <= bound).all()

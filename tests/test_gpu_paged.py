"""The caller-owned paged cache on the GPU: plan, append, attention, attention over selected pages, each against a plain
64-bit statement (tests/util_paged.py), and a run of them together."""
import math
import random

import pytest
import torch

from paper_2605_09649_b200 import binding
from util_paged import PAGE, Cache, attention, pages, plan, queries, slack

pytestmark = pytest.mark.gpu
DEV = "cuda"
I32 = torch.int32


def ints(x):
    return torch.tensor(x, dtype=I32, device=DEV)


def status_word():
    return torch.zeros(1, dtype=I32, device=DEV)


# ---------------------------------------------------------------- plan

def run_plan(old, keep, new, table, free, free_count, max_tokens, alias=False):
    t, f, st = ints(table), ints(free), status_word()
    o, n, fc = ints(old), ints(new), ints([free_count])
    k = None if keep is None else ints(keep)
    lens = o if alias else torch.full_like(o, -5)
    fco = fc if alias else torch.full_like(fc, -5)
    cu = torch.full((len(old) + 1,), -5, dtype=I32, device=DEV)
    slots, pos = (torch.full((max_tokens,), -5, dtype=I32, device=DEV) for _ in range(2))
    binding.paged_plan(o, k, n, t, f, fc, fco, lens, cu, slots, pos, st)
    return [t.tolist(), f.tolist(), fco.item(), lens.tolist(), cu.tolist(), slots.tolist(), pos.tolist()], st.item()


def random_plan(rng, n_req, longest, spare):
    old = [rng.choice([0, 1, 63, 64, 65, rng.randint(0, longest)]) for _ in range(n_req)]
    old = [min(o, longest) for o in old]
    new = [rng.choice([0, o, min(o + 1, longest), rng.randint(0, longest)]) for o in old]
    keep = [rng.randint(0, min(o, n)) for o, n in zip(old, new)]
    width = max(1, pages(longest)) + 1
    need = sum(max(0, pages(n) - pages(o)) for o, n in zip(old, new))
    ids = list(range(sum(pages(o) for o in old) + need + spare))
    rng.shuffle(ids)
    table, at = [], 0
    for o in old:
        table.append(ids[at:at + pages(o)] + [-3] * (width - pages(o)))
        at += pages(o)
    live = ids[at:]
    return old, keep, new, table, live + [-4] * (len(ids) - len(live)), len(live)


@pytest.mark.parametrize("n_req,longest,seed", [(1, 1, 0), (1, 64, 1), (1, 5000, 2), (7, 200, 3), (64, 700, 4), (300, 130, 5), (1025, 65, 6), (8192, 70, 7)])
@pytest.mark.parametrize("alias", [False, True])
def test_plan_equals_the_lists(n_req, longest, seed, alias):
    rng = random.Random(seed)
    for spare in (0, 5):
        old, keep, new, table, free, fc = random_plan(rng, n_req, longest, spare)
        for kp in (keep, None):
            tokens = sum(n - k for n, k in zip(new, keep if kp else [min(o, n) for o, n in zip(old, new)]))
            want = plan(old, kp, new, table, free, fc, tokens + 3)
            got, st = run_plan(old, kp, new, table, free, fc, tokens + 3, alias)
            assert st == 0
            for name, a, b in zip("table free count lens cu slots positions".split(), got, want):
                assert a == list(b) if isinstance(b, list) else a == b, name


def test_plan_refused_as_a_whole():
    old, keep, new = [70, 10, 0], [70, 9, 0], [140, 12, 65]
    table = [[5, 6, -3], [7, -3, -3], [-3, -3, -3]]
    free = [1, 2, 0, -4, -4, -4, -4, -4]
    cases = [
        (old, keep, new, table, free, 2, 200, binding.E_NOMEM),            # three pages are wanted
        (old, keep, new, table, free, 3, 136, binding.E_ARG),              # 70 + 3 + 65 new tokens
        (old, [71, 9, 0], new, table, free, 3, 200, binding.E_ARG),        # keep > old
        (old, [70, 13, 0], new, table, free, 3, 200, binding.E_ARG),       # keep > new
        ([70, -1, 0], keep, new, table, free, 3, 200, binding.E_ARG),
        (old, keep, [193, 12, 65], table, free, 3, 400, binding.E_ARG),    # longer than the table
        (old, keep, [2 ** 31 - 1, 12, 65], table, free, 3, 400, binding.E_ARG),
        (old, keep, new, table, free, 9, 200, binding.E_ARG),              # more free pages than pages
        (old, keep, new, table, free, -1, 200, binding.E_ARG),
    ]
    for o, k, n, t, f, fc, m, code in cases:
        got, st = run_plan(o, k, n, t, f, fc, m)
        assert st == code
        assert got == [t, f, fc, o, [0] * 4, [-1] * m, [-1] * m]


def test_plan_bad_page_in_the_free_list_or_table():
    got, st = run_plan([0, 3], None, [2, 5], [[-3], [99]], [50, 1], 1, 4)      # two pages exist
    assert st == binding.E_ARG
    assert got[0] == [[-1], [99]] and got[5] == [-1, -1, -1, -1]


def test_plan_bad_page_given_back():
    """The call that takes a bad entry from a table reports it, not the request that meets it on the stack later."""
    for bad in (-1, 5, 1 << 29, -(1 << 31)):
        got, st = run_plan([130, 3], None, [10, 3], [[0, bad, 2], [1, -3, -3]], [3, 4, -4, -4, -4], 2, 4)      # five pages exist
        assert st == binding.E_ARG
        assert got[0] == [[0, bad, 2], [1, -3, -3]] and got[1] == [3, 4, -1, 2, -4] and got[2] == 4
        assert got[3:] == [[10, 3], [0, 0, 0], [-1] * 4, [-1] * 4]
    got, st = run_plan([64, 0], None, [0, 65], [[7, -3], [-3, -3]], [1, -4, -4], 1, 65)        # given back and taken in one call
    assert st == binding.E_ARG
    assert got[0] == [[7, -3], [-1, 1]] and got[5] == [-1] * 64 + [64]


# ---------------------------------------------------------------- append

@pytest.mark.parametrize("H,d,dtype", [(2, 64, torch.float32), (8, 128, torch.bfloat16), (3, 8, torch.bfloat16), (1, 256, torch.float32), (5, 96, torch.bfloat16), (4, 200, torch.bfloat16)])
@pytest.mark.parametrize("stride", [False, True])
def test_append_writes_rows_and_bounds(H, d, dtype, stride):
    rng = random.Random(H * d)
    before, grow = [0, 1, 63, 64, 10, 120, 0], [64, 63, 1, 1, 0, 200, 130]
    n_pages = sum(pages(b + n) for b, n in zip(before, grow)) + 2
    ids = list(range(n_pages))
    rng.shuffle(ids)
    slots, full = [], []
    for b, n in zip(before, grow):
        mine, ids = ids[:pages(b + n)], ids[pages(b + n):]
        slots += [mine[p // PAGE] * PAGE + p % PAGE for p in range(b, b + n)]
        full += mine[b // PAGE:(b + n) // PAGE] if n else []
        if n:
            slots.insert(rng.randint(0, 1) * len(slots), -1)               # padding between requests and in front
    gen = torch.Generator().manual_seed(1)
    T = len(slots)
    kv = torch.randn(T, 2, H, d, generator=gen).to(dtype).to(DEV)
    k, v = (kv[:, 0], kv[:, 1]) if stride else (kv[:, 0].contiguous(), kv[:, 1].contiguous())
    kp, vp = (torch.randn(n_pages, H, PAGE, d, generator=gen).to(dtype).to(DEV) for _ in range(2))
    kb = torch.randn(n_pages, H, 2, d, generator=gen).to(dtype).to(DEV)
    want_k, want_v, want_b = kp.clone(), vp.clone(), kb.clone()
    for t, s in enumerate(slots):
        if s >= 0:
            want_k[s // PAGE, :, s % PAGE], want_v[s // PAGE, :, s % PAGE] = k[t], v[t]
    for p in full:
        want_b[p, :, 0], want_b[p, :, 1] = want_k[p].amin(1), want_k[p].amax(1)
    st = status_word()
    binding.paged_append(kp, vp, k, v, ints(slots), key_bounds=kb, status=st)
    assert st.item() == 0
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v) and torch.equal(kb, want_b)
    kp2, vp2 = kp.clone(), vp.clone()
    binding.paged_append(kp2, vp2, k, v, ints(slots))                      # without bounds
    assert torch.equal(kp2, want_k) and torch.equal(vp2, want_v)


def test_append_nan_keys_and_bad_slots():
    H, d = 2, 64
    kp, vp, kb = torch.zeros(2, H, PAGE, d, device=DEV), torch.zeros(2, H, PAGE, d, device=DEV), torch.zeros(2, H, 2, d, device=DEV)
    k = torch.randn(PAGE, H, d, device=DEV)
    k[5, 1, 7], k[6, 0, 3] = float("nan"), float("inf")
    st = status_word()
    binding.paged_append(kp, vp, k, k, torch.arange(PAGE, dtype=I32, device=DEV) + PAGE, key_bounds=kb, status=st)
    assert st.item() == 0
    assert torch.equal(kb[1].isnan(), torch.stack((kp[1].amin(1), kp[1].amax(1)), 1).isnan()) and kb[1].isnan().sum() == 2
    assert kb[1, 0, 1, 3] == float("inf") and (kb[0] == 0).all()
    slots = ints([3, 128, 4, -2, 5])                                       # 128 slots exist
    kp0 = kp.clone()
    binding.paged_append(kp, vp, k[10:15], k[10:15], slots, key_bounds=kb, status=st)
    assert st.item() == binding.E_ARG
    kp0[0, :, 3], kp0[0, :, 4], kp0[0, :, 5] = k[10], k[12], k[14]
    assert torch.equal(kp.nan_to_num(), kp0.nan_to_num())


# ---------------------------------------------------------------- attention

LAYOUTS = [(2, 2, 64, torch.float32), (1, 8, 128, torch.bfloat16), (4, 7, 128, torch.bfloat16), (2, 4, 64, torch.bfloat16), (3, 5, 96, torch.bfloat16),
           (2, 16, 64, torch.bfloat16), (1, 40, 128, torch.bfloat16), (1, 3, 256, torch.float32), (2, 1, 8, torch.bfloat16), (1, 20, 40, torch.float32),
           (8, 1, 128, torch.bfloat16), (1, 128, 128, torch.bfloat16)]
# (lengths, new tokens): empty requests, one entry, page borders, more new tokens than entries (rows that see nothing)
BATCHES = [([1], [1]), ([0, 5, 0], [0, 0, 3]), ([63, 64, 65, 1, 129], [1, 1, 1, 1, 1]), ([200, 64, 3, 130], [5, 4, 5, 2]), ([300, 7, 90], [150, 7, 33]), ([577], [300])]


def check_attention(lens, new, H, g, d, dtype, window=0, pad=0, stride=False, seed=0, max_new=None, scale=None, top=0, sink=0, recent=1, spread=1.0):
    c = Cache(lens, H, d, dtype, DEV, seed, spread=spread)
    q, cu = queries(new, H * g, d, dtype, DEV, seed, pad, stride=H * g * d + 16 if stride else 0)
    out = torch.full((q.shape[0], H * g, d), 7.0, dtype=dtype, device=DEV)
    st = status_word()
    ws = torch.full((binding.paged_workspace_bytes(H * g, H, d),), 255, dtype=torch.uint8, device=DEV)    # NaN everywhere
    if top:
        sel = torch.full((q.shape[0], H, top), -9, dtype=I32, device=DEV)
        binding.paged_sparse_attention(c.k, c.v, c.bounds, q, ints(cu), c.lens, c.table, top, sink_pages=sink, recent_pages=recent, scale=scale,
                                       out=out, selected=sel, workspace=ws, status=st)
    else:
        binding.paged_attention(c.k, c.v, q, ints(cu), c.lens, c.table, max(new) if max_new is None else max_new, scale=scale, window=window, out=out,
                                workspace=ws, status=st)
    want, bound, chosen = attention(c.k, c.v, q, cu, lens, c.table, d ** -0.5 if scale is None else scale, window, c.bounds, top, sink, recent)
    assert st.item() == 0
    T = cu[-1]
    if top:
        assert torch.equal(sel.cpu(), chosen)
    got = out.double().cpu()
    assert (got[T:] == 7.0).all()                                          # rows behind the last token are left alone
    off = (got[:T] - want[:T]).abs()
    assert torch.isfinite(got[:T]).all()
    assert (off <= bound[:T]).all(), f"off by up to {(off / bound[:T].clamp(min=1e-30)).max():.2f} of the bound"
    return out


@pytest.mark.parametrize("lens,new", BATCHES)
@pytest.mark.parametrize("H,g,d,dtype", LAYOUTS)
def test_attention_layouts_and_lengths(H, g, d, dtype, lens, new):
    check_attention(lens, new, H, g, d, dtype)


@pytest.mark.parametrize("window", [1, 2, 64, 100, 1000])
@pytest.mark.parametrize("H,g,d,dtype", [(2, 2, 64, torch.float32), (2, 4, 128, torch.bfloat16), (2, 4, 64, torch.bfloat16)])
def test_attention_window(H, g, d, dtype, window):
    check_attention([300, 64, 65, 0, 1], [1, 1, 1, 0, 1], H, g, d, dtype, window=window)
    check_attention([300, 7, 90, 64], [150, 7, 33, 66], H, g, d, dtype, window=window, pad=3)


@pytest.mark.parametrize("H,g,d,dtype", [(2, 2, 64, torch.float32), (4, 7, 128, torch.bfloat16), (2, 4, 64, torch.bfloat16)])
def test_attention_strided_queries_padding_and_scale(H, g, d, dtype):
    check_attention([200, 64, 3, 130], [1, 4, 3, 60], H, g, d, dtype, pad=5, stride=True, scale=0.3)
    check_attention([5000, 1], [1, 1], H, g, d, dtype, pad=1, stride=True)                      # one long request, shared out
    check_attention([5000, 2100], [3, 1], H, g, d, dtype, max_new=0)                           # the host knows nothing
    check_attention([200, 700], [90, 4], H, g, d, dtype, max_new=1)                            # ... or is wrong
    check_attention([400], [100], H, g, d, dtype, spread=6.0)                                  # large logits


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [0, 200])
def test_attention_logits_that_leap(d, window):
    """The reference of the softmax weights lags behind the maximum: logits that leap up (by far more than an exponent's range),
    fall, and rise slowly along the keys, in rows of one call."""
    H, g, n, new = 1, 4, 1500, 140
    c = Cache([n], H, d, torch.bfloat16, DEV, 8)
    q, cu = queries([new], H * g, d, torch.bfloat16, DEV, 8)
    u = torch.zeros(d)
    u[3] = 1.0
    q[:, :, 3] = torch.tensor([2.0, -2.0, 0.5, 0.0]).to(q.dtype).to(DEV)[None, :, None].squeeze(-1)
    steps = torch.zeros(n)
    steps[200:] = 40.0
    steps[450:] = 400.0
    steps[700:900] = -300.0
    steps[900:] = torch.linspace(-100, 900, n - 900)
    for e in range(n):
        c.k[c.table[0, e // PAGE].item(), :, e % PAGE, 3] = float(steps[e])
    out = binding.paged_attention(c.k, c.v, q, ints(cu), c.lens, c.table, new, window=window)
    want, bound, _ = attention(c.k, c.v, q, cu, [n], c.table, d ** -0.5, window)
    assert ((out.double().cpu() - want).abs() <= bound).all()


def test_attention_many_requests_and_mixed_batch():
    rng = random.Random(3)
    lens = [rng.randint(0, 150) for _ in range(1500)]
    new = [min(n, rng.choice([0, 1, 1, 1, 2])) for n in lens]
    check_attention(lens, new, 1, 2, 64, torch.bfloat16, pad=2)
    check_attention(lens[:1100], new[:1100], 1, 2, 32, torch.float32)
    lens = [rng.randint(300, 900) for _ in range(12)]
    check_attention(lens, [1, 1, 200, 1, 5, 300, 1, 0, 40, 1, 17, 1], 2, 4, 128, torch.bfloat16)


def test_attention_bad_requests_and_pages_are_skipped():
    H, g, d = 1, 2, 64
    for dtype in (torch.float32, torch.bfloat16):
        c = Cache([100, 100, 100, 100], H, d, dtype, DEV, 1)
        q, cu = queries([1, 1, 1, 1], H * g, d, dtype, DEV, 1)
        c.lens[1] = 64 * c.width + 1                                       # longer than its table row
        c.table[2, 0] = c.n_pages                                          # no such page: its entries do not count
        c.lens[3] = -1
        out, st = torch.full((4, H * g, d), 7.0, dtype=dtype, device=DEV), status_word()
        binding.paged_attention(c.k, c.v, q, ints(cu), c.lens, c.table, 1, out=out, status=st)
        assert st.item() == binding.E_ARG
        assert (out[1] == 7).all() and (out[3] == 7).all()
        want = torch.softmax(q[2].double() @ c.k[c.table[2, 1].item(), 0, :36].double().T / 8, -1) @ c.v[c.table[2, 1].item(), 0, :36].double()
        assert (out[2].double() - want).abs().max() < 2e-2
        st.zero_()
        for bad in ([0, 1, 2, 9, 4], [0, 2, 1, 3, 4], [-1, 1, 2, 3, 4]):   # offsets out of range or descending
            out.fill_(7.0)
            binding.paged_attention(c.k, c.v, q, ints(bad), ints([100] * 4), c.table.clamp(max=c.n_pages - 1), 1, out=out, status=st)
            assert st.item() == binding.E_ARG


@pytest.mark.parametrize("dtype,d,new", [(torch.bfloat16, 64, 140), (torch.bfloat16, 128, 140), (torch.bfloat16, 128, 3), (torch.bfloat16, 256, 40), (torch.float32, 64, 40)])
def test_attention_large_values(dtype, d, new):
    """Values up to 2^43 (randn, times 2^40), with logits that leap: no weight times a value overflows, whatever its reference is."""
    H, g, n = 1, 4, 900
    c = Cache([n], H, d, dtype, DEV, 18, spread=4.0)
    c.v *= 2.0 ** 40
    q, cu = queries([new], H * g, d, dtype, DEV, 18)
    out = binding.paged_attention(c.k, c.v, q, ints(cu), c.lens, c.table, new)
    want, bound, _ = attention(c.k, c.v, q, cu, [n], c.table, d ** -0.5)
    assert ((out.double().cpu() - want).abs() <= bound).all()


WIDE = [(2, 4, 256), (1, 8, 192), (3, 5, 136), (1, 40, 200)]                # head sizes above 128, bf16


@pytest.mark.parametrize("lens,new", BATCHES)
@pytest.mark.parametrize("H,g,d", WIDE)
def test_attention_wide_heads(H, g, d, lens, new):
    check_attention(lens, new, H, g, d, torch.bfloat16)


@pytest.mark.parametrize("H,g,d", WIDE)
def test_attention_wide_heads_shared_out(H, g, d):
    """Long requests, whose units several workers share: single tokens, drafts, a chunk, windows."""
    check_attention([5000, 1], [1, 1], H, g, d, torch.bfloat16, pad=1, stride=True)
    check_attention([4000, 2100], [3, 1], H, g, d, torch.bfloat16, max_new=0)
    check_attention([2500], [20], H, g, d, torch.bfloat16, window=1000)


@pytest.mark.parametrize("new", [[1, 1, 1], [5, 2, 3]])
@pytest.mark.parametrize("H,g,d,dtype", [(2, 2, 64, torch.float32), (1, 3, 256, torch.float32), (2, 4, 128, torch.bfloat16), (2, 4, 64, torch.bfloat16), (1, 7, 96, torch.bfloat16)])
def test_attention_window_over_shared_units(H, g, d, dtype, new):
    """Windows of many pages: their units are dealt out by pages, and a unit's pages are not as many as the line counts for it."""
    for window in (1500, 4031):
        check_attention([9000, 5000, 700], new, H, g, d, dtype, window=window)


def without_page(c, q, cu, lens, r_bad, page, scale):
    """(out, bound) in fp64 where the entries of one page of one request do not count."""
    H, d = c.k.shape[1], c.k.shape[3]
    g = q.shape[1] // H
    out, bound = (torch.zeros(q.shape, dtype=torch.float64) for _ in range(2))
    for r, total in enumerate(lens):
        at = torch.arange(total)
        keep = torch.ones(total, dtype=torch.bool) if r != r_bad else at // PAGE != page
        phys = torch.where(keep, c.table[r].cpu()[at // PAGE].long(), 0)
        for h in range(H):
            k, v = (torch.where(keep[:, None], x.cpu()[phys, h, at % PAGE].double(), 0.0) for x in (c.k, c.v))
            for t in range(cu[r], cu[r + 1]):
                see = keep & (at <= total - (cu[r + 1] - t))
                qq = q[t, h * g:(h + 1) * g].double().cpu()
                if not see.any():
                    continue
                w = torch.softmax((qq @ k.T * scale).masked_fill(~see, -math.inf), -1)
                o = w @ v
                out[t, h * g:(h + 1) * g] = o
                bound[t, h * g:(h + 1) * g] = slack(q.dtype, o, w @ v.abs(), (qq.abs() @ k.abs().T * scale).amax(-1, keepdim=True), total, d)
    return out, bound


@pytest.mark.parametrize("H,g,d,dtype", [(2, 2, 64, torch.float32), (2, 4, 128, torch.bfloat16), (2, 4, 40, torch.bfloat16), (1, 4, 256, torch.bfloat16)])
@pytest.mark.parametrize("new", [[5, 1], [100, 40], [200, 1]])
def test_attention_bad_page_of_a_chunk(H, g, d, dtype, new):
    """An entry of the table that is no page, first, in the middle and last, in drafts and chunks: its entries do not count, the rest does;
    what the cache's first page holds (NaN here) reaches nobody."""
    lens = [300, 129]
    for page, value in ((0, -1), (2, 1 << 29), (4, None)):
        c = Cache(lens, H, d, dtype, DEV, 31)
        q, cu = queries(new, H * g, d, dtype, DEV, 31)
        c.table[0, page] = c.n_pages if value is None else value
        spare = next(p for p in range(1, c.n_pages) if p not in c.table.flatten().tolist())
        c.k[spare], c.v[spare] = c.k[0], c.v[0]
        c.table[c.table == 0] = spare
        c.k[0], c.v[0] = float("nan"), float("nan")
        out, st = torch.full(q.shape, 7.0, dtype=dtype, device=DEV), status_word()
        binding.paged_attention(c.k, c.v, q, ints(cu), c.lens, c.table, max(new), out=out, status=st)
        want, bound = without_page(c, q, cu, lens, 0, page, d ** -0.5)
        assert st.item() == binding.E_ARG
        assert ((out.double().cpu() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_bad_offsets_leave_the_other_requests_right(dtype):
    H, g, d, lens = 1, 2, 64, [100, 90, 80, 70]
    c = Cache(lens, H, d, dtype, DEV, 1)
    q, _ = queries([1, 1, 1, 1], H * g, d, dtype, DEV, 1)
    # offsets, and the requests with good ones: (request, its rows); rows of no good request stay as they are
    cases = [([0, 1, 2, 9, 4], [(0, [0]), (1, [1])]),                      # request 2 ends behind the last row, request 3 descends
             ([0, 1, 3, 2, 4], [(0, [0]), (1, [1, 2]), (3, [2, 3])]),      # request 2 descends; row 2 is claimed twice
             ([-1, 1, 2, 3, 4], [(1, [1]), (2, [2]), (3, [3])]),           # request 0 begins in front of the first row
             ([5, 6, 2, 3, 4], [(2, [2]), (3, [3])])]                      # requests 0 and 1 lie behind the last row
    for cu, good in cases:
        out, st = torch.full(q.shape, 7.0, dtype=dtype, device=DEV), status_word()
        binding.paged_attention(c.k, c.v, q, ints(cu), c.lens, c.table, 1, out=out, status=st)
        assert st.item() == binding.E_ARG, cu
        owners = {}
        for r, rows in good:
            for row in rows:
                owners.setdefault(row, []).append(r)
        for row in range(4):
            if row not in owners:
                assert (out[row] == 7).all(), (cu, row)
            elif len(owners[row]) == 1:
                r = owners[row][0]
                mine = dict(good)[r]
                # the request by itself: its rows are the new tokens of a batch of one
                alone = Cache(lens, H, d, dtype, DEV, 1)
                want, bound, _ = attention(alone.k, alone.v, q[mine], [0, len(mine)], [lens[r]], alone.table[r:r + 1], d ** -0.5)
                i = mine.index(row)
                assert ((out[row].double().cpu() - want[i]).abs() <= bound[i]).all(), (cu, row)


# ---------------------------------------------------------------- attention over selected pages

@pytest.mark.parametrize("H,g,d,dtype", LAYOUTS)
@pytest.mark.parametrize("top,sink,recent", [(1, 0, 1), (4, 1, 2), (5, 0, 1), (3, 1, 2)])
def test_sparse_attention_layouts(H, g, d, dtype, top, sink, recent):
    check_attention([700, 64, 0, 1, 65, 257], [1, 1, 0, 1, 1, 1], H, g, d, dtype, top=top, sink=sink, recent=recent)
    check_attention([500, 6, 330], [5, 8, 70], H, g, d, dtype, top=top, sink=sink, recent=recent, pad=2, stride=True)


@pytest.mark.parametrize("H,g,d,dtype", [(1, 4, 128, torch.bfloat16), (2, 2, 64, torch.float32)])
def test_sparse_attention_long_context(H, g, d, dtype):
    check_attention([20000], [1], H, g, d, dtype, top=40, sink=2, recent=3)
    check_attention([9001, 4000, 12345], [1, 2, 1], H, g, d, dtype, top=33)
    check_attention([3000], [130], H, g, d, dtype, top=8, sink=1, recent=1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sparse_attention_ties_nan_and_infinite_bounds(dtype):
    H, g, d = 1, 1, 64
    c = Cache([64 * 40 + 3], H, d, dtype, DEV, 2)
    q, cu = queries([1], 1, d, dtype, DEV, 2)
    table = c.table[0].tolist()
    c.bounds[:] = 1.0                                                      # all scores equal: the lower pages win
    args = dict(sink_pages=0, recent_pages=1)
    call = lambda top: binding.paged_sparse_attention(c.k, c.v, c.bounds, q, ints(cu), c.lens, c.table, top, **args)[1][0, 0].tolist()
    assert call(6) == [0, 1, 2, 3, 4, 40]
    best = int(q[0, 0].float().argmax())
    c.bounds[table[30]] = float("nan")                                     # what cannot be bounded is read
    c.bounds[table[20], :, 1, best] = float("inf")
    c.bounds[table[10], :, :, best] = -float("inf")                        # the last to be taken
    assert call(4) == [0, 20, 30, 40]
    assert call(40) == [p for p in range(41) if p != 10]
    assert call(41) == list(range(41))
    c.bounds[:] = -0.0
    c.bounds[table[7]] = 0.0                                               # -0 and +0 are the same score
    assert call(3) == [0, 1, 40]


@pytest.mark.parametrize("step", [0.0, 1.0])
def test_sparse_attention_scores_that_only_64_bits_tell_apart(step):
    """More pages than the short list ranks, their scores equal (step 0) or apart by less than fp32 sums can tell: one small
    channel differs, beside channels that cancel to the same large sum."""
    H, g, d, n = 1, 2, 128, 700
    c = Cache([64 * n + 1], H, d, torch.bfloat16, DEV, 3)
    q = torch.ones(1, g, d, dtype=torch.bfloat16, device=DEV)
    q[0, :, 5] = 2.0 ** -20
    order = list(range(n))
    random.Random(1).shuffle(order)
    c.bounds[:] = 300.0
    c.bounds[:, :, :, 64:] = -299.0
    for rank, page in enumerate(order):
        c.bounds[c.table[0, page].item(), :, :, 5] = step * (rank % 233 + 1) / 256.0 + 1.0
    for top in (2, 100, 600, 700):
        sel = binding.paged_sparse_attention(c.k, c.v, c.bounds, q, ints([0, 1]), c.lens, c.table, top)[1][0, 0].tolist()
        u = {p: float(c.bounds[c.table[0, p].item(), 0, 1, 5]) for p in range(n)}
        want = sorted(sorted(range(n), key=lambda p: (-u[p], p))[:top - 1]) + [n]
        assert sel == want


def test_sparse_attention_tokens_that_share_a_unit():
    """Many tokens of few requests: several tokens walk the bounds together; some see fewer pages than they may select."""
    check_attention([420, 390, 130], [200, 101, 130], 8, 4, 64, torch.bfloat16, top=4, sink=1, recent=1, pad=3)
    check_attention([500, 260], [260, 255], 6, 7, 128, torch.bfloat16, top=3)
    check_attention([330], [329], 4, 16, 64, torch.bfloat16, top=2)


@pytest.mark.parametrize("H,g,d", WIDE)
@pytest.mark.parametrize("top,sink,recent", [(1, 0, 1), (4, 1, 2), (5, 0, 1)])
def test_sparse_attention_wide_heads(H, g, d, top, sink, recent):
    check_attention([700, 64, 0, 1, 65, 257], [1, 1, 0, 1, 1, 1], H, g, d, torch.bfloat16, top=top, sink=sink, recent=recent)
    check_attention([500, 6, 330], [5, 8, 70], H, g, d, torch.bfloat16, top=top, sink=sink, recent=recent, pad=2, stride=True)


def test_sparse_attention_wide_heads_over_long_contexts():
    check_attention([20000], [1], 1, 8, 256, torch.bfloat16, top=40, sink=2, recent=3)
    check_attention([9001, 4000, 12345], [1, 2, 1], 2, 4, 192, torch.bfloat16, top=33)
    check_attention([420, 390, 130], [200, 101, 130], 8, 2, 136, torch.bfloat16, top=4, sink=1, recent=1, pad=3)      # tokens share a unit


@pytest.fixture
def union_forced():
    binding.set_global_test_hooks(binding.TEST_UNION_OF_PAGES)
    yield
    binding.set_global_test_hooks(0)


@pytest.mark.parametrize("H,g,d", [(h, g, d) for h, g, d, dtype in LAYOUTS if dtype == torch.bfloat16])
@pytest.mark.parametrize("top,sink,recent", [(1, 0, 1), (4, 1, 2), (5, 0, 1)])
def test_sparse_attention_union_of_pages(union_forced, H, g, d, top, sink, recent):
    """The kernel for requests with many tokens, at sizes where it does not pay by itself."""
    check_attention([500, 6, 330], [70, 8, 64], H, g, d, torch.bfloat16, top=top, sink=sink, recent=recent, pad=2, stride=True)
    check_attention([700, 64, 65, 1], [66, 64, 1, 1], H, g, d, torch.bfloat16, top=top, sink=sink, recent=recent)


def test_sparse_attention_union_of_pages_over_long_contexts(union_forced):
    check_attention([3000], [130], 1, 4, 128, torch.bfloat16, top=8, sink=1, recent=1)
    check_attention([9001, 4000, 12345], [70, 2, 65], 1, 4, 64, torch.bfloat16, top=33)
    check_attention([420, 390, 130], [200, 101, 130], 2, 4, 64, torch.bfloat16, top=4, sink=1, recent=1, pad=3)


def launches(lens, new, H, g, d, top, dtype=torch.bfloat16, seed=11):
    c = Cache(lens, H, d, dtype, DEV, seed)
    q, cu = queries(new, H * g, d, dtype, DEV, seed)
    before = binding.kernel_launches()
    out, sel = binding.paged_sparse_attention(c.k, c.v, c.bounds, q, ints(cu), c.lens, c.table, top)
    return binding.kernel_launches() - before, out, sel


def test_sparse_attention_union_of_pages_only_where_it_pays():
    """A short chunk is served by the kernels that serve as many single tokens; a long one by those that the hook asks for, and right."""
    assert launches([6400], [40], 1, 4, 64, 4)[0] == launches([640] * 40, [1] * 40, 1, 4, 64, 4)[0]
    few, out, sel = launches([2200], [200], 8, 4, 64, 32)
    binding.set_global_test_hooks(binding.TEST_UNION_OF_PAGES)
    try:
        forced, same, _ = launches([2200], [200], 8, 4, 64, 32)
    finally:
        binding.set_global_test_hooks(0)
    assert few == forced and torch.equal(out, same)
    check_attention([2200], [200], 8, 4, 64, torch.bfloat16, top=32)


@pytest.mark.parametrize("forced", [False, True])
@pytest.mark.parametrize("H,g,d,dtype", [(2, 2, 64, torch.float32), (2, 4, 128, torch.bfloat16), (2, 4, 40, torch.bfloat16)])
def test_sparse_attention_bad_page(H, g, d, dtype, forced):
    """Among the pages that are always read, an entry that is no page counts for nothing; among the others it is chosen last."""
    lens, new = [300, 129], [80, 1]
    for page in (0, 2):
        c = Cache(lens, H, d, dtype, DEV, 32)
        q, cu = queries(new, H * g, d, dtype, DEV, 32)
        c.table[0, page] = 1 << 29
        st = status_word()
        binding.set_global_test_hooks(binding.TEST_UNION_OF_PAGES if forced else 0)
        try:
            out, sel = binding.paged_sparse_attention(c.k, c.v, c.bounds, q, ints(cu), c.lens, c.table, 5, sink_pages=1, status=st)
            out4, sel4 = binding.paged_sparse_attention(c.k, c.v, c.bounds, q, ints(cu), c.lens, c.table, 4, sink_pages=1, status=st)
        finally:
            binding.set_global_test_hooks(0)
        assert st.item() == binding.E_ARG
        want, bound = without_page(c, q, cu, lens, 0, page, d ** -0.5)     # five pages are all there are
        assert ((out.double().cpu() - want).abs() <= bound).all()
        if page == 2:                                                      # of pages 1 to 3 of a token on page 4 two are read, 2 is not
            late = sel4[36:80].cpu()                                       # (positions 256 to 299)
            assert (late == torch.tensor([0, 1, 3, 4], dtype=I32)).all()
            see = without_page(c, q, cu, lens, 0, page, d ** -0.5)
            assert ((out4[36:80].double().cpu() - see[0][36:80]).abs() <= see[1][36:80]).all()


def test_sparse_attention_chunk_among_idle_requests():
    """Requests without new tokens do not change which kernels serve a chunk."""
    alone, out, sel = launches([2200], [200], 8, 4, 64, 32)
    among, out2, sel2 = launches([2200] + [0] * 255, [200] + [0] * 255, 8, 4, 64, 32)
    assert among == alone and torch.equal(out2, out) and torch.equal(sel2, sel)


# ---------------------------------------------------------------- together

def serve(dtype, H, g, d, top, graph):
    """A continuous batch through plan, append and attention: requests start, draft, reject, end; every step's attention is
    compared with the history that each request really has."""
    rng, gen = random.Random(5), torch.Generator().manual_seed(5)
    R, W, n_pages, M = 5, 8, 30, 220
    st = status_word()
    k_pages, v_pages = (torch.full((n_pages, H, PAGE, d), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
    bounds = torch.full((n_pages, H, 2, d), float("nan"), dtype=dtype, device=DEV)
    table, free, count = torch.full((R, W), -1, dtype=I32, device=DEV), ints(list(range(n_pages))), ints([n_pages])
    lens, keep, new = ints([0] * R), ints([0] * R), ints([0] * R)
    cu, slots, pos = ints([0] * (R + 1)), ints([0] * M), ints([0] * M)
    k, v, q = (torch.zeros(M, n, d, dtype=dtype, device=DEV) for n in (H, H, H * g))
    out = torch.zeros(M, H * g, d, dtype=dtype, device=DEV)
    ws = torch.empty(binding.paged_workspace_bytes(H * g, H, d), dtype=torch.uint8, device=DEV)
    sel = torch.empty(M, H, max(top, 1), dtype=I32, device=DEV)

    def step():
        binding.paged_plan(lens, keep, new, table, free, count, count, lens, cu, slots, pos, st)
        binding.paged_append(k_pages, v_pages, k, v, slots, key_bounds=bounds, status=st)
        if top:
            binding.paged_sparse_attention(k_pages, v_pages, bounds, q, cu, lens, table, top, sink_pages=1, out=out, selected=sel, workspace=ws, status=st)
        else:
            binding.paged_attention(k_pages, v_pages, q, cu, lens, table, 0, out=out, workspace=ws, status=st)

    captured = None
    if graph:
        step()
        torch.cuda.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
    hist = [[torch.zeros(0, H, d)] * 2 for _ in range(R)]
    for it in range(14):
        kp, nw = [], []
        for r in range(R):
            n = hist[r][0].shape[0]
            kind = rng.random()
            if n == 0:
                kk, nn = 0, rng.choice([0, 1, 40, 64])
            elif kind < 0.1:
                kk = nn = 0
            elif kind < 0.5:
                kk = max(0, n - rng.randint(0, 4))
                nn = kk + rng.randint(1, 6)
            else:
                kk, nn = n, min(W * PAGE, n + rng.choice([1, 1, 30]))
            kp.append(kk), nw.append(nn)
        keep.copy_(ints(kp)), new.copy_(ints(nw))
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, generator=gen).to(dtype))
        captured.replay() if graph else step()
        assert st.item() == 0
        row, cl = 0, [0]
        for r in range(R):
            n = nw[r] - kp[r]
            for i, x in enumerate((k, v)):
                hist[r][i] = torch.cat((hist[r][i][:kp[r]], x[row:row + n].float().cpu()))
            row += n
            cl.append(row)
        assert cu.tolist() == cl and lens.tolist() == nw and count.item() == n_pages - sum(pages(n) for n in nw)
        live = [p for r in range(R) for p in table[r, :pages(nw[r])].tolist()]
        assert len(set(live + free[:count.item()].tolist())) == n_pages    # no page is lost or held twice
        # the reference reads the history, laid out in a cache of its own
        ref = Cache([len(h[0]) for h in hist], H, d, dtype, DEV, 9)
        for r in range(R):
            for e in range(nw[r]):
                p = ref.table[r, e // PAGE].item()
                ref.k[p, :, e % PAGE], ref.v[p, :, e % PAGE] = hist[r][0][e].to(dtype).to(DEV), hist[r][1][e].to(dtype).to(DEV)
        ref.bounds = torch.stack((ref.k.amin(2), ref.k.amax(2)), 2)
        want, bound, chosen = attention(ref.k, ref.v, q[:row], cl, nw, ref.table, d ** -0.5, 0, ref.bounds, top, 1 if top else 0, 1)
        assert ((out[:row].double().cpu() - want).abs() <= bound).all()
        if top:
            assert torch.equal(sel[:row].cpu(), chosen)


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("dtype,H,g,d", [(torch.float32, 2, 2, 32), (torch.bfloat16, 2, 4, 64)])
def test_serving_loop(dtype, H, g, d, top, graph):
    serve(dtype, H, g, d, top, graph)


def test_two_streams_at_once_and_repeatable():
    H, g, d, dtype = 2, 4, 128, torch.bfloat16
    c = Cache([3000, 40, 900], H, d, dtype, DEV, 4)
    q, cu = queries([2, 1, 150], H * g, d, dtype, DEV, 4)
    cu = ints(cu)
    first = binding.paged_attention(c.k, c.v, q, cu, c.lens, c.table, 150)
    firsts, sel = binding.paged_sparse_attention(c.k, c.v, c.bounds, q, cu, c.lens, c.table, 6)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(binding.paged_attention(c.k, c.v, q, cu, c.lens, c.table, 150) if i < 4 else
                        binding.paged_sparse_attention(c.k, c.v, c.bounds, q, cu, c.lens, c.table, 6)[0])
    torch.cuda.synchronize()
    for i, o in enumerate(outs):                                           # no atomics: the same bits every time
        assert torch.equal(o, first if i < 4 else firsts)


@pytest.mark.parametrize("dtype,n_pages", [(torch.bfloat16, 70000), (torch.float32, 35000)])
def test_pages_behind_32_bit_offsets(dtype, n_pages):
    """Arrays of more than 2^32 (bf16) and 2^31 elements, 9.2 GB each: pages anywhere in them give the bits that pages in a small
    cache give."""
    H, g, d = 8, 4, 128
    lens, new = [900, 130, 64], [70, 1, 3]
    c = Cache(lens, H, d, dtype, DEV, 6)
    q, cu = queries(new, H * g, d, dtype, DEV, 6)
    cu = ints(cu)
    far = n_pages - 1 - torch.arange(c.n_pages, device=DEV) * (n_pages // c.n_pages)
    far[-1] = 0
    k, v = (torch.empty(n_pages, H, PAGE, d, dtype=dtype, device=DEV) for _ in range(2))
    b = torch.empty(n_pages, H, 2, d, dtype=dtype, device=DEV)
    k[far], v[far], b[far] = c.k, c.v, c.bounds
    table = torch.where(c.table < c.n_pages, far[c.table.clamp(max=c.n_pages - 1).long()].to(I32), c.table)
    st = status_word()
    want = binding.paged_attention(c.k, c.v, q, cu, c.lens, c.table, 70)
    assert torch.equal(binding.paged_attention(k, v, q, cu, c.lens, table, 70, status=st), want)
    want, chosen = binding.paged_sparse_attention(c.k, c.v, c.bounds, q, cu, c.lens, c.table, 3)
    got, sel = binding.paged_sparse_attention(k, v, b, q, cu, c.lens, table, 3, status=st)
    assert torch.equal(got, want) and torch.equal(sel, chosen)
    x = torch.randn(PAGE + 1, H, d, device=DEV).to(dtype)
    slots = torch.arange(PAGE + 1, dtype=I32, device=DEV) + (n_pages - 1) * PAGE
    slots[PAGE] = 5
    binding.paged_append(k, v, x, -x, slots, key_bounds=b, status=st)
    assert torch.equal(k[n_pages - 1], x[:PAGE].transpose(0, 1)) and torch.equal(v[n_pages - 1], -x[:PAGE].transpose(0, 1))
    assert torch.equal(k[0, :, 5], x[PAGE]) and torch.equal(b[n_pages - 1, :, 1], x[:PAGE].amax(0)) and st.item() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sparse_attention_widest_table(dtype):
    check_attention([1 << 20], [1], 1, 2, 8, dtype, top=20, sink=1, recent=2)


def test_calls_that_share_a_workspace_in_turn():
    """Different calls one after the other on one stream, and two captured graphs, with one workspace: each gives what it gives alone."""
    H, g, d = 2, 4, 128
    c = Cache([3000, 40, 900, 2500], H, d, torch.bfloat16, DEV, 14)
    ws = torch.full((binding.paged_workspace_bytes(H * g, H, d),), 255, dtype=torch.uint8, device=DEV)
    calls = []
    for new, top in (([1, 1, 1, 1], 0), ([2, 1, 150, 300], 0), ([1, 1, 1, 1], 9), ([5, 5, 5, 5], 0), ([200, 1, 2, 130], 6)):
        q, cu = queries(new, H * g, d, torch.bfloat16, DEV, 14)
        cu, out = ints(cu), torch.empty_like(q)
        def call(q=q, cu=cu, out=out, new=new, top=top):
            if top:
                binding.paged_sparse_attention(c.k, c.v, c.bounds, q, cu, c.lens, c.table, top, out=out, workspace=ws)
            else:
                binding.paged_attention(c.k, c.v, q, cu, c.lens, c.table, max(new), out=out, workspace=ws)
            return out
        call()
        torch.cuda.synchronize()
        calls.append((call, call().clone(), out))
    graphs = []
    for half in (calls[:3], calls[3:]):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            for call, _, _ in half:
                call()
    for order in range(6):
        for _, _, out in calls:
            out.fill_(float("nan"))
        if order % 2:
            for graph in graphs:
                graph.replay()
        else:
            for call, _, _ in calls[order:] + calls[:order]:
                call()
        for _, want, out in calls:
            assert torch.equal(out, want)

"""Rows that share pages, dropped entries and moved rows on the GPU, each against lists (tests/util_paged_share.py), and a run of them
together with append and attention over a cache in 4 bits."""
import random

import pytest
import torch

from paper_2605_09649_b200 import binding
from util_paged import PAGE, pages
from util_paged4 import Cache4, attention, quantise, pack, values
from util_paged_share import Rows, compact, share

pytestmark = pytest.mark.gpu
DEV = "cuda"
I32 = torch.int32


def ints(x):
    return torch.tensor(x, dtype=I32, device=DEV)


def filled(n, v=-5):
    return torch.full((n,), v, dtype=I32, device=DEV)


def run_share(source, old, keep, new, table, refs, stack, n_pages, tokens, moves, in_place=False):
    t, rf, fr, fc = ints(table), ints(refs), ints(stack + [-4] * (n_pages - len(stack))), ints([len(stack)])
    out = torch.full_like(t, -5)
    ro, fo, co = (rf, fr, fc) if in_place else (filled(n_pages), filled(n_pages), filled(1))
    lens, cu, slots, pos = filled(len(old)), filled(len(old) + 1), filled(tokens), filled(tokens)
    src, dst, count, st = filled(moves), filled(moves), filled(1), torch.zeros(1, dtype=I32, device=DEV)
    binding.paged_share(ints(source), ints(old), ints(keep), ints(new), t, out, rf, ro, fr, fo, fc, co, lens, cu, slots, pos, src, dst, count, st)
    got = dict(table=out.tolist(), refs=ro.tolist(), free=fo.tolist(), count=co.item(), lens=lens.tolist(), cu=cu.tolist(), slots=slots.tolist(),
               positions=pos.tolist(), src=src.tolist(), dst=dst.tolist(), moves=count.item())
    return got, st.item()


def wishes(rng, s: Rows, grow):
    """(source, keep, new) of every row: ends, starts, goes on, takes back, forks from any place of any row."""
    R, cap = len(s.lens), s.width * PAGE
    source, keep, new = [], [], []
    for r in range(R):
        kind = rng.choice("end start on back fork fork tail".split())
        src, k = r, s.lens[r]
        if kind in ("end", "start"):
            src, k = rng.choice([-1, r]), 0
        elif kind == "back":
            k = rng.randint(0, s.lens[r])
        elif kind == "fork":
            src = rng.randrange(R)
            k = rng.choice([s.lens[src], rng.randint(0, s.lens[src])])
        elif kind == "tail":                                  # many rows of one source
            src = r // 4 * 4
            k = s.lens[src]
        n = 0 if kind == "end" else rng.choice([k, k + 1, k + rng.randint(0, grow)])
        source.append(src), keep.append(k), new.append(min(max(n, k), cap))
    return source, keep, new


def expect(want, s, new, tokens, moves):
    rows, refs, peak, live, lens, cu, slots, positions, mv = want
    return dict(table=[row + [-5] * (s.width - len(row)) for row in rows], refs=refs, free=peak, count=len(live), lens=lens, cu=cu,
                slots=slots + [-1] * (tokens - len(slots)), positions=positions + [-1] * (tokens - len(slots)),
                src=[a for a, _ in mv] + [-1] * (moves - len(mv)), dst=[b for _, b in mv] + [-1] * (moves - len(mv)), moves=len(mv))


@pytest.mark.parametrize("groups,per_group,longest,grow,seed", [(1, 1, 1, 3, 0), (1, 1, 5000, 70, 1), (1, 7, 300, 3, 2), (5, 4, 700, 1, 3), (16, 4, 130, 200, 4), (40, 8, 200, 1, 5),
                                                                (300, 4, 100, 2, 6), (2048, 4, 65, 1, 7), (2, 2, 200 * 64, 5, 8)])
@pytest.mark.parametrize("in_place", [False, True])
def test_share_equals_the_lists(groups, per_group, longest, grow, seed, in_place):
    rng = random.Random(seed)
    for _ in range(1 if groups > 1000 else 4):
        s = Rows(rng, groups, per_group, longest, spare=0)
        source, keep, new = wishes(rng, s, grow)
        room = sum(pages(n) for n in new)                     # enough, then exactly enough
        s.stack += [s.n_pages + i for i in range(room)]
        s.refs += [0] * room
        s.n_pages += room
        tokens, moves = sum(new) - sum(keep) + 3, 63 * len(new) + 2
        want = share(source, s.lens, keep, new, s.table, s.refs, s.stack, s.n_pages, s.width)
        got, st = run_share(source, s.lens, keep, new, s.table, s.refs, s.stack, s.n_pages, tokens, moves, in_place)
        assert st == 0
        e = expect(want, s, new, tokens, moves)
        got["free"] = got["free"][:len(e["free"])]
        for name in e:
            assert got[name] == e[name], name
        spare = len(want[3])
        if spare:                                             # with the lowest `spare` pages of the stack gone it is exactly enough
            gone = s.stack[:spare]
            stack = s.stack[spare:]
            want = share(source, s.lens, keep, new, s.table, s.refs, stack, s.n_pages, s.width)
            if want != "nomem":
                got, st = run_share(source, s.lens, keep, new, s.table, s.refs, stack, s.n_pages, tokens, moves, in_place)
                assert st == 0 and got["table"] == [row + [-5] * (s.width - len(row)) for row in want[0]] and got["refs"] == want[1] and got["count"] == len(want[3])
                assert not set(gone) & {p for row in want[0] for p in row}


def test_share_refused_as_a_whole():
    rng = random.Random(3)
    s = Rows(rng, 3, 4, 300, spare=4)
    R = len(s.lens)
    base = dict(source=list(range(R)), keep=list(s.lens), new=[n + 1 for n in s.lens])

    def attempt(code, tokens=R + 2, moves=64 * R, stack=None, **kw):
        a = {k: list(v) for k, v in base.items()}
        for name, (i, v) in kw.items():
            a[name][i] = v
        stack = s.stack if stack is None else stack
        for in_place in (False, True):
            got, st = run_share(a["source"], s.lens, a["keep"], a["new"], s.table, s.refs, stack, s.n_pages, tokens, moves, in_place)
            assert st == code
            if code:
                assert got["table"] == [row[:pages(n)] + [-5] * (s.width - pages(n)) for row, n in zip(s.table, s.lens)]
                assert got["refs"] == s.refs and got["count"] == len(stack) and got["free"][:len(stack)] == stack and got["lens"] == s.lens
                assert got["cu"] == [0] * (R + 1) and got["slots"] == got["positions"] == [-1] * tokens and got["src"] == got["dst"] == [-1] * moves and got["moves"] == 0

    longest = max(range(R), key=lambda r: s.lens[r])
    plain = share(base["source"], s.lens, base["keep"], base["new"], s.table, s.refs, s.stack, s.n_pages, s.width)
    assert plain == "nomem"                                   # (and nothing is wrong with the lengths)
    attempt(binding.E_NOMEM)
    attempt(binding.E_ARG, source=(0, R))
    attempt(binding.E_ARG, source=(0, -2))
    attempt(binding.E_ARG, keep=(longest, s.lens[longest] + 1))
    attempt(binding.E_ARG, keep=(0, -1))
    attempt(binding.E_ARG, new=(longest, s.lens[longest] - 1))
    attempt(binding.E_ARG, new=(0, s.width * PAGE + 1))
    attempt(binding.E_ARG, new=(0, 2 ** 31 - 1))
    attempt(binding.E_ARG, source=(longest, -1))              # nothing to keep entries of
    attempt(binding.E_ARG, tokens=R - 1)
    attempt(binding.E_NOMEM, stack=[], new=(longest, s.width * PAGE), tokens=s.width * PAGE + R)
    # forks of a partly filled page: every row goes on from the longest one, so all but one copy its rows
    n = s.lens[longest] - (0 if s.lens[longest] % PAGE else 1)
    fork = dict(source=[longest] * R, keep=[n] * R, new=[n + 1] * R)
    base.update(fork)
    attempt(binding.E_NOMEM, stack=[])
    attempt(binding.E_ARG, moves=(R - 1) * (n % PAGE) - 1, stack=s.stack + [p for p in range(s.n_pages) if s.refs[p] == 0 and p not in s.stack])


def test_share_bad_pages_are_latched():
    table = [[0, 99, -9], [1, -9, -9], [-9, -9, -9]]
    got, st = run_share([0, 1, 0], [100, 64, 0], [100, 0, 100], [101, 0, 102], table, [1, 1, 0, 0], [2, 3], 4, 4, 200)
    assert st == binding.E_ARG
    assert got["table"][0] == [0, -1, -5] and got["table"][2] == [0, -1, -5] and got["slots"] == [-1, -1, -1, -1]
    assert got["refs"] == [2, 0, 0, 0] and got["count"] == 3 and got["free"][:3] == [2, 3, 1] and got["moves"] == 0
    got, st = run_share([0], [0], [0], [130], [[-9, -9, -9]], [0, 0, 0], [7, -3, 1], 3, 130, 0)      # a stack that holds no pages
    assert st == binding.E_ARG
    assert got["table"][0] == [1, -1, -1]


# ---------------------------------------------------------------- compact

def bits_of(kept, width, junk=None):
    words = [[0] * width for _ in kept]
    for row, keep in zip(words, kept):
        for e in keep:
            if e < width * PAGE:
                row[e // PAGE] |= 1 << (e % PAGE)
    return torch.tensor([[w - (1 << 64) if w >> 63 else w for w in row] for row in words], dtype=torch.int64, device=DEV)


def run_compact(lens, kept, table, refs, stack, n_pages, width, moves, in_place=False):
    t, fr, fc = ints(table), ints(stack + [-4] * (n_pages - len(stack))), ints([len(stack)])
    rf = None if refs is None else ints(refs)
    out = torch.full_like(t, -5)
    ro, fo, co = (rf, fr, fc) if in_place else (None if refs is None else filled(n_pages), filled(n_pages), filled(1))
    n, src, dst, count, st = filled(len(lens)), filled(moves), filled(moves), filled(1), torch.zeros(1, dtype=I32, device=DEV)
    binding.paged_compact(ints(lens), bits_of(kept, width), t, out, rf, ro, fr, fo, fc, co, n, src, dst, count, st)
    return dict(table=out.tolist(), refs=None if refs is None else ro.tolist(), free=fo.tolist(), count=co.item(), lens=n.tolist(), src=src.tolist(), dst=dst.tolist(),
                moves=count.item()), st.item()


def random_kept(rng, n):
    kind = rng.choice("all none front end thin half one first".split())
    if kind == "all":
        return list(range(n + 5))
    if kind == "none":
        return list(range(n, n + 70))
    if kind == "front":
        return list(range(rng.randint(0, n)))
    if kind == "end":
        return list(range(rng.randint(0, n), n))
    if kind == "one":
        return [rng.randint(0, n)] if n else []
    if kind == "first":
        return [e for e in range(n) if e != rng.randint(0, n)]
    return [e for e in range(n + 9) if rng.random() < (0.05 if kind == "thin" else 0.5)]


@pytest.mark.parametrize("groups,per_group,longest,seed,width", [(1, 1, 1, 0, None), (1, 1, 5000, 1, None), (3, 2, 700, 2, None), (20, 4, 300, 3, None), (500, 3, 150, 4, None),
                                                                 (4096, 2, 66, 5, None), (2, 1, 300 * 64, 6, None), (2, 1, 900, 7, 2500), (70, 1, 200, 8, 2100)])
@pytest.mark.parametrize("with_refs", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_compact_equals_the_lists(groups, per_group, longest, seed, width, with_refs, in_place):
    rng = random.Random(seed)
    for _ in range(1 if groups > 1000 else 4):
        s = Rows(rng, groups, per_group, longest, spare=0, shared=with_refs, holders=with_refs, width=width)
        kept = [random_kept(rng, n) for n in s.lens]
        room = sum(pages(n) for n in s.lens) + 1
        s.stack += [s.n_pages + i for i in range(room)]
        s.refs += [0] * room
        s.n_pages += room
        refs, moves = s.refs if with_refs else None, sum(s.lens) + 3
        want = compact(s.lens, kept, s.table, refs, s.stack, s.n_pages, s.width)
        rows, wrefs, live, lens, mv, memory = want
        got, st = run_compact(s.lens, kept, s.table, refs, s.stack, s.n_pages, s.width, moves, in_place)
        assert st == 0
        assert got["lens"] == lens
        assert got["table"] == [row + [-5] * (s.width - len(row)) for row in rows]
        assert got["refs"] == wrefs and got["count"] == len(live) and got["free"][:len(memory)] == memory
        assert got["moves"] == len(mv) and got["src"] == [a for a, _ in mv] + [-1] * (moves - len(mv)) and got["dst"] == [b for _, b in mv] + [-1] * (moves - len(mv))


@pytest.mark.parametrize("rows,longest,width,seed", [(16, 130 * 64, 140, 0), (17, 2000, 260, 1), (40, 260 * 64, 300, 2), (150, 900, 130, 3), (513, 100, 129, 4)])
def test_compact_of_rows_by_several_warps(rows, longest, width, seed):
    rng = random.Random(seed)
    s = Rows(rng, rows, 1, longest, spare=0, shared=False, holders=False, width=width)
    kept = [random_kept(rng, n) for n in s.lens]
    room = sum(pages(n) for n in s.lens)
    stack, n_pages = s.stack + [s.n_pages + i for i in range(room)], s.n_pages + room
    after, _, live, lens, mv, memory = compact(s.lens, kept, s.table, None, stack, n_pages, width)
    got, st = run_compact(s.lens, kept, s.table, None, stack, n_pages, width, len(mv))
    assert st == 0 and got["lens"] == lens and got["count"] == len(live) and got["free"][:len(memory)] == memory
    assert got["table"] == [row + [-5] * (width - len(row)) for row in after]
    assert got["moves"] == len(mv) and got["src"] == [a for a, _ in mv] and got["dst"] == [b for _, b in mv]


def test_compact_refused_as_a_whole():
    table, lens, kept = [[3, 1, 5], [0, -9, -9]], [150, 20], [list(range(2, 150)), [3, 4]]
    refs, stack = [1, 1, 0, 1, 0, 1, 0, 0], [2, 4, 6, 7]
    for code, change in ((0, {}), (binding.E_ARG, dict(lens=[193, 20])), (binding.E_ARG, dict(lens=[-1, 20])), (binding.E_NOMEM, dict(stack=[2, 4, 6])),
                         (binding.E_ARG, dict(moves=149)), (binding.E_ARG, dict(count=-1)), (binding.E_ARG, dict(count=9))):
        n, stk, moves = change.get("lens", lens), change.get("stack", stack), change.get("moves", 150)
        t, fr, fc, rf = ints(table), ints(stk + [-4] * (8 - len(stk))), ints([change.get("count", len(stk))]), ints(refs)
        out, fo, co, ro, lo = torch.full_like(t, -5), filled(8), filled(1), filled(8), filled(2)
        src, dst, mc, st = filled(moves), filled(moves), filled(1), torch.zeros(1, dtype=I32, device=DEV)
        binding.paged_compact(ints(n), bits_of(kept, 3), t, out, rf, ro, fr, fo, fc, co, lo, src, dst, mc, st)
        assert st.item() == code
        if code:
            assert lo.tolist() == n and ro.tolist() == refs and co.item() == change.get("count", len(stk)) and mc.item() == 0
            assert src.tolist() == dst.tolist() == [-1] * moves
            assert out.tolist()[1] == [0, -5, -5] and out.tolist()[0][:pages(max(n[0], 0))] == table[0][:pages(max(n[0], 0))][:3]
        else:
            assert lo.tolist() == [148, 2] and mc.item() == 150


# ---------------------------------------------------------------- move

@pytest.mark.parametrize("n_moves", [0, 1, 63, 64, 65, 700])
def test_move_copies_rows_of_every_array(n_moves):
    """bf16 and fp32 pages, codes and scales of several row sizes and head counts, odd rows; more arrays than one launch takes."""
    rng = random.Random(n_moves)
    n_pages = 30
    slots = rng.sample(range(n_pages * PAGE), 2 * n_moves)
    src, dst = slots[:n_moves], slots[n_moves:]
    if n_moves > 20:                                          # runs, as the calls before list them; skipped pairs
        src[:15] = range(500, 515)
        dst[:15] = [x for x in range(700, 715)]
        rest = [x for x in range(n_pages * PAGE) if not 500 <= x < 515 and not 700 <= x < 715]
        rng.shuffle(rest)
        src[15:], dst[15:] = rest[:n_moves - 15], rest[n_moves - 15:2 * (n_moves - 15)]
        src[17] = dst[17] = -1
    shapes = [(8, 128, torch.bfloat16), (2, 64, torch.float32), (8, 64, torch.uint8), (8, 8, torch.uint8), (3, 2, torch.uint8), (1, 12, torch.uint8), (5, 3, torch.uint8), (2, 256, torch.float32),
              (4, 16, torch.uint8)]
    for copies in (1, 15):
        arrays = [torch.randint(0, 256, (n_pages, h, PAGE, w * t.itemsize), dtype=torch.uint8, device=DEV).view(t) for h, w, t in shapes * copies]
        before = [a.view(torch.uint8).clone() for a in arrays]
        st = torch.zeros(1, dtype=I32, device=DEV)
        binding.paged_move(arrays, ints(src + [7, 7]), ints(dst + [9, 9]), ints([n_moves]), status=st)
        assert st.item() == 0
        s, d = (torch.tensor([x for x in v if x >= 0], dtype=torch.long, device=DEV) for v in (src, dst))
        for a, b in zip(arrays, before):
            want = b.clone()
            want[d // PAGE, :, d % PAGE] = b[s // PAGE, :, s % PAGE]
            assert torch.equal(a.view(torch.uint8), want)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64), (torch.bfloat16, 8), (torch.float32, 256)])
def test_move_makes_bounds_of_completed_pages(dtype, d):
    H, n_pages = 3, 8
    gen = torch.Generator().manual_seed(d)
    k = torch.randn(n_pages, H, PAGE, d, generator=gen).to(dtype)
    k[5, 1, 7, 2] = float("nan")
    k = k.to(DEV)
    arrays, bounds = [k, k.clone(), k.clone()], [torch.full((n_pages, H, 2, d), 5.0, dtype=dtype, device=DEV), None, torch.full((n_pages, H, 2, d), 5.0, dtype=dtype, device=DEV)]
    # page 1 entirely, page 2 its last rows only, page 3 not its last row
    src = [5 * PAGE + e for e in range(64)] + [4 * PAGE + e for e in range(10, 40)] + [6 * PAGE, 6 * PAGE + 1]
    dst = [1 * PAGE + e for e in range(64)] + [2 * PAGE + e for e in range(34, 64)] + [3 * PAGE, 3 * PAGE + 62]
    st = torch.zeros(1, dtype=I32, device=DEV)
    binding.paged_move(arrays, ints(src + [-1] * 40), ints(dst + [-1] * 40), ints([len(src)]), key_bounds=bounds, status=st)
    assert st.item() == 0
    for a, b in ((arrays[0], bounds[0]), (arrays[2], bounds[2])):
        for p in range(n_pages):
            if p not in (1, 2):
                assert (b[p] == 5).all()
                continue
            lo, hi = a[p].float().amin(1), a[p].float().amax(1)
            assert torch.equal(torch.nan_to_num(b[p, :, 0].float(), nan=9e9), torch.nan_to_num(lo, nan=9e9))
            assert torch.equal(torch.nan_to_num(b[p, :, 1].float(), nan=9e9), torch.nan_to_num(hi, nan=9e9))


def test_move_makes_bounds_of_arrays_with_different_heads():
    gen, n_pages = torch.Generator().manual_seed(1), 6
    arrays = [torch.randn(n_pages, h, PAGE, 64, generator=gen).to(DEV, torch.bfloat16) for h in (1, 9, 4, 16)]
    bounds = [torch.full((n_pages, a.shape[1], 2, 64), 7.0, dtype=a.dtype, device=DEV) for a in arrays]
    src, dst = list(range(100)), [3 * PAGE + e for e in range(20, 120)]
    binding.paged_move(arrays, ints(src), ints(dst), ints([100]), key_bounds=bounds)
    for a, b in zip(arrays, bounds):
        assert torch.equal(b[3, :, 0], a[3].amin(1)) and torch.equal(b[3, :, 1], a[3].amax(1))
        assert (b[[0, 1, 2, 4, 5]] == 7).all()


def test_move_skips_what_does_not_exist():
    a = torch.arange(2 * PAGE, dtype=torch.float32, device=DEV).view(2, 1, PAGE, 1).expand(2, 1, PAGE, 4).contiguous()
    for pair in ((-1, 5), (5, -1), (128, 3), (3, 128), (-7, 2), (1 << 30, 4)):
        b, st = a.clone(), torch.zeros(1, dtype=I32, device=DEV)
        binding.paged_move([b], ints([pair[0], 70]), ints([pair[1], 9]), ints([2]), status=st)
        want = a.clone()
        want[0, 0, 9] = a[1, 0, 6]
        assert st.item() == binding.E_ARG and torch.equal(b, want)
    for count in (-3, 3):                                     # more pairs than there is room for, fewer than none
        b, st = a.clone(), torch.zeros(1, dtype=I32, device=DEV)
        binding.paged_move([b], ints([70, 71]), ints([9, 10]), ints([count]), status=st)
        assert st.item() == binding.E_ARG and torch.equal(b[0, 0, 9], a[1, 0, 6] if count > 0 else a[0, 0, 9])


def test_move_takes_rows_by_shape_where_a_dimension_is_one():
    """One head: its stride says nothing about the rows."""
    a = torch.randn(4, PAGE, 1, 128, device=DEV).transpose(1, 2)
    assert a.is_contiguous() and a.stride(1) != PAGE * 128
    want = a.clone()
    want[3, :, 9] = a[1, :, 6]
    binding.paged_move([a], ints([PAGE + 6]), ints([3 * PAGE + 9]), ints([1]))
    assert torch.equal(a, want)


# ---------------------------------------------------------------- together

def test_fork_append_attend_compact_over_a_cache_in_4_bits():
    """Two prompts are appended, forked into samples, grown over several steps (rows that share a partly filled page get their own), thinned by
    keep bits and grown again, in two layers, on a stream of their own; at every step attention equals that over a dense copy of each request."""
    H, g, d, layers, width = 2, 4, 64, 2, 8
    n_pages, R, cap = 60, 6, width * PAGE
    gen = torch.Generator().manual_seed(0)
    stream = torch.cuda.Stream()
    arrays = [[torch.zeros(n_pages, H, PAGE, w, dtype=torch.uint8, device=DEV) for w in (d // 2, d // 16, d // 2, d // 16)] for _ in range(layers)]
    caches = [binding.Paged4Cache(*a) for a in arrays]
    flat = [x for a in arrays for x in a]
    state = dict(table=torch.full((R, width), -9, dtype=I32, device=DEV), refs=filled(n_pages, 0), free=torch.arange(n_pages, dtype=I32, device=DEV), fc=ints([n_pages]),
                 lens=filled(R, 0))
    dense = [[[] for _ in range(R)] for _ in range(layers)]   # per layer and row: [(k, v)] fp64 values per entry
    mirror = [0] * R
    st = torch.zeros(1, dtype=I32, device=DEV)
    ws = torch.empty(binding.paged4_workspace_bytes(H * g, H, d), dtype=torch.uint8, device=DEV)

    def step(source, keep, new):
        tokens = sum(new) - sum(keep)
        cu, slots, pos = filled(R + 1), filled(tokens), filled(tokens)
        src, dst, count = filled(64 * R), filled(64 * R), filled(1)
        out, ro, fo, co, lo = torch.full_like(state["table"], -9), filled(n_pages), filled(n_pages), filled(1), filled(R)
        binding.paged_share(ints(source), state["lens"], ints(keep), ints(new), state["table"], out, state["refs"], ro, state["free"], fo, state["fc"], co, lo, cu, slots, pos,
                            src, dst, count, st)
        binding.paged_move(flat, src, dst, count, status=st)
        state.update(table=out, refs=ro, free=fo, fc=co, lens=lo)
        old = [list(map(list, dense[l])) for l in range(layers)]
        cul = [0]
        for r in range(R):
            cul.append(cul[-1] + new[r] - keep[r])
        for l in range(layers):
            kv = torch.randn(tokens, 2, H, d, generator=gen).to(torch.bfloat16)
            dev = kv.to(DEV)
            binding.paged4_append(caches[l], dev[:, 0], dev[:, 1], slots, status=st)
            vals = []
            for x in range(2):
                codes, scale = quantise(kv[:, x], torch.zeros(H))
                vals.append(values(pack(codes)[:, :, None], scale.to(torch.uint8)[:, :, None], torch.zeros(H))[:, :, 0])
            for r in range(R):
                dense[l][r] = (old[l][source[r]][:keep[r]] if source[r] >= 0 else []) + [(vals[0][t], vals[1][t]) for t in range(cul[r], cul[r + 1])]
        mirror[:] = new
        attend(cu, cul)

    def attend(cu, cul):
        for l in range(layers):
            q = torch.randn(cul[-1], H * g, d, generator=gen).to(torch.bfloat16).to(DEV)
            out = binding.paged4_attention(caches[l], q, cu, state["lens"], state["table"], 0, workspace=ws, status=st)
            k = torch.zeros(R * width, H, PAGE, d, dtype=torch.float64)
            v, table = torch.zeros_like(k), torch.arange(R * width).view(R, width)
            for r in range(R):
                for e, (a, b) in enumerate(dense[l][r]):
                    k[r * width + e // PAGE, :, e % PAGE], v[r * width + e // PAGE, :, e % PAGE] = a, b
            want, bound = attention(k, v, q, cul, list(mirror), table, d ** -0.5)
            assert ((out.double().cpu() - want).abs() <= bound).all()
        assert st.item() == 0

    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step([-1] * R, [0] * R, [100, 64, 0, 0, 0, 0])                          # two prompts
        step([0, 1, 0, 0, 1, -1], [100, 64, 100, 90, 64, 0], [101, 65, 101, 95, 64, 3])      # samples, one from an earlier place
        step([2, 1, 2, 0, 0, 5], [101, 65, 101, 101, 64, 3], [102, 66, 103, 102, 130, 4])    # beams
        kept = [[e for e in range(n) if (e * 7 + r) % 3] for r, n in enumerate(mirror)]
        out, ro, fo, co, lo = torch.full_like(state["table"], -9), filled(n_pages), filled(n_pages), filled(1), filled(R)
        src, dst, count = filled(sum(mirror)), filled(sum(mirror)), filled(1)
        binding.paged_compact(state["lens"], bits_of(kept, width), state["table"], out, state["refs"], ro, state["free"], fo, state["fc"], co, lo, src, dst, count, st)
        binding.paged_move(flat, src, dst, count, status=st)
        state.update(table=out, refs=ro, free=fo, fc=co, lens=lo)
        for l in range(layers):
            dense[l] = [[row[e] for e in keep] for row, keep in zip(dense[l], kept)]
        mirror[:] = [len(keep) for keep in kept]
        step(list(range(R)), list(mirror), [n + 2 for n in mirror])
        step([0, 0, 0, 3, 4, -1], [10, 60, mirror[0], 0, 0, 0], [11, 64, mirror[0] + 70, 0, 1, 0])
    torch.cuda.synchronize()
    held = {p for row, n in zip(state["table"].tolist(), mirror) for p in row[:pages(n)]}
    assert state["fc"].item() + len(held) == n_pages and not held & set(state["free"].tolist()[:state["fc"].item()])
    assert [r > 0 for r in state["refs"].tolist()] == [p in held for p in range(n_pages)]


def test_captured_share_and_compact_replay():
    """One captured graph serves every step: lengths and keep bits are changed in place between the replays."""
    R, width, n_pages = 4, 6, 64
    s = dict(source=ints([0, 0, 0, 0]), old=ints([70, 0, 0, 0]), keep=ints([70] * 4), new=ints([71] * 4), table=ints([[5, 9] + [0] * 4] + [[0] * 6] * 3))
    refs = [0] * n_pages
    refs[5] = refs[9] = 1
    free = [p for p in range(n_pages) if p not in (5, 9)]
    args = [s["source"], s["old"], s["keep"], s["new"], s["table"], torch.zeros_like(s["table"]), ints(refs), filled(n_pages), ints(free + [0, 0]), filled(n_pages), ints([62]), filled(1),
            filled(R), filled(R + 1), filled(16), filled(16), filled(256), filled(256), filled(1), filled(1, 0)]
    binding.paged_share(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.paged_share(*args)
    for keep, new in (([70] * 4, [71] * 4), ([64] * 4, [65, 64, 66, 64]), ([10, 20, 70, 0], [11, 24, 70, 0])):
        s["keep"].copy_(ints(keep)), s["new"].copy_(ints(new))
        graph.replay()
        torch.cuda.synchronize()
        want = share([0] * 4, [70, 0, 0, 0], keep, new, [[5, 9] + [0] * 4] + [[0] * 6] * 3, refs, free, n_pages, width)
        assert [row[:pages(n)] for row, n in zip(args[5].tolist(), new)] == want[0] and args[7].tolist() == want[1] and args[11].item() == len(want[3])
        assert args[18].item() == len(want[8]) and args[19].item() == 0

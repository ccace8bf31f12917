"""Calls on one table after another on the GPU: a table of the plan that goes over to counted pages, keep bits as the selection writes them, what
positions and windows mean after entries were dropped."""
import random

import pytest
import torch

from paper_2605_09649_b200 import binding
from test_gpu_paged_share import DEV, I32, filled, ints, run_compact, run_share
from util_paged import PAGE, pages
from util_paged4 import Cache4, attention, values
from util_paged_share import share

pytestmark = pytest.mark.gpu


def test_compact_takes_the_bits_that_the_selection_writes():
    """The highest scores of each row's entries, by trimkv_select_topk row by row, kept by trimkv_paged_compact."""
    lens, budget, width, n_pages = [700, 64, 130, 5], [200, 64, 7, 3], 12, 40
    gen = torch.Generator().manual_seed(1)
    scores = [torch.randn(n, generator=gen) for n in lens]
    bits = torch.zeros(len(lens), width, dtype=torch.int64, device=DEV)
    for r, (s, k) in enumerate(zip(scores, budget)):
        words, _ = binding.select_topk(s.to(DEV), k)
        bits[r, :words.numel()] = words
    order = list(range(n_pages))
    random.Random(1).shuffle(order)
    table, at = [], 0
    for n in lens:
        table.append(order[at:at + pages(n)] + [-9] * (width - pages(n)))
        at += pages(n)
    kept = [sorted(torch.topk(s, k).indices.tolist()) for s, k in zip(scores, budget)]
    moves = sum(lens)
    got, st = run_compact(lens, kept, table, None, order[at:], n_pages, width, moves)
    assert st == 0
    t, fr, fc = ints(table), ints(order[at:] + [-4] * at), ints([n_pages - at])
    out, fo, co, lo = torch.full_like(t, -5), filled(n_pages), filled(1), filled(len(lens))
    src, dst, count, status = filled(moves), filled(moves), filled(1), torch.zeros(1, dtype=I32, device=DEV)
    binding.paged_compact(ints(lens), bits, t, out, None, None, fr, fo, fc, co, lo, src, dst, count, status)
    assert status.item() == 0 and lo.tolist() == budget
    assert out.tolist() == got["table"] and src.tolist() == got["src"] and dst.tolist() == got["dst"] and fo.tolist()[:co.item()] == got["free"][:got["count"]]


def test_positions_and_windows_count_entries_after_compact():
    """A row that keeps 40 of 200 entries goes on at position 40, and a window of 30 is its newest 30 entries, whatever tokens they were."""
    H, g, d, width = 1, 4, 64, 4
    c = Cache4([200], H, d, seed=40, spare=6, width=width)
    kept = list(range(0, 200, 5))
    held = c.table[0].tolist()
    free = [p for p in range(c.n_pages) if p not in held]
    t, n_pages = c.table.clone(), c.n_pages
    bits = torch.zeros(1, width, dtype=torch.int64)
    for e in kept:
        bits[0, e // PAGE] |= (1 << e % PAGE) - (1 << 64 if e % PAGE == 63 else 0)
    refs = ints([1 if p in held else 0 for p in range(n_pages)])
    out, ro, fo, co, lo = torch.full_like(t, -5), filled(n_pages), filled(n_pages), filled(1), filled(1)
    src, dst, count = filled(64), filled(64), filled(1)
    st = torch.zeros(1, dtype=I32, device=DEV)
    binding.paged_compact(c.lens, bits.to(DEV), t, out, refs, ro, ints(free + [-4] * len(held)), fo, ints([len(free)]), co, lo, src, dst, count, st)
    flat = [c.arrays[i] for i in (0, 1, 3, 4)]
    binding.paged_move(flat, src, dst, count, status=st)
    table2, ro2, fo2, co2, lo2 = torch.full_like(t, -5), filled(n_pages), filled(n_pages), filled(1), filled(1)
    cu, slots, pos = filled(2), filled(2), filled(2)
    binding.paged_share(ints([0]), lo, lo, lo + 2, out, table2, ro, ro2, fo, fo2, co, co2, lo2, cu, slots, pos, src, dst, count, st)
    assert pos.tolist() == [40, 41] and lo2.tolist() == [42] and st.item() == 0
    kv = torch.randn(2, 2, H, d, device=DEV, dtype=torch.bfloat16)
    binding.paged4_append(c.cache(), kv[0], kv[1], slots, status=st)
    k, v = values(*c.arrays[:3]), values(*c.arrays[3:])
    page = int(table2[0, 0])
    old = c.table[0].tolist()
    for i, e in enumerate(kept):                              # (c.k and c.v: as the cache was)
        assert torch.equal(k[page, 0, i], c.k[old[e // PAGE], 0, e % PAGE]) and torch.equal(v[page, 0, i], c.v[old[e // PAGE], 0, e % PAGE])
    q = torch.randn(2, g, d, device=DEV, dtype=torch.bfloat16)
    got = binding.paged4_attention(c.cache(), q, cu, lo2, table2, 2, window=30, status=st)
    want, bound = attention(k, v, q, [0, 2], [42], table2, d ** -0.5, 30)
    assert st.item() == 0 and ((got.double().cpu() - want).abs() <= bound).all()


def test_a_table_of_the_plan_goes_over_with_counts_of_one():
    """Three requests are planned; their pages are counted once each; from there on rows are forked and ended by counts."""
    lens, width, n_pages = [130, 64, 5, 0], 5, 12
    table, free, count = torch.full((4, width), -9, dtype=I32, device=DEV), torch.arange(n_pages, dtype=I32, device=DEV), ints([n_pages])
    out, cu, slots, st = filled(4), filled(5), filled(sum(lens)), torch.zeros(1, dtype=I32, device=DEV)
    binding.paged_plan(ints([0] * 4), None, ints(lens), table, free, count, count, out, cu, slots, None, st)
    rows, stack = table.tolist(), free.tolist()[:count.item()]
    refs = [0] * n_pages
    for row, n in zip(rows, lens):
        for p in row[:pages(n)]:
            refs[p] += 1
    assert st.item() == 0 and max(refs) == 1 and sum(refs) + len(stack) == n_pages
    for source, keep, new in (([0, 0, -1, 0], [130, 128, 0, 100], [131, 130, 0, 128]), ([-1, 1, 0, 3], [0, 64, 60, 5], [0, 65, 61, 5])):
        want = share(source, lens, keep, new, rows, refs, stack, n_pages, width)
        got, status = run_share(source, lens, keep, new, rows, refs, stack, n_pages, sum(new) - sum(keep), 63 * 4)
        assert status == 0 and [row[:pages(n)] for row, n in zip(got["table"], new)] == want[0] and got["refs"] == want[1]
        assert got["free"][:got["count"]] == want[3] and got["positions"] == want[6 + 1] and got["moves"] == len(want[8])
        rows, refs, stack, lens = got["table"], got["refs"], got["free"][:got["count"]], got["lens"]


def test_compact_says_when_more_pages_come_back_than_there_are():
    """Two rows hold a page without counts: it comes back twice, and the stack has no room for the second."""
    got, st = run_compact([64, 64], [[], []], [[3], [3]], None, [0, 1, 2], 4, 1, 0)
    assert st == binding.E_ARG and got["count"] == 4 and got["free"] == [0, 1, 2, 3] and got["lens"] == [0, 0]
    got, st = run_compact([64, 64], [[], []], [[3], [2]], None, [0, 1], 4, 1, 0)
    assert st == 0 and got["count"] == 4 and got["free"] == [0, 1, 3, 2]

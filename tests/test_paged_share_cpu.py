"""Shared, compacted and moved pages without a GPU: refusals of the C entry points, the binding's checks, and invariants of the lists that
the GPU tests compare with."""
import ctypes as C
import random

import pytest
import torch

from paper_2605_09649_b200 import binding
from util_paged import PAGE, pages
from util_paged_share import Rows, compact, share

OK16 = 1 << 20            # an aligned address that is never followed
OUT = OK16 + 4096


def share_args(**kw):
    a = dict(n_req=2, source=OK16, old=OK16, keep=OK16, new=OK16, table=OK16, table_out=OUT, width=4, refs=OK16, refs_out=OK16, free=OK16, free_out=OK16, n_pages=4,
             count=OK16, count_out=OK16, max_tokens=4, lens=OUT, cu=OUT, slots=OUT, positions=OUT, max_moves=4, src=OUT, dst=OUT, moves=OUT, status=OK16, stream=None)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


def compact_args(**kw):
    a = dict(n_req=2, lens_in=OK16, bits=OK16, table=OK16, table_out=OUT, width=4, refs=OK16, refs_out=OK16, free=OK16, free_out=OK16, n_pages=4, count=OK16, count_out=OK16,
             lens=OUT, max_moves=4, src=OUT, dst=OUT, moves=OUT, status=OK16, stream=None)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


def refused(fn, args, code=binding.E_ARG):
    assert getattr(binding.lib(), fn)(*args) == code, binding.last_error()
    assert binding.last_error()


SHARED = [dict(n_req=0), dict(n_req=8193), dict(width=0), dict(width=16385), dict(n_pages=0), dict(n_pages=(1 << 24) + 1), dict(max_moves=-1), dict(max_moves=(1 << 30) + 1), dict(table=None),
          dict(table_out=None), dict(table_out=OK16), dict(refs_out=None), dict(refs=None), dict(free=None), dict(free_out=None), dict(count=None), dict(count_out=None), dict(lens=None),
          dict(src=None), dict(dst=None), dict(moves=None), dict(table=OK16 + 2), dict(refs=OK16 + 1), dict(src=OUT + 2), dict(status=OK16 + 3)]


@pytest.mark.parametrize("kw", SHARED + [dict(max_tokens=-1), dict(max_tokens=(1 << 30) + 1), dict(source=None), dict(old=None), dict(keep=None), dict(new=None), dict(cu=None), dict(slots=None),
                                         dict(source=OK16 + 2), dict(positions=OUT + 2)])
def test_share_refusals(kw):
    refused("trimkv_paged_share", share_args(**kw))


@pytest.mark.parametrize("kw", SHARED + [dict(lens_in=None), dict(bits=None), dict(bits=OK16 + 4)])
def test_compact_refusals(kw):
    refused("trimkv_paged_compact", compact_args(**kw))


def rows(n=1, **kw):
    a = (binding.PagedRows * max(n, 1))()
    for x in a:
        x.pages, x.key_bounds, x.heads, x.row_bytes, x.dtype = OK16, None, 2, 128, 0
    for name, v in kw.items():
        setattr(a[max(n, 1) - 1], name, v)
    return a


def move_args(arrays=None, **kw):
    a = dict(n=1, arrays=C.cast(rows() if arrays is None else arrays, C.c_void_p), n_pages=4, max_moves=4, src=OK16, dst=OK16, count=OK16, status=OK16, stream=None)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


@pytest.mark.parametrize("kw", [dict(n=-1), dict(n=1025), dict(arrays=0), dict(n_pages=0), dict(n_pages=(1 << 24) + 1), dict(max_moves=-1), dict(max_moves=(1 << 30) + 1), dict(src=None),
                                dict(dst=None), dict(count=None), dict(src=OK16 + 2), dict(count=OK16 + 1), dict(status=OK16 + 2)])
def test_move_refusals(kw):
    refused("trimkv_paged_move", move_args(**kw))


@pytest.mark.parametrize("kw", [dict(pages=None), dict(pages=OK16 + 8), dict(heads=0), dict(heads=1025), dict(row_bytes=0), dict(row_bytes=4097), dict(reserved=1), dict(key_bounds=OK16 + 4),
                                dict(key_bounds=OK16, dtype=2), dict(key_bounds=OK16, row_bytes=24)])
def test_move_refuses_bad_arrays(kw):
    for n in (1, 3):                                          # the last of them
        refused("trimkv_paged_move", move_args(rows(n, **kw), n=n))


def test_nothing_to_move_is_no_error():
    L = binding.lib()
    assert L.trimkv_paged_move(*move_args(n=0, arrays=0)) == binding.OK
    assert L.trimkv_paged_move(*move_args(max_moves=0, src=None, dst=None, count=None)) == binding.OK


def test_descriptions_and_packed_bytes_agree():
    raw = binding._pack_rows(1, 2, 3, 4, 5, 6)
    assert len(raw) == C.sizeof(binding.PagedRows)
    r = binding.PagedRows.from_buffer_copy(raw)
    assert [getattr(r, name) for name, _ in r._fields_] == [1, 2, 3, 4, 5, 6]


def test_binding_refuses_host_tensors():
    t = torch.zeros(4, dtype=torch.int32)
    for fn, n in ((binding.paged_share, 19), (binding.paged_compact, 14)):
        with pytest.raises(ValueError, match="CUDA"):
            fn(*[t] * n)
    with pytest.raises(ValueError, match="CUDA"):
        binding.paged_move([t], t, t, t)


@pytest.mark.parametrize("seed", range(30))
def test_lists_neither_lose_nor_double_a_page(seed):
    """Counts equal holders, the stack holds exactly the pages without one, no page is written by two rows, moves go to fresh pages."""
    rng = random.Random(seed)
    s = Rows(rng, rng.randint(1, 5), rng.randint(1, 5), rng.choice([3, 200, 500]), spare=0)
    assert sorted(s.stack) == [p for p in range(s.n_pages) if s.refs[p] == 0]
    R = len(s.lens)
    source = [rng.randrange(-1, R) for _ in range(R)]
    keep = [0 if x < 0 else rng.choice([s.lens[x], rng.randint(0, s.lens[x])]) for x in source]
    new = [k + rng.randint(0, 70) for k in keep]
    new = [min(n, s.width * PAGE) for n in new]
    room = sum(pages(n) for n in new)
    n_pages, refs, stack = s.n_pages + room, s.refs + [0] * room, s.stack + list(range(s.n_pages, s.n_pages + room))
    after, got, _, live, _, _, slots, _, moves = share(source, s.lens, keep, new, s.table, refs, stack, n_pages, s.width)
    count = [0] * n_pages
    for p in s.outside + [p for row in after for p in row]:
        count[p] += 1
    assert got == count and sorted(live) == [p for p in range(n_pages) if count[p] == 0]
    assert len(set(slots)) == len(slots) and all(count[x // PAGE] == 1 for x in slots)
    assert len({b for _, b in moves}) == len(moves) and not {a for a, _ in moves} & {b for _, b in moves}
    old_pages = {p for row, n in zip(s.table, s.lens) for p in row[:pages(n)]}
    assert all(a // PAGE in old_pages and count[a // PAGE] for a, _ in moves)
    kept = [[e for e in range(n) if rng.random() < 0.6] for n in new]
    room = sum(pages(n) for n in new)
    n2, refs, stack = n_pages + room, got + [0] * room, live + list(range(n_pages, n_pages + room))
    rows2, got2, live2, lens2, moves2, _ = compact(new, kept, [row + [-9] * s.width for row in after], refs, stack, n2, s.width)
    count = [0] * n2
    for p in s.outside + [p for row in rows2 for p in row]:
        count[p] += 1
    assert got2 == count and sorted(live2) == [p for p in range(n2) if count[p] == 0] and lens2 == [len(k) for k in kept]
    assert not {a // PAGE for a, _ in moves2} & {b // PAGE for _, b in moves2}


@pytest.mark.parametrize("name", ["source", "old", "keep", "new"])
def test_lengths_are_not_written_over_what_is_read(name):
    refused("trimkv_paged_share", share_args(**{name: OUT}))


def test_kept_lengths_are_not_written_over_what_is_read():
    refused("trimkv_paged_compact", compact_args(lens_in=OUT))

"""Plain statements, by lists, of rows that share pages, of dropped entries and of moved rows."""
from __future__ import annotations

import random

from util_paged import PAGE, pages


def share(source, old, keep, new, table, refs, stack, n_pages, width):
    """(rows, refs, stack after the pushes, stack, lens, cu, slots, positions, moves) or the reason of the refusal ("arg", "nomem")."""
    R, cap = len(old), width * PAGE
    for r in range(R):
        s = source[r]
        if not -1 <= s < R or not 0 <= old[r] <= cap or not 0 <= new[r] <= cap:
            return "arg"
        if not 0 <= keep[r] <= min(old[s] if s >= 0 else 0, new[r]):
            return "arg"
    refs = list(refs)
    held = [table[r][:pages(old[r])] for r in range(R)]
    for p in (p for row in held for p in row):
        refs[p] -= 1
    rows, last = [], [None] * R                               # last: the partly filled page that the row will write
    for r in range(R):
        row = list(held[source[r]][:pages(keep[r])]) if source[r] >= 0 else []
        if keep[r] % PAGE and new[r] > keep[r]:
            last[r] = row.pop()
        for p in row:
            refs[p] += 1
        rows.append(row)
    others = list(refs)
    moves_of = [None] * R
    for r in range(R):
        p = last[r]
        if p is None:
            continue
        if others[p] == 0 and refs[p] == 0:                   # nobody else goes on with it, and no lower row writes it
            refs[p] = 1
            rows[r].append(p)
        else:
            moves_of[r] = p
    pushed = []
    for p in (p for row in held for p in row):
        if refs[p] == 0 and p not in pushed:
            pushed.append(p)
    peak = stack + pushed
    need = sum(pages(n) - len(row) for n, row in zip(new, rows))
    if len(peak) > n_pages:
        return "arg"
    if need > len(peak):
        return "nomem"
    live = list(peak)
    for r in range(R):
        while len(rows[r]) < pages(new[r]):
            rows[r].append(live.pop())
            refs[rows[r][-1]] = 1
    cu, slots, positions, moves = [0], [], [], []
    for r in range(R):
        positions += range(keep[r], new[r])
        slots += [rows[r][p // PAGE] * PAGE + p % PAGE for p in range(keep[r], new[r])]
        cu.append(len(slots))
        if moves_of[r] is not None:
            moves += [(moves_of[r] * PAGE + e, rows[r][keep[r] // PAGE] * PAGE + e) for e in range(keep[r] % PAGE)]
    return rows, refs, peak, live, list(new), cu, slots, positions, moves


def compact(lens, kept, table, refs, stack, n_pages, width):
    """(rows, refs, stack, lens, moves, stack's memory) or the reason of the refusal; kept: per row the entries kept, ascending."""
    if any(not 0 <= n <= width * PAGE for n in lens):
        return "arg"
    refs = None if refs is None else list(refs)
    fc, taken = len(stack), 0
    rows, moves, gone = [], [], []
    for r, n in enumerate(lens):
        keep = [e for e in kept[r] if e < n]
        first = next((i for i, e in enumerate(keep) if i != e), len(keep))
        stay = pages(len(keep)) if first == len(keep) else first // PAGE
        row = table[r][:stay]
        for _ in range(pages(len(keep)) - stay):
            taken += 1
            if taken > fc:
                return "nomem"
            row.append(stack[fc - taken])
        if first < len(keep):
            moves += [(table[r][keep[i] // PAGE] * PAGE + keep[i] % PAGE, row[i // PAGE] * PAGE + i % PAGE) for i in range(stay * PAGE, len(keep))]
        gone += table[r][stay:pages(n)]
        if refs is not None:
            for p in row[stay:]:
                refs[p] = 1
        rows.append(row)
    back = list(gone)
    if refs is not None:
        for p in gone:
            refs[p] -= 1
        back = []
        for p in gone:
            if refs[p] == 0 and p not in back:
                back.append(p)
    live = stack[:fc - taken] + back
    return rows, refs, live, [len([e for e in kept[r] if e < n]) for r, n in enumerate(lens)], moves, live + stack[len(live):]


class Rows:
    """Random rows that share pages: groups hold a prompt's full pages together, some pages have a holder outside the table."""

    def __init__(self, rng: random.Random, groups, per_group, longest, spare, shared=True, holders=True, width=None):
        self.rows, self.lens, used = [], [], 0
        for _ in range(groups):
            prompt = rng.randint(0, longest) // PAGE * PAGE if shared else 0
            common = list(range(used, used + prompt // PAGE))
            used += len(common)
            for _ in range(per_group):
                n = rng.choice([prompt, prompt + 1, rng.randint(prompt, max(prompt, longest)), 0])
                row = [] if n < prompt else list(common)
                mine = pages(n) - len(row)
                self.rows.append(row + list(range(used, used + mine)))
                self.lens.append(n)
                used += mine
        self.width = width or pages(longest) + 2
        self.n_pages = used + spare
        name = list(range(self.n_pages))
        rng.shuffle(name)
        self.rows = [[name[p] for p in row] for row in self.rows]
        self.stack = [name[p] for p in range(used, self.n_pages)]
        self.refs = [0] * self.n_pages
        for p in (p for row in self.rows for p in row):
            self.refs[p] += 1
        self.outside = []
        if holders:
            for p in sorted({p for row in self.rows for p in row}):
                if rng.random() < 0.1:
                    self.refs[p] += 1
                    self.outside.append(p)
        # (a prompt that no row holds any more is free)
        lost = [p for p in range(self.n_pages) if self.refs[p] == 0 and p not in self.stack]
        self.stack = lost + self.stack
        self.table = [row + [-9] * (self.width - len(row)) for row in self.rows]

"""Plain 64-bit statements of the paged-cache operators and the error bounds their tests use."""
from __future__ import annotations

import math

import torch

PAGE = 64


def pages(n: int) -> int:
    return (n + PAGE - 1) // PAGE


def plan(old, keep, new, table, free, free_count, max_tokens):
    """The plan by lists: (table, free, free_count, lens, cu_new, slot_map, positions) or None where it is refused."""
    width = len(table[0])
    keep = [min(o, n) for o, n in zip(old, new)] if keep is None else keep
    if any(not 0 <= k <= min(o, n) or max(o, n) > width * PAGE for o, k, n in zip(old, keep, new)):
        return None
    table, free = [list(t) for t in table], list(free)
    stack = free[:free_count]
    for r, (o, n) in enumerate(zip(old, new)):
        stack += table[r][pages(n):pages(o)]
    if len(stack) > len(free) or len(stack) < sum(max(0, pages(n) - pages(o)) for o, n in zip(old, new)):
        return None
    free = stack + free[len(stack):]
    for r, (o, n) in enumerate(zip(old, new)):
        for p in range(pages(o), pages(n)):
            table[r][p] = stack.pop()
    cu, slots, pos = [0], [], []
    for r, (k, n) in enumerate(zip(keep, new)):
        pos += range(k, n)
        slots += [table[r][p // PAGE] * PAGE + p % PAGE for p in range(k, n)]
        cu.append(len(pos))
    if len(pos) > max_tokens:
        return None
    pad = [-1] * (max_tokens - len(pos))
    return table, free, len(stack), list(new), cu, slots + pad, pos + pad


def select(q, bounds, npages, top, sink, recent):
    """Pages that a token reads: q [g, d], bounds [pages, 2, d] in fp64, npages up to its own."""
    if npages <= top:
        return list(range(npages))
    u = torch.maximum(q[:, None] * bounds[None, :, 0], q[:, None] * bounds[None, :, 1]).sum(-1).amax(0)
    free = list(range(sink, npages - recent))
    key = {p: (math.inf if u[p] != u[p] else u[p].item()) for p in free}
    nan_first = sorted(free, key=lambda p: (not bool(u[p] != u[p]), -key[p], p))
    return sorted(list(range(sink)) + list(range(npages - recent, npages)) + nan_first[:top - sink - recent])


def attention(k_pages, v_pages, q, cu, lens, table, scale, window=0, bounds=None, top=0, sink=0, recent=1):
    """(out, bound, selected) in fp64 on the CPU.  bound: largest distance of a correct kernel's output; see `slack`."""
    dt = q.dtype
    k_pages, v_pages, qd = k_pages.double().cpu(), v_pages.double().cpu(), q.double().cpu()
    table = table.cpu().tolist()
    H, d = k_pages.shape[1], k_pages.shape[3]
    T, Hq = q.shape[0], q.shape[1]
    g = Hq // H
    out = torch.full((T, Hq, d), math.nan, dtype=torch.float64)
    bound = torch.zeros_like(out)
    chosen = torch.full((T, H, max(top, 1)), -9, dtype=torch.int32)
    for r, total in enumerate(lens):
        n = cu[r + 1] - cu[r]
        for j in range(n):
            t, pos = cu[r] + j, total - n + j
            for h in range(H):
                rows = slice(h * g, (h + 1) * g)
                qq = qd[t, rows]
                if top:
                    np_ = pos // PAGE + 1 if pos >= 0 else 0
                    b = bounds[[table[r][p] for p in range(np_)], h].double().cpu() if np_ else None
                    sel = select(qq, b, np_, top, sink, recent)
                    chosen[t, h] = torch.tensor(sel + [-1] * (top - len(sel)))
                else:
                    sel = range(pages(pos + 1)) if pos >= 0 else []
                at = [(p, e) for p in sel for e in range(PAGE) if p * PAGE + e <= pos and (not window or p * PAGE + e > pos - window)]
                if not at:
                    out[t, rows] = 0.0
                    continue
                phys = torch.tensor([table[r][p] for p, _ in at])
                off = torch.tensor([e for _, e in at])
                k, v = k_pages[phys, h, off], v_pages[phys, h, off]
                x = qq @ k.T * scale
                wgt = torch.softmax(x, -1)
                o = wgt @ v
                out[t, rows] = o
                bound[t, rows] = slack(dt, o, wgt @ v.abs(), (qq.abs() @ k.abs().T * scale).amax(-1, keepdim=True), len(at), d)
    return out, bound, chosen


def slack(dt, o, mass, logit, n, d):
    """How far a correct output may be from o.  mass = sum w |v|, logit = max over keys of sum |q k| scale, n keys.
    The final rounding takes half a step of o.  A logit is a sum of d products in fp32 and one scaling: off by
    (d + 2) 2^-24 logit; a weight is its exponential, off by twice that (numerator and sum), the 7.5e-5 of the kernels'
    polynomial 2^x (bf16 only; 2 steps of fp32 otherwise), and the n-term fp32 sums.  bf16 rounds every weight before
    it meets V: half a step each, in the numerator and (kernels that sum the rounded weights) in the sum.  Tensor cores
    may truncate instead of rounding a sum's terms: counted by a factor of two on the fp32 terms."""
    step = torch.finfo(dt).eps / 2
    fp32 = 2 * (2 * (d + 2) * logit + n + 16) * 2.0 ** -24
    weights = 2 * step + 1.5e-4 if dt == torch.bfloat16 else 4 * 2.0 ** -24
    return step * o.abs() + (fp32 + weights) * mass + 1e-30


class Cache:
    """A paged cache filled for tests: requests of the given lengths over shuffled pages; everything that no request holds is
    NaN (rows behind the last entry, spare pages), table entries behind the last page are out of range."""

    def __init__(self, lens, H, d, dtype, device="cuda", seed=0, spare=3, width=None, spread=1.0):
        gen = torch.Generator().manual_seed(seed)
        self.n_pages = sum(pages(n) for n in lens) + spare
        self.width = width or max(1, max(pages(n) for n in lens))
        k = torch.full((self.n_pages, H, PAGE, d), math.nan)
        v = torch.full((self.n_pages, H, PAGE, d), math.nan)
        order = torch.randperm(self.n_pages, generator=gen)
        table = torch.full((len(lens), self.width), 1 << 29, dtype=torch.int32)
        at = 0
        bounds = torch.full((self.n_pages, H, 2, d), math.nan)
        for r, n in enumerate(lens):
            for p in range(pages(n)):
                phys = int(order[at])
                at += 1
                table[r, p] = phys
                m = min(PAGE, n - p * PAGE)
                k[phys, :, :m] = torch.randn(H, m, d, generator=gen) * spread + torch.randn(H, 1, d, generator=gen)
                v[phys, :, :m] = torch.randn(H, m, d, generator=gen)
        k, v = k.to(dtype), v.to(dtype)
        for r, n in enumerate(lens):
            for p in range(n // PAGE):
                phys = int(table[r, p])
                bounds[phys, :, 0], bounds[phys, :, 1] = k[phys].float().amin(1), k[phys].float().amax(1)
        self.k, self.v, self.bounds, self.table = (x.to(device) for x in (k, v, bounds.to(dtype), table))
        self.lens = torch.tensor(lens, dtype=torch.int32, device=device)


def queries(new, Hq, d, dtype, device="cuda", seed=0, pad=0, stride=0):
    """(q, cu_new list): q rows `stride` elements apart where > 0; pad rows of NaN behind the last token."""
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    gen = torch.Generator().manual_seed(seed + 77)
    q = torch.full((cu[-1] + pad, Hq, d), math.nan)
    q[:cu[-1]] = torch.randn(cu[-1], Hq, d, generator=gen) * 1.5
    q = q.to(dtype)
    if stride:
        wide = torch.full((q.shape[0], stride), math.nan, dtype=dtype)
        wide[:, :Hq * d] = q.flatten(1)
        return wide.to(device)[:, :Hq * d].unflatten(1, (Hq, d)), cu
    return q.to(device), cu

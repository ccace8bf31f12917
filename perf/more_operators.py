"""Cases of the paged cache held in 4 bits and of the operators that share, compact and move pages.

4-bit cache: k_codes, v_codes uint8 [n_pages, H, 64, d / 2] (channel 2 i in the low half of byte i), k_scales, v_scales e4m3
[n_pages, H, 64, d / 16], k_shift, v_shift int32 [H].  Sixteen channels of an entry share a scale; a value is
e2m1(code) * scale * 2^shift.  Tables, lengths and slot maps are those of the other paged operators (perf/operators.py).

Sharing: rows of a block table hold pages together and page_refs counts the holders.  With `own` set the calls go to
paper_2605_09649_b200.binding; otherwise the same results come from elementary torch operations in fp32.
"""
import math
import random

import torch

own = False

PAGE = 64
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)      # magnitudes of the eight codes


def listed():
    return [
        # one token for each of 32 dialogues, rounded into the cache and read back
        {"name": "append decode 32", "op": "append", "requests": 32, "length": 2304, "new": 1, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "ragged": False, "shift": False, "lens": 1},
        # prompt chunks of 32 dialogues
        {"name": "append chunks 32x512", "op": "append", "requests": 32, "length": 2048, "new": 512, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "ragged": True, "shift": True, "lens": 2},
        # a small fp32 model's prompt
        {"name": "attention f32 512", "op": "attention", "requests": 1, "length": 512, "new": 512, "kv_heads": 2, "group": 2, "head_dim": 64, "dtype": "f32", "ragged": False, "shift": False, "window": 0, "lens": 3},
        # single tokens over 32K contexts: the bandwidth case
        {"name": "attention decode 8x32k", "op": "attention", "requests": 8, "length": 32768, "new": 1, "kv_heads": 8, "group": 4, "head_dim": 128, "dtype": "bf16", "ragged": False, "shift": True, "window": 0, "lens": 4},
        # drafted tokens scored in one call, 32 dialogues of different lengths
        {"name": "attention drafts 32x5", "op": "attention", "requests": 32, "length": 2304, "new": 5, "kv_heads": 8, "group": 4, "head_dim": 128, "dtype": "bf16", "ragged": True, "shift": True, "window": 0, "lens": 5},
        # prompt chunks of 512 deep inside 16K contexts
        {"name": "attention chunks 4x512", "op": "attention", "requests": 4, "length": 16384, "new": 512, "kv_heads": 8, "group": 4, "head_dim": 128, "dtype": "bf16", "ragged": False, "shift": True, "window": 0, "lens": 6},
        # a step of a beam search: 16 prompts of 4 beams, each beam goes on from any of its prompt's beams
        {"name": "share beams 16x4", "op": "share", "mix": "beams", "groups": 16, "rows": 4, "length": 2304, "new": 1, "lens": 7},
        # 16 samples each of 8 prompts of up to 16K begin
        {"name": "share samples 8x16", "op": "share", "mix": "samples", "groups": 8, "rows": 16, "length": 16384, "new": 1, "lens": 8},
        # one request of 4K drops half of its entries
        {"name": "compact 1x4k", "op": "compact", "groups": 1, "rows": 1, "length": 4096, "keep": 0.5, "refs": False, "lens": 9},
        # 32 requests of up to 32K, two to a prompt, keep an eighth
        {"name": "compact 32x32k", "op": "compact", "groups": 16, "rows": 2, "length": 32768, "keep": 0.125, "refs": True, "lens": 10},
        # the last pages of 32 forked requests, in all 32 layers
        {"name": "move forks 32x32 layers", "op": "move", "mode": "forks", "copies": 32, "layers": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "bounds": False, "lens": 11},
        # 4 requests of up to 4K keep a quarter of their entries, in 8 layers whose key bounds are kept too
        {"name": "move kept 4x4k 8 layers", "op": "move", "mode": "kept", "copies": 4, "length": 4096, "keep": 0.25, "layers": 8, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "bounds": True, "lens": 12},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "attention", "share", "compact", "move"])
    c = {"op": op, "lens": rng.randrange(1 << 30)}
    if op == "share":
        mix = rng.choice(["beams", "samples", "serve"])
        groups = _log(rng, 1, 32)
        rows = _log(rng, 1, max(1, 128 // groups))
        return {**c, "mix": mix, "groups": groups, "rows": rows, "length": _log(rng, 8, 16384), "new": rng.choice([1, 1, 5, _log(rng, 1, 128)])}
    if op == "compact":
        groups = _log(rng, 1, 16)
        return {**c, "groups": groups, "rows": rng.randint(1, 2), "length": _log(rng, 70, 32768), "keep": rng.choice([0.03, 0.125, 0.5, 0.9]), "refs": rng.random() < 0.7}
    heads, group = rng.choice([(8, 4), (4, 7), (8, 8), (2, 2), (1, 8), (3, 5), (8, 1), (2, 16)])
    c["kv_heads"], c["head_dim"] = heads, rng.choice([128, 128, 128, 64, 64, 96, 32, 256])
    c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "move":
        wide = max(1, heads * c["head_dim"] // 1024)
        mode = rng.choice(["forks", "kept"])
        c = {**c, "mode": mode, "layers": _log(rng, 1, 16 // wide), "bounds": rng.random() < 0.5}
        if mode == "forks":
            return {**c, "copies": _log(rng, 1, 32)}
        return {**c, "copies": rng.randint(1, 4), "length": _log(rng, 64, 2048), "keep": rng.choice([0.1, 0.25, 0.6])}
    c["ragged"], c["shift"] = rng.random() < 0.7, rng.random() < 0.5
    if op == "append":
        new = _log(rng, 1, 512)
        r = _log(rng, 1, max(1, 4096 // new))
        return {**c, "requests": r, "new": new, "length": new + _log(rng, 1, 2048)}
    c["group"] = group
    kind = rng.choice(["decode", "decode", "drafts", "chunk"])
    if kind == "chunk":
        new, length = _log(rng, 32, 1024), _log(rng, 64, 8192)
        r = _log(rng, 1, max(1, min(8, (1 << 22) // (new * max(new, length)))))
        if c["dtype"] == "f32":
            new, length, r = min(new, 256), min(length, 2048), min(r, 2)
    else:
        new = 1 if kind == "decode" else rng.randint(2, 9)
        length = _log(rng, 1, 32768)
        r = _log(rng, 1, max(1, min(64, 131072 // length)))
        if c["dtype"] == "f32":
            length, r = min(length, 8192), min(r, 8)
    return {**c, "requests": r, "new": new, "length": max(length, new), "window": rng.choice([0, 0, 0, _log(rng, 16, 4096)])}


# ---------------------------------------------------------------- host-side facts of a case

def _lengths(case):
    """(cached tokens after the call, new tokens) of each request: a property of the case, not of the seed."""
    rng = random.Random(case["lens"])
    lens, new = [], []
    for _ in range(case["requests"]):
        n, total = case["new"], case["length"]
        if case["ragged"]:
            n = rng.randint((n + 1) // 2, n)
            total = rng.randint(max(n, total // 4), total)
        new.append(n)
        lens.append(total)
    return lens, new


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _cumulative(counts):
    total = [0]
    for n in counts:
        total.append(total[-1] + n)
    return total


def _shared_rows(case):
    """(rows of page numbers, lengths, pages in use): the requests of a group hold the full pages of their prompt together."""
    rng = random.Random(case["lens"])
    rows, lens, used = [], [], 0
    samples = case.get("mix") == "samples"
    for _ in range(case["groups"]):
        total = rng.randint((case["length"] + 1) // 2, case["length"])
        prompt = total if samples else rng.randint(0, total)
        shared = list(range(used, used + prompt // PAGE))
        used += len(shared)
        for i in range(case["rows"]):
            if samples and i > 0:
                rows.append([])
                lens.append(0)
                continue
            n = total if samples or case.get("mix") == "beams" else rng.randint(prompt, total)
            mine = _pages(n) - len(shared)
            rows.append(shared + list(range(used, used + mine)))
            lens.append(n)
            used += mine
    return rows, lens, used


def _shares(case):
    """(source, old, keep, new) of each row of a share, and the rows before it."""
    rows, old, used = _shared_rows(case)
    rng = random.Random(case["lens"] + 1)
    n_rows = len(rows)
    source, keep = list(range(n_rows)), list(old)
    new = [o + case["new"] for o in old]
    for r in range(n_rows):
        first = r - r % case["rows"]
        if case["mix"] == "beams":
            source[r] = rng.randrange(first, first + case["rows"])
        elif case["mix"] == "samples":
            source[r] = first
        else:
            kind = rng.random()
            if kind < 0.1:                                    # ends
                source[r], keep[r], new[r] = -1, 0, 0
                continue
            if kind < 0.2:                                    # another request takes its place
                source[r], keep[r] = -1, 0
                new[r] = rng.randint(1, min(case["length"], 16 * case["new"]))
                continue
            if kind < 0.4:                                    # goes on from another request, from some way back
                source[r] = rng.randrange(n_rows)
                keep[r] = rng.randint(0, old[source[r]])
                new[r] = keep[r] + rng.randint(0, case["new"])
                continue
            if kind < 0.6:                                    # takes drafts back
                keep[r] = max(0, old[r] - rng.randint(0, 70))
                new[r] = keep[r] + case["new"]
                continue
        keep[r] = old[source[r]]
        new[r] = keep[r] + case["new"]
    return rows, used, source, old, keep, new


def _move_counts(case):
    rng = random.Random(case["lens"])
    if case["mode"] == "forks":
        return [rng.randint(1, PAGE - 1) for _ in range(case["copies"])]
    return [rng.randint((case["length"] + 1) // 2, case["length"]) for _ in range(case["copies"])]


# ---------------------------------------------------------------- inputs

def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _quantise(x, shift):
    """Codes and scales of x [..., H, n, d] (fp32), shift [H]: the definition in elementary operations."""
    y = torch.ldexp(x, -shift[:, None, None])
    y = y.unflatten(-1, (-1, 16))
    scale = (y.abs().amax(-1) / 6).clamp(max=448).to(torch.float8_e4m3fn)
    s, t = scale.float()[..., None], y.abs()
    code = torch.zeros_like(y, dtype=torch.uint8)
    for i, mid in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):      # halves go to the even code
        code += (t >= mid * s) if i % 2 else (t > mid * s)
    code = torch.where(s > 0, code, 0) | (torch.signbit(y).to(torch.uint8) << 3)
    code = code.flatten(-2)
    return code[..., ::2] | (code[..., 1::2] << 4), scale


def _values(codes, scales, shift):
    """fp32 values of codes [..., H, n, d / 2]; all of them are exact."""
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=DEV)
    x = level[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return torch.ldexp(x * scales.float().repeat_interleave(16, -1), shift[:, None, None])


def _cache(case, lens, gen):
    """A cache in use: pages in no order, all rows written (rows past a request's end hold what earlier requests left)."""
    h, d = case["kv_heads"], case["head_dim"]
    width = max(1, max(_pages(n) for n in lens))
    n_pages = sum(_pages(n) for n in lens) + 3
    rng = random.Random(case["lens"] + 2)
    s = {"k_shift": None, "v_shift": None}
    channel = torch.exp2(torch.randn(h, 1, d, generator=gen, device=DEV) * 0.7)      # some channels of keys are larger than others
    for x in "kv":
        shift = [rng.randint(-4, 4) if case["shift"] else 0 for _ in range(h)]
        shift = _ints(shift)
        codes = torch.empty(n_pages, h, PAGE, d // 2, dtype=torch.uint8, device=DEV)
        scales = torch.empty(n_pages, h, PAGE, d // 16, dtype=torch.float8_e4m3fn, device=DEV)
        for p in range(0, n_pages, 512):
            v = torch.randn(min(512, n_pages - p), h, PAGE, d, generator=gen, device=DEV)
            if x == "k":
                v *= channel
            codes[p:p + 512], scales[p:p + 512] = _quantise(v, shift if case["shift"] else shift * 0)
        s[x + "_codes"], s[x + "_scales"] = codes, scales
        if case["shift"]:
            s[x + "_shift"] = shift
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.zeros(len(lens), width, dtype=torch.int32, device=DEV)
    first = 0
    for r, n in enumerate(lens):
        table[r, :_pages(n)] = order[first:first + _pages(n)]
        first += _pages(n)
    return {**s, "table": table}


def _rows_state(rows, lens, used, extra, width, gen):
    """Block table of rows of page numbers in a random numbering, page_refs and a stack of free pages."""
    n_pages = used + extra
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.zeros(len(rows), width, dtype=torch.int32)
    for r, row in enumerate(rows):
        table[r, :len(row)] = torch.tensor(row, dtype=torch.int32)
    table = order[table.to(DEV).long()].contiguous()
    count = [0] * n_pages
    for row in rows:
        for p in row:
            count[p] += 1
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[order.long()] = _ints(count)
    free = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    free[:extra] = order[used:]
    zeros = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    return {"table": table, "table_out": torch.zeros_like(table), "page_refs": refs, "refs_out": zeros.clone(), "free": free, "free_out": zeros,
            "free_count": _ints([extra]), "free_count_out": _ints([0]), "lens": _ints([0] * len(rows)), "old": _ints(lens)}


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"case": case, "status": torch.zeros(1, dtype=torch.int32, device=DEV)}
    if case["op"] == "share":
        rows, used, source, old, keep, new = _shares(case)
        extra = sum(_pages(n) - k // PAGE for n, k in zip(new, keep)) + 8
        s.update(_rows_state(rows, old, used, extra, max(1, _pages(max(old + new))), gen))
        tokens = sum(n - k for n, k in zip(new, keep))
        return {**s, "source": _ints(source), "keep": _ints(keep), "new": _ints(new), "cu_new": _ints([0] * (len(old) + 1)),
                "slot_map": _ints([0] * (tokens + 5)), "positions": _ints([0] * (tokens + 5)),
                "move_src": _ints([0] * (PAGE * len(old))), "move_dst": _ints([0] * (PAGE * len(old))), "move_count": _ints([0])}
    if case["op"] == "compact":
        rows, lens, used = _shared_rows(case)
        width = max(1, _pages(max(lens)))
        extra = sum(_pages(n) for n in lens) + 8
        s.update(_rows_state(rows, lens, used, extra, width, gen))
        if not case["refs"]:                                  # every page has one holder: the rows of a group get pages of their own
            order = torch.randperm(used + extra, generator=gen, device=DEV).to(torch.int32)
            at = 0
            for r, n in enumerate(lens):
                s["table"][r, :_pages(n)] = order[at:at + _pages(n)]
                at += _pages(n)
            s["free"][:used + extra - at] = order[at:]
            s["free_count"] = _ints([used + extra - at])
            s["page_refs"] = s["refs_out"] = None
        keep = torch.rand(len(lens), width * PAGE, generator=gen, device=DEV) < case["keep"]
        at = torch.arange(width * PAGE, device=DEV)
        keep |= (at < 4) | ((at >= s["old"][:, None] - 32) & (at < s["old"][:, None]))
        s["keep_bits"] = (keep.unflatten(1, (width, PAGE)).long() << torch.arange(PAGE, device=DEV)).sum(-1)
        room = sum(min(n, int(1.25 * case["keep"] * n) + 128) for n in lens)
        return {**s, "move_src": _ints([0] * room), "move_dst": _ints([0] * room), "move_count": _ints([0])}
    if case["op"] == "move":
        counts, rng = _move_counts(case), random.Random(case["lens"] + 3)
        src, dst, used = [], [], 0
        kept = [n if case["mode"] == "forks" else max(1, int(case["keep"] * n)) for n in counts]
        for n, k in zip(counts, kept):
            src += [used * PAGE + e for e in (range(n) if case["mode"] == "forks" else sorted(rng.sample(range(n), k)))]
            used += _pages(n)
        for k in kept:
            dst += [used * PAGE + e for e in range(k)]
            used += _pages(k)
        order = torch.randperm(used + 3, generator=gen, device=DEV)
        src, dst = (torch.tensor(x, device=DEV) for x in (src, dst))
        src, dst = ((order[x // PAGE] * PAGE + x % PAGE).to(torch.int32) for x in (src, dst))
        pad = torch.full((PAGE,), -1, dtype=torch.int32, device=DEV)
        shape = (used + 3, case["kv_heads"], PAGE, case["head_dim"])
        arrays = [torch.randn(shape, generator=gen, device=DEV).to(DTYPES[case["dtype"]]) for _ in range(2 * case["layers"])]
        bounds = [torch.zeros(shape[0], shape[1], 2, shape[3], dtype=a.dtype, device=DEV) if case["bounds"] and i % 2 == 0 else None for i, a in enumerate(arrays)]
        return {**s, "arrays": arrays, "bounds": bounds, "move_src": torch.cat((src, pad)), "move_dst": torch.cat((dst, pad)), "move_count": _ints([src.numel()])}
    lens, new = _lengths(case)
    s.update(_cache(case, lens, gen))
    tokens, h, d, dtype = sum(new), case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
    if case["op"] == "append":
        slots = []
        for r, (total, n) in enumerate(zip(lens, new)):
            row = s["table"][r].tolist()
            slots += [row[p // PAGE] * PAGE + p % PAGE for p in range(total - n, total)]
        s["slot_map"] = _ints(slots)
        size = torch.exp2(torch.randn(1, 1, h, d, generator=gen, device=DEV) * 0.7)
        kv = (torch.randn(tokens, 2, h, d, generator=gen, device=DEV) * size).to(dtype)
        s["k"], s["v"] = kv[:, 0], kv[:, 1]                  # views of one projection's output
        s["k_read"], s["v_read"] = (torch.zeros(tokens, h, d, dtype=dtype, device=DEV) for _ in range(2))
        return s
    hq = h * case["group"]
    s["q"] = (1.5 * torch.randn(tokens, hq, d, generator=gen, device=DEV)).to(dtype)
    s["cu_new"], s["lens"] = _ints(_cumulative(new)), _ints(lens)
    s["out"] = torch.zeros(tokens, hq, d, dtype=dtype, device=DEV)
    if own:                                                  # scratch that a serving program keeps beside its cache
        from paper_2605_09649_b200 import binding

        s["workspace"] = torch.empty(binding.paged4_workspace_bytes(hq, h, d), dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------- plain forms

def _shift(s, x):
    return s[x + "_shift"] if s[x + "_shift"] is not None else torch.zeros(s["case"]["kv_heads"], dtype=torch.int32, device=DEV)


def _plain_append(s):
    slot = s["slot_map"].long()
    page, off = slot // PAGE, slot % PAGE
    out = {}
    for x in "kv":
        codes, scales = _quantise(s[x].float().transpose(0, 1), _shift(s, x))
        s[x + "_codes"][page, :, off] = codes.transpose(0, 1)
        s[x + "_scales"].view(torch.uint8)[page, :, off] = scales.view(torch.uint8).transpose(0, 1)
        back = s[x + "_scales"].view(torch.uint8)[page, :, off].view(torch.float8_e4m3fn)
        out[x] = _values(s[x + "_codes"][page, :, off][:, :, None], back[:, :, None], _shift(s, x))[:, :, 0].to(s[x].dtype)
    return out


def _plain_attention(s):
    case = s["case"]
    scale, n, h, g = case["head_dim"] ** -0.5, case["new"], case["kv_heads"], case["group"]
    cu, lens = s["cu_new"].long(), s["lens"].long()
    j = torch.arange(n, device=DEV)
    rows = (cu[:-1, None] + j).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][rows].float().unflatten(2, (h, g)).permute(0, 2, 3, 1, 4)                # [R, H, g, n, d]
    pos = lens[:, None] - (cu[1:] - cu[:-1])[:, None] + j
    table = s["table"].long()
    k, v = (_values(s[x + "_codes"][table], s[x + "_scales"].view(torch.uint8)[table].view(torch.float8_e4m3fn), _shift(s, x)).transpose(1, 2).flatten(2, 3)[:, :, None]
            for x in "kv")
    key = torch.arange(k.shape[3], device=DEV)
    mask = key <= pos[..., None]
    if case["window"]:
        mask &= key > pos[..., None] - case["window"]
    x = torch.where(mask[:, None, None], q @ k.transpose(-1, -2) * scale, -torch.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -torch.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(total == 0, 1.0, total)
    token = torch.arange(s["q"].shape[0], device=DEV)
    r = torch.searchsorted(cu[1:].contiguous(), token, right=True)
    return {"out": o.permute(0, 3, 1, 2, 4)[r, token - cu[r]].flatten(1, 2).to(s["q"].dtype)}


def _count_pages(pages, mask, n):
    """How often each of n pages stands where mask is true."""
    return torch.zeros(n + 1, dtype=torch.int32, device=DEV).index_add_(0, torch.where(mask, pages, n).flatten(), mask.flatten().int())[:n]


def _first_place(pages, mask, n):
    """The lowest place (of the flattened arrays) of each page where mask is true."""
    place = torch.arange(pages.numel(), device=DEV)
    first = torch.full((n + 1,), pages.numel(), device=DEV)
    return first.scatter_reduce_(0, torch.where(mask, pages, n).flatten(), place, "amin")[:n]


def _rank(mask):
    """Place of each true value among the true values, in order."""
    return mask.flatten().cumsum(0).view_as(mask) - 1


def _put(target, at, value, mask):
    """target with target[at] = value where mask is true."""
    n = target.numel()
    longer = torch.cat((target, target.new_zeros(1)))
    longer[torch.where(mask, at, n).flatten()] = value.expand(mask.shape).flatten().to(target.dtype)
    return longer[:n]


def _live(s):
    """free_out with the live part of the stack copied in."""
    at = torch.arange(s["free"].numel(), device=DEV)
    return torch.where(at < s["free_count"], s["free"], s["free_out"])


def _plain_share(s):
    i32 = torch.int32
    source, old, keep, new, table = s["source"].long(), s["old"].long(), s["keep"].long(), s["new"].long(), s["table"].long()
    n, (rows, width) = s["page_refs"].numel(), table.shape
    row, col = torch.arange(rows, device=DEV), torch.arange(width, device=DEV)
    had, kept, has = (old + PAGE - 1) // PAGE, (keep + PAGE - 1) // PAGE, (new + PAGE - 1) // PAGE
    from_row = table[source.clamp(min=0)]
    held = col < had[:, None]
    writes = (keep % PAGE != 0) & (new > keep)
    last = from_row.gather(1, (keep // PAGE).clamp(max=width - 1)[:, None])[:, 0]
    stay = (col < kept[:, None]) & ~(writes[:, None] & (col == (keep // PAGE)[:, None]))
    refs = s["page_refs"] - _count_pages(table, held, n) + _count_pages(from_row, stay, n)
    in_place = writes & (refs[last] == 0) & (_first_place(last, writes, n)[last] == row)
    refs = refs + _count_pages(last, in_place, n)
    copied = writes & ~in_place
    back = held & (refs[table] == 0) & (_first_place(table, held, n)[table] == row[:, None] * width + col)
    free = _put(_live(s), s["free_count"] + _rank(back), table, back)
    n_back = back.sum()
    begin = kept - copied.long()
    take = (col >= begin[:, None]) & (col < has[:, None])
    page = free[(s["free_count"] + n_back - 1 - _rank(take)).clamp(0, n - 1)].long()
    out = torch.where(take, page, from_row)
    refs = refs + _count_pages(page, take, n)
    grow = new - keep
    cu = torch.cat((grow.new_zeros(1), grow.cumsum(0)))
    token = torch.arange(s["slot_map"].numel(), device=DEV)
    r = torch.searchsorted(cu[1:].contiguous(), token, right=True).clamp(max=rows - 1)
    pos = keep[r] + token - cu[r]
    real = token < cu[-1]
    slot = out[r, (pos // PAGE).clamp(0, width - 1)] * PAGE + pos % PAGE
    entry = torch.arange(PAGE, device=DEV)
    move = copied[:, None] & (entry < (keep % PAGE)[:, None])
    none = torch.full_like(s["move_src"], -1)
    copy = out.gather(1, (keep // PAGE).clamp(max=width - 1)[:, None])
    return {"table": torch.where(col < has[:, None], out, s["table_out"]).to(i32), "refs": refs.to(i32), "free": free,
            "free_count": (s["free_count"] + n_back - take.sum()).to(i32), "lens": new.to(i32), "cu_new": cu.to(i32),
            "slot_map": torch.where(real, slot, -1).to(i32), "positions": torch.where(real, pos, -1).to(i32),
            "move_src": _put(none, _rank(move), last[:, None] * PAGE + entry, move), "move_dst": _put(none, _rank(move), copy * PAGE + entry, move),
            "move_count": move.sum()[None].to(i32)}


def _plain_compact(s):
    i32 = torch.int32
    lens, table = s["old"].long(), s["table"].long()
    n, (rows, width) = s["free"].numel(), table.shape
    row, col, entry = (torch.arange(x, device=DEV) for x in (rows, width, width * PAGE))
    inside = entry < lens[:, None]
    keep = ((s["keep_bits"][..., None] >> torch.arange(PAGE, device=DEV)) & 1).flatten(1).bool() & inside
    count = keep.sum(1)
    first = torch.where(inside & ~keep, entry, width * PAGE).amin(1)
    moves = torch.where(keep, entry, -1).amax(1) > first
    begin = torch.where(moves, first // PAGE, (count + PAGE - 1) // PAGE)       # pages that stay
    had, has = (lens + PAGE - 1) // PAGE, (count + PAGE - 1) // PAGE
    gone = (col >= begin[:, None]) & (col < had[:, None])
    refs = torch.ones(n, dtype=i32, device=DEV) if s["page_refs"] is None else s["page_refs"]
    refs = refs - _count_pages(table, gone, n)
    back = gone & (refs[table] == 0) & (_first_place(table, gone, n)[table] == row[:, None] * width + col)
    take = (col >= begin[:, None]) & (col < has[:, None])
    page = s["free"][(s["free_count"] - 1 - _rank(take)).clamp(0, n - 1)].long()
    out = torch.where(take, page, table)
    left = s["free_count"] - take.sum()
    free = _put(_live(s), left + _rank(back), table, back)
    move = keep & (entry >= (begin * PAGE)[:, None]) & moves[:, None]
    rank = keep.cumsum(1) - 1
    none = torch.full_like(s["move_src"], -1)
    source = table.repeat_interleave(PAGE, 1) * PAGE + entry % PAGE
    target = out.gather(1, (rank // PAGE).clamp(min=0)) * PAGE + rank % PAGE
    result = {"table": torch.where(col < has[:, None], out, s["table_out"]).to(i32), "free": free, "free_count": (left + back.sum()).to(i32),
              "lens": count.to(i32), "move_src": _put(none, _rank(move), source, move), "move_dst": _put(none, _rank(move), target, move),
              "move_count": move.sum()[None].to(i32)}
    if s["page_refs"] is not None:
        result["refs"] = (refs + _count_pages(page, take, n)).to(i32)
    return result


def _plain_move(s):
    real = torch.arange(s["move_src"].numel(), device=DEV) < s["move_count"]
    # (pairs behind the last repeat the first one)
    src, dst = (torch.where(real, s[x], s[x][0]).long() for x in ("move_src", "move_dst"))
    full = torch.zeros(s["arrays"][0].shape[0], device=DEV).index_put_((dst // PAGE,), (dst % PAGE == PAGE - 1).float(), accumulate=True) > 0
    for a, b in zip(s["arrays"], s["bounds"]):
        a[dst // PAGE, :, dst % PAGE] = a[src // PAGE, :, src % PAGE]
        if b is not None:
            b.copy_(torch.where(full[:, None, None, None], torch.stack((a.amin(2), a.amax(2)), 2), b))
    return s["arrays"] + [b for b in s["bounds"] if b is not None]


# ---------------------------------------------------------------- the framework's calls

def _own(s):
    from paper_2605_09649_b200 import binding

    case = s["case"]
    if case["op"] == "share":
        binding.paged_share(s["source"], s["old"], s["keep"], s["new"], s["table"], s["table_out"], s["page_refs"], s["refs_out"], s["free"], s["free_out"],
                            s["free_count"], s["free_count_out"], s["lens"], s["cu_new"], s["slot_map"], s["positions"], s["move_src"], s["move_dst"],
                            s["move_count"], s["status"])
        return {"table": s["table_out"], "refs": s["refs_out"], "free": s["free_out"], "free_count": s["free_count_out"], "lens": s["lens"],
                "cu_new": s["cu_new"], "slot_map": s["slot_map"], "positions": s["positions"], "move_src": s["move_src"], "move_dst": s["move_dst"],
                "move_count": s["move_count"]}
    if case["op"] == "compact":
        binding.paged_compact(s["old"], s["keep_bits"], s["table"], s["table_out"], s["page_refs"], s["refs_out"], s["free"], s["free_out"],
                              s["free_count"], s["free_count_out"], s["lens"], s["move_src"], s["move_dst"], s["move_count"], status=s["status"])
        result = {"table": s["table_out"], "free": s["free_out"], "free_count": s["free_count_out"], "lens": s["lens"], "move_src": s["move_src"],
                  "move_dst": s["move_dst"], "move_count": s["move_count"]}
        return {**result, "refs": s["refs_out"]} if s["page_refs"] is not None else result
    if case["op"] == "move":
        binding.paged_move(s["arrays"], s["move_src"], s["move_dst"], s["move_count"], key_bounds=s["bounds"], status=s["status"])
        return s["arrays"] + [b for b in s["bounds"] if b is not None]
    cache = binding.Paged4Cache(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], s["k_shift"], s["v_shift"])
    if case["op"] == "append":
        binding.paged4_append(cache, s["k"], s["v"], s["slot_map"], status=s["status"])
        binding.paged4_read(cache, s["slot_map"], s["k_read"], s["v_read"], status=s["status"])
        return {"k": s["k_read"], "v": s["v_read"]}
    binding.paged4_attention(cache, s["q"], s["cu_new"], s["lens"], s["table"], case["new"], window=case["window"], out=s["out"],
                             workspace=s["workspace"], status=s["status"])
    return {"out": s["out"]}


PLAIN = {"append": _plain_append, "attention": _plain_attention, "share": _plain_share, "compact": _plain_compact, "move": _plain_move}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------- work and exact values

def work(case):
    if case["op"] == "share":
        rows, used, source, old, keep, new = _shares(case)
        n, tokens = len(old), sum(b - a for a, b in zip(keep, new))
        # lengths and sources in; lengths and offsets out; the rows' entries read and written, their pages' counts and what changes hands;
        # slot and position per token
        return {"bytes": 16 * n + 8 * n + 8 * sum(_pages(x) for x in new) + 8 * used + 8 * tokens + 8 * PAGE * n + 16, "flops": 0}
    if case["op"] == "compact":
        _, lens, used = _shared_rows(case)
        words = sum(_pages(n) for n in lens)
        room = sum(min(n, int(1.25 * case["keep"] * n) + 128) for n in lens)
        # keep bits and table entries in; moved rows, the new table and the stack out
        return {"bytes": 12 * words + 8 * room + 8 * int(case["keep"] * words) + 12 * words, "flops": 0}
    if case["op"] == "move":
        counts = _move_counts(case)
        moved = sum(counts) if case["mode"] == "forks" else sum(max(1, int(case["keep"] * n)) for n in counts)
        row = case["kv_heads"] * case["head_dim"] * DTYPES[case["dtype"]].itemsize
        full = 0 if case["mode"] == "forks" else sum(max(1, int(case["keep"] * n)) // PAGE for n in counts)
        bounds = case["layers"] * full * 2 * row if case["bounds"] else 0
        return {"bytes": 2 * case["layers"] * moved * 2 * row + 8 * moved + bounds, "flops": 2 * PAGE * full * case["layers"] * case["kv_heads"] * case["head_dim"] if case["bounds"] else 0}
    lens, new = _lengths(case)
    h, d, size = case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]].itemsize
    row = h * (d // 2 + d // 16)                             # of k, and of v
    tokens = sum(new)
    if case["op"] == "append":
        # k and v in, their rows out; the rows in again and their values out
        return {"bytes": tokens * (2 * h * d * size + 2 * row + 2 * row + 2 * h * d * size + 8), "flops": 4 * tokens * h * d}
    hq, w = h * case["group"], case["window"] or 1 << 30
    read = sum(t - max(0, t - n + 1 - w) for t, n in zip(lens, new))
    seen = sum(min(p + 1, w) for t, n in zip(lens, new) for p in range(t - n, t))
    return {"bytes": 2 * tokens * hq * d * size + 4 * (len(lens) + sum(_pages(t) for t in lens)) + 2 * read * row, "flops": 4 * d * hq * seen}


def _nearest(x, table):
    """Place of the nearest of an ascending table (fp64); halves go to the even place."""
    mid = (table[1:] + table[:-1]) / 2
    at = torch.bucketize(x.contiguous(), mid)
    odd_half = (at % 2 == 1) & (x == mid[at.clamp(max=mid.numel() - 1)])
    return at + odd_half.long()


def _exact_values(codes, scales, shift):
    sign = 1.0 - 2.0 * (codes.long() >> 3 & 1).double()
    return sign * torch.tensor(LEVELS, dtype=torch.float64, device=DEV)[codes.long() & 7] * scales * torch.exp2(shift.double())


def _exact_share(s, case):
    rows, used, source, old, keep, new = _shares(case)
    table, refs, stack = s["table"].tolist(), s["page_refs"].tolist(), s["free"].tolist()
    live = stack[:s["free_count"].item()]
    before = [row[:_pages(o)] for row, o in zip(table, old)]
    for p in (p for row in before for p in row):
        refs[p] -= 1
    after, asks = [], []
    for r in range(len(old)):
        row = before[source[r]][:_pages(keep[r])] if source[r] >= 0 else []
        asks.append(bool(keep[r] % PAGE and new[r] > keep[r]))
        for p in row[:len(row) - asks[r]]:
            refs[p] += 1
        after.append(row)
    others, copies = list(refs), {}
    for r in range(len(old)):
        if asks[r]:
            p = after[r].pop()
            if others[p] == 0 and refs[p] == 0:
                refs[p] = 1
                after[r].append(p)
            else:
                copies[r] = p
    peak = list(live)
    pushed = set()
    for p in (p for row in before for p in row):
        if refs[p] == 0 and p not in pushed:
            pushed.add(p)
            peak.append(p)
    live = list(peak)
    src, dst, slots, positions, cu = [], [], [], [], [0]
    for r in range(len(old)):
        while len(after[r]) < _pages(new[r]):
            after[r].append(live.pop())
            refs[after[r][-1]] = 1
    for r in range(len(old)):
        if r in copies:
            src += [copies[r] * PAGE + e for e in range(keep[r] % PAGE)]
            dst += [after[r][keep[r] // PAGE] * PAGE + e for e in range(keep[r] % PAGE)]
        positions += range(keep[r], new[r])
        slots += [after[r][p // PAGE] * PAGE + p % PAGE for p in range(keep[r], new[r])]
        cu.append(len(slots))
    none = lambda x, n: _ints(x + [-1] * (n - len(x)))
    width, n = len(table[0]), len(stack)
    return {"table": _ints([row + [0] * (width - len(row)) for row in after]), "refs": _ints(refs), "free": _ints(peak + [0] * (n - len(peak))),
            "free_count": _ints([len(live)]), "lens": _ints(new), "cu_new": _ints(cu), "slot_map": none(slots, s["slot_map"].numel()),
            "positions": none(positions, s["positions"].numel()), "move_src": none(src, s["move_src"].numel()),
            "move_dst": none(dst, s["move_dst"].numel()), "move_count": _ints([len(src)])}


def _exact_compact(s):
    table, lens, bits, stack = s["table"].tolist(), s["old"].tolist(), s["keep_bits"].tolist(), s["free"].tolist()
    fc = s["free_count"].item()
    refs = None if s["page_refs"] is None else s["page_refs"].tolist()
    live, taken = stack[:fc], 0
    after, counts, src, dst, gone = [], [], [], [], []
    for r, n in enumerate(lens):
        kept = [e for e in range(n) if bits[r][e // PAGE] >> (e % PAGE) & 1]
        first = next((i for i, e in enumerate(kept) if e != i), len(kept))          # kept[:first] stay where they are
        stay = _pages(len(kept)) if first == len(kept) else first // PAGE
        row = table[r][:stay]
        while len(row) < _pages(len(kept)):
            taken += 1
            row.append(live[fc - taken])
            if refs is not None:
                refs[row[-1]] += 1
        if first < len(kept):
            for i in range(stay * PAGE, len(kept)):
                src.append(table[r][kept[i] // PAGE] * PAGE + kept[i] % PAGE)
                dst.append(row[i // PAGE] * PAGE + i % PAGE)
        gone += table[r][stay:_pages(n)]
        after.append(row)
        counts.append(len(kept))
    back = []
    if refs is None:
        back = gone
    else:
        for p in gone:
            refs[p] -= 1
        for p in gone:
            if refs[p] == 0 and p not in back:
                back.append(p)
    left = fc - taken
    free = live[:left] + back
    free += live[len(free):] if len(free) < fc else []
    none = lambda x: _ints(x + [-1] * (s["move_src"].numel() - len(x)))
    result = {"table": _ints([row + [0] * (len(table[0]) - len(row)) for row in after]), "free": _ints(free + [0] * (len(stack) - len(free))),
              "free_count": _ints([left + len(back)]), "lens": _ints(counts), "move_src": none(src), "move_dst": none(dst), "move_count": _ints([len(src)])}
    if refs is not None:
        result["refs"] = _ints(refs)
    return result


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "share":
        return _exact_share(s, case)
    if case["op"] == "compact":
        return _exact_compact(s)
    if case["op"] == "move":
        n = s["move_count"].item()
        src, dst = s["move_src"][:n].long(), s["move_dst"][:n].long()
        arrays, bounds = [], []
        whole = dst[dst % PAGE == PAGE - 1] // PAGE
        for a, b in zip(s["arrays"], s["bounds"]):
            flat = a.double().transpose(1, 2).reshape(-1, a.shape[1], a.shape[3])
            flat[dst] = flat[src]
            arrays.append(flat.view(a.shape[0], PAGE, a.shape[1], a.shape[3]).transpose(1, 2))
            if b is not None:
                b = b.double()
                b[whole] = torch.stack((arrays[-1][whole].min(2).values, arrays[-1][whole].max(2).values), 2)
                bounds.append(b)
        return arrays + bounds
    h, d = case["kv_heads"], case["head_dim"]
    shifts = {x: s[x + "_shift"] if s[x + "_shift"] is not None else torch.zeros(h, device=DEV) for x in "kv"}
    if case["op"] == "append":
        bits = torch.arange(127, device=DEV)                 # of the e4m3 numbers from 0 to 448
        e4m3 = torch.where(bits < 8, bits * 2.0 ** -9, (1 + (bits % 8).double() / 8) * torch.exp2((bits // 8).double() - 7))
        out = {}
        for x in "kv":
            y = s[x].double().unflatten(-1, (-1, 16)) * torch.exp2(-shifts[x].double())[:, None, None]
            scale = e4m3[_nearest(y.abs().max(-1, keepdim=True).values / 6, e4m3)]
            code = _nearest((y.abs() / torch.where(scale > 0, scale, 1.0)) * (scale > 0), torch.tensor(LEVELS, dtype=torch.float64, device=DEV))
            out[x] = (_exact_values(code, scale, shifts[x][:, None, None]) * torch.sign(y)).flatten(-2)
        return out
    lens, new = _lengths(case)
    cu, g = _cumulative(new), case["group"]
    out = torch.zeros(cu[-1], h * g, d, dtype=torch.float64, device=DEV)
    for r, (t, n) in enumerate(zip(lens, new)):
        pages = s["table"][r, :_pages(t)].long()
        pos, at = torch.arange(t - n, t, device=DEV), torch.arange(t, device=DEV)
        seen = (at <= pos[:, None]) & (at > pos[:, None] - (case["window"] or 1 << 30))
        for head in range(h):
            kv = []
            for x in "kv":
                byte = s[x + "_codes"][pages, head].reshape(-1, d // 2)[:t]
                code = torch.stack((byte % 16, byte // 16), -1).reshape(t, d)
                scale = s[x + "_scales"].view(torch.uint8)[pages, head].view(torch.float8_e4m3fn).reshape(-1, d // 16)[:t].double().repeat_interleave(16, 1)
                kv.append(_exact_values(code, scale, shifts[x][head]))
            q = s["q"][cu[r]:cu[r + 1], head * g:(head + 1) * g].double()
            x = torch.einsum("ngd,kd->gnk", q, kv[0]) / math.sqrt(d)
            x = torch.softmax(x.masked_fill(~seen, -float("inf")), -1)
            out[cu[r]:cu[r + 1], head * g:(head + 1) * g] = torch.einsum("gnk,kd->ngd", x, kv[1])
    return {"out": out}

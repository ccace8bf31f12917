"""Cases of the paged-cache operators: block tables and slot maps, the append, causal attention over the cache, and
attention over the pages that each query selects.

The cache is the caller's: k_pages and v_pages [n_pages, H, 64, d], key_bounds [n_pages, H, 2, d] (channelwise smallest
and largest key of each full page), a block table [requests, width] of physical pages, and lengths on the device.  With
`own` set the calls go to paper_2605_09649_b200.binding; otherwise the same results come from elementary torch operations
in fp32 (fp64 for the page scores, whose order decides which pages are read).
"""
import math
import random

import torch

own = False

PAGE = 64
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
WORKSPACE_BYTES = 160 << 20        # scratch that a serving program keeps beside its cache


def listed():
    return [
        # a decode step of a continuous batch: one token for most requests, drafts taken back, requests that end or start
        {"name": "plan decode 64", "op": "plan", "requests": 64, "length": 32768, "new": 8, "mix": "serve", "lens": 1},
        # admission of many prompts at once: 256 requests, up to 1024 tokens each
        {"name": "plan prompts 256", "op": "plan", "requests": 256, "length": 2048, "new": 1024, "mix": "grow", "lens": 2},
        # one token for each of 32 dialogues (8 KV heads of 128)
        {"name": "append decode 32", "op": "append", "requests": 32, "length": 2304, "new": 1, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "ragged": False, "lens": 3},
        # prompt chunks of 32 dialogues
        {"name": "append chunks 32x512", "op": "append", "requests": 32, "length": 2048, "new": 512, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "ragged": True, "lens": 4},
        # a small fp32 model's prompt
        {"name": "attention f32 512", "op": "attention", "requests": 1, "length": 512, "new": 512, "kv_heads": 2, "group": 2, "head_dim": 64, "dtype": "f32", "ragged": False, "window": 0, "lens": 5},
        # single tokens over vision-language prompts, 7 query heads per KV head
        {"name": "attention decode 4x16k", "op": "attention", "requests": 4, "length": 16384, "new": 1, "kv_heads": 4, "group": 7, "head_dim": 128, "dtype": "bf16", "ragged": True, "window": 0, "lens": 6},
        # single tokens over 32K contexts: the bandwidth case
        {"name": "attention decode 8x32k", "op": "attention", "requests": 8, "length": 32768, "new": 1, "kv_heads": 8, "group": 4, "head_dim": 128, "dtype": "bf16", "ragged": False, "window": 0, "lens": 7},
        # drafted tokens scored in one call, 32 dialogues of different lengths
        {"name": "attention drafts 32x5", "op": "attention", "requests": 32, "length": 2304, "new": 5, "kv_heads": 8, "group": 4, "head_dim": 128, "dtype": "bf16", "ragged": True, "window": 0, "lens": 8},
        # prompt chunks of 512 deep inside 16K contexts
        {"name": "attention chunks 4x512", "op": "attention", "requests": 4, "length": 16384, "new": 512, "kv_heads": 8, "group": 4, "head_dim": 128, "dtype": "bf16", "ragged": False, "window": 0, "lens": 9},
        # one token over a 128K context, 64 of its 2048 pages read
        {"name": "pages decode 1x128k", "op": "pages", "requests": 1, "length": 131072, "new": 1, "kv_heads": 8, "group": 8, "head_dim": 128, "dtype": "bf16", "ragged": False, "top": 64, "sink": 1, "recent": 2, "lens": 10},
        # single tokens of 32 requests over contexts of up to 16K, 32 pages read
        {"name": "pages decode 32x16k", "op": "pages", "requests": 32, "length": 16384, "new": 1, "kv_heads": 8, "group": 4, "head_dim": 128, "dtype": "bf16", "ragged": True, "top": 32, "sink": 1, "recent": 2, "lens": 11},
        # a chunk's tokens, each with its own 32 pages
        {"name": "pages chunk 2x128", "op": "pages", "requests": 2, "length": 16384, "new": 128, "kv_heads": 8, "group": 4, "head_dim": 128, "dtype": "bf16", "ragged": True, "top": 32, "sink": 1, "recent": 1, "lens": 12},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "append", "attention", "attention", "pages"])
    c = {"op": op, "lens": rng.randrange(1 << 30)}
    if op == "plan":
        r = _log(rng, 1, 512)
        return {**c, "requests": r, "length": _log(rng, 64, 32768), "new": _log(rng, 1, max(1, min(4096, 131072 // r))), "mix": rng.choice(["serve", "grow"])}
    c["kv_heads"], c["group"] = rng.choice([(8, 4), (4, 7), (8, 8), (2, 2), (1, 8), (3, 5), (8, 1), (2, 16)])
    c["head_dim"] = rng.choice([128, 128, 128, 64, 64, 96, 256])
    c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
    c["ragged"] = rng.random() < 0.7
    if op == "append":
        del c["group"]
        new = _log(rng, 1, 1024)
        r = _log(rng, 1, max(1, 4096 // new))
        return {**c, "requests": r, "new": new, "length": new + _log(rng, 1, 2048)}
    if op == "attention":
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
    new = rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 8, 96)])
    length = _log(rng, 256, 65536 if new == 1 else 16384)
    r = _log(rng, 1, max(1, min(32, 262144 // (length * max(1, new // 2)))))
    top = rng.choice([8, 16, 32, 33, 48])
    return {**c, "requests": r, "new": new, "length": max(length, new), "top": top, "sink": rng.randint(0, 2), "recent": rng.randint(1, 3)}


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


def _resizes(case):
    """(old, keep, new) lengths of each request of a plan."""
    rng = random.Random(case["lens"])
    old, keep, new = [], [], []
    for _ in range(case["requests"]):
        o = rng.randint(0, case["length"] - case["new"]) if case["length"] > case["new"] else 0
        k, n = o, o + rng.randint((case["new"] + 1) // 2, case["new"])
        if case["mix"] == "serve":
            kind = rng.random()
            if kind < 0.1:                                   # the request ends
                k = n = 0
            elif kind < 0.2:                                 # a request starts
                o = k = 0
                n = rng.randint(1, case["length"])
                n = min(n, 16 * case["new"])
            elif kind < 0.5:                                 # rejected drafts are taken back first
                k = max(0, o - rng.randint(0, case["new"]))
                n = k + rng.randint(1, case["new"])
            else:
                n = o + 1
        old.append(o), keep.append(k), new.append(n)
    return old, keep, new


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _cumulative(counts):
    total = [0]
    for n in counts:
        total.append(total[-1] + n)
    return total


def _cache(case, lens, gen):
    """A cache in use: pages in no order, all rows written (rows past a request's end hold what earlier requests left)."""
    h, d, dtype = case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
    width = max(1, max(_pages(n) for n in lens))
    n_pages = sum(_pages(n) for n in lens) + 3
    # keys of a page share a direction of their own, so that pages differ in what they are good for
    k = torch.randn(n_pages, h, PAGE, d, generator=gen, device=DEV, dtype=torch.float32)
    k += 0.7 * torch.randn(n_pages, h, 1, d, generator=gen, device=DEV, dtype=torch.float32)
    k = k.to(dtype)
    v = torch.randn(n_pages, h, PAGE, d, generator=gen, device=DEV, dtype=torch.float32).to(dtype)
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.zeros(len(lens), width, dtype=torch.int32, device=DEV)
    first = 0
    for r, n in enumerate(lens):
        table[r, :_pages(n)] = order[first:first + _pages(n)]
        first += _pages(n)
    return {"k_pages": k, "v_pages": v, "key_bounds": torch.stack((k.amin(2), k.amax(2)), 2).contiguous(), "table": table}


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"case": case, "status": torch.zeros(1, dtype=torch.int32, device=DEV)}
    if case["op"] == "plan":
        old, keep, new = _resizes(case)
        width = max(1, _pages(max(old + new)))
        used = sum(_pages(n) for n in old)
        n_pages = used + sum(max(0, _pages(n) - _pages(o)) for n, o in zip(new, old)) + 8
        order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
        table = torch.zeros(len(old), width, dtype=torch.int32, device=DEV)
        first = 0
        for r, n in enumerate(old):
            table[r, :_pages(n)] = order[first:first + _pages(n)]
            first += _pages(n)
        free = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        free[:n_pages - used] = order[used:]
        tokens = sum(n - k for n, k in zip(new, keep))
        return {**s, "old": _ints(old), "keep": _ints(keep), "new": _ints(new), "table": table, "free": free, "free_count": _ints([n_pages - used]),
                "free_count_out": _ints([0]), "lens": _ints([0] * len(old)), "cu_new": _ints([0] * (len(old) + 1)),
                "slot_map": _ints([0] * (tokens + 5)), "positions": _ints([0] * (tokens + 5))}
    lens, new = _lengths(case)
    s.update(_cache(case, lens, gen))
    tokens, h, d, dtype = sum(new), case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
    if case["op"] == "append":
        slots = []
        for r, (total, n) in enumerate(zip(lens, new)):
            row = s["table"][r].tolist()
            slots += [row[p // PAGE] * PAGE + p % PAGE for p in range(total - n, total)]
        s["slot_map"] = _ints(slots)
        kv = torch.randn(tokens, 2, h, d, generator=gen, device=DEV, dtype=torch.float32).to(dtype)
        s["k"], s["v"] = kv[:, 0], kv[:, 1]                  # views of one projection's output
        return s
    hq = h * case["group"]
    s["q"] = (1.5 * torch.randn(tokens, hq, d, generator=gen, device=DEV, dtype=torch.float32)).to(dtype)
    s["cu_new"], s["lens"] = _ints(_cumulative(new)), _ints(lens)
    s["out"] = torch.zeros(tokens, hq, d, dtype=dtype, device=DEV)
    s["workspace"] = torch.empty(WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    if case["op"] == "pages":
        s["selected"] = torch.zeros(tokens, h, case["top"], dtype=torch.int32, device=DEV)
    return s


# ---------------------------------------------------------------- plain forms

def _plain_plan(s):
    old, keep, new, table, free = s["old"].long(), s["keep"].long(), s["new"].long(), s["table"], s["free"]
    width, slots = table.shape[1], s["slot_map"].numel()
    page = torch.arange(width, device=DEV)
    had, has = (old + PAGE - 1) // PAGE, (new + PAGE - 1) // PAGE
    back = (page >= has[:, None]) & (page < had[:, None])          # returned to the free list, in table order
    take = (page >= had[:, None]) & (page < has[:, None])          # taken from its end, in table order
    back_at = back.flatten().cumsum(0).view_as(back) - 1 + s["free_count"]
    n_back, n_take = back.sum(), take.sum()
    stack = torch.cat((free, free.new_zeros(1)))
    stack[torch.where(back, back_at, free.numel()).flatten()] = table.flatten()
    stack = stack[:-1]
    take_at = s["free_count"] + n_back - 1 - (take.flatten().cumsum(0).view_as(take) - 1)
    table = torch.where(take, stack[take_at.clamp(0, free.numel() - 1)], table)
    grow = new - keep
    cu = torch.cat((grow.new_zeros(1), grow.cumsum(0)))
    token = torch.arange(slots, device=DEV)
    r = torch.searchsorted(cu[1:].contiguous(), token, right=True).clamp(max=old.numel() - 1)
    pos = keep[r] + token - cu[r]
    slot = table[r, (pos // PAGE).clamp(0, width - 1)] * PAGE + pos % PAGE
    real = token < cu[-1]
    i32 = torch.int32
    return {"table": table, "free": stack, "free_count": (s["free_count"] + n_back - n_take).to(i32), "lens": new.to(i32), "cu_new": cu.to(i32),
            "slot_map": torch.where(real, slot, -1).to(i32), "positions": torch.where(real, pos, -1).to(i32)}


def _plain_append(s):
    slot = s["slot_map"].long()
    page, off = slot // PAGE, slot % PAGE
    s["k_pages"][page, :, off] = s["k"]
    s["v_pages"][page, :, off] = s["v"]
    done = torch.zeros(s["k_pages"].shape[0], device=DEV).index_put_((page,), (off == PAGE - 1).float(), accumulate=True) > 0
    bounds = torch.stack((s["k_pages"].amin(2), s["k_pages"].amax(2)), 2)
    s["key_bounds"].copy_(torch.where(done[:, None, None, None], bounds, s["key_bounds"]))
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "key_bounds": s["key_bounds"]}


def _padded(s):
    """Queries as [R, H, g, n, d] in fp32, positions [R, n], and the way back to rows."""
    case = s["case"]
    n, h, g = case["new"], case["kv_heads"], case["group"]
    cu, lens = s["cu_new"].long(), s["lens"].long()
    count = cu[1:] - cu[:-1]
    j = torch.arange(n, device=DEV)
    rows = (cu[:-1, None] + j).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][rows].float().unflatten(2, (h, g)).permute(0, 2, 3, 1, 4)
    pos = lens[:, None] - count[:, None] + j
    token = torch.arange(s["q"].shape[0], device=DEV)
    r = torch.searchsorted(cu[1:].contiguous(), token, right=True)
    return q, pos, r, token - cu[r]


def _softmax_times(x, mask, v):
    x = torch.where(mask, x, -torch.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -torch.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    return (p @ v) / torch.where(total == 0, 1.0, total)


def _plain_attention(s):
    case = s["case"]
    scale = case["head_dim"] ** -0.5
    q, pos, r, j = _padded(s)
    kv = [t[s["table"]].float().transpose(1, 2).flatten(2, 3)[:, :, None] for t in (s["k_pages"], s["v_pages"])]
    key = torch.arange(kv[0].shape[3], device=DEV)
    mask = key <= pos[..., None]
    if case["window"]:
        mask &= key > pos[..., None] - case["window"]
    o = _softmax_times(q @ kv[0].transpose(-1, -2) * scale, mask[:, None, None], kv[1])
    return {"out": o.permute(0, 3, 1, 2, 4)[r, j].flatten(1, 2).to(s["q"].dtype)}


def _plain_pages(s):
    case = s["case"]
    top, scale = case["top"], case["head_dim"] ** -0.5
    q, pos, r, j = _padded(s)
    lo, hi = (s["key_bounds"][s["table"]][:, :, :, i].double().permute(0, 2, 3, 1)[:, :, None] for i in (0, 1))
    score = (q.double().clamp(min=0) @ hi + q.double().clamp(max=0) @ lo).amax(2)             # [R, H, n, pages]
    score = torch.nn.functional.pad(score, (0, max(0, top - score.shape[-1])), value=-torch.inf)
    page = torch.arange(score.shape[-1], device=DEV)
    last = (pos // PAGE)[:, None, :, None]
    score = torch.where((page < case["sink"]) | (page > last - case["recent"]), torch.inf, score)
    score = torch.where(page > last, -torch.inf, score)
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :top]
    best = torch.where(best > last, 1 << 30, best).sort(-1).values
    selected = torch.where(best == 1 << 30, -1, best)[r, :, j]                                # [T, H, top]
    physical = s["table"][r[:, None, None], selected.clamp(min=0)]
    head = torch.arange(case["kv_heads"], device=DEV)[:, None]
    k, v = (t[physical, head].float().flatten(2, 3) for t in (s["k_pages"], s["v_pages"]))   # [T, H, top * 64, d]
    at = selected[..., None] * PAGE + torch.arange(PAGE, device=DEV)
    mask = ((selected >= 0)[..., None] & (at <= pos[r, j][:, None, None, None])).flatten(2)
    x = q.permute(0, 3, 1, 2, 4)[r, j] @ k.transpose(-1, -2) * scale
    o = _softmax_times(x, mask[:, :, None], v)
    return {"out": o.flatten(1, 2).to(s["q"].dtype), "selected": selected.to(torch.int32)}


# ---------------------------------------------------------------- the framework's calls

def _own(s):
    from paper_2605_09649_b200 import binding

    case = s["case"]
    if case["op"] == "plan":
        binding.paged_plan(s["old"], s["keep"], s["new"], s["table"], s["free"], s["free_count"], s["free_count_out"], s["lens"], s["cu_new"],
                           s["slot_map"], s["positions"], s["status"])
        return {"table": s["table"], "free": s["free"], "free_count": s["free_count_out"], "lens": s["lens"], "cu_new": s["cu_new"],
                "slot_map": s["slot_map"], "positions": s["positions"]}
    if case["op"] == "append":
        binding.paged_append(s["k_pages"], s["v_pages"], s["k"], s["v"], s["slot_map"], key_bounds=s["key_bounds"], status=s["status"])
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "key_bounds": s["key_bounds"]}
    if case["op"] == "attention":
        binding.paged_attention(s["k_pages"], s["v_pages"], s["q"], s["cu_new"], s["lens"], s["table"], case["new"], window=case["window"],
                                out=s["out"], workspace=s["workspace"], status=s["status"])
        return {"out": s["out"]}
    binding.paged_sparse_attention(s["k_pages"], s["v_pages"], s["key_bounds"], s["q"], s["cu_new"], s["lens"], s["table"], case["top"],
                                   sink_pages=case["sink"], recent_pages=case["recent"], out=s["out"], selected=s["selected"],
                                   workspace=s["workspace"], status=s["status"])
    return {"out": s["out"], "selected": s["selected"]}


PLAIN = {"plan": _plain_plan, "append": _plain_append, "attention": _plain_attention, "pages": _plain_pages}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------- work and exact values

def work(case):
    if case["op"] == "plan":
        old, keep, new = _resizes(case)
        tokens = sum(n - k for n, k in zip(new, keep))
        moved = sum(abs(_pages(n) - _pages(o)) for n, o in zip(new, old))
        # lengths in; lengths, offsets out; an entry read and one written per page that changes hands; slot and position per token
        return {"bytes": 12 * len(old) + 8 * len(old) + 8 * moved + 8 * tokens + 16, "flops": 0}
    lens, new = _lengths(case)
    h, d, size = case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]].itemsize
    row = h * d * size
    if case["op"] == "append":
        done = sum(t // PAGE - (t - n) // PAGE for t, n in zip(lens, new))
        # rows of a completed page that were there before the call are read once more for its bounds
        before = sum((t - n) % PAGE for t, n in zip(lens, new) if t // PAGE > (t - n) // PAGE)
        return {"bytes": sum(new) * (4 * row + 4) + before * row + done * 2 * row, "flops": 2 * PAGE * done * h * d}
    hq, tokens = h * case["group"], sum(new)
    io = 2 * tokens * hq * d * size + 4 * (len(lens) + sum(_pages(t) for t in lens))
    if case["op"] == "attention":
        w = case["window"] or 1 << 30
        read = sum(t - max(0, t - n + 1 - w) for t, n in zip(lens, new))
        seen = sum(min(p + 1, w) for t, n in zip(lens, new) for p in range(t - n, t))
        return {"bytes": io + 2 * read * row, "flops": 4 * d * hq * seen}
    # a page that several tokens of a request select is read once; tokens together select as many pages as there are
    count = [[min(case["top"], p // PAGE + 1) for p in range(t - n, t)] for t, n in zip(lens, new)]
    read = sum(min(sum(c), _pages(t)) for c, t in zip(count, lens))
    scored = sum(p // PAGE for t, n in zip(lens, new) for p in range(t - n, t))
    full = sum((t - 1) // PAGE for t in lens)
    keys = sum(PAGE * (c - 1) + p % PAGE + 1 for cs, t, n in zip(count, lens, new) for c, p in zip(cs, range(t - n, t)))
    return {"bytes": io + 4 * tokens * h * case["top"] + 2 * full * row + 2 * PAGE * read * row, "flops": hq * d * (4 * keys + 2 * scored)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "plan":
        old, keep, new = _resizes(case)
        table, stack = s["table"].tolist(), s["free"].tolist()
        live = stack[:s["free_count"].item()]
        for r in range(len(old)):
            live += table[r][_pages(new[r]):_pages(old[r])]
        after = live + stack[len(live):]
        slots, positions, cu = [], [], [0]
        for r in range(len(old)):
            for p in range(_pages(old[r]), _pages(new[r])):
                table[r][p] = live.pop()
        for r in range(len(old)):
            positions += range(keep[r], new[r])
            slots += [table[r][p // PAGE] * PAGE + p % PAGE for p in range(keep[r], new[r])]
            cu.append(len(slots))
        pad = [-1] * (s["slot_map"].numel() - len(slots))
        return {"table": _ints(table), "free": _ints(after), "free_count": _ints([len(live)]), "lens": _ints(new), "cu_new": _ints(cu),
                "slot_map": _ints(slots + pad), "positions": _ints(positions + pad)}
    lens, new = _lengths(case)
    cu = _cumulative(new)
    h = case["kv_heads"]
    if case["op"] == "append":
        k, v, b = s["k_pages"].double(), s["v_pages"].double(), s["key_bounds"].double()
        for r, (t, n) in enumerate(zip(lens, new)):
            p = torch.arange(t - n, t, device=DEV)
            physical = s["table"][r].long()[p // PAGE]
            rows = slice(cu[r], cu[r + 1])
            k[physical, :, p % PAGE], v[physical, :, p % PAGE] = s["k"][rows].double(), s["v"][rows].double()
            full = s["table"][r].long()[(t - n) // PAGE:t // PAGE]
            b[full, :, 0], b[full, :, 1] = k[full].min(2).values, k[full].max(2).values
        return {"k_pages": k, "v_pages": v, "key_bounds": b}
    d, g = case["head_dim"], case["group"]
    out = torch.zeros(cu[-1], h * g, d, dtype=torch.float64, device=DEV)
    chosen = torch.full((cu[-1], h, case.get("top", 1)), -1, dtype=torch.int32, device=DEV)
    for r, (t, n) in enumerate(zip(lens, new)):
        pages = s["table"][r, :_pages(t)].long()
        pos = torch.arange(t - n, t, device=DEV)
        at = torch.arange(_pages(t) * PAGE, device=DEV)
        for head in range(h):
            k, v = (x[pages, head].double().reshape(-1, d) for x in (s["k_pages"], s["v_pages"]))
            q = s["q"][cu[r]:cu[r + 1], head * g:(head + 1) * g].double()
            seen = (at <= pos[:, None])
            if case["op"] == "attention":
                seen = seen & (at > pos[:, None] - (case["window"] or 1 << 30))
            else:
                b = s["key_bounds"][pages, head].double()
                own_page = pos // PAGE
                index = torch.arange(len(pages), device=DEV)
                forced = (index < case["sink"]) | (index > own_page[:, None] - case["recent"])
                score = torch.stack([torch.maximum(q[i, :, None] * b[:, 0], q[i, :, None] * b[:, 1]).sum(-1).max(0).values for i in range(n)])
                score[forced] = float("inf")
                score[index > own_page[:, None]] = -float("inf")
                order = torch.argsort(score, dim=1, descending=True, stable=True)[:, :case["top"]]
                keep = torch.zeros_like(score, dtype=torch.bool).scatter_(1, order, True) & (index <= own_page[:, None])
                seen = seen & keep.repeat_interleave(PAGE, 1)
                rank = keep.cumsum(1) - 1
                token, page = keep.nonzero(as_tuple=True)
                chosen[cu[r] + token, head, rank[token, page]] = page.to(torch.int32)
            x = torch.einsum("ngd,kd->gnk", q, k) / math.sqrt(d)
            x = torch.softmax(x.masked_fill(~seen, -float("inf")), -1)
            out[cu[r]:cu[r + 1], head * g:(head + 1) * g] = torch.einsum("gnk,kd->ngd", x, v)
    return {"out": out} if case["op"] == "attention" else {"out": out, "selected": chosen}

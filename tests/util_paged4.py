"""Plain 64-bit statements of the operators of the paged cache in 4 bits and the error bounds their tests use."""
from __future__ import annotations

import random

import torch

from util_paged import PAGE, pages

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
# the e4m3 numbers of the bytes 0 .. 126 (127: NaN), written out from sign / 4 bits of exponent (bias 7) / 3 bits of mantissa
E4M3 = torch.tensor([(b % 8) * 2.0 ** -9 if b < 8 else (1 + b % 8 / 8) * 2.0 ** (b // 8 - 7) for b in range(127)], dtype=torch.float64)


def nearest(x, table):
    """Place of the nearest number of an ascending table, halves to the even place; x >= 0."""
    mid = (table[1:] + table[:-1]) / 2
    at = torch.bucketize(x, mid)
    return at + ((at % 2 == 1) & (x == mid[at.clamp(max=mid.numel() - 1)])).long()


def quantise(x, shift):
    """(codes [..., H, d] 0 .. 15, scale bytes [..., H, d / 16]) of x [..., H, d], shift [H], on the CPU."""
    y = x.double() * torch.exp2(-shift.double())[:, None]
    y = y.unflatten(-1, (-1, 16))
    amax = y.abs().amax(-1)
    bad = torch.isnan(y).any(-1)
    quotient = (amax.float() / 6).double()                   # in fp32, as it is defined
    byte = torch.where(bad, 127, nearest(torch.where(bad, 0.0, quotient), E4M3))
    s = torch.cat((E4M3, torch.zeros(1, dtype=torch.float64)))[byte][..., None]
    code = torch.where(s > 0, nearest(torch.nan_to_num(y.abs(), nan=0.0) / torch.where(s > 0, s, 1.0), LEVELS), 0)
    return (code + 8 * (y < 0)).flatten(-2), byte


def values(codes, scale_bytes, shift):
    """fp64 values of packed codes [..., H, n, d / 2] and scale bytes [..., H, n, d / 16] (any device), on the CPU."""
    codes, scale_bytes = codes.cpu().long(), scale_bytes.view(torch.uint8).cpu().long()
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    table = torch.cat((E4M3, torch.tensor([float("nan")], dtype=torch.float64)))
    scale = table[scale_bytes & 127] * (1 - 2 * (scale_bytes >> 7))
    return (LEVELS[code & 7] * (1 - 2 * (code >> 3)) * scale.repeat_interleave(16, -1)) * torch.exp2(shift.double().cpu())[:, None, None]


def pack(codes):
    codes = codes.to(torch.uint8)
    return codes[..., ::2] | codes[..., 1::2] << 4


class Cache4:
    """A cache in 4 bits filled for tests: requests of the given lengths over shuffled pages; everything that no request holds has
    NaN scales, table entries behind the last page are out of range.  k, v: the values in fp64 on the CPU."""

    def __init__(self, lens, H, d, device="cuda", seed=0, spare=3, width=None, spread=1.0, shift=0):
        gen = torch.Generator().manual_seed(seed)
        rng = random.Random(seed)
        self.n_pages = sum(pages(n) for n in lens) + spare
        self.width = width or max(1, max(pages(n) for n in lens))
        order = torch.randperm(self.n_pages, generator=gen)
        table = torch.full((len(lens), self.width), 1 << 29, dtype=torch.int32)
        owner = torch.zeros(self.n_pages, dtype=torch.long)   # entries of each page in use
        at = 0
        for r, n in enumerate(lens):
            for p in range(pages(n)):
                table[r, p] = int(order[at])
                owner[order[at]] = min(PAGE, n - p * PAGE)
                at += 1
        unused = torch.arange(PAGE) >= owner[:, None]
        arrays = []
        for x in range(2):
            sh = torch.tensor([rng.randint(-shift, shift) for _ in range(H)], dtype=torch.int32)
            val = torch.randn(self.n_pages, H, PAGE, d, generator=gen)
            if x == 0:
                val = val * spread + torch.randn(self.n_pages, H, 1, d, generator=gen)
            codes, scale = quantise(val.transpose(1, 2), torch.zeros(H))
            codes, scale = pack(codes.transpose(1, 2)), scale.transpose(1, 2).to(torch.uint8)
            scale = torch.where(unused[:, None, :, None], 127, scale).to(torch.uint8)
            arrays += [codes.contiguous(), scale.contiguous(), sh]
        self.k, self.v = values(*arrays[:3]), values(*arrays[3:])
        arrays = [a.to(device) for a in arrays]
        self.arrays = arrays                                  # k codes, scales, shift, v codes, scales, shift
        self.table, self.lens = table.to(device), torch.tensor(lens, dtype=torch.int32, device=device)

    def cache(self):
        from paper_2605_09649_b200 import binding

        kc, ks, ksh, vc, vs, vsh = self.arrays
        return binding.Paged4Cache(kc, ks, vc, vs, ksh, vsh)


def attention(k, v, q, cu, lens, table, scale, window=0):
    """(out, bound) in fp64 on the CPU; k, v [n_pages, H, 64, d] fp64.  bound: largest distance of a correct kernel's output."""
    table = table.cpu().tolist()
    dt, T, Hq, d = q.dtype, q.shape[0], q.shape[1], q.shape[2]
    H = k.shape[1]
    g = Hq // H
    qd = q.double().cpu()
    out = torch.full((T, Hq, d), float("nan"), dtype=torch.float64)
    bound = torch.zeros_like(out)
    for r, total in enumerate(lens):
        n = cu[r + 1] - cu[r]
        if n == 0:
            continue
        rows = slice(cu[r], cu[r + 1])
        pos = torch.arange(total - n, total)
        phys = torch.tensor(table[r][:pages(total)], dtype=torch.long)
        at = torch.arange(total)
        sees = (at <= pos[:, None]) & ((at > pos[:, None] - window) if window else torch.ones(n, total, dtype=torch.bool))
        for h in range(H):
            kk, vv = (x[phys, h].reshape(-1, d)[:total] for x in (k, v))
            qq = qd[rows, h * g:(h + 1) * g]                  # [n, g, d]
            x = torch.where(sees[:, None], qq @ kk.T * scale, -torch.inf)
            top = x.amax(-1, keepdim=True) if total else torch.full(x.shape[:-1] + (1,), -torch.inf)
            w = torch.exp(x - torch.where(top == -torch.inf, 0.0, top))
            norm = w.sum(-1, keepdim=True)
            w = w / torch.where(norm > 0, norm, 1.0)
            o = w @ vv
            logit = torch.where(sees[:, None], qq.abs() @ kk.abs().T * scale, 0.0).amax(-1, keepdim=True) if total else torch.zeros(n, g, 1)
            biggest = torch.where(sees[:, None, :, None], vv.abs(), 0.0).amax(2) if total else torch.zeros(n, 1, d)
            out[rows, h * g:(h + 1) * g] = o
            bound[rows, h * g:(h + 1) * g] = slack(dt, o, w @ vv.abs(), logit, biggest, total, d)
    return out, bound


def slack(dt, o, mass, logit, biggest, n, d):
    """How far a correct output may be from o.  mass = sum w |v|, logit = max over keys of sum |q k| scale, biggest = max |v|, n keys.
    The final rounding takes half a step of o.  The cache's values enter exactly.  A logit is a sum of d products in fp32 and two
    scalings: off by (d + 2) 2^-24 logit; a weight is its exponential, off by twice that (numerator and sum), and the n-term fp32
    sums; tensor cores may truncate instead of rounding a sum's terms: counted by a factor of two.  bf16: a weight is rounded to fp16,
    2^-11 of it, or 2^-32 of the row's largest weight where it is that small (each of n), and a polynomial 2^x may be off by
    7.5e-5, numerator and sum.  fp32: q and weights in two fp16 parts, 2^-22 each; 2^x good to 2 steps of fp32; what two
    parts cannot hold of a small weight is 2^-32 of the largest.  q: 2^-35 of the row's largest value, within the fp32 terms."""
    step = torch.finfo(dt).eps / 2
    fp32 = 2 * (2 * (d + 2) * logit + n + 16) * 2.0 ** -24
    weights = 2.0 ** -11 + 1.5e-4 if dt == torch.bfloat16 else 2 * (2.0 ** -22 * (1 + logit) + 4 * 2.0 ** -24)
    return step * o.abs() + (fp32 + weights) * mass + n * 2.0 ** -32 * biggest + 1e-30

"""Definitions for the tests of caches in 8 bits with a scale for each page and head, and of the plan: on the CPU, one thing after
the other."""
import math
import random

import torch


def block_scale(top):
    """The least m 2^e with m = 4, 5, 6, 7 and 127 m 2^e >= top, at least 2^-126; 0 for 0, NaN for what is not finite."""
    if not math.isfinite(top):
        return math.nan
    if top == 0.0:
        return 0.0
    e = math.frexp(top)[1] - 14
    while True:
        for m in (4, 5, 6, 7):
            if 127 * m * 2.0**e >= top:
                return max(m * 2.0**e, 2.0**-126)
        e += 1


class Blocks:
    """An int8 cache whose pages hold `kvs[b]` tokens of each sequence, under scales of 3 significant bits that differ by up to
    2^spread; rows of nobody hold codes of their own, pages of nobody are under NaN."""

    def __init__(self, kvs, H, D, page, layout="head", seed=0, spare=2, device="cuda", spread=3, room=0, cancel=False):
        g = torch.Generator().manual_seed(seed)
        r = random.Random(seed)
        self.kvs, self.lens, self.H, self.D, self.page = list(kvs), list(kvs), H, D, page
        B, need = len(kvs), [-(-n // page) for n in kvs]
        self.n_pages = sum(need) + spare
        ids = list(range(self.n_pages))
        r.shuffle(ids)
        M = max(max(need), -(-room // page), 1) + (0 if room else 1)
        self.table_cpu = torch.full((B, M), -1, dtype=torch.int32)
        there, at = torch.zeros(self.n_pages, dtype=torch.bool), 0
        for b, n in enumerate(need):
            self.table_cpu[b, :n] = torch.tensor(ids[at:at + n], dtype=torch.int32)
            there[ids[at:at + n]] = True
            at += n
        self.codes, self.scales, self.stored, self.scale = {}, {}, {}, {}
        for n in ("k", "v"):
            x = torch.randn((self.n_pages, H, page, D), generator=g)
            if cancel and n == "v":  # rows of one sign and of the other in turn: sums far smaller than their terms
                x = 3.0 * (1 - 2 * (torch.arange(page) % 2))[:, None] + 0.2 * x
            codes = (30 * x).round().clamp(-127, 127).to(torch.int8)
            m, e = torch.randint(4, 8, (self.n_pages, H), generator=g), torch.randint(0, spread + 1, (self.n_pages, H), generator=g)
            scale = torch.ldexp(m.float(), -e - 6)
            scale[~there] = math.nan
            self.codes[n], self.scales[n] = codes, scale
            self.scale[n] = scale.to(device)
            if layout == "token":  # [n_pages, page, H, D]
                store = codes.transpose(1, 2).contiguous().to(device).transpose(1, 2)
            elif layout == "joint":  # k and v of a page beside each other, with room between rows
                pad = torch.zeros((self.n_pages, 2, H, page, D + 16), dtype=torch.int8, device=device)
                store = pad[:, int(n == "v"), :, :, :D]
                store.copy_(codes)
            else:
                store = codes.to(device)
            self.stored[n] = store
        self.page_table = self.table_cpu.to(device)
        self.kv_len = torch.tensor(self.kvs, dtype=torch.int32, device=device)

    def args(self):
        return self.stored["k"], self.stored["v"], self.page_table, self.kv_len

    def scale_args(self):
        return dict(k_scale=self.scale["k"], v_scale=self.scale["v"])

    exps = scale_args

    def sequence(self, n, b, length=None):
        """fp64 [H, length, D] of sequence b as the CPU's codes and scales say; zeros where the table names no page."""
        length = self.kvs[b] if length is None else length
        out = torch.zeros((self.H, length, self.D), dtype=torch.float64)
        for p in range(-(-length // self.page)):
            rows = min(self.page, length - p * self.page)
            i = self.table_cpu[b, p].item() if p < self.table_cpu.shape[1] else -1
            if 0 <= i < self.n_pages:
                out[:, p * self.page:p * self.page + rows] = self.codes[n][i, :, :rows].double() * self.scales[n][i].double()[:, None, None]
        return out

    def write(self, qs, k, v):
        """Writes new tokens (CPU) into the CPU's codes and scales."""
        at = 0
        for b, n in enumerate(qs):
            kv, cap = self.lens[b], self.table_cpu.shape[1] * self.page
            for p in range(max(kv - n, 0) // self.page, -(-min(kv, cap) // self.page)):
                lo, first, hi = p * self.page, max(p * self.page, kv - n, 0), min((p + 1) * self.page, kv, cap)
                i = self.table_cpu[b, p].item()
                if hi <= first or not 0 <= i < self.n_pages:
                    continue
                for name, x in (("k", k), ("v", v)):
                    for h in range(self.H):
                        rows = x[at + first - (kv - n):at + hi - (kv - n), h].double()
                        top = math.nan if rows.isnan().any() else rows.abs().max().item()
                        need, had = block_scale(top), self.scales[name][i, h].item() if first > lo else 0.0
                        codes = self.codes[name][i, h]
                        if need > had and first > lo:
                            codes[:first - lo] = torch.round(codes[:first - lo].double() * had / need).to(torch.int8)
                        scale = need if need > had or math.isnan(need) else had
                        self.scales[name][i, h] = scale
                        some = scale > 0
                        codes[first - lo:hi - lo] = torch.round(rows / scale).to(torch.int8) if some else 0
            at += n

    def same(self, what=""):
        """The GPU's codes and scales are the CPU's, bit for bit (a NaN is a NaN)."""
        for n in ("k", "v"):
            got, want = self.scale[n].cpu(), self.scales[n]
            assert ((got == want) | (got.isnan() & want.isnan())).all(), f"{what}: scales of {n}"
            off = (self.stored[n].cpu() != self.codes[n])
            assert not off.any(), f"{what}: {off.sum().item()} codes of {n}"


def tolerance(pages, q, qs, causal=1, window=0, scale=0.0, weight=2.0**-11):
    """out [T,Hq,D], lse [Hq,T] in 64 bits on the CPU, and how far a right kernel may be off each.

    Logits: products of queries (bf16) and codes are exact in fp32; D sums, the start, the scale, its product with the query's
    power of two and with log2 e, and the difference to the reference: d = (D + 8) 2^-24 scale max_j sum |q k_j|.  exp2 is good to
    2^-22.  Weights are rounded to f16 (`weight` 2^-11; below 2^-14, where the largest is at least 2^7, to steps of 2^-24), of few
    rows to a sum of two bf16 (2^-16); n of them and of their products are added, 2^-24 each; values of 3 significant bits times a
    code are exact.  The quotient is rounded to bf16 (2^-8).  With A = sum p |v|:
      |out - exact| <= (weight + 2 d + n 2^-23 + 2^-20) A + 2^-32 sum |v| + 2^-8 (1 + 2^-6) |out|
      |lse - exact| <= d + n 2^-24 + 2^-22 (1 + |lse|)."""
    T, Hq, D = q.shape
    G = Hq // pages.H
    scale = scale or 1.0 / math.sqrt(D)
    out, tol = torch.zeros((T, Hq, D), dtype=torch.float64), torch.zeros((T, Hq, D), dtype=torch.float64)
    lse, ltol = torch.full((Hq, T), -math.inf, dtype=torch.float64), torch.zeros((Hq, T), dtype=torch.float64)
    at = 0
    for b, n in enumerate(qs):
        kv, there = pages.lens[b], pages.kvs[b]
        if n and kv > 0:
            k, v = pages.sequence("k", b, there), pages.sequence("v", b, there)
            p = torch.arange(kv - n, kv)
            hi = ((p // causal + 1) * causal).clamp_max(kv).masked_fill(p < 0, 0) if causal else torch.full_like(p, kv)
            lo = (hi - window).clamp_min(0) if window else torch.zeros_like(hi)
            j = torch.arange(there)
            hidden = (j < lo[:, None]) | (j >= hi[:, None])
            some = (hi.clamp_max(there) > lo)[:, None]
            for h in range(Hq):
                x, kh, vh = q[at:at + n, h].double(), k[h // G], v[h // G]
                s = (x @ kh.t() * scale).masked_fill(hidden, -math.inf)
                l = torch.logsumexp(s, -1)
                w = torch.exp(s - torch.where(some[:, 0], l, 0.0)[:, None])
                d = (D + 8) * 2.0**-24 * scale * (x.abs() @ kh.abs().t()).masked_fill(hidden, 0.0).amax(-1)
                o = w @ vh
                small = 2.0**-32 * (~hidden).double() @ vh.abs()
                out[at:at + n, h] = o
                tol[at:at + n, h] = ((weight + 2 * d[:, None] + there * 2.0**-23 + 2.0**-20) * (w @ vh.abs()) + small
                                     + 2.0**-8 * (1 + 2.0**-6) * o.abs())
                lse[h, at:at + n] = l
                ltol[h, at:at + n] = d + there * 2.0**-24 + 2.0**-22 * (1 + torch.where(some[:, 0], l.abs(), 0.0))
        at += n
    return out, lse, tol, ltol


def plan(add, kv, keep, table, free, n_free, page, T):
    """heart_cache_plan of lists (`table` of lists): request after request, page after page.  Returns new ones."""
    B, M, n_pages = len(kv), len(table[0]), len(free)
    table, free = [list(t) for t in table], list(free)
    up = lambda n: -(-n // page)  # noqa: E731
    kv = [min(max(n, 0), M * page) for n in kv]
    keep = [min(max(k, 0), n) for k, n in zip(keep, kv)]
    first = min(max(n_free, 0), n_pages)
    back = [(b, p) for b in range(B) for p in range(up(keep[b]), up(kv[b]))]
    top = min(first + len(back), n_pages)
    for j, (b, p) in enumerate(back):
        if top - 1 - j >= first:
            free[top - 1 - j] = table[b][p]
        table[b][p] = -1
    asked = tokens = 0
    cu, slots, positions, left = [0], [-1] * T, [-1] * T, top
    for b in range(B):
        n, had = max(add[b], 0), up(keep[b])
        fits = n > 0 and keep[b] + n <= M * page
        need = up(keep[b] + n) - had if fits else 0
        asked += need
        paged = fits and (need == 0 or asked <= top)
        tokens += n if paged else 0
        if not paged or tokens > T:
            n = need = 0
        for p in range(had, had + need):
            left -= 1
            table[b][p] = free[left]
        for i in range(n):
            pos = keep[b] + i
            at = table[b][pos // page]
            positions[cu[-1] + i] = pos
            if 0 <= at < n_pages:
                slots[cu[-1] + i] = at * page + pos % page
        kv[b] = keep[b] + n
        cu.append(cu[-1] + n)
    return dict(cu_q=cu, slots=slots, positions=positions, kv_len=kv, page_table=table, free_pages=free[:left], n_free=[left])

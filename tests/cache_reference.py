"""Attention over a paged cache in 64 bits on the GPU, for caches too large for the definition on the CPU, with derived tolerances."""
import math
import random

import torch

E4M3 = torch.float8_e4m3fn
FILL = 0x55  # what a workspace holds before a call


class Pages:
    """Pages of random tokens in random order; rows behind a sequence's last token, and pages of nobody, hold NaN.  `room`: tokens
    that the page table has room for (at least those of the longest sequence)."""

    def __init__(self, kvs, H, D, page=64, kind="bf16", seed=0, room=0, cancel=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = random.Random(seed)
        self.kvs, self.H, self.D, self.page, self.kind = list(kvs), H, D, page, kind
        self.lens = self.kvs  # (kv_len, which may be more than there is room for)
        need = [-(-n // page) for n in kvs]
        n_pages, M = sum(need) + 2, max(max(need), -(-room // page), 1)
        ids = list(range(n_pages))
        r.shuffle(ids)
        table, there, at = [], torch.zeros((n_pages, page), dtype=torch.bool), 0
        for b, n in enumerate(need):
            mine = ids[at:at + n]
            table.append(mine + [-1] * (M - n))
            for p, i in enumerate(mine):
                there[i, :kvs[b] - p * page] = True
            at += n
        self.cap, self.n_pages = M * page, n_pages
        self.page_table = torch.tensor(table, dtype=torch.int32, device="cuda")
        self.kv_len = torch.tensor(self.kvs, dtype=torch.int32, device="cuda")
        gone = ~there.cuda()[:, None, :, None]
        self.stored, self.exp = {}, {}
        for n in ("k", "v"):
            x = torch.randn((n_pages, H, page, D), generator=g, device="cuda")
            if cancel and n == "v":  # rows of one sign and of the other in turn: sums far smaller than their terms
                x = 8.0 * (1 - 2 * (torch.arange(page, device="cuda") % 2))[:, None] + 2.0**-4 * x
            if kind == "e4m3":
                self.exp[n] = torch.randint(125, 130, (n_pages, H, page), generator=g, device="cuda", dtype=torch.uint8)
                self.exp[n].masked_fill_(gone[..., 0], 255)
                self.stored[n] = x.clamp(-400, 400).masked_fill_(gone, math.nan).to(E4M3)
            else:
                self.exp[n], self.stored[n] = None, x.masked_fill_(gone, math.nan).bfloat16()

    def args(self):
        return self.stored["k"], self.stored["v"], self.page_table, self.kv_len

    def exps(self):
        return dict(k_exp=self.exp["k"], v_exp=self.exp["v"])

    def sequence(self, n, b):
        """fp64 [H, tokens, D] of sequence b."""
        kv = self.kvs[b]
        ids = self.page_table[b, :-(-kv // self.page)].long()
        x = self.stored[n].view(torch.uint8)[ids].view(self.stored[n].dtype).float().double()
        if self.kind == "e4m3":
            x = x * torch.exp2(self.exp[n][ids].double() - 127.0)[..., None]
        return x.permute(1, 0, 2, 3).flatten(1, 2)[:, :kv]


def reference(pages, q, qs, causal=1, window=0, scale=0.0, chain=None, weight=2.0**-8):
    """out [T,Hq,D], lse [Hq,T] of q, and how far a right kernel may be off each.

    d: error of a logit.  The products of bf16 values are exact; their sum of D terms, the start from the reference, its
    subtraction and the scaling add D + 8 roundings of 2^-24 of scale sum |q k|.  exp2 is good to 2^-22.  A weight and its
    product are added at most `chain` times (keys of a part, and parts; all keys by default), 2^-24 each, in numerator and
    denominator.  `weight`: rounding of a weight (bf16 2^-8; a sum of two bf16 2^-16: the second is at most 2^-8 of the first, and rounded
    to 2^-8 of itself).  The quotient is rounded to bf16 (2^-8).  With A = sum p |v|:
      |out - exact| <= (weight + 2 d + 2 chain 2^-24 + 2^-20) A + 2^-8 (1 + 2^-6) |out|
      |lse - exact| <= d + chain 2^-24 + 2^-22 (1 + |lse|)."""
    T, Hq, D = q.shape
    G = Hq // pages.H
    scale = scale or 1.0 / math.sqrt(D)
    z = dict(dtype=torch.float64, device="cuda")
    out, tol = torch.zeros((T, Hq, D), **z), torch.zeros((T, Hq, D), **z)
    lse, ltol = torch.full((Hq, T), -math.inf, **z), torch.zeros((Hq, T), **z)
    at = 0
    for b, n in enumerate(qs):
        kv, there = pages.lens[b], pages.kvs[b]
        if n and kv:
            k, v = pages.sequence("k", b), pages.sequence("v", b)
            p = torch.arange(kv - n, kv, device="cuda")
            hi = ((p // causal + 1) * causal).clamp_max(kv).masked_fill(p < 0, 0) if causal else torch.full_like(p, kv)
            lo = (hi - window).clamp_min(0) if window else torch.zeros_like(hi)
            j = torch.arange(there, device="cuda")
            hidden = (j < lo[:, None]) | (j >= hi[:, None])
            some = (hi.clamp_max(there) > lo)[:, None]
            c = there if chain is None else chain
            for h in range(Hq):
                x, kh, vh = q[at:at + n, h].double(), k[h // G], v[h // G]
                s = (x @ kh.t() * scale).masked_fill(hidden, -math.inf)
                l = torch.logsumexp(s, -1)
                w = torch.exp(s - torch.where(some[:, 0], l, 0.0)[:, None])
                d = (D + 8) * 2.0**-24 * scale * (x.abs() @ kh.abs().t()).masked_fill(hidden, 0.0).amax(-1)
                o = w @ vh
                out[at:at + n, h] = o
                tol[at:at + n, h] = (weight + 2 * d[:, None] + c * 2.0**-23 + 2.0**-20) * (w @ vh.abs()) + 2.0**-8 * (1 + 2.0**-6) * o.abs()
                lse[h, at:at + n] = l
                ltol[h, at:at + n] = d + c * 2.0**-24 + 2.0**-22 * (1 + torch.where(some[:, 0], l.abs(), 0.0))
        at += n
    return out, lse, tol, ltol


def near(got, want, tol, what):
    got = got.double()
    ok = (got == want) | ((got - want).abs() <= tol)
    worst = ((got - want).abs() - tol).masked_fill(ok, 0.0)
    assert ok.all(), f"{what}: {(~ok).sum().item()} of {ok.numel()} off, worst by {worst.nan_to_num(nan=math.inf).max().item():.3g}"

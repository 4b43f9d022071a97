"""Inputs, definitions in 64 bits and derived tolerances for the tests of the paged key/value cache."""
import math
import random

import torch

E4M3 = torch.float8_e4m3fn


def e4m3_values(x):
    """fp64 rows of x [..., D] as 8-bit rows stand for them, and the exponent bytes: from the format (4 significant bits, steps
    of 2^-9 at least, largest 448) and the rule of the exponent (least power of two, 2^-126 at least, 1 for zeros)."""
    x = x.double()
    finite = torch.isfinite(x)
    top = torch.where(finite, x.abs(), 0.0).amax(-1, keepdim=True)
    m, e = torch.frexp(top)  # top = m 2^e, 1/2 <= m < 1; 448 = 7/8 * 2^9
    e = torch.where(top > 0, torch.where(m <= 0.875, e - 9, e - 8).clamp_min(-126), 0)
    unit = torch.exp2(e.double())
    y = torch.where(finite, x, 0.0) / unit
    step = torch.exp2((torch.frexp(y.abs())[1] - 1 - 3).clamp_min(-9).double())
    val = torch.round(y / step) * step  # (ties to even)
    return torch.where(finite, val * unit, math.nan), (e[..., 0] + 127).to(torch.uint8)


class Cache:
    """A cache on `device` whose pages hold `kvs[b]` random tokens of each sequence; everything else holds garbage."""

    def __init__(self, kvs, H, D, page, kind="bf16", layout="head", seed=0, spare=2, device="cuda", gain=1.0):
        g = torch.Generator().manual_seed(seed)
        r = random.Random(seed)
        self.kvs, self.H, self.D, self.page, self.kind = list(kvs), H, D, page, kind
        B = len(kvs)
        need = [-(-n // page) for n in kvs]
        self.n_pages = sum(need) + spare
        ids = list(range(self.n_pages))
        r.shuffle(ids)
        M = max(max(need), 1) + 1
        table = torch.full((B, M), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = torch.tensor(ids[at:at + n], dtype=torch.int32)
            at += n
        shape = (self.n_pages, H, page, D)
        self.value, self.stored, self.exp = {}, {}, {}
        for n in ("k", "v"):
            x = torch.full(shape, math.nan, dtype=torch.float64)
            for b in range(B):
                for p in range(need[b]):
                    rows = min(page, kvs[b] - p * page)
                    y = torch.randn((H, rows, D), generator=g) * torch.exp(0.5 * torch.randn((H, rows, 1), generator=g)) * gain
                    x[table[b, p].item(), :, :rows] = y.bfloat16().double()
            if kind == "e4m3":
                there = ~torch.isnan(x).any(-1)
                val, exp = e4m3_values(torch.where(there[..., None], x, 0.0))
                codes = torch.ldexp(val, 127 - exp.int().unsqueeze(-1)).float().to(E4M3).view(torch.uint8)
                codes[~there] = 0x7F
                exp[~there] = 255
                self.value[n], store, self.exp[n] = val, codes.view(E4M3), exp.to(device)
            else:
                self.value[n], store, self.exp[n] = x, x.bfloat16(), None
            if layout == "token":  # [n_pages, page, H, D]
                store = store.transpose(1, 2).contiguous().to(device).transpose(1, 2)
            elif layout == "joint":  # k and v of a page beside each other, with room between rows
                pad = torch.zeros((self.n_pages, 2, H, page, D + 16), dtype=torch.uint8).to(device)
                pad = pad.view(E4M3) if kind == "e4m3" else pad.bfloat16()
                i = int(n == "v")
                pad.view(torch.uint8)[:, i, :, :, :D] = store.to(device).view(torch.uint8) if kind == "e4m3" else 0
                if kind != "e4m3":
                    pad[:, i, :, :, :D] = store.to(device)
                store = pad[:, i, :, :, :D]
            else:
                store = store.to(device)
            self.stored[n] = store
        self.table_cpu = table
        self.page_table = table.to(device)
        self.kv_len = torch.tensor(list(kvs), dtype=torch.int32, device=device)

    def args(self):
        return self.stored["k"], self.stored["v"], self.page_table, self.kv_len

    def exps(self):
        return dict(k_exp=self.exp["k"], v_exp=self.exp["v"])

    def sequence(self, n, b, length=None):
        """fp64 [H, length, D] of sequence b; zeros where the table names no page."""
        length = self.kvs[b] if length is None else length
        out = torch.zeros((self.H, length, self.D), dtype=torch.float64)
        for p in range(-(-length // self.page)):
            rows = min(self.page, length - p * self.page)
            i = self.table_cpu[b, p].item() if p < self.table_cpu.shape[1] else -1
            if 0 <= i < self.n_pages:
                out[:, p * self.page:p * self.page + rows] = self.value[n][i, :, :rows]
        return out


def seen(p, kv, causal, window):
    hi = kv if causal == 0 else (min(kv, (p // causal + 1) * causal) if p >= 0 else 0)
    return (max(0, hi - window) if window else 0), hi


def attention(cache, q, qs, causal, window, scale=None):
    """fp64 out [T,Hq,D], lse [Hq,T] of q (CPU), and how far a right kernel may be off each.

    Logits: products of bf16 values are exact in fp32; a sum of D of them in any order is off by at most D 2^-24 sum |q k|, the
    scaling by three roundings, the difference to the reference exponent by one more: d = scale (D + 4) 2^-24 max_j sum |q k_j|
    + 2^-24 * 4 |s|max.  exp2 is good to 2^-22, so weights are off by a factor 1 + d + 2^-22; they are rounded to bf16 (2^-8),
    the n of them summed in fp32 (n 2^-24), and the quotient rounded to bf16 (2^-8).  With A = sum p |v|:
      |out - exact| <= (2^-8 + 2 d + n 2^-23 + 2^-20) A + 2^-8 |out| (1 + 2^-6)
      |lse - exact| <= d + n 2^-24 + 2^-22 + 2^-22 |lse|."""
    T, Hq, D = q.shape
    G = Hq // cache.H
    scale = scale or 1.0 / math.sqrt(D)
    out = torch.zeros((T, Hq, D), dtype=torch.float64)
    lse = torch.full((Hq, T), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    at = 0
    for b, n in enumerate(qs):
        kv = cache.kvs[b]
        k, v = cache.sequence("k", b), cache.sequence("v", b)
        j = torch.arange(kv)
        lim = [seen(kv - n + i, kv, causal, window) for i in range(n)]
        if n:
            lo, hi = torch.tensor(lim).unbind(1)
            vis = (j >= lo[:, None]) & (j < hi[:, None])
        for h in range(Hq if n else 0):
            x = q[at:at + n, h].double()
            kh, vh = k[h // G], v[h // G]
            s = torch.where(vis, x @ kh.t() * scale, -math.inf)
            some = vis.any(1)
            w = torch.softmax(torch.where(some[:, None], s, 0.0), -1) * some[:, None] if kv else s
            o, A = w @ vh, w @ vh.abs()
            mag = torch.where(vis, x.abs() @ kh.abs().t(), 0.0).amax(-1) * scale if kv else torch.zeros(n, dtype=torch.float64)
            d = (D + 8) * 2.0**-24 * mag
            out[at:at + n, h] = o
            tol[at:at + n, h] = (2.0**-8 + 2 * d[:, None] + kv * 2.0**-23 + 2.0**-20) * A + 2.0**-8 * (1 + 2.0**-6) * o.abs()
            l = torch.where(some, torch.logsumexp(s, -1), -math.inf) if kv else torch.full((n,), -math.inf, dtype=torch.float64)
            lse[h, at:at + n] = l
            ltol[h, at:at + n] = d + kv * 2.0**-24 + 2.0**-22 + 2.0**-22 * torch.where(some, l.abs(), 0.0) if kv else 0.0
        at += n
    return out, lse, tol, ltol


def assert_near(got, want, tol, what):
    got = got.double().cpu()
    assert torch.isfinite(got).all() or not torch.isfinite(want).all(), f"{what}: not finite"
    same = (got == want) | ((got - want).abs() <= tol)
    worst = ((got - want).abs() - tol)[~same]
    assert same.all(), f"{what}: {(~same).sum().item()} of {same.numel()} off, worst by {worst.max().item():.3g}"


def ends(qs, device="cuda"):
    return torch.tensor([sum(qs[:b]) for b in range(len(qs) + 1)], dtype=torch.int32, device=device)

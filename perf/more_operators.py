"""Timed cases of the cache's plan and of the cache in 8 bits under a scale for each page and head.

A case is a dict of plain values.  `op` says what one pass calls:

  plan    heart_cache_plan: pages, token ranges, slots and positions of a step's new tokens, from the requests' lengths
  write   heart_cache_write of a chunk into an int8 cache, then heart_cache_read of it, so that the output is the values that
          the codes stand for
  read    heart_cache_read of an int8 cache: the cached tokens as the [B,H,N,D] tensors of pooling and block-sparse attention
  attn    heart_cache_attn over an int8 cache, which holds the chunk already

plan: B requests that have up to `kv` tokens and get up to `q` new ones; of every 100, `ended` have ended (their pages go back, a
few begin anew) and `undone` take back some tokens; `spare`: free pages for so many percent of what is asked for; `room`:
new tokens the outputs hold (0: all).  The others: B sequences of up to `q` new tokens and `kv` cached ones (with them);
`ragged`: lengths that differ, made from `mix`.  `page` tokens a page, pages in random order.  `causal`: 0 a row sees the whole
cache, n it sees the blocks of n positions up to its own; `window`: only the last so many of those.

Where `own` is false the operators are computed from torch operations in 32 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_FRAME = 30 * 52  # tokens of a latent frame at 480P


def _case(name, op, *, B=1, q=1, kv=1, ragged=False, Hq=1, Hkv=1, D=128, page=64, causal=1, window=0, lse=False, ended=0, undone=0,
          spare=130, room=0, mix=1):
    c = {"op": op, "B": B, "q": q, "kv": kv, "page": page, "ragged": ragged, "mix": mix}
    if op == "plan":
        c.update(ended=ended, undone=undone, spare=spare, room=room)
    else:
        c.update(Hq=Hq, Hkv=Hkv, D=D, causal=causal, window=window, lse=lse)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decoding step of a few requests: latency alone
        _case("plan_tokens_few", "plan", B=3, q=1, kv=700, page=16, ragged=True),
        # a serving batch whose drafts were in part refused; some requests have ended and others took their places
        _case("plan_drafts_batch", "plan", B=256, q=8, kv=9000, page=32, ragged=True, ended=9, undone=60, mix=2),
        # prompts of many requests come in, more than there are pages for
        _case("plan_prompts", "plan", B=1500, q=1021, kv=2000, page=64, ragged=True, ended=30, undone=5, spare=70, mix=3),
        # the tokens of one decoding step, into pages that are begun
        _case("write_tokens", "write", B=64, q=1, kv=500, ragged=True, Hkv=8, page=16, mix=5),
        # a later chunk of a clip: three latent frames behind three others
        _case("write_frames", "write", q=3 * _FRAME, kv=6 * _FRAME, Hkv=40, page=64),
        # the whole cached clip for the sparse path
        _case("read_clip", "read", kv=21 * _FRAME, Hkv=12, page=64),
        # a ragged batch, rows behind the last token left alone
        _case("read_ragged", "read", B=7, kv=4099, ragged=True, Hkv=5, D=64, page=16, mix=6),
        # one new token after a short prompt, two heads: latency alone
        _case("attn_token_small", "attn", kv=1000, Hq=2, Hkv=2, D=64, page=16),
        # a serving batch that decodes: ragged lengths, five query heads a key head
        _case("attn_tokens_batch", "attn", B=64, kv=8192, ragged=True, Hq=40, Hkv=8, page=16, mix=2),
        # drafted tokens that are verified together, sliding window, head dimension 64
        _case("attn_drafts_window", "attn", B=16, q=8, kv=16384, ragged=True, Hq=24, Hkv=3, D=64, page=32, window=4096, lse=True,
              mix=3),
        # prompts taken in by chunks, ragged
        _case("attn_prompts_ragged", "attn", B=6, q=2048, kv=12000, ragged=True, Hq=40, Hkv=8, page=32, lse=True, mix=4),
        # three latent frames of a clip that is generated chunk by chunk, frame after frame: Wan2.1-14B heads at 480P, the largest
        _case("attn_frames_wan14b", "attn", q=3 * _FRAME, kv=21 * _FRAME, Hq=40, Hkv=40, page=64, causal=_FRAME),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: from one token of a short sequence to the chunks of a clip."""
    op = rng.choice(["plan", "plan", "write", "write", "read", "attn", "attn", "attn"])
    page, mix = rng.choice([16, 32, 64, 128, 256]), rng.randrange(1 << 20)
    if op == "plan":
        B = _log(rng, 1, 4000)
        q = _log(rng, 1, min(4680, max(2, 800_000 // B)))
        return _case("", op, B=B, q=q, kv=_log(rng, 16, max(32, min(60000, 4_000_000 // B))), page=page, ragged=rng.random() < 0.8,
                     ended=rng.choice([0, 3, 25]), undone=rng.choice([0, 0, 50]), spare=rng.choice([60, 100, 130, 400]),
                     room=rng.choice([0, 0, 0, max(1, B * q // 3)]), mix=mix)
    D, Hkv, G = rng.choice([64, 128, 128]), rng.choice([1, 2, 3, 4, 5, 8, 12]), rng.choice([1, 1, 2, 4, 5, 8])
    form = rng.choice(["token", "token", "draft", "chunk", "chunk"])
    if form == "token":
        q, B = 1, _log(rng, 1, 64)
    elif form == "draft":
        q, B = rng.randint(2, 16), _log(rng, 1, 16)
    else:
        q, B = _log(rng, 64, 4680), _log(rng, 1, 6)
    kv = max(q, _log(rng, 64, 65536 if form != "chunk" else 32768))
    # (no more than the largest listed case: scores of the padded batch, elements of the padded cache)
    while B > 1 and (B * Hkv * G * q * kv > 40 * 4680 * 32760 // 2 or B * Hkv * kv * D > 40 * 32760 * 128):
        B -= 1
    while B * Hkv * kv * D > 40 * 32760 * 128 and kv > q:
        kv = max(q, kv * 3 // 4)
    return _case("", op, B=B, q=q, kv=kv, ragged=rng.random() < 0.6, Hq=Hkv * G, Hkv=Hkv, D=D, page=page,
                 causal=rng.choice([1, 1, 0, rng.randint(16, 1600)]) if form == "chunk" else 1,
                 window=rng.choice([0, 0, 0, _log(rng, 16, 8192)]), lse=rng.random() < 0.3, mix=mix)


# ---- inputs -------------------------------------------------------------------------------------

def _lengths(case):
    """(new tokens, cached tokens) of every sequence: a function of the case alone."""
    if not case["ragged"]:
        return [case["q"]] * case["B"], [case["kv"]] * case["B"]
    rng = random.Random(case["mix"])
    qs, kvs = [case["q"]], [case["kv"]]
    for _ in range(case["B"] - 1):
        n = rng.randint(1, case["q"])
        qs.append(n)
        kvs.append(max(n, _log(rng, max(1, case["kv"] // 32), case["kv"])))
    return qs, kvs


def _requests(case):
    """(new tokens, cached tokens, tokens kept) of every request, tokens the outputs hold, pages a request can have, free pages."""
    rng, P = random.Random(case["mix"] + 77), case["page"]
    add, kv = _lengths({**case, "B": case["B"]})
    keep = list(kv)
    for b in range(case["B"]):
        x = rng.randrange(100)
        if x < case["ended"]:
            keep[b] = 0
            if rng.random() < 0.4:
                add[b] = 0
        elif x < case["ended"] + case["undone"]:
            keep[b] = max(0, kv[b] - rng.randint(1, max(1, case["q"])))
    pages = max(-(-(case["kv"] + case["q"]) // P), 1)
    asked = sum(-(-(k + n) // P) - -(-k // P) for k, n in zip(keep, add))
    back = sum(-(-n // P) - -(-k // P) for n, k in zip(kv, keep))
    free = max(asked * case["spare"] // 100 - back, 0) + 1
    return add, kv, keep, case["room"] or max(sum(add), 1), pages, free


_STEP = 0x1FFFFF  # the bits of a float behind the third significant one


def _scale_of(top):
    """Scales of blocks whose largest magnitudes are `top` (fp32): of 3 significant bits, the least with 127 scale >= top."""
    up = ((top / 127.0).contiguous().view(torch.int32) + _STEP & ~_STEP).view(torch.float32)
    up = torch.where(top > 0, up.clamp_min(2.0 ** -126), 0.0)
    return torch.where(torch.isfinite(top), up, math.nan)


def _to_codes(x, scale):
    """Codes of fp32 x under scales of its shape: the nearest multiple, ties to even."""
    some = scale > 0
    return torch.where(some, torch.round(x / torch.where(some, scale, 1.0)), 0.0).to(torch.int8)


def _random_pages(need, spare, r):
    order = list(range(sum(need) + spare))
    r.shuffle(order)
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n])
        at += n
    return table, order[at:]


def _prepare_plan(case, seed):
    add, kv, keep, T, pages, free = _requests(case)
    r = random.Random(9_000_011 * seed + 29)
    B, P = case["B"], case["page"]
    table, rest = _random_pages([-(-n // P) for n in kv], free, r)
    i32 = dict(dtype=torch.int32, device="cuda")
    n_pages = sum(len(t) for t in table) + free
    st = {"case": case, "add": torch.tensor(add, **i32), "kv_len": torch.tensor(kv, **i32), "keep": torch.tensor(keep, **i32),
          "page_table": torch.tensor([t + [-1] * (pages - len(t)) for t in table], **i32),
          "free_pages": torch.tensor(rest + [-1] * (n_pages - free), **i32), "n_free": torch.tensor([free], **i32), "T": T}
    if own:
        import paper_2605_14513_amd as heart

        st["workspace"] = torch.empty(heart.heart_cache_plan_workspace_bytes(B, pages, T), dtype=torch.uint8, device="cuda")
        st["cu_q"], st["positions"] = torch.empty(B + 1, **i32), torch.empty(T, **i32)
        st["slots"] = torch.empty(T, dtype=torch.int64, device="cuda")
    return st


def prepare(case, seed):
    if case["op"] == "plan":
        return _prepare_plan(case, seed)
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(9_000_011 * seed + 23)
    r = random.Random(seed)
    B, Hq, Hkv, D, P = (case[n] for n in ("B", "Hq", "Hkv", "D", "page"))
    qs, kvs = _lengths(case)
    T = sum(qs)
    i32 = dict(dtype=torch.int32, device=dev)
    need = [-(-n // P) for n in kvs]
    pages, rest = _random_pages(need, 3, r)
    n_pages = sum(need) + 3
    st = {"case": case, "page_table": torch.tensor([p + [-1] * (max(need) - len(p)) for p in pages], **i32),
          "kv_len": torch.tensor(kvs, **i32),
          "cu_q": torch.tensor([sum(qs[:b]) for b in range(B + 1)], **i32) if case["ragged"] else None}
    # rows that a page holds: in writing, those before the new ones
    there = [0] * n_pages
    for p, n, kv in zip(pages, qs, kvs):
        kv -= n if case["op"] == "write" else 0
        for i, page in enumerate(p):
            there[page] = min(max(kv - i * P, 0), P)
    there = torch.tensor(there, **i32)[:, None, None, None] > torch.arange(P, device=dev)[None, None, :, None]

    # keys are normalised rows whose channels differ, values rows of differing size, as projections leave them
    gain = torch.exp(0.4 * torch.randn((Hkv, 1, D), generator=g, device=dev))

    def rows(n, *shape):
        x = torch.randn(shape, generator=g, device=dev)
        if n == "k":
            return x.mul_(gain.transpose(0, 1) if len(shape) == 3 else gain)
        return x.mul_(torch.exp(0.25 * torch.randn(shape[:-1] + (1,), generator=g, device=dev)))

    st["q"] = (1.2 * torch.randn((T, Hq, D), generator=g, device=dev)).bfloat16()
    for n in ("k", "v"):
        st[n] = rows(n, T, Hkv, D).bfloat16()  # the new tokens, where they are written
        x = rows(n, n_pages, Hkv, P, D).bfloat16().float().mul_(there)
        st[n + "_scale"] = _scale_of(x.abs().amax((2, 3)))
        st[n + "_cache"] = _to_codes(x, st[n + "_scale"][:, :, None, None])
        del x
        if case["op"] != "attn":
            st[n + "_out"] = torch.zeros((B, Hkv, max(kvs), D), dtype=torch.bfloat16, device=dev)
    if own and case["op"] == "attn":
        import paper_2605_14513_amd as heart

        st["workspace"] = torch.empty(
            heart.heart_cache_attn_workspace_bytes(st["q"], st["k_cache"], st["page_table"]), dtype=torch.uint8, device=dev)
    return st


# ---- the plain forms ----------------------------------------------------------------------------

def _plain_plan(st):
    P, T, table, free = st["case"]["page"], st["T"], st["page_table"], st["free_pages"]
    B, M = table.shape
    dev, n_pages = table.device, free.shape[0]
    up = lambda x: torch.div(x + P - 1, P, rounding_mode="floor")  # noqa: E731
    kv = st["kv_len"].long().clamp(0, M * P)
    k = torch.minimum(st["keep"].long().clamp_min(0), kv)
    own_p, kept = up(kv), up(k)
    cols = torch.arange(M, device=dev)
    gone = (cols >= kept[:, None]) & (cols < own_p[:, None])
    n_gone = gone.sum()
    first = st["n_free"].long().clamp(0, n_pages)
    top = torch.clamp_max(first + n_gone, n_pages)
    # pages that go back, the first of them on top
    order = torch.cumsum(gone.flatten().long(), 0) - 1
    to = top - 1 - order
    at = torch.where(gone.flatten() & (to >= first), to, n_pages)
    grown = torch.cat([free, free.new_zeros(1)])
    grown.scatter_(0, at, table.flatten())
    free.copy_(grown[:n_pages])
    # who gets its tokens
    want = st["add"].long().clamp_min(0)
    fits = (k + want <= M * P) & (want > 0)
    need = torch.where(fits, up(k + want) - kept, 0)
    paged = fits & ((need == 0) | (torch.cumsum(need, 0) <= top))
    given = paged & (torch.cumsum(torch.where(paged, want, 0), 0) <= T)
    n = torch.where(given, want, 0)
    need = torch.where(given, need, 0)
    before = torch.cumsum(need, 0) - need
    cu = torch.cat([n.new_zeros(1), torch.cumsum(n, 0)])
    new = (cols >= kept[:, None]) & (cols < (kept + need)[:, None])
    take = (top - 1 - (before[:, None] + cols - kept[:, None])).clamp(0, n_pages - 1)
    table.copy_(torch.where(new, free[take], torch.where(gone, -1, table)))
    st["n_free"].copy_(top - need.sum())
    st["kv_len"].copy_(k + n)
    # the tokens
    t = torch.arange(T, device=dev)
    b = (torch.searchsorted(cu, t, right=True) - 1).clamp(0, B - 1)
    pos = k[b] + t - cu[b]
    some = t < cu[B]
    pos = torch.where(some, pos, 0)
    page = table[b, torch.div(pos, P, rounding_mode="floor")].long()
    slots = torch.where(some & (page >= 0) & (page < n_pages), page * P + pos % P, -1)
    return {"cu_q": cu.int(), "slots": slots, "positions": torch.where(some, pos, -1).int(), "kv_len": st["kv_len"],
            "page_table": table, "free_pages": free, "n_free": st["n_free"]}


def _tokens(st):
    """Of every new token: its sequence, its place among the sequence's new tokens, its position in the cache."""
    case, B = st["case"], st["case"]["B"]
    T, dev = st["q"].shape[0], st["q"].device
    cu = st["cu_q"].long() if st["cu_q"] is not None else torch.arange(B + 1, device=dev) * case["q"]
    b = torch.searchsorted(cu, torch.arange(T, device=dev), right=True) - 1
    i = torch.arange(T, device=dev) - cu[b]
    n = cu[1:] - cu[:-1]
    return b, i, st["kv_len"].long()[b] - n[b] + i, cu, n


def _gather(st, n):
    """fp32 [B, Hkv, tokens, D] of the pages of every sequence."""
    at = st["page_table"].long().clamp_min(0)
    x = st[n + "_cache"][at].float() * st[n + "_scale"][at][:, :, :, None, None]
    B, M, H, P, D = x.shape
    return x.transpose(1, 2).reshape(B, H, M * P, D)


def _plain_write(st):
    b, _, pos, _, _ = _tokens(st)
    P, n_pages = st["case"]["page"], st["k_cache"].shape[0]
    page, off = st["page_table"].long()[b, torch.div(pos, P, rounding_mode="floor")], pos % P
    first = torch.full((n_pages,), P, device=b.device).scatter_reduce_(0, page, off, "amin")  # of a page's new rows
    begun = ((first > 0) & (first < P))[:, None]
    old = (torch.arange(P, device=b.device) < first[:, None])[:, None, :, None]
    for n in ("k", "v"):
        x = st[n].float()
        H, D = x.shape[1:]
        top = torch.zeros((n_pages, H), device=x.device).scatter_reduce_(0, page[:, None].expand(-1, H), x.abs().amax(-1), "amax")
        had = torch.where(begun, st[n + "_scale"], 0.0)
        scale = torch.maximum(_scale_of(top), had)
        touched = (first < P)[:, None]
        grew = (begun & (scale > had))[:, :, None, None] & old
        c = st[n + "_cache"]
        again = _to_codes(c.float() * had[:, :, None, None], scale[:, :, None, None].expand(-1, -1, P, D))
        c.copy_(torch.where(grew, again, c))
        st[n + "_scale"].copy_(torch.where(touched, scale, st[n + "_scale"]))
        c[page, :, off] = _to_codes(x, scale[page][:, :, None].expand(-1, -1, D))


def _plain_read(st):
    N = st["k_out"].shape[2]
    there = (torch.arange(N, device=st["k"].device)[None] < st["kv_len"][:, None])[:, None, :, None]
    return {n: torch.where(there, _gather(st, n)[:, :, :N].bfloat16(), st[n + "_out"]) for n in ("k", "v")}


def _plain_attn(st):
    case = st["case"]
    Hq, Hkv, D, causal, window = (case[n] for n in ("Hq", "Hkv", "D", "causal", "window"))
    G, nq = Hq // Hkv, case["q"]
    b, i, _, cu, n = _tokens(st)
    dev = b.device
    kv = st["kv_len"].long()[:, None]
    k, v = _gather(st, "k"), _gather(st, "v")
    N = k.shape[2]
    key = torch.arange(N, device=dev)
    v = torch.where((key < kv)[:, None, :, None], v, 0.0)
    # the batch padded to its longest chunk: rows (query head of a key head, token)
    pad = (cu[:-1, None] + torch.arange(nq, device=dev)).clamp_max(st["q"].shape[0] - 1)
    q = st["q"][pad].float().reshape(-1, nq, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(-1, Hkv, G * nq, D)
    p = kv - n[:, None] + torch.arange(nq, device=dev)
    hi = torch.where(p >= 0, torch.minimum(kv, (p // causal + 1) * causal), 0) if causal else kv.expand_as(p)
    lo = (hi - window).clamp_min(0) if window else torch.zeros_like(hi)
    hidden = ((key < lo[:, :, None]) | (key >= hi[:, :, None]))[:, None].repeat(1, 1, G, 1)
    s = (q @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(D)).masked_fill_(hidden, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    s.sub_(m).exp_()
    total = s.sum(-1, keepdim=True)
    o = (s @ v) / torch.where(total > 0, total, 1.0)
    back = lambda x: x.reshape(-1, Hkv, G, nq, x.shape[-1]).permute(0, 3, 1, 2, 4).reshape(-1, nq, Hq, x.shape[-1])[b, i]  # noqa: E731
    out = {"out": back(o).bfloat16()}
    if case["lse"]:
        out["lse"] = back(m + total.log())[..., 0].t().contiguous()
    return out


def _run_plain(st):
    op = st["case"]["op"]
    if op == "plan":
        return _plain_plan(st)
    if op == "attn":
        return _plain_attn(st)
    if op == "write":
        _plain_write(st)
    return _plain_read(st)


# ---- the framework's calls ----------------------------------------------------------------------

def _run_own(st):
    import paper_2605_14513_amd as heart

    case, op = st["case"], st["case"]["op"]
    if op == "plan":
        cu, slots, positions = heart.heart_cache_plan(st["add"], st["kv_len"], st["page_table"], st["free_pages"], st["n_free"],
                                                      case["page"], keep=st["keep"], cu_q=st["cu_q"], slots=st["slots"],
                                                      positions=st["positions"], workspace=st["workspace"])
        return {"cu_q": cu, "slots": slots, "positions": positions, "kv_len": st["kv_len"], "page_table": st["page_table"],
                "free_pages": st["free_pages"], "n_free": st["n_free"]}
    kw = dict(k_scale=st["k_scale"], v_scale=st["v_scale"])
    cache = (st["k_cache"], st["v_cache"], st["page_table"], st["kv_len"])
    if op == "attn":
        lse = torch.empty((case["Hq"], st["q"].shape[0]), dtype=torch.float32, device=st["q"].device) if case["lse"] else None
        out = heart.heart_cache_attn(st["q"], *cache, cu_q=st["cu_q"], causal=case["causal"], window=case["window"], lse=lse,
                                     workspace=st["workspace"], **kw)
        return {"out": out, "lse": lse} if case["lse"] else {"out": out}
    if op == "write":
        heart.heart_cache_write(st["k"], st["v"], *cache, cu_q=st["cu_q"], **kw)
    k, v = heart.heart_cache_read(*cache, k=st["k_out"], v=st["v_out"], **kw)
    return {"k": k, "v": v}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- definitions --------------------------------------------------------------------------------

def _exact_plan(case, seed):
    """Request after request, page after page, with the list as a stack."""
    st = _prepare_plan(case, seed)
    P, T = case["page"], st["T"]
    table = st["page_table"].cpu().numpy().copy()
    free = st["free_pages"].cpu().numpy().copy()
    add, kv, keep = (st[n].tolist() for n in ("add", "kv_len", "keep"))
    B, M = table.shape
    stack = free[:st["n_free"].item()].tolist()
    back = []
    for b in range(B):
        keep[b] = min(keep[b], kv[b])
        for p in range(-(-keep[b] // P), -(-kv[b] // P)):
            back.append(int(table[b, p]))
            table[b, p] = -1
    stack += back[::-1]
    free[:len(stack)] = stack
    slots, positions = np.full(T, -1, np.int64), np.full(T, -1, np.int32)
    cu, asked, left, given = [0], 0, T, len(stack)
    for b in range(B):
        n, had = max(add[b], 0), -(-keep[b] // P)
        want = -(-(keep[b] + n) // P) - had if n and keep[b] + n <= M * P else 0
        asked += want
        fits = 0 < n <= M * P - keep[b] and (want == 0 or asked <= given)
        left -= n if fits else 0
        if not fits or left < 0:
            n = 0
        else:
            for p in range(had, had + want):
                table[b, p] = stack.pop()
            pos = np.arange(keep[b], keep[b] + n)
            slots[cu[-1]:cu[-1] + n] = table[b, pos // P].astype(np.int64) * P + pos % P
            positions[cu[-1]:cu[-1] + n] = pos
        kv[b] = keep[b] + n
        cu.append(cu[-1] + n)
    as_is = lambda x, t: torch.as_tensor(np.asarray(x), dtype=t, device="cuda")  # noqa: E731
    return {"cu_q": as_is(cu, torch.int32), "slots": as_is(slots, torch.int64), "positions": as_is(positions, torch.int32),
            "kv_len": as_is(kv, torch.int32), "page_table": as_is(table, torch.int32), "free_pages": as_is(free, torch.int32),
            "n_free": as_is([len(stack)], torch.int32)}


def _block_scale(top):
    """fp64, from the definition: m 2^e with m = 4, 5, 6, 7, the least that is at least top / 127."""
    if top == 0.0:
        return 0.0
    m, e = math.frexp(top / 127.0)  # (127 m 2^e has ten bits: a quotient that is one of them is exact)
    return max(math.ldexp(math.ceil(m * 8), e - 3), 2.0 ** -126)


def _sequence(st, n, b, length):
    """fp64 [Hkv, length, D] of sequence b, page after page."""
    ids = st["page_table"][b, :-(-length // st["case"]["page"])].long()
    x = st[n + "_cache"][ids].double() * st[n + "_scale"][ids].double()[:, :, None, None]
    return x.permute(1, 0, 2, 3).flatten(1, 2)[:, :length]


def _exact_write(st, qs, kvs):
    """fp64 sequences after the write: every page that new tokens are in, head after head."""
    P, whole, at = st["case"]["page"], {"k": [], "v": []}, 0
    for b, (q, kv) in enumerate(zip(qs, kvs)):
        for n in ("k", "v"):
            x = _sequence(st, n, b, kv).clone()
            new = st[n][at:at + q].double().transpose(0, 1)
            for p in range((kv - q) // P, -(-kv // P)):
                lo, first, hi = p * P, max(p * P, kv - q), min(p * P + P, kv)
                rows = new[:, first - (kv - q):hi - (kv - q)]
                top = rows.abs().amax((1, 2)).tolist()
                had = st[n + "_scale"][int(st["page_table"][b, p])].tolist() if first > lo else [0.0] * len(top)
                unit = torch.tensor([max(_block_scale(t), h) for t, h in zip(top, had)], dtype=torch.float64, device=x.device)
                unit = unit[:, None, None]
                some = torch.where(unit > 0, unit, 1.0)
                x[:, lo:first] = torch.round(x[:, lo:first] / some) * unit
                x[:, first:hi] = torch.round(rows / some) * unit
            whole[n].append(x)
        at += q
    return whole


def exact(case, seed):
    op = case["op"]
    if op == "plan":
        return _exact_plan(case, seed)
    st = prepare(case, seed)
    qs, kvs = _lengths(case)
    Hq, Hkv, D = (case[n] for n in ("Hq", "Hkv", "D"))
    G, T, dev = Hq // Hkv, sum(qs), "cuda"
    if op == "write" and sum(-(-q // case["page"]) + 1 for q in qs) > 5000:
        return None
    if op != "attn":
        whole = _exact_write(st, qs, kvs) if op == "write" else {n: [_sequence(st, n, b, kvs[b]) for b in range(case["B"])] for n in "kv"}
        got = {}
        for n in ("k", "v"):
            got[n] = torch.zeros((case["B"], Hkv, max(kvs), D), dtype=torch.float64, device=dev)
            for b in range(case["B"]):
                got[n][b, :, :kvs[b]] = whole[n][b]
        return got
    out = torch.zeros((T, Hq, D), dtype=torch.float64, device=dev)
    lse = torch.full((Hq, T), -math.inf, dtype=torch.float64, device=dev)
    start = 0
    for b in range(case["B"]):
        p = torch.arange(kvs[b] - qs[b], kvs[b], device=dev)
        hi = torch.full_like(p, kvs[b]) if not case["causal"] else ((p // case["causal"] + 1) * case["causal"]).clamp_max(kvs[b])
        lo = (hi - case["window"]).clamp_min(0) if case["window"] else torch.zeros_like(hi)
        j = torch.arange(kvs[b], device=dev)
        seen = (j >= lo[:, None]) & (j < hi[:, None])
        at = slice(start, start + qs[b])
        start += qs[b]
        k, v = _sequence(st, "k", b, kvs[b]), _sequence(st, "v", b, kvs[b])
        for h in range(Hq):
            s = torch.where(seen, st["q"][at, h].double() @ k[h // G].t() / math.sqrt(D), -math.inf)
            lse[h, at] = torch.logsumexp(s, -1)
            out[at, h] = torch.softmax(s, -1) @ v[h // G]
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def work(case):
    op, P = case["op"], case["page"]
    if op == "plan":
        add, kv, keep, T, _, _ = _requests(case)
        moved = sum(-(-n // P) - -(-k // P) for n, k in zip(kv, keep)) + sum(-(-(k + n) // P) - -(-k // P) for n, k in zip(add, keep))
        return {"bytes": 20.0 * case["B"] + 12.0 * T + 8.0 * moved, "flops": 0.0}
    qs, kvs = _lengths(case)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    T, tokens = sum(qs), sum(kvs)
    blocks = sum(-(-n // P) for n in kvs)
    read = 2.0 * Hkv * (tokens * 3 * D + 4 * blocks)
    if op == "read":
        return {"bytes": read, "flops": 0.0}
    if op == "write":
        return {"bytes": 2.0 * T * Hkv * 3 * D + read, "flops": 0.0}
    pairs = keys = 0
    for n, kv in zip(qs, kvs):
        first = None
        for p in range(kv - n, kv):
            hi = min(kv, (p // case["causal"] + 1) * case["causal"]) if case["causal"] else kv
            lo = max(0, hi - case["window"]) if case["window"] else 0
            first = lo if first is None else first
            pairs += hi - lo
        keys += kv - first
    moved = 2.0 * Hkv * (keys * D + 4 * keys / P) + 4.0 * T * Hq * D + (4.0 * T * Hq if case["lse"] else 0.0)
    return {"bytes": moved, "flops": 4.0 * D * Hq * pairs}

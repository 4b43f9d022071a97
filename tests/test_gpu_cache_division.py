"""heart_cache_attn in every way that it divides keys, against attention in 64 bits; each test looks at what the call left in its
workspace, so that it is known to have gone that way."""
import math

import pytest
import torch

import cache_rules as rules
import paper_2605_14513_amd as heart
from cache_reference import FILL, Pages, near, reference

pytestmark = pytest.mark.gpu


def new_q(T, Hq, D, seed=1):
    return torch.randn((T, Hq, D), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


def cu_of(cu):
    return torch.tensor(cu, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kind,D", [("bf16", 128), ("e4m3", 64)])
@pytest.mark.parametrize("cu,T,H,G", [
    ([0, 800, 0, 800, 0], 800, 8, 8),            # tiles of 128 rows, more of them than workgroups
    ([0, 600, 200, 400], 600, 2, 4), ([0] + [300, 200] * 35, 300, 2, 16),
    ([0, 3, 1, 4], 5, 2, 2)])                     # few rows
def test_ranges_that_fall_leave_tokens_out(cu, T, H, G, kind, D):
    """No result is made of what the workspace held: with divided keys no token of such a call is attended.  (The records that are
    there before the call are of two parts in the workspace, so that a launch that went by them would stay in it.)"""
    B = len(cu) - 1
    c = Pages([4000 - 10 * b for b in range(B)], H, D, 64, kind)
    q = new_q(T, H * G, D)
    n = heart.heart_cache_attn_workspace_bytes(q, c.stored["k"], c.page_table)
    ws = torch.zeros(n // 4, dtype=torch.int32, device="cuda")
    if not rules.few(B, H, T, H * G):
        assert rules.mode(B, H, T, H * G, c.cap)[0] == "parts"
        ws[:4 * rules.PLACES] = torch.tensor([0, 2, 1, 0], dtype=torch.int32).repeat(rules.PLACES)
    out, lse = torch.full_like(q, 7.0), torch.full((H * G, T), 7.0, device="cuda")
    print(f"cache_attn ranges {cu[:5]} T={T} H={H} G={G} {kind} D={D}", flush=True)
    heart.heart_cache_attn(q, *c.args(), cu_q=cu_of(cu), out=out, lse=lse, workspace=ws, **c.exps())
    torch.cuda.synchronize()
    assert (out == 7.0).all() and (lse == 7.0).all()
    # without a workspace: rows of a sequence that has them, or left as they were
    heart.heart_cache_attn(q, *c.args(), cu_q=cu_of(cu), out=out, lse=lse, workspace=None, **c.exps())
    torch.cuda.synchronize()
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("cu", [[0, 9, 2, 3], [0, 40, 0, 40], [30, 10, 20, 5], [0, 7, -3, 12], [5, 2**31 - 1, 3, 4], [-(2**31), 20, 1, 40]])
def test_writing_by_ranges_that_fall_stays_behind_the_last_token(cu, kind):
    """A token goes to a place among its sequence's new ones, or nowhere."""
    c = Pages([100, 130, 90], 2, 64, 16, kind, room=300)
    # (every position of the table has a page, so that one behind the last token could be written)
    c.page_table = torch.arange(3 * 19, dtype=torch.int32, device="cuda").reshape(3, 19)
    store = torch.zeros((57, 2, 16, 64), dtype=torch.uint8 if kind == "e4m3" else torch.bfloat16, device="cuda")
    k, v = store.clone(), store.clone()
    e = dict.fromkeys(("k_exp", "v_exp"))
    if kind == "e4m3":
        e = {n: torch.zeros((57, 2, 16), dtype=torch.uint8, device="cuda") for n in e}
    x = torch.ones((40, 2, 64), dtype=torch.bfloat16, device="cuda")
    print(f"cache_write ranges {cu} {kind}", flush=True)
    heart.heart_cache_write(x, x, *((t.view(torch.float8_e4m3fn) if kind == "e4m3" else t) for t in (k, v)), c.page_table, c.kv_len,
                            cu_q=cu_of(cu), **e)
    torch.cuda.synchronize()
    for t in (k, v):
        there = (t != 0).any(-1).any(1).reshape(3, 19 * 16)
        for b, kv in enumerate(c.kvs):
            n = cu[b + 1] - cu[b]
            assert not there[b, kv:].any() and not there[b, :max(kv - max(n, 0), 0)].any(), (b, there[b].nonzero().flatten().tolist())


def run(c, q, qs, causal, window, what, **kw):
    """A call on a workspace that is full of FILL, beside the definition; (out, lse, workspace)."""
    T, Hq, D = q.shape
    n = heart.heart_cache_attn_workspace_bytes(q, c.stored["k"], c.page_table)
    ws = torch.full((n,), FILL, dtype=torch.uint8, device="cuda")
    cu = cu_of([sum(qs[:b]) for b in range(len(qs) + 1)])
    out = torch.full((T, Hq, D), math.nan, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((Hq, T), math.nan, device="cuda")
    print(f"cache_attn {what} B={len(qs)} T={T} Hq={Hq} H={c.H} D={D} {c.kind} page={c.page} kv<={max(c.kvs)} causal={causal} "
          f"window={window}", flush=True)
    heart.heart_cache_attn(q, *c.args(), cu_q=cu, causal=causal, window=window, out=out, lse=lse, workspace=ws, **c.exps())
    torch.cuda.synchronize()
    want, want_lse, tol, ltol = reference(c, q, qs, causal, window, **kw)
    near(out, want, tol, "out")
    near(lse, want_lse, ltol, "lse")
    again, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
    heart.heart_cache_attn(q, *c.args(), cu_q=cu, causal=causal, window=window, out=again, lse=lse2, **c.exps())
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    return out, lse, ws


def ragged(B, top, seed, empty=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.exp(torch.rand(B, generator=g) * math.log(top)).int().tolist()
    x[0] = top
    if empty and B > 4:
        x[1], x[2], x[3] = 0, 1, 129
    return x


def shares_test(c, G, qs, causal, window, mode, what):
    """Few rows: the flags that the call leaves are those of the parts that the rules give."""
    s = rules.shares_of(qs, c.lens, c.H, G, c.cap, causal, window, c.D, c.kind)
    assert s.mode == mode
    stages, parts = s.longest()
    # (a part's keys are dealt to four wavefronts; the sums of wavefronts and parts)
    q = new_q(sum(qs), c.H * G, c.D)
    _, _, ws = run(c, q, qs, causal, window, what, chain=stages * rules.FEW_STAGE // 4 + 64 + 4 + parts, weight=2.0**-16)
    flags = ws[:2 * rules.FEW_PLACES * 8].view(torch.int64).tolist()
    used = [i for i, x in enumerate(flags) if x == 0]
    assert used == sorted(s.slots()) and all(x == int.from_bytes(bytes([FILL] * 8), "little") for x in flags if x)
    return s, q


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,H,G,B,top,causal,window", [
    (128, 8, 5, 64, 6000, 1, 0),      # decoding, ragged: equal shares that cross tiles and sequences
    (64, 8, 2, 64, 6000, 1, 0),
    (128, 16, 1, 20, 9000, 0, 0),     # shares shorter than tiles: tiles of many parts
    (64, 12, 16, 40, 5000, 1, 3000),  # windows
    (128, 8, 3, 100, 5000, 1, 0),     # more than 64 sequences
    (64, 4, 1, 256, 4000, 1, 1500)])
def test_few_rows_in_shares(D, H, G, B, top, causal, window, kind):
    kvs = ragged(B, top, B + D)
    kvs = [k if i % 3 else max(k, top // 2) for i, k in enumerate(kvs)]
    kvs[1:4] = [0, 1, 129]
    c = Pages(kvs, H, D, 32, kind, seed=B, room=top + 200)
    qs = [1] * B
    qs[B // 2] = 0
    s, _ = shares_test(c, G, qs, causal, window, "shares", "shares")
    # (shares that end one tile and begin the next leave two parts)
    slots = set(s.slots())
    assert any(2 * i in slots and 2 * i + 1 in slots for i in range(rules.FEW_PLACES))


@pytest.mark.parametrize("kind,D", [("bf16", 128), ("e4m3", 64)])
def test_one_long_sequence_in_shares(kind, D):
    """More than 64 parts a tile; and drafts, of one tile and of several in one sequence."""
    for G, qs, kvs in ((3, [1], [66000]), (2, [5, 1, 0, 20], [50000, 24000, 100, 9000])):
        c = Pages(kvs, 8, D, 256, kind, seed=G)
        shares_test(c, G, qs, 1, 0, "shares", "long")


@pytest.mark.parametrize("kind,D", [("bf16", 128), ("e4m3", 128), ("bf16", 64)])
def test_few_rows_in_parts(kind, D):
    """The same look at calls of parts of 2, 4 and 8 stages."""
    for B, H, top in ((3, 2, 5000), (20, 4, 3000), (100, 2, 2500), (60, 8, 900)):
        c = Pages(ragged(B, top, B), H, D, 16, kind, seed=B)
        shares_test(c, 2, [1] * B, 1, 0, "parts", "parts")


@pytest.mark.parametrize("kvs,H,past", [([66000], 8, False), ([9000] * 48, 12, True)])
def test_loads_past_the_caches(kvs, H, past):
    """Shares of calls that read more than 80 MB, where loads go past the caches, and of one that reads less (by the shares' length,
    of which half a stage of 64 keys is 8 KB)."""
    c = Pages(kvs, H, 64, 64, "e4m3", seed=H)
    s, _ = shares_test(c, 1, [1] * len(kvs), 1, 0, "shares", "loads")
    assert (s.total * 8192 > 80 << 20) == past


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_replays_in_shares_follow_their_lengths(kind):
    """A captured call: shares, parts and shares again as the lengths go, with eager calls on the same workspace between them."""
    B, H, G, D, top = 64, 8, 2, 64, 5000
    c = Pages([top] * B, H, D, 64, kind, seed=4)
    q = new_q(B, H * G, D)
    out = torch.zeros_like(q)
    ws = torch.full((heart.heart_cache_attn_workspace_bytes(q, c.stored["k"], c.page_table),), FILL, dtype=torch.uint8, device="cuda")

    def call(o):
        heart.heart_cache_attn(q, *c.args(), out=o, workspace=ws, **c.exps())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    modes = []
    lens = [[top] * B, ragged(B, 200, 1), ragged(B, top, 2), [top - 3 * b for b in range(B)], [17] * B, [top] * B]
    for i, kv in enumerate(lens):
        modes.append(rules.shares_of([1] * B, kv, H, G, c.cap, 1, 0, D, kind).mode)
        c.kvs = c.lens = kv
        c.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        q.copy_(new_q(B, H * G, D, seed=i))
        print(f"replay {i} {modes[-1]}", flush=True)
        out.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        got, eager = out.clone(), torch.zeros_like(out)
        want, _, tol, _ = reference(c, q, [1] * B, weight=2.0**-16)
        near(got, want, tol, f"replay {i}")
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(got, eager)
    assert set(modes) == {"shares", "parts"}, modes


def records_of(ws):
    """(first part, parts, distance) of the records that a call has written."""
    x = ws[:rules.PLACES * 16].view(torch.int32).reshape(-1, 4).cpu()
    fill = int.from_bytes(bytes([FILL] * 4), "little")
    return {i: tuple(r[:3]) for i, r in enumerate(x.tolist()) if r != [fill] * 4}


def parts_written(ws, D):
    """Numbers of the parts of whose first rows something has been written."""
    n = 64 * (D // 2) + 128
    x = ws[rules.PLACES * 16:].view(torch.int32).reshape(-1, 4 * n)
    fill = int.from_bytes(bytes([FILL] * 4), "little")
    return set((x[:, :n] != fill).any(1).nonzero().flatten().tolist())


def parts_test(c, G, qs, causal, window, expect, what):
    """Tiles of 128 rows: the mode by the rules, records and parts by what the workspace holds after the call."""
    B, T, Hq = len(qs), sum(qs), c.H * G
    assert not rules.few(B, c.H, T, Hq)
    got = rules.mode(B, c.H, T, Hq, c.cap)
    assert got[:2] == expect, got
    _, _, ws = run(c, new_q(T, Hq, c.D), qs, causal, window, what)
    if got[0] == "whole":
        assert ws.numel() == 0 or (ws == FILL).all()
        return None
    records = records_of(ws)
    seqs = rules.sequences([sum(qs[:b]) for b in range(B + 1)], c.lens, T, c.cap)
    tiles = [rules.tiles_of(rules.TILE, G, s) for s in seqs]
    if got[0] == "parts":
        cu = [sum(qs[:b]) for b in range(B + 1)]
        assert set(records) == {(rules.tile_start(rules.TILE, G, cu, b) + m) * c.H + h for b in range(B) for m in range(tiles[b]) for h in range(c.H)}
    slots = [r[0] + i * r[2] for r in records.values() for i in range(r[1])]
    assert len(slots) == len(set(slots))
    divided = {r[0] + i * r[2] for r in records.values() if r[1] > 1 for i in range(r[1])}
    assert divided == parts_written(ws, c.D)
    return records, slots, got


@pytest.mark.parametrize("kind,D", [("bf16", 128), ("e4m3", 64), ("bf16", 64), ("e4m3", 128)])
@pytest.mark.parametrize("H,G,qs,kvs,causal", [
    (8, 1, [8400], [8401], 0),                  # an eighth of the heads an XCD
    (3, 4, [5500], [5500], 0),                  # heads in turn
    (5, 3, [3000, 0, 500, 3500], [6000, 30, 500, 9000], 40),
    (16, 2, [2300], [9000], 300)])
def test_a_last_round_of_tiles_is_divided(H, G, qs, kvs, causal, kind, D):
    c = Pages(kvs, H, D, 64, kind, seed=H, room=5200)
    records, slots, (_, _, whole, tail) = parts_test(c, G, qs, causal, 0, ("tail", 1), "last round")
    n = rules.most_items(rules.TILE, len(qs), H, sum(qs), H * G) - whole
    assert tail > 1 and max(records) < n and max(r[1] for r in records.values()) > 1
    assert all(r[2] == n and r[0] == i for i, r in records.items())


@pytest.mark.parametrize("kind,D", [("bf16", 128), ("e4m3", 64), ("bf16", 64), ("e4m3", 128)])
@pytest.mark.parametrize("H,G,qs,kvs,causal,window", [
    (8, 8, [590], [9000], 1, 0), (4, 2, [1500, 2000, 700, 300], [9000, 7000, 8000, 300], 1, 0),
    (8, 1, [2000, 1900, 1000], [9000, 9000, 5000], 0, 7000)])
def test_parts_in_two_rounds(H, G, qs, kvs, causal, window, kind, D):
    c = Pages(kvs, H, D, 128, kind, seed=H, room=5200)
    records, slots, _ = parts_test(c, G, qs, causal, window, ("parts", 2), "two rounds")
    assert len(slots) > rules.PLACES and max(slots) < 2 * rules.PLACES


@pytest.mark.parametrize("kind,D", [("bf16", 128), ("e4m3", 64), ("bf16", 64), ("e4m3", 128)])
@pytest.mark.parametrize("B,H,G,n,top,window", [(65, 2, 4, 8, 5000, 0), (100, 2, 4, 9, 3000, 800), (256, 1, 5, 7, 6000, 0), (130, 1, 2, 40, 5500, 0)])
def test_parts_of_many_sequences(B, H, G, n, top, window, kind, D):
    """65 to 256 sequences on tiles of 128 rows, some without new tokens, some shorter than their new tokens."""
    kvs = ragged(B, top, B)
    qs = [(n * (1 + i % 3)) // 2 for i in range(B)]
    qs[5] = 0
    c = Pages(kvs, H, D, 16, kind, seed=B)
    records, slots, got = parts_test(c, G, qs, 1, window, rules.mode(B, H, sum(qs), H * G, c.cap)[:2], "many sequences")
    assert got[0] == "parts" and max(r[1] for r in records.values()) > 2


@pytest.mark.parametrize("kind,D", [("bf16", 128), ("e4m3", 64)])
def test_a_round_of_parts_and_tiles_that_are_not_divided(kind, D):
    """A table with little room: one round of parts, or none."""
    c = Pages([3000, 2800, 100], 8, D, 64, kind)
    records, slots, _ = parts_test(c, 2, [100, 700, 90], 1, 0, ("parts", 1), "one round")
    assert max(r[1] for r in records.values()) > 1 and len(slots) <= rules.PLACES
    c = Pages([3100], 16, D, 64, kind)
    parts_test(c, 2, [2300], 1, 0, ("whole", 1), "whole")

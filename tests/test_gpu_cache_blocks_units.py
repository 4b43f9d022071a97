"""heart_cache_attn over int8 caches on tiles of 128 and of 256 rows: the unit of v's values in f16, which is known from the scales of a
part's first 64 stages and, of longer parts, from a look at all others."""
import pytest
import torch

import cache_rules as rules
import paper_2605_14513_amd as heart
from cache_blocks_reference import Blocks, tolerance
from cache_reference import FILL
from cache_testlib import assert_near
from test_gpu_cache_blocks_attn import new_q
from test_gpu_cache_division import records_of

pytestmark = pytest.mark.gpu

LOOKED_AT = 63 * rules.STAGE  # from this key of a part on the scales of v are looked at one by one
WIDE, WIDE_PLACES = 256, 256


def divide_wide(n_items):
    """The last round of tiles of 256 rows: (mode, tiles that are not divided, parts of the others, rounds that it takes)."""
    r, before = n_items % WIDE_PLACES, n_items // WIDE_PLACES
    if n_items < WIDE_PLACES or n_items > rules.TAIL_ROUNDS * WIDE_PLACES or r == 0:
        return "whole", n_items, 1, before + (r > 0)
    best, least, p = 1, 1e9, 1
    while p <= 8 and r * p <= 2 * WIDE_PLACES:
        cost = -(-r * p // WIDE_PLACES) / p + (0.03 * p * r / WIDE_PLACES + 0.02 if p > 1 else 0.0)
        if cost < least:
            least, best = cost, p
        p += 1
    return ("whole", n_items, 1, before + 1) if best == 1 else ("tail", n_items - r, best, before + least)


def wide(B, H, D, T, Hq, room, divided=True):
    """(mode, tiles not divided, parts, tiles) where a call has tiles of 256 rows, else None; not within 4 % of the rule's edge."""
    if D != 128 or T * (Hq // H) < 4 * WIDE * B or room <= rules.BRIEF:
        return None
    n = rules.most_items(WIDE, B, H, T, Hq)
    mode, whole, parts, cost = divide_wide(n)
    if not divided:
        mode, whole, parts, cost = "whole", n, 1, -(-n // WIDE_PLACES)
    full = 7 * n / (6 * WIDE_PLACES * cost)
    assert not 0.96 < full < 1.04, full
    return (mode, whole, parts, n) if full > 1 else None


def attend(c, q, n, B=1, window=0, causal=1, workspace="auto", what=""):
    print(f"cache_attn int8 {what} B={B} n={n} kvs={c.kvs} H={c.H} D={c.D} page={c.page} causal={causal} window={window} "
          f"workspace={workspace if not torch.is_tensor(workspace) else workspace.numel()}", flush=True)
    lse = torch.zeros((q.shape[1], q.shape[0]), device="cuda")
    out = heart.heart_cache_attn(q.cuda(), *c.args(), causal=causal, window=window, lse=lse, workspace=workspace, **c.scale_args())
    torch.cuda.synchronize()
    return out, lse


def near_definition(c, q, qs, out, lse, heads, causal=1, window=0, rows=None):
    """Some heads (one query head a key head) against the definition in 64 bits; `rows`: of one sequence some, which all see the same."""
    one = Blocks(c.kvs, 1, c.D, c.page, seed=0, device="cpu")
    one.table_cpu, one.n_pages = c.table_cpu, c.n_pages
    if rows is not None:
        assert causal == 0 and len(qs) == 1
        q, out, lse, qs = q[rows], out[rows], lse[:, rows], [len(rows)]
    for h in heads:
        for w in ("k", "v"):
            one.codes[w], one.scales[w] = c.codes[w][:, h:h + 1], c.scales[w][:, h:h + 1]
        want, want_lse, tol, ltol = tolerance(one, q[:, h:h + 1], qs, causal, window)
        assert_near(out[:, h:h + 1], want, tol, f"out of head {h}")
        assert_near(lse[h:h + 1], want_lse, ltol, f"lse of head {h}")


def hot_pages(kv, page, key0):
    """Pages, one a head, whose v is to be far above all others (None: no page): the last one, those around the key from which scales
    are looked at one by one, one far behind it, one that the first stages have, all from that key on."""
    at = [kv - 1] + [key0 + LOOKED_AT + d for d in (0, 16, 32, 48, 64, 256, 512, 1000)] + [key0 + 700]
    return [[min(p, kv - 1) // page] for p in at] + [list(range(-(-(key0 + LOOKED_AT) // page), -(-kv // page))), []]


def raise_v(c, hot, by):
    """Scales of v of pages `hot[h]` (of sequence 0) 2^by times what they are, heads in turn."""
    for h in range(c.H):
        for p in hot[h % len(hot)]:
            c.scales["v"][c.table_cpu[0, p], h] *= 2.0**by
    c.scale["v"].copy_(c.scales["v"])


# (Under the unit of the first 64 stages alone a scale that is 2^10 times another is 2^11 units at least, and times a code of 40 there
# is no f16 for it: infinities and NaN.)
@pytest.mark.parametrize("workspace", ["auto", None])
@pytest.mark.parametrize("kv,window", [(6000, 0), (9137, 0), (9300, 5003), (10000, 6001)])
@pytest.mark.parametrize("D,page,by", [(64, 16, 11), (128, 256, 12), (128, 16, 10), (64, 256, 10)])
def test_larger_scales_of_v_behind_the_first_stages(D, page, by, kv, window, workspace):
    n = 100
    c = Blocks([kv], 12, D, page, seed=kv + D, spread=2)
    key0 = (kv - n + 1 - window) // rules.STAGE * rules.STAGE if window else 0
    raise_v(c, hot_pages(kv, page, key0), by)
    q = new_q(n, 12, D)
    out, lse = attend(c, q, n, window=window, workspace=workspace, what=f"v up by 2^{by}")
    near_definition(c, q, [n], out, lse, range(12), window=window)


@pytest.mark.parametrize("D,H,page", [(64, 80, 16), (64, 80, 256), (128, 72, 16), (128, 72, 256)])
def test_larger_scales_of_v_in_parts_of_more_than_64_stages(D, H, page):
    """147 stages; the tiles of the last round, of 128 rows and of 256, in two parts."""
    n, kv = 1024, 9400
    c = Blocks([kv], H, D, page, seed=D, spread=2)
    raise_v(c, hot_pages(kv, page, 0) + hot_pages(kv, page, 74 * rules.STAGE), 10)
    q = new_q(n, H, D)
    tiles = wide(1, H, D, n, H, c.table_cpu.shape[1] * page)
    if D == 64:
        tiles = rules.most_items(rules.TILE, 1, H, n, H)
        assert rules.mode(1, H, n, H, kv) == ("tail", 1, 512, 2)
        tiles = ("tail", 512, 2, tiles)
    mode, whole, parts, tiles = tiles
    assert (mode, parts) == ("tail", 2)
    ws = torch.full((heart.heart_cache_attn_workspace_bytes(q, c.stored["k"], c.page_table),), FILL, dtype=torch.uint8, device="cuda")
    out, lse = attend(c, q, n, causal=0, workspace=ws, what="divided, v up")
    records = records_of(ws)
    assert records and set(records.values()) == {(i, 2, tiles - whole) for i in records}
    # (heads of the last round are the last ones)
    near_definition(c, q, [n], out, lse, list(range(0, 24, 5)) + list(range(H - 24, H)), causal=0, rows=list(range(0, n, 41)))


@pytest.mark.parametrize("page,kv,window", [(16, 6000, 0), (256, 9137, 0), (16, 9300, 5003)])
def test_larger_scales_of_v_in_tiles_of_256_rows(page, kv, window):
    H, n = 48, 1024
    c = Blocks([kv], H, 128, page, seed=page, spread=2)
    assert wide(1, H, 128, n, H, c.table_cpu.shape[1] * page)[0] == "whole"
    raise_v(c, hot_pages(kv, page, (kv - window) // rules.STAGE * rules.STAGE if window else 0), 10)
    q = new_q(n, H, 128)
    for workspace in ("auto", None):
        out, lse = attend(c, q, n, window=window, causal=0, workspace=workspace, what="wide, v up")
        near_definition(c, q, [n], out, lse, range(12), causal=0, window=window, rows=list(range(0, n, 41)))

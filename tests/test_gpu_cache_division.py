"""heart_cache_attn in every way that it divides keys, against attention in 64 bits; each test looks at what the call left in its
workspace, so that it is known to have gone that way."""
import math

import pytest
import torch

import cache_rules as rules
import paper_2605_14513_amd as heart
from cache_reference import Pages

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

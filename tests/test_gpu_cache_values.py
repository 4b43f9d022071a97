"""heart_cache_attn on values at the ends of the formats: NaN and infinities among what is seen, exponents of rows, weights that
cancel."""
import math

import pytest
import torch

import paper_2605_14513_amd as heart
from cache_reference import E4M3, Pages, near, reference
from cache_testlib import e4m3_values

pytestmark = pytest.mark.gpu


def new_q(T, Hq, D, seed=1):
    return torch.randn((T, Hq, D), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


def place(c, b, j):
    """Page and row of token j of sequence b."""
    return c.page_table[b, j // c.page].item(), j % c.page


# (few rows in parts, 128-row tiles in parts; with and without a workspace)
@pytest.mark.parametrize("workspace", ["auto", None])
@pytest.mark.parametrize("n", [2, 150])
@pytest.mark.parametrize("kind,D", [("bf16", 128), ("bf16", 64), ("e4m3", 128)])
def test_logits_that_are_not_finite(kind, D, n, workspace):
    """A query with NaN among its logits gives NaN in out and in the log-sum-exp, not what one without keys gives; so does +inf; a
    key whose logit is -inf has weight 0.  Other queries, and heads, get what they get without."""
    H, G, kvs = 2, 2, [3000, 700]
    c = Pages(kvs, H, D, 32, kind)
    q = new_q(2 * n, H * G, D).abs()  # (signs: an infinite k gives an infinite logit)
    q[n + 1, 3, D // 2] = math.nan
    want, want_lse, tol, ltol = reference(c, q.nan_to_num(0.0), [n, n])
    bad = torch.zeros((2 * n, H * G), dtype=torch.bool, device="cuda")
    bad[n + 1, 3] = True
    sees = torch.arange(n, device="cuda")
    for b, h, j, x in ((0, 0, kvs[0] - 1, math.nan), (0, 1, kvs[0] - n, math.inf), (1, 0, 5, -math.inf)):
        page, row = place(c, b, j)
        if kind == "e4m3":  # (no infinities in the format)
            if x == -math.inf:
                continue
            c.stored["k"][page, h, row] = math.nan
        else:
            c.stored["k"][page, h, row] = x
        if x == -math.inf:  # the definition without that key
            k, v = (c.sequence(m, 1)[h][torch.arange(kvs[1]) != j] for m in "kv")
            for i in range(n):
                for g in range(G):
                    s = k[:kvs[1] - n + i] @ q[n + i, h * G + g].double() / math.sqrt(D)
                    want[n + i, h * G + g] = torch.softmax(s, 0) @ v[:kvs[1] - n + i]
                    want_lse[h * G + g, n + i] = torch.logsumexp(s, 0)
        else:
            bad[b * n:(b + 1) * n, h * G:(h + 1) * G] |= (kvs[b] - n + sees >= j)[:, None]
    print(f"cache_attn not finite {kind} D={D} n={n} workspace={workspace}", flush=True)
    out, lse = torch.zeros_like(q), torch.zeros((H * G, 2 * n), device="cuda")
    heart.heart_cache_attn(q, *c.args(), out=out, lse=lse, workspace=workspace, **c.exps())
    torch.cuda.synchronize()
    assert out[bad].isnan().all() and lse.t()[bad].isnan().all()
    near(out[~bad], want[~bad], tol[~bad], "out")
    near(lse.t()[~bad], want_lse.t()[~bad], ltol.t()[~bad], "lse")


@pytest.mark.parametrize("D", [64, 128])
def test_rows_under_every_exponent(D):
    """Exponent bytes 0 to 254 are powers of two from 2^-127 on: read back, and attended by few rows and by many.  Every sequence
    is one token whose v is a row under one exponent, so that out is that row; k is such a row too and q is zero."""
    B, page = 255, 16
    codes = (torch.arange(B * D, device="cuda") * 7 % 127).to(torch.uint8).reshape(B, D) | (torch.arange(D, device="cuda") % 2 * 128).to(torch.uint8)
    exp = torch.arange(B, device="cuda", dtype=torch.uint8)
    value = codes.view(E4M3).double() * torch.exp2(exp.double() - 127)[:, None]
    want = value.bfloat16()  # (beyond the largest bf16: infinities)
    store = torch.zeros((B, 1, page, D), dtype=torch.uint8, device="cuda")
    e = torch.full((B, 1, page), 255, dtype=torch.uint8, device="cuda")
    store[:, 0, 0], e[:, 0, 0] = codes, exp
    plain = torch.full_like(e, 127)
    table = torch.arange(B, dtype=torch.int32, device="cuda")[:, None].contiguous()
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    print(f"cache_read, cache_attn exponents D={D}", flush=True)
    k, v = heart.heart_cache_read(store.view(E4M3), store.view(E4M3), table, one, n=1, k_exp=e, v_exp=e)
    normal = (value.abs() >= 2.0**-126) | (value == 0)  # (those below may be read as zero)
    for x in (k, v):
        assert ((x[:, 0, 0] == want) | (~normal & (x[:, 0, 0] == 0))).all()
    here = slice(0, 240)  # (2^8 sum |v| has to stay below 2^128)
    for G in (1, 40):  # few rows, and tiles of 128
        q = torch.zeros((B, G, D), dtype=torch.bfloat16, device="cuda")
        out = heart.heart_cache_attn(q, store.view(E4M3), store.view(E4M3), table, one, k_exp=plain, v_exp=e)
        for g in range(G):
            assert ((out[here, g] == want[here]) | (~normal[here] & (out[here, g] == 0))).all(), g
        # (as k: a query along one element has that logit)
        q[:, :, 0] = 1.0
        lse = torch.zeros((G, B), device="cuda")
        heart.heart_cache_attn(q, store.view(E4M3), store.view(E4M3), table, one, k_exp=e, v_exp=plain, lse=lse, scale=1.0)
        s = value[here, 0]
        assert ((lse[:, here] - s).abs() <= 2.0**-20 * s.abs() + 2.0**-100).all()


@pytest.mark.parametrize("kind,D", [("bf16", 64), ("e4m3", 128)])
@pytest.mark.parametrize("n", [3, 70])
def test_windows_of_lengths_beyond_the_page_table(kind, D, n):
    """kv_len past the room of the table: a window reaches back from the position, not from the last key that there is room for."""
    c = Pages([256, 256, 256], 2, D, 16, kind)
    c.lens = [256 + n // 2, 300, 1000]
    c.kv_len = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    q = new_q(3 * n, 4, D)
    for causal, window in ((1, 60), (0, 60), (0, 0), (64, 100), (1, 30), (1, 0), (1, 2000)):
        want, want_lse, tol, ltol = reference(c, q, [n] * 3, causal, window)
        assert causal == 0 or window != 60 or n != 70 or (want_lse == -math.inf).any()
        for workspace in ("auto", None):
            print(f"cache_attn beyond the table {kind} D={D} n={n} causal={causal} window={window} workspace={workspace}", flush=True)
            lse = torch.zeros((4, 3 * n), device="cuda")
            out = heart.heart_cache_attn(q, *c.args(), causal=causal, window=window, lse=lse, workspace=workspace, **c.exps())
            near(out, want, tol, "out")
            near(lse, want_lse, ltol, "lse")


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [64, 128])
def test_weights_of_few_rows_are_two_bf16(D, kind):
    """Columns of v that the weights of all rows cancel: out is next to nothing beside sum p |v|, so what is left of a weight's
    rounding shows.  (On the CPU: weights of one bf16 would be outside the tolerance.)"""
    n, G = 40, 8
    c = Pages([n], 1, D, 16, kind, seed=D)
    q = (0.25 * new_q(1, G, D).float()).bfloat16()
    k = c.sequence("k", 0)[0].cpu()
    s = q[0].double().cpu() @ k.t() / math.sqrt(D)
    p = torch.softmax(s, -1)
    g = torch.Generator().manual_seed(2)
    v = torch.randn((n, D), generator=g, dtype=torch.float64)
    v = v - torch.linalg.pinv(p) @ (p @ v)
    if kind == "e4m3":
        v, exp = e4m3_values(v)
        codes = torch.ldexp(v, 127 - exp.int()[:, None]).float().to(E4M3).view(torch.uint8)
    else:
        v = v.bfloat16().double()
    for j in range(n):
        page, row = place(c, 0, j)
        if kind == "e4m3":
            c.stored["v"].view(torch.uint8)[page, 0, row], c.exp["v"][page, 0, row] = codes[j].cuda(), exp[j].cuda()
        else:
            c.stored["v"][page, 0, row] = v[j].bfloat16().cuda()
    want, _, tol, _ = reference(c, q, [1], weight=2.0**-16)
    w = torch.exp(s - s.amax(-1, keepdim=True))
    one = (w.float().bfloat16().double() @ v) / w.sum(-1, keepdim=True)
    assert ((one - want[0].cpu()).abs() > tol[0].cpu()).float().mean() > 0.2
    print(f"cache_attn weights {kind} D={D}", flush=True)
    for workspace in ("auto", None):
        near(heart.heart_cache_attn(q, *c.args(), workspace=workspace, **c.exps()), want, tol, "out")

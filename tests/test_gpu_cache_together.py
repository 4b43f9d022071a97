"""The cache's calls as they are used: together with each other and with the sparse path, captured and replayed, on other
streams, at addresses beyond 4 GiB, with as little and as much as the arguments allow."""
import math

import pytest
import torch

import oracle
import paper_2605_14513_amd as heart
from cache_testlib import Cache, assert_near, attention, e4m3_values, ends
from heart_testlib import u16

pytestmark = pytest.mark.gpu


def empty_cache(B, H, D, page, tokens, kind):
    """k_cache, v_cache, exponents, page_table for up to `tokens` tokens of B sequences, pages dealt out in turn."""
    M = -(-tokens // page)
    n = B * M + 1
    dt = torch.bfloat16 if kind == "bf16" else torch.float8_e4m3fn
    k, v = (torch.zeros((n, H, page, D), dtype=torch.uint8 if kind == "e4m3" else dt, device="cuda").view(dt) for _ in range(2))
    exps = {x: torch.zeros((n, H, page), dtype=torch.uint8, device="cuda") if kind == "e4m3" else None for x in ("k_exp", "v_exp")}
    table = torch.tensor([[n - 1 - (m * B + b) for m in range(M)] for b in range(B)], dtype=torch.int32, device="cuda")
    return k, v, exps, table


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,block", [(64, 64), (128, 128)])
def test_a_clip_in_chunks_and_the_sparse_path(kind, D, block):
    """A clip written chunk by chunk, frames of `span` tokens: every chunk attends frame after frame as it is there; at the end
    the clip is read back, pooled, and block-sparse attention over all of its blocks agrees with the cache's."""
    H, span, frames = 3, 70, 7
    N = span * frames
    g = torch.Generator().manual_seed(D)
    q, k, v = (torch.randn((N, H, D), generator=g).bfloat16() for _ in range(3))
    kc, vc, exps, table = empty_cache(1, H, D, 32, N, kind)
    ref = Cache([N], H, D, 32, "bf16", device="cpu")  # (the definition's inputs: what the cache stands for)
    stands = {}
    for n, x in (("k", k), ("v", v)):
        stands[n] = e4m3_values(x)[0] if kind == "e4m3" else x.double()
    ref.sequence = lambda n, b, length=None: stands[n][:ref.kvs[0]].transpose(0, 1)
    at = 0
    for n in (2 * span, span, 3 * span, span):
        kv_len = torch.tensor([at + n], dtype=torch.int32, device="cuda")
        part = slice(at, at + n)
        heart.heart_cache_write(k[part].cuda(), v[part].cuda(), kc, vc, table, kv_len, **exps)
        out = heart.heart_cache_attn(q[part].cuda(), kc, vc, table, kv_len, causal=span, **exps)
        at += n
        ref.kvs = [at]
        want, _, tol, _ = attention(ref, q[part], [n], span, 0)
        assert_near(out, want, tol, f"chunk that ends at {at}")
    rk, rv = heart.heart_cache_read(kc, vc, table, kv_len, n=N, **exps)
    assert torch.equal(rk[0].transpose(0, 1).double().cpu(), stands["k"]) and torch.equal(rv[0].transpose(0, 1).double().cpu(), stands["v"])
    qq = q.cuda().transpose(0, 1)[None]
    qb, kb, _, _ = heart.heart_pool_qk(qq, rk, block)
    oqb, _ = oracle.pool(u16(qq.contiguous()), block)
    assert torch.allclose(qb.cpu(), torch.from_numpy(oqb), atol=1e-5)
    Nb = qb.shape[2]
    tau = torch.ones(H, device="cuda")  # (keeps every block)
    _, idx, cnt = heart.heart_mask_topp(qb, kb, tau)
    assert (cnt == Nb).all()
    sparse = heart.heart_block_sparse_attn(qq, rk, rv, block, idx, cnt)
    whole = heart.heart_cache_attn(q.cuda(), kc, vc, table, kv_len, causal=0, **exps)
    want, _, tol, _ = attention(ref, q, [N], 0, 0)
    assert_near(whole, want, tol, "whole clip")
    assert_near(sparse[0].transpose(0, 1), want, tol, "whole clip, block-sparse")


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,H,Hq", [(1, 2, 8), (40, 3, 3)])
def test_captured_steps_follow_their_lengths(kind, n, H, Hq):
    """A step of writing and attention, captured once: every replay follows the lengths and tokens that are there then, with
    eager calls on the same workspace between the replays."""
    B, D, page = 3, 64, 16
    kc, vc, exps, table = empty_cache(B, H, D, page, 3000, kind)
    g = torch.Generator().manual_seed(n)
    lens = [torch.tensor(x, dtype=torch.int32) for x in ([900, 40, n], [901, 41 + n, 700], [902, 2900, 701 + n], [903, 2901, n])]
    # (what is there before: tokens of random values everywhere)
    x = [torch.randn((B * 3000, H, D), generator=g).bfloat16().cuda() for _ in range(2)]
    heart.heart_cache_write(*x, kc, vc, table, torch.full((B,), 3000, dtype=torch.int32, device="cuda"), **exps)
    q, k, v = (torch.zeros((B * n, h, D), dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H))
    kv_len = torch.full((B,), n, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros((Hq, B * n), device="cuda")
    ws = torch.full((heart.heart_cache_attn_workspace_bytes(q, kc, table),), 255, dtype=torch.uint8, device="cuda")

    def step(o, l):
        heart.heart_cache_write(k, v, kc, vc, table, kv_len, **exps)
        heart.heart_cache_attn(q, kc, vc, table, kv_len, out=o, lse=l, workspace=ws, **exps)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out, lse)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, lse)
    for i, x in enumerate(lens + lens[:2]):
        kv_len.copy_(x)
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g))
        print(f"replay {i} lengths {x.tolist()}", flush=True)
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        eager, eager_lse = torch.zeros_like(out), torch.zeros_like(lse)
        step(eager, eager_lse)
        torch.cuda.synchronize()
        assert torch.equal(got, eager) and torch.equal(got_lse, eager_lse)
        alone = heart.heart_cache_attn(q, kc, vc, table, kv_len, workspace=None, **exps)
        assert (alone.float() - got.float()).abs().max() <= 2.0**-6 * max(1.0, got.float().abs().max().item())


def test_captured_calls_share_a_workspace():
    """Two captured calls of different shapes on one workspace, replayed in turn: each gives what it gives alone."""
    caches = [Cache([4000, 300], 2, 128, 32, "bf16", seed=1), Cache([2500, 2600], 2, 128, 16, "e4m3", seed=2)]
    qs = [torch.randn((2 * n, 8, 128), generator=torch.Generator().manual_seed(n)).bfloat16().cuda() for n in (1, 30)]
    want = [heart.heart_cache_attn(q, *c.args(), **c.exps()) for q, c in zip(qs, caches)]
    need = max(heart.heart_cache_attn_workspace_bytes(q, c.stored["k"], c.page_table) for q, c in zip(qs, caches))
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    out = [torch.zeros_like(q) for q in qs]
    graphs = [torch.cuda.CUDAGraph() for _ in qs]
    for i, c in enumerate(caches):
        with torch.cuda.graph(graphs[i]):
            heart.heart_cache_attn(qs[i], *c.args(), out=out[i], workspace=ws, **c.exps())
    for turn in (0, 1, 0, 0, 1, 1, 0):
        out[turn].zero_()
        graphs[turn].replay()
        torch.cuda.synchronize()
        assert torch.equal(out[turn], want[turn]), turn


def test_two_streams_at_once():
    """Calls that overlap, each with a workspace of its own, give what they give alone."""
    caches = [Cache([4000, 300], 2, 128, 32, "bf16", seed=1), Cache([2500, 2600], 2, 64, 16, "e4m3", seed=2)]
    qs = [torch.randn((2, 8, c.D), generator=torch.Generator().manual_seed(i)).bfloat16().cuda() for i, c in enumerate(caches)]
    want = [heart.heart_cache_attn(q, *c.args(), **c.exps()) for q, c in zip(qs, caches)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(heart.heart_cache_attn(qs[i], *caches[i].args(), **caches[i].exps()))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_more_sequences_than_are_divided():
    """Beyond 256 sequences a workgroup has a whole tile."""
    B = 300
    kvs = [1 + (37 * i) % 130 for i in range(B)]
    c = Cache(kvs, 1, 64, 16, "e4m3", seed=5)
    q = torch.randn((B, 3, 64), generator=torch.Generator().manual_seed(1)).bfloat16()
    assert heart.heart_cache_attn_workspace_bytes(q, c.stored["k"], c.page_table) == 0
    for cu in (None, ends([1] * B)):
        out = heart.heart_cache_attn(q.cuda(), *c.args(), cu_q=cu, **c.exps())
        want, _, tol, _ = attention(c, q, [1] * B, 1, 0)
        assert_near(out, want, tol, "out")


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_caches_beyond_4_gib(kind):
    """Pages whose elements (and, of codes, exponents' rows) lie more than 2^32 bytes behind the first."""
    H, page, D = 8, 256, 128
    esz = 2 if kind == "bf16" else 1
    n = (9 << 30) // (H * page * D * esz)
    dt = torch.bfloat16 if kind == "bf16" else torch.float8_e4m3fn
    kc, vc = (torch.empty((n, H, page, D * esz), dtype=torch.uint8, device="cuda").view(dt) for _ in range(2))
    exps = {x: torch.empty((n, H, page), dtype=torch.uint8, device="cuda") if kind == "e4m3" else None for x in ("k_exp", "v_exp")}
    table = torch.tensor([[n - 1, 0, n // 2 + 1, 3]], dtype=torch.int32, device="cuda")
    N = 700
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn((N, H, D), generator=g).bfloat16() for _ in range(3))
    kv_len = torch.tensor([N], dtype=torch.int32, device="cuda")
    heart.heart_cache_write(k.cuda(), v.cuda(), kc, vc, table, kv_len, **exps)
    stands = {m: e4m3_values(x)[0] if kind == "e4m3" else x.double() for m, x in (("k", k), ("v", v))}
    rk, rv = heart.heart_cache_read(kc, vc, table, kv_len, n=N, **exps)
    assert torch.equal(rk[0].transpose(0, 1).double().cpu(), stands["k"]) and torch.equal(rv[0].transpose(0, 1).double().cpu(), stands["v"])
    ref = Cache([N], H, D, 32, "bf16", device="cpu")
    ref.sequence = lambda m, b, length=None: stands[m].transpose(0, 1)
    for rows in (slice(N - 1, N), slice(N - 200, N)):  # (single tokens, and chunks)
        out = heart.heart_cache_attn(q[rows].cuda(), kc, vc, table, kv_len, **exps)
        want, _, tol, _ = attention(ref, q[rows], [q[rows].shape[0]], 1, 0)
        assert_near(out, want, tol, "out")


def test_sequences_without_anything():
    """No new tokens at all though the tensors hold some; negative lengths; out stays as it was, or is zero."""
    c = Cache([50, 20], 2, 64, 16, "bf16", seed=1)
    for T, Hq in ((3, 4), (400, 2)):
        q = torch.randn((T, Hq, 64), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
        out = torch.full_like(q, 3.0)
        heart.heart_cache_attn(q, *c.args(), cu_q=torch.zeros(3, dtype=torch.int32, device="cuda"), out=out)
        assert (out == 3.0).all()
        c2 = (c.stored["k"], c.stored["v"], c.page_table, torch.tensor([-5, -(2**31)], dtype=torch.int32, device="cuda"))
        lse = torch.zeros((Hq, T), device="cuda")
        heart.heart_cache_attn(q, *c2, cu_q=ends([1, T - 1]), out=out, lse=lse)
        assert (out == 0.0).all() and (lse == -math.inf).all()
        before = c.stored["k"].clone()
        heart.heart_cache_write(q[:, :2].contiguous(), q[:, :2].contiguous(), *c2, cu_q=ends([1, T - 1]))
        assert torch.equal(before.view(torch.int16), c.stored["k"].view(torch.int16))


def test_tensors_of_another_device_are_refused():
    c = Cache([20], 1, 64, 16)
    q = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    native = heart.binding._native()
    k, v, table, lens = c.args()
    with pytest.raises(ValueError, match="current device"):
        native.cache_attn(q, k, v, table, lens, None, None, None, 1, 0, 0.0, torch.empty_like(q), None, None, 1, 0)

"""The plan, the int8 cache and its attention as they are used: step after step of a serving loop, captured and replayed, on other
streams, at addresses beyond 4 GiB."""
import random

import pytest
import torch

import paper_2605_14513_amd as heart
from cache_blocks_reference import Blocks, plan, tolerance
from cache_testlib import assert_near

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rand(T, H, D, seed, gain=1.0):
    return (gain * torch.randn((T, H, D), generator=torch.Generator().manual_seed(seed))).bfloat16()


@pytest.mark.parametrize("D,page,T", [(64, 16, 150), (128, 32, 9000)])
def test_a_serving_loop(D, page, T):
    """Prompts, single tokens, drafts of which some are taken back, requests that end and others in their places, more than there
    are pages for: every array and code after every step as the definitions say, and what the new tokens attend to."""
    B, M, H, G, n_pages = 5, 12, 2, 3, 22
    c = Blocks([0] * B, H, D, page, seed=D, spare=n_pages, room=M * page)
    table = [[-1] * M for _ in range(B)]
    free = list(range(n_pages))
    random.Random(D).shuffle(free)
    n_free, kv = n_pages, [0] * B
    s = dict(kv_len=i32(kv), page_table=i32(table), free_pages=i32(free), n_free=i32([n_free]))
    for n in "kv":  # (as an allocation finds them)
        c.scale[n].fill_(float("nan"))
        c.scales[n].fill_(float("nan"))
    steps = [([40, 17, 0, 100, 1], None), ([1, 1, 33, 1, 1], None), ([4, 4, 4, 4, 4], None), ([2, 5, 1, 1, 3], [41, 18, 37, 103, 6]),
             ([1, 70, 1, 200, 1], [43, 0, 38, 0, 9]), ([8, 8, 8, 8, 8], None), ([0, 1, 0, 1, 500], [0, 10**6, 0, -4, 3]), ([60, 1, 60, 1, 60], None)]
    refused = 0
    for i, (add, keep) in enumerate(steps):
        print(f"step {i} add {add} keep {keep} lengths {kv}", flush=True)
        want = plan(add, kv, kv if keep is None else keep, table, free, n_free, page, T)
        cu, slots, pos = heart.heart_cache_plan(i32(add), *s.values(), page, n=T, keep=None if keep is None else i32(keep))
        torch.cuda.synchronize()
        assert cu.tolist() == want["cu_q"] and slots.tolist() == want["slots"] and pos.tolist() == want["positions"]
        assert s["kv_len"].tolist() == want["kv_len"] and s["page_table"].tolist() == want["page_table"]
        assert s["n_free"].tolist() == want["n_free"] and s["free_pages"].tolist()[:want["n_free"][0]] == want["free_pages"]
        table, kv, n_free = want["page_table"], want["kv_len"], want["n_free"][0]
        free = want["free_pages"] + [-1] * (n_pages - n_free)
        qs = [b - a for a, b in zip(want["cu_q"], want["cu_q"][1:])]
        refused += sum(q == 0 for q, a in zip(qs, add) if a > 0)
        # the step's tensors have room for T tokens, as a captured one's
        N = sum(qs) + 7
        q, k, v = rand(N, H * G, D, 3 * i), rand(N, H, D, 3 * i + 1, 1.0 + i % 3), rand(N, H, D, 3 * i + 2, 0.5 + i % 2)
        c.table_cpu = torch.tensor(table, dtype=torch.int32)
        c.kvs = c.lens = kv
        c.write(qs, k, v)
        cache = (c.stored["k"], c.stored["v"], s["page_table"], s["kv_len"])
        heart.heart_cache_write(k.cuda(), v.cuda(), *cache, cu_q=cu, **c.scale_args())
        out = heart.heart_cache_attn(q.cuda(), *cache, cu_q=cu, **c.scale_args())
        rk, rv = heart.heart_cache_read(*cache, **c.scale_args())
        torch.cuda.synchronize()
        c.same(f"step {i}")
        want_out, _, tol, _ = tolerance(c, q, qs)
        assert_near(out[:sum(qs)], want_out[:sum(qs)], tol[:sum(qs)], f"out of step {i}")
        for b in range(B):
            for n, x in (("k", rk), ("v", rv)):
                assert torch.equal(x[b, :, :kv[b]].cpu(), c.sequence(n, b).float().bfloat16()), (i, b, n)
        # (slots are where the tokens are)
        t = torch.tensor([x for x in want["slots"] if x >= 0])
        codes = c.stored["k"].cpu()[t // page, :, t % page]
        scale = c.scales["k"][t // page]
        assert ((codes * scale[:, :, None] - k[:len(t)].float()).abs() <= scale[:, :, None] / 2).all()
    assert refused >= (2 if page == 16 else 1)  # (so that there were some)


@pytest.mark.parametrize("B,n,T", [(3, 1, 8), (3, 40, 160), (300, 1, 7000)])
def test_captured_steps(B, n, T):
    """Plan, writing and attention captured as one graph: every replay follows the additions and lengths that are there then, with
    the same step run eagerly on copies of the state in between."""
    H, G, D, page, M = 2, 2, 64, 16, 40
    n_pages = min(B, 40) * 30
    r = random.Random(B)
    free = list(range(n_pages))
    r.shuffle(free)
    s = dict(kv_len=i32([0] * B), page_table=torch.full((B, M), -1, dtype=torch.int32, device="cuda"), free_pages=i32(free), n_free=i32([n_pages]))
    cache = dict(k_cache=torch.zeros((n_pages, H, page, D), dtype=torch.int8, device="cuda"), v_cache=torch.zeros((n_pages, H, page, D), dtype=torch.int8, device="cuda"))
    scales = dict(k_scale=torch.full((n_pages, H), float("nan"), device="cuda"), v_scale=torch.full((n_pages, H), float("nan"), device="cuda"))
    add, keep = i32([0] * B), i32([0] * B)
    q, k, v = (torch.zeros((T, h, D), dtype=torch.bfloat16, device="cuda") for h in (H * G, H, H))
    outs = dict(cu_q=i32([0] * (B + 1)), slots=torch.zeros(T, dtype=torch.int64, device="cuda"), positions=i32([0] * T))
    out, lse = torch.zeros_like(q), torch.zeros((H * G, T), device="cuda")
    ws = torch.empty(max(heart.heart_cache_attn_workspace_bytes(q, cache["k_cache"], s["page_table"]), 16), dtype=torch.uint8, device="cuda")
    plan_ws = torch.empty(max(heart.heart_cache_plan_workspace_bytes(B, M, T), 16), dtype=torch.uint8, device="cuda")

    def step(s, cache, scales, outs, out, lse):
        heart.heart_cache_plan(add, *s.values(), page, keep=keep, workspace=plan_ws, **outs)
        args = (*cache.values(), s["page_table"], s["kv_len"])
        heart.heart_cache_write(k, v, *args, cu_q=outs["cu_q"], **scales)
        heart.heart_cache_attn(q, *args, cu_q=outs["cu_q"], out=out, lse=lse, workspace=ws, **scales)

    copy = lambda: [{m: x.clone() for m, x in d.items()} for d in (s, cache, scales, outs)] + [out.clone(), lse.clone()]  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*copy())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(s, cache, scales, outs, out, lse)
    g = torch.Generator().manual_seed(B + n)
    for i in range(7):
        lens = s["kv_len"].tolist()
        add.copy_(i32([r.randint(0, 2 * n) if i % 2 else n for _ in range(B)]))
        keep.copy_(i32([r.choice([x, x, max(0, x - n), 0 if i > 2 else x]) for x in lens]))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g))
        eager = copy()
        step(*eager)
        torch.cuda.synchronize()
        print(f"replay {i}", flush=True)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager[:4], (s, cache, scales, outs)):
            for m in a:
                x, y = a[m], b[m]
                assert ((x == y) | ((x != x) & (y != y))).all(), (i, m)
        m = outs["cu_q"][-1].item()
        assert m > 0 and torch.equal(eager[4][:m], out[:m]) and torch.equal(eager[5][:, :m], lse[:, :m]), i
        assert torch.isfinite(out[:m]).all()


def test_two_streams_at_once():
    """Calls that overlap, each with a workspace and a cache of its own, give what they give alone."""
    caches = [Blocks([4000, 300], 2, 128, 32, seed=1), Blocks([2500, 2600], 2, 64, 16, seed=2)]
    qs = [rand(2 * n, 8, c.D, i).cuda() for i, (c, n) in enumerate(zip(caches, (1, 60)))]
    kv = [rand(2 * n, 2, c.D, 5 + i).cuda() for i, (c, n) in enumerate(zip(caches, (1, 60)))]
    step = lambda i: (heart.heart_cache_write(kv[i], kv[i], *caches[i].args(), **caches[i].scale_args()),  # noqa: E731
                      heart.heart_cache_attn(qs[i], *caches[i].args(), **caches[i].scale_args()))[1]
    want = [step(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(step(i))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_captured_calls_share_a_workspace():
    """Captured calls of three kernels on one workspace, replayed in turn: each gives what it gives alone."""
    caches = [Blocks([4000, 300], 2, 128, 32, seed=1), Blocks([2500, 2600], 2, 128, 16, seed=2), Blocks([900, 700], 2, 128, 16, seed=3)]
    qs = [rand(2 * n, 8, 128, n).cuda() for n in (1, 30, 8)]
    want = [heart.heart_cache_attn(q, *c.args(), **c.scale_args()) for q, c in zip(qs, caches)]
    need = max(heart.heart_cache_attn_workspace_bytes(q, c.stored["k"], c.page_table) for q, c in zip(qs, caches))
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    out = [torch.zeros_like(q) for q in qs]
    graphs = [torch.cuda.CUDAGraph() for _ in qs]
    for i, c in enumerate(caches):
        with torch.cuda.graph(graphs[i]):
            heart.heart_cache_attn(qs[i], *c.args(), out=out[i], workspace=ws, **c.scale_args())
    for turn in (0, 1, 2, 0, 0, 2, 1, 1, 0, 2):
        out[turn].zero_()
        graphs[turn].replay()
        torch.cuda.synchronize()
        assert torch.equal(out[turn], want[turn]), turn


def test_caches_beyond_4_gib():
    """Pages whose codes lie more than 2^32 bytes behind the first."""
    H, page, D = 8, 256, 128
    n = (9 << 30) // (H * page * D)
    kc, vc = (torch.empty((n, H, page, D), dtype=torch.int8, device="cuda") for _ in range(2))
    scales = dict(k_scale=torch.empty((n, H), device="cuda"), v_scale=torch.empty((n, H), device="cuda"))
    ids = [n - 1, 0, n // 2 + 1]
    table = i32([ids])
    N = 700
    c = Blocks([N], H, D, page, seed=1, room=768, device="cpu")  # (the same pages in the definition's small cache)
    c.table_cpu = torch.tensor([[0, 1, 2]], dtype=torch.int32)
    q, k, v = rand(N, H, D, 1), rand(N, H, D, 2), rand(N, H, D, 3)
    c.write([N], k, v)
    kv_len = i32([N])
    heart.heart_cache_write(k.cuda(), v.cuda(), kc, vc, table, kv_len, **scales)
    torch.cuda.synchronize()
    for m, (store, scale) in {"k": (kc, scales["k_scale"]), "v": (vc, scales["v_scale"])}.items():
        for i, page_id in enumerate(ids):
            rows = min(page, N - i * page)
            assert torch.equal(store[page_id, :, :rows].cpu(), c.codes[m][i, :, :rows]) and torch.equal(scale[page_id].cpu(), c.scales[m][i])
    rk, _ = heart.heart_cache_read(kc, vc, table, kv_len, n=N, **scales)
    assert torch.equal(rk[0].cpu(), c.sequence("k", 0).float().bfloat16())
    for rows in (slice(N - 1, N), slice(N - 200, N)):  # (single tokens, and chunks)
        m = rows.stop - rows.start
        out = heart.heart_cache_attn(q[rows].cuda(), kc, vc, table, kv_len, **scales)
        want, _, tol, _ = tolerance(c, q[rows], [m])
        assert_near(out, want, tol, "out")


def test_tensors_of_another_device_are_refused():
    c = Blocks([20], 1, 64, 16)
    q = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    native = heart.binding._native()
    k, v, table, lens = c.args()
    with pytest.raises(ValueError, match="current device"):
        native.cache_attn(q, k, v, table, lens, None, c.scale["k"], c.scale["v"], 1, 0, 0.0, torch.empty_like(q), None, None, 1, 0)
    with pytest.raises(ValueError, match="current device"):
        native.cache_plan(lens, lens, table, lens, lens, 16, None, i32([0, 0]), torch.zeros(1, dtype=torch.int64, device="cuda"), lens, None, 1, 0)

"""heart_cache_plan against the definition, request after request: whole numbers, so all of them are equal."""
import random

import pytest
import torch

import paper_2605_14513_amd as heart
from cache_blocks_reference import plan

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def state(B, M, page, r, spare, full=0.5):
    """Requests that have pages in random order, and a list of `spare` others."""
    kv = [r.choice([0, r.randint(0, M * page), min(M * page, page * r.randint(0, M))]) if r.random() > full * 0.1 else M * page for _ in range(B)]
    need = [-(-n // page) for n in kv]
    n_pages = sum(need) + spare + r.randint(0, 3)
    ids = list(range(n_pages))
    r.shuffle(ids)
    table, at = [], 0
    for n in need:
        table.append(ids[at:at + n] + [-1] * (M - n))
        at += n
    return kv, table, ids[at:at + spare] + [-7] * (n_pages - spare), spare


def check(add, kv, keep, table, free, n_free, page, T, what="", workspace="auto", passes=2):
    print(f"cache_plan B={len(kv)} max_pages={len(table[0])} page={page} n_pages={len(free)} n_free={n_free} T={T} {what}", flush=True)
    want = plan(add, kv, kv if keep is None else keep, table, free, n_free, page, T)
    s = dict(kv_len=i32(kv), page_table=i32(table), free_pages=i32(free), n_free=i32([n_free]))
    k = None if keep is None else i32(keep)
    for i in range(passes):
        cu, slots, pos = heart.heart_cache_plan(i32(add), *s.values(), page, n=T, keep=k, workspace=workspace)
        torch.cuda.synchronize()
        got = dict(cu_q=cu, slots=slots, positions=pos, **s)
        for n, w in want.items():
            g = got[n].tolist()
            if n == "free_pages":
                g = g[:len(w)]
            assert g == w, f"{n} of pass {i}"
        if keep is None:
            break  # (what was new is kept; else the second pass takes back what the first gave)
    return s


@pytest.mark.parametrize("B,M,page,T", [
    (1, 1, 16, 1), (1, 1, 16, 0), (1, 500, 64, 4680), (2, 9, 16, 40), (64, 20, 16, 300), (65, 20, 32, 4000), (1023, 6, 16, 3000), (1024, 5, 32, 6000),
    (1024, 6, 16, 6001), (1025, 6, 16, 3000), (3000, 4, 16, 9000), (4096, 3, 16, 9000), (4097, 3, 16, 9000), (9000, 2, 16, 20000), (2, 140000, 16, 50), (17, 200, 256, 30000), (300, 300, 16, 5000), (5, 3, 128, 2)])
def test_random_requests(B, M, page, T):
    for seed in range(4):
        r = random.Random(1000 * B + 10 * M + seed)
        spare = r.choice([0, 1, B // 2 + 1, 3 * B, 20 * B])
        kv, table, free, n_free = state(B, M, page, r, spare)
        most = max(1, 2 * T // B)
        add = [r.choice([0, 1, r.randint(0, most), -5]) for _ in range(B)]
        keep = [r.choice([n, n, 0, r.randint(0, n)]) for n in kv]
        check(add, kv, keep, table, free, n_free, page, T, f"seed {seed}")
        check(add, kv, None, table, free, n_free, page, T, f"seed {seed}, all kept")


@pytest.mark.parametrize("B", [5, 1200])
def test_order_of_refusals(B):
    """Behind the first request that finds too few pages only those that need none are granted; behind the first without room
    for its tokens none; a request beyond the table takes nothing from the others."""
    page, M = 16, 4
    kv = [16] * B
    table = [[b, -1, -1, -1] for b in range(B)]
    free = list(range(B, B + 3)) + [-1] * B
    add = [0] * B
    add[:5] = [17, 100, 40, 0, 1]
    kv[4] = 15
    s = check(add, kv, None, table, free, 3, page, 100)
    assert s["kv_len"][:5].tolist() == [33, 16, 16, 16, 16] and s["n_free"].item() == 1
    add[:5] = [5, 5, 5, 1, 1]
    kv[4] = 16
    s = check(add, kv, None, table, free, 3, page, 11)
    assert s["kv_len"][:5].tolist() == [21, 21, 16, 16, 16]


@pytest.mark.parametrize("B,T", [(7, 50), (1100, 4000), (7, 20000), (4200, 3000)])
def test_arrays_that_hold_anything(B, T):
    """Lengths, lists and tables of no sense: as the definition, and nothing outside the arrays is touched."""
    page, M, n_pages = 16, 6, 40
    big = 2**31 - 1
    for seed in range(6):
        r = random.Random(seed + B)
        odd = lambda: r.choice([0, 1, -1, 5, 17, 96, 97, big, -big - 1, r.randint(-100, 200)])  # noqa: E731
        kv, keep, add = ([odd() for _ in range(B)] for _ in range(3))
        table = [[r.choice([-1, 0, 39, 40, big, -big - 1, r.randint(0, 39)]) for _ in range(M)] for _ in range(B)]
        free = [r.choice([0, 39, 40, -1, big, r.randint(0, 39)]) for _ in range(n_pages)]
        n_free = r.choice([-3, 0, 5, 40, 41, big, -big - 1])
        print(f"cache_plan anything B={B} T={T} seed {seed}", flush=True)
        want = plan(add, kv, keep, table, free, n_free, page, T)
        # every array in the middle of a larger one
        hold = {}

        def inside(name, x, dtype=torch.int32):
            x = torch.tensor(x, dtype=dtype, device="cuda")
            whole = torch.full((x.numel() + 256,), 1234567, dtype=dtype, device="cuda")
            whole[128:128 + x.numel()] = x.flatten()
            hold[name] = whole
            return whole[128:128 + x.numel()].view(x.shape)

        a = {n: inside(n, x) for n, x in (("add", add), ("kv_len", kv), ("page_table", table), ("free_pages", free), ("n_free", [n_free]), ("keep", keep))}
        outs = dict(cu_q=inside("cu_q", [0] * (B + 1)), slots=inside("slots", [0] * T, torch.int64), positions=inside("positions", [0] * T))
        need = heart.heart_cache_plan_workspace_bytes(B, M, T)
        ws = inside("workspace", [0] * (need // 4)).view(torch.uint8) if need else None
        heart.heart_cache_plan(a["add"], a["kv_len"], a["page_table"], a["free_pages"], a["n_free"], page, keep=a["keep"], workspace=ws, **outs)
        torch.cuda.synchronize()
        got = dict(a, **outs)
        for n, w in want.items():
            g = got[n].tolist()
            assert (g[:len(w)] if n == "free_pages" else g) == w, n
        for n, whole in hold.items():
            assert (whole[:128] == 1234567).all() and (whole[-128:] == 1234567).all(), n
        assert got["add"].tolist() == add and got["keep"].tolist() == keep


def test_keep_may_be_the_lengths():
    for B in (9, 1100, 4200):
        r = random.Random(B)
        kv, table, free, n_free = state(B, 8, 16, r, 5 * B)
        add = [r.randint(0, 3) for _ in range(B)]
        want = plan(add, kv, kv, table, free, n_free, 16, 9 * B)
        s = dict(kv_len=i32(kv), page_table=i32(table), free_pages=i32(free), n_free=i32([n_free]))
        cu, slots, pos = heart.heart_cache_plan(i32(add), *s.values(), 16, n=9 * B, keep=s["kv_len"])
        assert cu.tolist() == want["cu_q"] and slots.tolist() == want["slots"] and s["kv_len"].tolist() == want["kv_len"]


def test_outputs_that_are_not_asked_for():
    """The library's call without slots and positions."""
    lib = heart.load_library()
    for B, T in ((4, 30), (4, 20000)):
        r = random.Random(B)
        kv, table, free, n_free = state(B, 8, 16, r, 50)
        add = [3] * B
        want = plan(add, kv, kv, table, free, n_free, 16, T)
        s = [i32(kv), i32(table), i32(free), i32([n_free])]
        cu, a = torch.zeros(B + 1, dtype=torch.int32, device="cuda"), i32(add)
        ws = torch.empty(heart.heart_cache_plan_workspace_bytes(B, 8, T) + 16, dtype=torch.uint8, device="cuda")
        rc = lib.heart_cache_plan(B, 8, 16, len(free), T, None, a.data_ptr(), *[x.data_ptr() for x in s], cu.data_ptr(), None, None, ws.data_ptr(),
                                  ws.numel(), torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        torch.cuda.synchronize()
        assert cu.tolist() == want["cu_q"] and s[1].tolist() == want["page_table"] and s[3].item() == want["n_free"][0]


@pytest.mark.parametrize("B,T", [(6, 60), (1100, 5000), (4200, 9000)])
def test_captured_plans_follow_the_lengths(B, T):
    """A plan captured once and replayed: lengths, additions and refusals of every replay are those that are there then, with
    eager plans on the same workspace in between."""
    page, M = 16, 12
    r = random.Random(B)
    kv, table, free, n_free = state(B, M, page, r, 6 * B)
    s = dict(kv_len=i32(kv), page_table=i32(table), free_pages=i32(free), n_free=i32([n_free]))
    add, keep = i32([0] * B), i32(kv)
    ws = torch.empty(max(heart.heart_cache_plan_workspace_bytes(B, M, T), 16), dtype=torch.uint8, device="cuda")
    outs = dict(cu_q=i32([0] * (B + 1)), slots=torch.zeros(T, dtype=torch.int64, device="cuda"), positions=i32([0] * T))
    run = lambda st, o: heart.heart_cache_plan(add, *st.values(), page, keep=keep, workspace=ws, **o)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run({n: x.clone() for n, x in s.items()}, outs)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(s, outs)
    for step in range(6):
        now = [r.randint(0, 9) for _ in range(B)]
        lens = s["kv_len"].tolist()
        kept = [r.choice([n, n, n, max(0, n - 3), 0]) for n in lens]
        add.copy_(i32(now))
        keep.copy_(i32(kept))
        want = plan(now, lens, kept, s["page_table"].tolist(), s["free_pages"].tolist(), s["n_free"].item(), page, T)
        copy = {n: x.clone() for n, x in s.items()}
        run(copy, {n: x.clone() for n, x in outs.items()})
        print(f"cache_plan replay {step}", flush=True)
        graph.replay()
        torch.cuda.synchronize()
        for n, w in want.items():
            g = dict(outs, **s)[n].tolist()
            assert (g[:len(w)] if n == "free_pages" else g) == w, (n, step)


def test_refused_tensors():
    B = 3
    s = [i32([0] * B), i32([0] * B), i32([[0] * 4] * B), i32([0] * 9), i32([0])]
    call = lambda a, **kw: heart.heart_cache_plan(*a, 16, **{"n": 5, **kw})  # noqa: E731
    call(s)
    for i, bad, error, text in ((0, i32([0] * 2), ValueError, "add"), (1, i32([0] * 4), ValueError, "kv_len"), (0, s[0].long(), TypeError, "int32"),
                                (1, s[1].float(), TypeError, "int32"), (2, s[2].t().contiguous().t(), ValueError, "contiguous"),
                                (3, s[3][::2], ValueError, "contiguous"), (3, s[2], ValueError, "n_pages"), (4, i32([0, 0]), ValueError, "n_free"),
                                (0, s[0].cpu(), TypeError, "GPU"), (3, None, TypeError, "free_pages")):
        a = list(s)
        a[i] = bad
        with pytest.raises(error, match=text):
            call(a)
    for kw, error, text in ((dict(keep=i32([0])), ValueError, "keep"), (dict(cu_q=i32([0] * 3)), ValueError, "cu_q"),
                            (dict(slots=i32([0] * 5)), TypeError, "int64"), (dict(positions=torch.zeros(5, device="cuda")), TypeError, "int32"),
                            (dict(n=-1, slots=None), (ValueError, RuntimeError), "negative")):
        with pytest.raises(error, match=text):
            call(s, **kw)
    with pytest.raises(heart.HeartError, match="workspace"):
        call(s, n=20000, workspace=None)
    with pytest.raises(heart.HeartError, match="page must be"):
        heart.heart_cache_plan(*s, 17, n=5)
    with pytest.raises(TypeError, match="page"):
        heart.heart_cache_plan(*s, 16.0, n=5)

"""heart_cache_write and heart_cache_read on int8 caches: codes and scales bit for bit, and nothing else touched."""
import math

import pytest
import torch

import paper_2605_14513_amd as heart
from cache_blocks_reference import Blocks
from cache_testlib import ends

pytestmark = pytest.mark.gpu


def tokens(T, H, D, seed, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, H, D), generator=g) * torch.exp(0.5 * torch.randn((T, H, 1), generator=g)) * gain
    return x.bfloat16()


def write(c, qs, k, v, cu=True, what=""):
    print(f"cache_write int8 qs={qs} kvs={c.lens} H={c.H} D={c.D} page={c.page} {what}", flush=True)
    c.write(qs, k.cpu(), v.cpu())
    heart.heart_cache_write(k.cuda(), v.cuda(), *c.args(), cu_q=ends(qs) if cu is True else cu if cu is not False else None, **c.scale_args())
    torch.cuda.synchronize()
    c.same(what)


def read_back(c, n=None):
    """The values that the CPU's codes and scales stand for, rounded once; rows behind a sequence as they were."""
    B, N = len(c.kvs), n if n is not None else max(max(c.kvs), 1)
    k, v = (torch.full((B, c.H, N, c.D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    heart.heart_cache_read(*c.args(), k=k, v=v, **c.scale_args())
    torch.cuda.synchronize()
    for name, got in (("k", k), ("v", v)):
        for b, kv in enumerate(c.kvs):
            m = min(kv, N)
            want = c.sequence(name, b, kv)[:, :m].float().bfloat16()
            assert ((got[b, :, :m].cpu() == want) | (want.isnan() & got[b, :, :m].cpu().isnan())).all(), (name, b)
            assert (got[b, :, m:] == 7.0).all(), (name, b)


@pytest.mark.parametrize("layout", ["head", "token", "joint"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_write_and_read(page, D, layout):
    """Begun pages whose scale grows and whose does not, whole pages, a token in one page, two pages, many."""
    kvs = [1, page, page + 1, 3 * page - 1, 2 * page + 5, 700, 16]
    qs = [1, page, 2, page + 7, 1, 333, 0]
    c = Blocks(kvs, 3, D, page, layout, seed=page + D)
    for gain, seed in ((0.2, 1), (30.0, 2), (2.0, 3)):  # (scales: as they were, larger, and as the second time)
        write(c, qs, tokens(sum(qs), 3, D, seed, gain), tokens(sum(qs), 3, D, seed + 9, gain), what=f"{layout} gain {gain}")
    read_back(c)
    read_back(c, n=page + 3)
    read_back(c, n=1)


@pytest.mark.parametrize("H,T", [(1, 1), (5, 1), (40, 1), (2, 77), (1, 4097)])
def test_equal_chunks_without_ranges(H, T):
    for B in (1, 3, 70):
        if B * T * H > 20000:
            continue
        c = Blocks([T + 13 * b for b in range(B)], H, 64, 16, seed=B)
        write(c, [T] * B, tokens(B * T, H, 64, B), tokens(B * T, H, 64, B + 1), cu=False)


def test_tokens_one_by_one():
    """A sequence that grows by single tokens of rising and falling size, through begun pages and new ones."""
    H, D, page, n = 2, 128, 16, 40
    c = Blocks([0], H, D, page, seed=4, room=64, spare=5)
    c.table_cpu[0] = torch.tensor([4, 1, 3, 0], dtype=torch.int32)
    c.page_table.copy_(c.table_cpu)
    for i in range(n):
        c.kvs[0] = c.lens[0] = i + 1
        c.kv_len.fill_(i + 1)
        write(c, [1], tokens(1, H, D, i, gain=2.0 ** (i % 7 - 3)), tokens(1, H, D, 100 + i, gain=1.0 + i / 9), cu=False, what=f"token {i}")
    read_back(c)


def test_strided_tokens():
    """k and v as slices of one projection's output, heads with room between them."""
    c = Blocks([50, 20], 3, 64, 32, seed=2)
    x = tokens(30, 9, 80, 5).cuda()
    k, v = x[:, :3, :64], x[:, 5:8, 16:]
    write(c, [20, 10], k, v)


def test_values_at_the_ends():
    """Rows of zeros, a token of zeros behind others and before them, halves (ties), the smallest and largest numbers, NaN and
    infinities: of the pages and heads they are in."""
    H, D, page = 8, 64, 16
    c = Blocks([24, 30], H, D, page, seed=3)
    k, v = tokens(18, H, D, 1), tokens(18, H, D, 2)
    k[:, 0] = 0.0                                              # (also: a begun page keeps its scale)
    k[:, 1] = (torch.arange(D) - 31.5).bfloat16() * 2.0**-3     # ties under scales that are powers of two
    k[0, 1, 0] = 127.0 * 2.0**-3
    k[:, 2] *= 2.0**-130
    k[:, 3] = 3.3895e38
    k[4, 4, 7], k[6, 5, 0], v[17, 6, 3] = math.nan, math.inf, -math.inf
    v[:, 7] = -0.0
    v[:, 2] = 2.0**-133
    write(c, [8, 10], k, v, what="ends")
    assert c.scales["k"].isnan().any() and (c.scales["k"] == 2.0**-126).any()
    read_back(c)
    # (a page keeps a NaN until its first token is written anew)
    write(c, [1, 1], tokens(2, H, D, 5), tokens(2, H, D, 6), what="after")
    write(c, [24, 30], tokens(54, H, D, 7), tokens(54, H, D, 8), what="anew")
    assert not any(c.scales[n][c.table_cpu[b, :2]].isnan().any() for n in "kv" for b in range(2))
    read_back(c)


def test_a_page_of_zeros_and_then_more():
    c = Blocks([16], 2, 128, 16, seed=1)
    zero = torch.zeros((16, 2, 128), dtype=torch.bfloat16)
    write(c, [16], zero, zero)
    assert (c.scales["k"][c.table_cpu[0, 0]] == 0).all()
    read_back(c)
    write(c, [4], tokens(4, 2, 128, 3), tokens(4, 2, 128, 4))
    read_back(c)


def test_places_that_are_none():
    """Negative positions, positions behind the page table, pages that the table does not name or that are none: not written,
    read as zeros; tokens behind the last range left out."""
    H, D, page = 2, 64, 16
    c = Blocks([70, 40, 8, 33], H, D, page, seed=6)
    cap = c.table_cpu.shape[1] * page
    c.table_cpu[0, 1], c.table_cpu[1, 2], c.table_cpu[3, 0] = -1, c.n_pages, -(2**31)
    c.page_table.copy_(c.table_cpu)
    c.lens = [70, 40, 8, cap + 9]
    c.kv_len.copy_(torch.tensor(c.lens))
    qs = [60, 30, 20, 40]
    k, v = tokens(sum(qs) + 13, H, D, 1), tokens(sum(qs) + 13, H, D, 2)
    write(c, qs, k, v, what="none")
    c.lens = c.kvs = [70, 40, 8, 33]
    c.kv_len.copy_(torch.tensor(c.lens))
    read_back(c)


def test_ranges_that_fall_or_leave_the_tensors():
    """Memory outside what the table names for these sequences stays as it was, whatever the ranges say."""
    H, D, page = 2, 64, 16
    for cu in ([0, 30, 10, 40], [5, 3, 2, 1], [-7, 4, 90, 95], [0, 2**31 - 1, 8, 16], [-(2**31), 5, 5, 40]):
        c = Blocks([33, 20, 48], H, D, page, seed=8, spare=6)
        before = {n: (c.stored[n].clone(), c.scale[n].clone()) for n in "kv"}
        x = tokens(40, H, D, 1).cuda()
        print(f"cache_write int8 ranges {cu}", flush=True)
        heart.heart_cache_write(x, x, *c.args(), cu_q=torch.tensor(cu, dtype=torch.int32, device="cuda"), **c.scale_args())
        torch.cuda.synchronize()
        named = torch.zeros(c.n_pages, dtype=torch.bool)
        named[c.table_cpu[c.table_cpu >= 0].long()] = True
        for n in "kv":
            assert torch.equal(c.stored[n][~named], before[n][0][~named])
            assert (c.scale[n][~named].isnan()).all()


@pytest.mark.parametrize("D,page", [(64, 16), (128, 256)])
def test_reading_much(D, page):
    """More codes than are read through the caches, by the room of the outputs."""
    H, N = 33, 2 * (81 << 20) // (2 * 33 * D * 2) + 5
    c = Blocks([700, 0], H, D, page, seed=D, room=N)
    k, v = (torch.full((2, H, N, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    print(f"cache_read int8 of room for {N} tokens, H={H} D={D}", flush=True)
    heart.heart_cache_read(*c.args(), k=k, v=v, **c.scale_args())
    torch.cuda.synchronize()
    for name, got in (("k", k), ("v", v)):
        assert torch.equal(got[0, :, :700].cpu(), c.sequence(name, 0).float().bfloat16())
        assert (got[0, :, 700:] == 7.0).all() and (got[1] == 7.0).all()


def test_no_tokens():
    c = Blocks([5, 0], 1, 64, 16, seed=1)
    x = torch.zeros((0, 1, 64), dtype=torch.bfloat16, device="cuda")
    heart.heart_cache_write(x, x, *c.args(), **c.scale_args())
    write(c, [0, 0], tokens(3, 1, 64, 1), tokens(3, 1, 64, 2))
    read_back(c, n=9)


@pytest.mark.parametrize("bad,error,text", [
    (dict(k_scale=None), TypeError, "k_scale"), (dict(v_scale=None), TypeError, "v_scale"),
    (dict(k_scale="half"), TypeError, "float32"), (dict(v_scale="page"), ValueError, "n_pages,H"), (dict(v_scale="strided"), ValueError, "contiguous"),
    (dict(k_cache="bf16"), ValueError, "only an int8"), (dict(v_cache="bf16"), TypeError, "v_cache")])
def test_refused_caches(bad, error, text):
    c = Blocks([20], 2, 64, 16, seed=1)
    a, kw = list(c.args()), c.scale_args()
    s = kw["k_scale"]
    what = {"half": s.half(), "page": s[:, :, None].expand(-1, -1, 16).contiguous(), "strided": s.t().contiguous().t(),
            "bf16": a[0].bfloat16(), None: None}
    for n, x in bad.items():
        if n in kw:
            kw[n] = what[x]
        else:
            a[0 if n == "k_cache" else 1] = what[x]
    x = tokens(1, 2, 64, 1).cuda()
    with pytest.raises(error, match=text):
        heart.heart_cache_write(x, x, *a, **kw)
    with pytest.raises(error, match=text):
        heart.heart_cache_read(*a, **kw)
    with pytest.raises(error, match=text):
        heart.heart_cache_attn(x, *a, workspace=None, **kw)

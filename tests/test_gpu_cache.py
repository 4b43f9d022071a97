"""heart_cache_write and heart_cache_read: exact values, and nothing else touched."""
import math

import pytest
import torch

import paper_2605_14513_amd as heart
from cache_testlib import Cache, e4m3_values, ends

pytestmark = pytest.mark.gpu


def bits(x):
    return x.contiguous().view(torch.uint8 if x.element_size() == 1 else torch.int16).cpu()


def write(cache, qs, k, v, cu=True, cu_q=None):
    """The call, and the cache as it has to be after it (codes and exponents, by token)."""
    want = {n: (bits(cache.stored[n]).clone(), None if cache.exp[n] is None else cache.exp[n].cpu().clone()) for n in "kv"}
    at = 0
    for b, n in enumerate(qs):
        for i in range(n):
            p = cache.kv_len[b].item() - n + i
            page = cache.table_cpu[b, p // cache.page].item() if 0 <= p < cache.table_cpu.shape[1] * cache.page else -1
            if not 0 <= page < cache.n_pages:
                continue
            for name, x in (("k", k), ("v", v)):
                row = x[at + i].cpu()
                if cache.kind == "e4m3":
                    val, exp = e4m3_values(row)
                    codes = torch.ldexp(val, 127 - exp.int().unsqueeze(-1)).float().to(torch.float8_e4m3fn)
                    want[name][0][page, :, p % cache.page] = codes.view(torch.uint8)
                    want[name][1][page, :, p % cache.page] = exp
                else:
                    want[name][0][page, :, p % cache.page] = row.view(torch.int16)
        at += n
    print(f"cache_write qs={qs} kvs={cache.kv_len.tolist()} H={cache.H} D={cache.D} page={cache.page} {cache.kind}", flush=True)
    heart.heart_cache_write(k, v, *cache.args(), cu_q=cu_q if cu_q is not None else ends(qs) if cu else None, **cache.exps())
    torch.cuda.synchronize()
    for n in "kv":
        got = bits(cache.stored[n])
        if cache.kind == "e4m3":  # (a NaN is a NaN)
            nan = (got & 0x7F == 0x7F) & (want[n][0] & 0x7F == 0x7F)
            assert ((got == want[n][0]) | nan).all(), n
            assert torch.equal(cache.exp[n].cpu(), want[n][1]), n + "_exp"
        else:
            assert torch.equal(got, want[n][0]), n


def rows(T, H, D, seed=3):
    g = torch.Generator().manual_seed(seed)
    x = [torch.randn((T, H, D), generator=g) * torch.exp(3 * torch.randn((T, H, 1), generator=g)) for _ in range(2)]
    return [y.bfloat16().cuda() for y in x]


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kvs,qs", [([1], [1]), ([17], [17]), ([100, 3, 40], [33, 3, 0]), ([0, 50, 0, 16], [0, 1, 0, 16]),
                                    ([40] * 70, [1] * 70), ([300], [250]), ([5, 9], [8, 2])])
def test_write(kvs, qs, D, kind):
    write(Cache(kvs, 3, D, 16, kind, seed=len(kvs)), qs, *rows(sum(qs), 3, D))


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("layout", ["head", "token", "joint"])
def test_write_pages_and_layouts(page, layout, kind):
    write(Cache([300, 65], 2, 64, page, kind, layout, seed=page), [40, 40], *rows(80, 2, 64), cu=False)


def test_write_takes_strided_rows():
    big = torch.randn((30, 9, 128), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    write(Cache([64], 3, 128, 16, "e4m3"), [30], big[:, :3], big[:, 4:7])
    write(Cache([64], 1, 128, 16, "bf16"), [30], big[:, :1], big[:, 8:])


def test_write_leaves_out_what_has_no_place():
    """Tokens behind the last sequence, positions below 0 or beyond the table, pages that are none."""
    cache = Cache([40, 64], 2, 64, 16, "bf16", seed=6)
    k, v = rows(60, 2, 64)
    write(cache, [20, 10], k, v)  # 30 tokens are nobody's
    cache.kv_len.copy_(torch.tensor([7, 90]))  # (positions -3 .., and up to 89 of 80)
    write(cache, [10, 30], k, v)
    cache.table_cpu[0, 0], cache.table_cpu[1, 3] = cache.n_pages, -7
    cache.page_table = cache.table_cpu.cuda()
    cache.kv_len.copy_(torch.tensor([30, 64]))
    write(cache, [30, 30], k, v)


def test_write_many_short_sequences():
    """More sequences than a wavefront has lanes, sequences without new tokens among them."""
    kvs = [1 + i % 5 for i in range(200)]
    qs = [i % 3 if i % 3 <= kvs[i] else 1 for i in range(200)]
    write(Cache(kvs, 1, 64, 16, "bf16"), qs, *rows(sum(qs), 1, 64))


def test_write_values_next_to_borders():
    """Zeros, the ends of bf16, subnormal numbers, rows at 448 of a power of two, ties, NaN and infinities."""
    D = 64
    x = torch.zeros((10, 1, D), dtype=torch.float64)
    x[1, 0] = torch.ldexp(1.75 + torch.arange(D) / 128.0, torch.tensor(3)).clamp_max(15.9)   # above 1.75: one power more
    x[2, 0, 0], x[2, 0, 1:] = 448.0, torch.arange(1, D) / 16.0
    x[3, 0, 0], x[3, 0, 1:] = 450.0, torch.arange(1, D) * 7.0                                # (450 rounds to 448 in bf16)
    x[4, 0] = torch.ldexp(torch.ones(D, dtype=torch.float64), -133 + torch.arange(D) % 9)     # subnormal numbers of bf16
    x[5, 0] = 3.3895e38
    x[5, 0, 1::2] = 1e-38
    x[6, 0, 0], x[6, 0, 1:] = 256.0, (torch.arange(1, D) + 0.5) * 2.0**-9                     # ties in the smallest steps
    x[7, 0, 0], x[7, 0, 1:] = 256.0, 16.0 + torch.arange(1, D) / 4.0                          # ties
    x[8, 0] = torch.arange(D) - 20.0
    x[8, 0, 3], x[8, 0, 4], x[8, 0, 5] = math.nan, math.inf, -math.inf
    x[9, 0] = math.inf
    x = x.bfloat16().cuda()
    write(Cache([10], 1, D, 16, "e4m3"), [10], x, -x)


def expect_read(cache, N):
    out = {}
    for n in "kv":
        y = torch.full((len(cache.kvs), cache.H, N, cache.D), 9.0, dtype=torch.float64)
        for b in range(len(cache.kvs)):
            m = min(cache.kvs[b], N)
            y[b, :, :m] = cache.sequence(n, b, m)
        out[n] = y.bfloat16()
    return out


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kvs,N", [([1], 1), ([0], 5), ([100, 0, 17], 100), ([300, 63], 130), ([64, 16], 200), ([200], 13)])
def test_read(kvs, N, D, kind):
    """Rows behind the last token stay as they were, also where N is past the page table's room."""
    cache = Cache(kvs, 2, D, 16, kind, seed=N)
    k, v = (torch.full((len(kvs), 2, N, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    print(f"cache_read kvs={kvs} N={N} D={D} {kind}", flush=True)
    heart.heart_cache_read(*cache.args(), k=k, v=v, **cache.exps())
    torch.cuda.synchronize()
    want = expect_read(cache, N)
    assert torch.equal(bits(k), bits(want["k"])) and torch.equal(bits(v), bits(want["v"]))


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("layout", ["head", "token", "joint"])
def test_read_pages_and_layouts(page, layout, kind):
    """Also into token-major outputs."""
    cache = Cache([300, 129], 3, 64, page, kind, layout, seed=1)
    k, v = (torch.full((2, 300, 3, 64), 9.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2) for _ in range(2))
    heart.heart_cache_read(*cache.args(), k=k, v=v, **cache.exps())
    want = expect_read(cache, 300)
    assert torch.equal(bits(k), bits(want["k"])) and torch.equal(bits(v), bits(want["v"]))
    a, b = heart.heart_cache_read(*cache.args(), n=7, **cache.exps())
    assert a.shape == (2, 3, 7, 64) and torch.equal(bits(a), bits(want["k"][:, :, :7])) and torch.equal(bits(b), bits(want["v"][:, :, :7]))


def test_read_of_pages_that_are_none_gives_zeros():
    cache = Cache([80], 2, 64, 16, "e4m3")
    cache.table_cpu[0, 1], cache.table_cpu[0, 3] = -1, cache.n_pages
    cache.page_table = cache.table_cpu.cuda()
    k, v = heart.heart_cache_read(*cache.args(), n=80, **cache.exps())
    want = expect_read(cache, 80)
    assert torch.equal(bits(k), bits(want["k"])) and torch.equal(bits(v), bits(want["v"]))


def test_every_code_reads_as_its_value():
    """All codes under all exponents whose values are normal numbers of bf16."""
    D, page = 64, 256
    cache = Cache([page * 4], 1, D, page, "e4m3", spare=0)
    for q in range(4):
        i = cache.table_cpu[0, q].item()
        codes = torch.arange(64 * q, 64 * q + 64, dtype=torch.uint8)
        cache.stored["k"].view(torch.uint8)[i, 0] = codes.cuda()
        cache.exp["k"][i, 0] = torch.arange(page).clamp(10, 240).to(torch.uint8).cuda()
    k, _ = heart.heart_cache_read(*cache.args(), **cache.exps(), n=4 * page)
    for q in range(4):
        val = torch.arange(64 * q, 64 * q + 64, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
        exp = torch.arange(page).clamp(10, 240).double() - 127
        want = (val[None] * torch.exp2(exp)[:, None]).bfloat16()
        got = k[0, 0, q * page:(q + 1) * page].cpu()
        assert ((got == want) | (got.isnan() & want.isnan())).all()


def test_no_tokens():
    cache = Cache([20], 2, 64, 16)
    before = bits(cache.stored["k"])
    x = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    heart.heart_cache_write(x, x, *cache.args())
    k, v = heart.heart_cache_read(*cache.args(), n=0)
    assert k.shape == v.shape == (1, 2, 0, 64) and torch.equal(before, bits(cache.stored["k"]))


# what the binding refuses of tensors on the GPU (nothing is launched)
@pytest.mark.parametrize("change,error,text", [
    (dict(k_cache="half"), TypeError, "k_cache"), (dict(v_cache="e4m3"), TypeError, "v_cache"), (dict(v_cache="few"), ValueError, "v_cache"),
    (dict(v_cache="columns"), ValueError, "contiguous D"), (dict(k_exp="bytes"), ValueError, "no exponents"),
    (dict(page_table="long"), TypeError, "page_table"), (dict(page_table="columns"), ValueError, "page_table"),
    (dict(kv_len="few"), ValueError, "kv_len"), (dict(cu_q="few"), ValueError, "cu_q"), (dict(cu_q="long"), TypeError, "cu_q"),
    (dict(x="float"), TypeError, "dtype"), (dict(x="heads"), ValueError, "heads|H"), (dict(x="width"), ValueError, "D"),
    (dict(x="columns"), ValueError, "contiguous D"), (dict(x="cpu"), TypeError, "GPU"), (dict(x="none"), TypeError, "GPU")])
def test_refusals_of_the_binding(change, error, text):
    c = Cache([20, 30], 2, 64, 16)
    a = dict(zip(("k_cache", "v_cache", "page_table", "kv_len"), c.args()))
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    more = {}
    for name, how in change.items():
        t = x if name == "x" else ends([2, 2]) if name == "cu_q" else a.get(name)
        y = {"half": lambda: t.half(), "e4m3": lambda: t.to(torch.float8_e4m3fn), "few": lambda: t[:-1].contiguous(),
             "columns": lambda: t.transpose(-1, -2).contiguous().transpose(-1, -2), "long": lambda: t.long(),
             "bytes": lambda: torch.zeros((c.n_pages, 2, 16), dtype=torch.uint8, device="cuda"), "float": lambda: t.float(),
             "heads": lambda: t[:, :1].expand(4, 3, 64).contiguous(), "width": lambda: t[..., :32].contiguous(),
             "cpu": lambda: t.cpu(), "none": lambda: None}[how]()
        if name == "x":
            x = y
        elif name in a:
            a[name] = y
        else:
            more[name] = y
    cache = tuple(a.values())
    with pytest.raises(error, match=text):
        heart.heart_cache_write(x, x, *cache, **more)
    if "x" not in change:
        q = torch.zeros((4, 6, 64), dtype=torch.bfloat16, device="cuda")
        with pytest.raises(error, match=text):
            heart.heart_cache_attn(q, *cache, workspace=None, **more)
        if "cu_q" not in change:
            with pytest.raises(error, match=text):
                heart.heart_cache_read(*cache, k=torch.zeros((2, 2, 5, 64), dtype=torch.bfloat16, device="cuda"),
                                       v=torch.zeros((2, 2, 5, 64), dtype=torch.bfloat16, device="cuda"), **more)


def test_refusals_of_exponents():
    c = Cache([20, 30], 2, 64, 16, "e4m3")
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    e = c.exps()
    for bad, error in ((None, TypeError), (e["k_exp"].int(), TypeError), (e["k_exp"][:-1].contiguous(), ValueError),
                       (e["k_exp"].transpose(0, 1).contiguous().transpose(0, 1), ValueError)):
        with pytest.raises(error, match="k_exp"):
            heart.heart_cache_write(x, x, *c.args(), k_exp=bad, v_exp=e["v_exp"])


def test_refusals_of_outputs():
    c = Cache([20, 30], 2, 64, 16)
    q = torch.zeros((4, 4, 64), dtype=torch.bfloat16, device="cuda")
    for kw, error in ((dict(out=q[:3]), ValueError), (dict(out=q.float()), TypeError), (dict(lse=torch.zeros((4, 5), device="cuda")), ValueError),
                      (dict(lse=torch.zeros((4, 4), device="cuda").double()), TypeError), (dict(lse=torch.zeros(4, 8, device="cuda")[:, ::2]), ValueError),
                      (dict(workspace=torch.zeros(100, dtype=torch.uint8, device="cuda")), heart.HeartError), (dict(workspace=q.cpu()), TypeError),
                      (dict(causal=-1), heart.HeartError), (dict(causal=1.5), TypeError), (dict(window=2.0), TypeError)):
        with pytest.raises(error):
            heart.heart_cache_attn(q, *c.args(), **kw)
    with pytest.raises(heart.HeartError, match="multiple"):
        heart.heart_cache_attn(q[:, :3], *c.args())
    with pytest.raises(heart.HeartError, match="multiple of B"):
        heart.heart_cache_attn(q[:3], *c.args())
    k = torch.zeros((2, 2, 5, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (k[:1], k[:, :1], k[..., :32], k[0]):
        with pytest.raises(ValueError, match="k and v"):
            heart.heart_cache_read(*c.args(), k=bad, v=bad)

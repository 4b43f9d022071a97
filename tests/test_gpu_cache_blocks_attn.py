"""heart_cache_attn over int8 caches, against the definition in 64 bits with derived tolerances."""
import math

import pytest
import torch

import paper_2605_14513_amd as heart
from cache_blocks_reference import Blocks, tolerance
from cache_testlib import assert_near, ends

pytestmark = pytest.mark.gpu


def new_q(T, Hq, D, seed=1):
    return torch.randn((T, Hq, D), generator=torch.Generator().manual_seed(seed)).bfloat16()


def check(c, q, qs, causal=1, window=0, scale=0.0, workspace="auto", cu=True, weight=2.0**-11, what=""):
    print(f"cache_attn int8 B={len(qs)} qs={qs[:6]} kvs={c.lens[:6]} Hq={q.shape[1]} H={c.H} D={c.D} page={c.page} causal={causal} window={window} "
          f"workspace={workspace} {what}", flush=True)
    T, Hq, D = q.shape
    if T * (Hq // c.H) <= 16 * len(qs):  # (few rows: weights of two bf16, scales in fp32)
        weight = 2.0**-16
    want, want_lse, tol, ltol = tolerance(c, q, qs, causal, window, scale, weight)
    out = torch.full((T, Hq, D), 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((Hq, T), 5.0, device="cuda")
    heart.heart_cache_attn(q.cuda(), *c.args(), cu_q=ends(qs) if cu else None, causal=causal, window=window, scale=scale, out=out, lse=lse,
                           workspace=workspace, **c.scale_args())
    torch.cuda.synchronize()
    n = sum(qs)
    assert_near(out[:n], want[:n], tol[:n], "out")
    assert_near(lse[:, :n], want_lse[:, :n], ltol[:, :n], "lse")
    assert (out[n:] == 5.0).all() and (lse[:, n:] == 5.0).all()
    return out


@pytest.mark.parametrize("workspace", ["auto", None])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("D", [64, 128])
def test_single_tokens(D, page, workspace):
    for kvs, H, G in (([1], 1, 1), ([1000], 2, 1), ([700, 1, 16, 129, 333], 2, 5), ([5000, 17], 1, 16), ([60] * 70, 1, 2)):
        c = Blocks(kvs, H, D, page, seed=len(kvs) + page)
        check(c, new_q(len(kvs), H * G, D), [1] * len(kvs), workspace=workspace, cu=len(kvs) % 2 == 0)


@pytest.mark.parametrize("workspace", ["auto", None])
@pytest.mark.parametrize("page,layout", [(16, "token"), (32, "joint"), (64, "head"), (128, "token"), (256, "head")])
@pytest.mark.parametrize("D", [64, 128])
def test_chunks(D, page, layout, workspace):
    for kvs, qs, H, G in (([200], [200], 2, 1), ([900, 64, 33], [40, 64, 1], 1, 3), ([1500, 700], [257, 0], 2, 2), ([37], [37], 3, 8)):
        c = Blocks(kvs, H, D, page, layout, seed=page)
        check(c, new_q(sum(qs) + 3, H * G, D), qs, workspace=workspace)


@pytest.mark.parametrize("n", [1, 5, 90])
@pytest.mark.parametrize("causal,window", [(0, 0), (1, 1), (1, 50), (0, 64), (70, 0), (70, 100), (3, 7), (1000, 33), (2**30, 0), (1, 2**31 - 1)])
def test_masks(n, causal, window):
    c = Blocks([n, 300, 777], 2, 64, 32, seed=n)
    check(c, new_q(3 * n, 4, 64), [n] * 3, causal, window, cu=False)


@pytest.mark.parametrize("workspace", ["auto", None])
@pytest.mark.parametrize("n", [2, 60])
def test_rows_without_keys_and_lengths_that_are_none(n, workspace):
    """More new tokens than cached ones (positions below 0), lengths of 0 and below, lengths beyond the table with windows that
    reach back from the position."""
    c = Blocks([n - 1, 0, 40, 256, 256], 2, 128, 16, seed=5, room=256)
    c.lens = [n - 1, 0, -3, 300, 2**31 - 1]
    c.kv_len.copy_(torch.tensor(c.lens))
    for causal, window in ((1, 0), (0, 0), (1, 30), (1, 60), (64, 100)):
        want_q = new_q(5 * n, 4, 128)
        c2 = c.lens
        c.lens = [n - 1, 0, 0, 300, 2**31 - 1]  # (a negative length is none: positions are those of length 0)
        check(c, want_q, [n] * 5, causal, window, workspace=workspace)
        c.lens = c2


def test_pages_that_are_none_read_as_zeros():
    for n, G in ((1, 2), (50, 3)):
        c = Blocks([300, 100], 2, 64, 16, seed=4)
        c.table_cpu[0, 2], c.table_cpu[0, 18], c.table_cpu[1, 0] = -1, c.n_pages, 2**31 - 1
        c.table_cpu[c.table_cpu == 0] = -1  # (page 0, whose scales such a page must not get, is under NaN)
        c.page_table.copy_(c.table_cpu)
        for w in ("k", "v"):
            c.scales[w][0] = math.nan
            c.scale[w][0] = math.nan
        check(c, new_q(2 * n, 2 * G, 64), [n, n])


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("spread", [0, 12, 20])
def test_scales_of_very_different_size(n, spread):
    """Blocks whose scales differ by up to 2^spread, as they come, and all of them far from one."""
    for shift in (0, 40, -40):
        c = Blocks([900, 200], 2, 64, 16, seed=spread, spread=spread)
        c.scales["v"] *= 2.0**shift
        c.scale["v"].copy_(c.scales["v"])
        c.scales["k"] *= 2.0**-shift
        c.scale["k"].copy_(c.scales["k"])
        q = (new_q(2 * n, 4, 64).float() * 2.0**shift).bfloat16()
        check(c, q, [n, n], what=f"spread {spread} shift {shift}")


@pytest.mark.parametrize("n", [1, 40])
def test_scales_of_zero(n):
    """Blocks of zeros: keys whose logits are 0, values that are 0; a cache of nothing else."""
    c = Blocks([300, 90], 2, 64, 32, seed=2)
    for w in ("k", "v"):
        for b, ps in ((0, (1, 4)), (1, (0, 1, 2))):
            for p in ps:
                c.scales[w][c.table_cpu[b, p]] = 0.0
        c.scale[w].copy_(c.scales[w])
    for causal, window in ((1, 0), (1, 20), (0, 0)):
        check(c, new_q(2 * n, 4, 64), [n, n], causal, window)


@pytest.mark.parametrize("n", [1, 40])
def test_scales_of_seven_bits(n):
    """Scales that another program wrote: values have up to 14 bits, and are rounded to f16 too."""
    c = Blocks([500, 90], 2, 128, 16, seed=2)
    g = torch.Generator().manual_seed(1)
    for w in ("k", "v"):
        c.scales[w] = torch.randint(64, 128, c.scales[w].shape, generator=g).float() * 2.0**-11
        c.scale[w].copy_(c.scales[w])
    check(c, new_q(2 * n, 4, 128), [n, n], weight=2.0**-10)


@pytest.mark.parametrize("n", [2, 150])
@pytest.mark.parametrize("workspace", ["auto", None])
def test_what_is_not_finite(n, workspace):
    """A scale that is NaN: the queries of its head that see the page get NaN, no others but those of tiles that hold them; a query
    with NaN gets NaN."""
    H, G, kvs = 2, 2, [3000, 700]
    for w in ("k", "v"):
        c = Blocks(kvs, H, 64, 32, seed=1)
        q = new_q(2 * n, H * G, 64)
        q[n + 1, 3, 5] = math.nan
        bad_page = c.table_cpu[0, kvs[0] // 32 - 3].item()
        c.scale[w][bad_page, 0] = math.nan
        print(f"cache_attn int8 NaN scale of {w} n={n} workspace={workspace}", flush=True)
        out, lse = torch.zeros_like(q).cuda(), torch.zeros((H * G, 2 * n), device="cuda")
        heart.heart_cache_attn(q.cuda(), *c.args(), out=out, lse=lse, workspace=workspace, **c.scale_args())
        torch.cuda.synchronize()
        out, lse = out.cpu(), lse.cpu()
        sees = kvs[0] - n + torch.arange(n) >= (kvs[0] // 32 - 3) * 32
        assert out[:n][sees][:, :G].isnan().all() and out[n + 1, 3].isnan().all() and lse[3, n + 1].isnan()
        assert w == "v" or lse[:G, :n][:, sees].isnan().all()
        want, want_lse, tol, ltol = tolerance(c, q.nan_to_num(0.0), [n, n], weight=2.0**-11)
        ok = torch.ones((2 * n, H * G), dtype=torch.bool)
        ok[:n, :G] = False
        ok[n + 1, 3] = False
        assert_near(out[ok], want[ok], tol[ok], "out")
        assert_near(lse.t()[ok], want_lse.t()[ok], ltol.t()[ok], "lse")


@pytest.mark.parametrize("D,room", [(64, 1024), (128, 512), (64, 1040), (128, 528)])
def test_short_sequences(D, room):
    """All keys of a tile at once, where the page tables have room for no more, and one page more: empty and full sequences, windows,
    pages that are none, a scale that is NaN, many sequences."""
    for B, H, G, n in ((4, 3, 1, 1), (4, 3, 5, 3), (5, 1, 16, 1), (200, 1, 1, 1), (3, 2, 8, 7)):
        kvs = [room, 0, 1, room - 17, 33][:B] + [1 + 37 * b % room for b in range(5, B)]
        kvs = [max(0, k - 16) if room % 64 else k for k in kvs]
        c = Blocks(kvs, H, D, 16, seed=B, room=room)
        for causal, window in ((1, 0), (1, 45), (0, 0), (100, 0)):
            check(c, new_q(B * n, H * G, D), [n] * B, causal, window, cu=B % 2 == 0)
        c.table_cpu[0, 5], c.table_cpu[min(3, B - 1), 0] = -1, c.n_pages
        c.page_table.copy_(c.table_cpu)
        check(c, new_q(B * n, H * G, D), [n] * B, workspace=None)
        for w in ("k", "v"):
            bad = Blocks(kvs, H, D, 16, seed=B, room=room)
            bad.scale[w][bad.table_cpu[0, 7], 0] = math.nan
            out = heart.heart_cache_attn(new_q(B * n, H * G, D).cuda(), *bad.args(), **bad.scale_args()).cpu()
            assert out[:n, :G].isnan().all() and not out[n:].isnan().any() and not out[:, G:].isnan().any()


@pytest.mark.parametrize("scale", [2.0, 1e-3])
@pytest.mark.parametrize("n", [1, 40])
def test_logits_far_apart(n, scale):
    """References that move often: keys that grow along the sequence; and hardly any difference at all."""
    c = Blocks([1200], 1, 64, 16, seed=9, spread=0)
    for p in range(-(-1200 // 16)):
        c.scales["k"][c.table_cpu[0, p]] = 2.0 ** (p // 12 - 8)
    c.scale["k"].copy_(c.scales["k"])
    check(c, new_q(n, 4, 64), [n], scale=scale, workspace=None)
    check(c, new_q(n, 4, 64), [n], scale=scale)


def test_weights_down_to_the_smallest():
    """One key far above many: what the many weigh, 2^-21 to 2^-27 of it each, is not lost."""
    N, D = 4000, 64
    for n, G in ((20, 1), (1, 1)):
        for below in (14.6, 17.3, 18.7):  # of the natural logarithm
            c = Blocks([N], 1, D, 16, seed=3, spread=0)
            for w in ("k", "v"):
                c.codes[w][:] = 0
                c.scales[w][:] = 2.0**-4
            first = c.table_cpu[0, 0].item()
            c.codes["k"][first, 0, 0, 0] = 64               # k = 4 along the first axis
            c.codes["v"][:, 0, :, 1], c.codes["v"][first, 0, 0, 0], c.codes["v"][first, 0, 0, 1] = 127, 100, 0
            for w in ("k", "v"):
                c.stored[w].copy_(c.codes[w])
                c.scale[w].copy_(c.scales[w])
            q = torch.zeros((n, G, D), dtype=torch.bfloat16)
            q[:, :, 0] = below / 4
            out = check(c, q, [n], causal=0, scale=1.0)
            some = out[:, :, 1].double().cpu()
            p = torch.softmax(torch.cat([q[0, 0, :1].double() * 4, torch.zeros(N - 1, dtype=torch.float64)]), 0)
            want = 127 / 16 * p[1:].sum()
            assert ((some - want).abs() <= 2.0**-4 * want).all(), (n, below, some[0, 0].item(), want.item())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 100])
def test_columns_that_the_weights_cancel(D, n):
    """Rows of v of one sign and of the other in turn: out is far smaller than its terms, so a weight's rounding shows."""
    c = Blocks([2000], 1, D, 16, seed=D, cancel=True, spread=0)
    q = (0.25 * new_q(n, 8, D).float()).bfloat16()
    check(c, q, [n], causal=0)


@pytest.mark.parametrize("D", [64, 128])
def test_either_kernel_around_its_limits(D):
    """Rows, tiles and keys on either side of what the kernel for few rows takes of int8 (tables with room for just so many)."""
    for B, n, kv, H, G, room in ((1, 64, 700, 2, 1, 0), (1, 65, 700, 2, 1, 0), (2, 16, 4096, 1, 4, 4096), (2, 16, 4096, 1, 4, 4097),
                                 (2, 4, 600, 2, 5, 0), (20, 16, 300, 8, 4, 0), (64, 16, 200, 2, 4, 0), (65, 16, 200, 2, 4, 0), (3, 17, 48, 1, 1, 0), (1, 512, 700, 2, 1, 0),
                                 (1, 513, 700, 2, 1, 0), (2, 100, 130, 3, 5, 0), (1, 300, 1024, 2, 1, 1024)):
        c = Blocks([max(n, kv - 11 * b) for b in range(B)], H, D, 16, seed=n, room=room)
        for ws in ("auto", None):
            check(c, new_q(B * n, H * G, D), [n] * B, cu=B % 2 == 0, workspace=ws)


# (44 heads of five tiles of 256 rows: one round that is nearly full, where the page table has room for more than 5120 tokens)
@pytest.mark.parametrize("B,n,kvs,G,page,causal,window", [
    (1, 1024, [1100], 1, 16, 1, 0), (1, 1037, [1037], 1, 64, 1, 0), (1, 1024, [1029], 1, 16, 0, 0), (1, 1024, [1203], 1, 32, 300, 0),
    (1, 1024, [2047], 1, 16, 1, 77), (1, 257, [1016], 4, 128, 100, 130), (1, 1024, [4093], 1, 16, 1, 0), (2, 1100, [1111, 1100], 1, 16, 1, 0)])
def test_wide_tiles(B, n, kvs, G, page, causal, window):
    """Tiles of 256 rows give the same bits as those of 128 (the same cache under a page table with less room); lengths that end inside
    the sixteen rows of two wavefronts among them."""
    H, D = 44 if B == 1 else 24, 128
    c = Blocks(kvs, H, D, page, seed=n, room=5200, spread=9)
    q = new_q(B * n, H * G, D)
    out, lse = torch.zeros((2, B * n, H * G, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, H * G, B * n), device="cuda")
    short = c.page_table[:, :-(-max(kvs) // page)].contiguous()
    for i, table in enumerate((c.page_table, short)):
        print(f"cache_attn int8 wide B={B} n={n} kvs={kvs} G={G} page={page} causal={causal} window={window} room {table.shape[1] * page}", flush=True)
        heart.heart_cache_attn(q.cuda(), c.stored["k"], c.stored["v"], table, c.kv_len, causal=causal, window=window, out=out[i], lse=lse[i],
                               workspace=None, **c.scale_args())
        torch.cuda.synchronize()
    assert torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1])
    some = [0, H * G - 1]  # (the definition of two heads)
    one = Blocks(kvs, H, D, page, seed=n, room=5200, spread=9, device="cpu")
    for h in some:
        for w in ("k", "v"):
            one.codes[w], one.scales[w] = c.codes[w][:, h // G:h // G + 1], c.scales[w][:, h // G:h // G + 1]
        one.H = 1
        want, want_lse, tol, ltol = tolerance(one, q[:, h:h + 1], [n] * B, causal, window)
        assert_near(out[0][:, h:h + 1], want, tol, "out")
        assert_near(lse[0][h:h + 1], want_lse, ltol, "lse")


@pytest.mark.parametrize("H,n,kv,causal,window", [(60, 1100, 4200, 1, 0), (60, 1030, 4199, 500, 3000), (55, 1281, 2600, 0, 0)])
def test_wide_tiles_of_a_divided_round(H, n, kv, causal, window):
    """300 and 330 tiles of 256 rows: those of the last round are divided and added up, the others have the bits that they have
    undivided."""
    D = 128
    c = Blocks([kv], H, D, 64, seed=n, room=5200, spread=5)
    q = new_q(n, H, D)
    need = heart.heart_cache_attn_workspace_bytes(q, c.stored["k"], c.page_table)
    assert need > 0
    got = []
    for ws in (torch.full((need,), 0x55, dtype=torch.uint8, device="cuda"), None):
        print(f"cache_attn int8 wide, last round H={H} n={n} kv={kv} causal={causal} window={window} workspace={ws is not None}", flush=True)
        lse = torch.zeros((H, n), device="cuda")
        got.append((heart.heart_cache_attn(q.cuda(), *c.args(), causal=causal, window=window, lse=lse, workspace=ws, **c.scale_args()), lse))
        torch.cuda.synchronize()
    differ = (got[0][0] != got[1][0]).any(-1).float().mean().item()
    assert 0 < differ < 0.5
    one = Blocks([kv], 1, D, 64, seed=n, room=5200, device="cpu")
    one.table_cpu = c.table_cpu
    for h in (0, H // 2, H - 1):
        for w in ("k", "v"):
            one.codes[w], one.scales[w] = c.codes[w][:, h:h + 1], c.scales[w][:, h:h + 1]
        want, want_lse, tol, ltol = tolerance(one, q[:, h:h + 1], [n], causal, window)
        for out, lse in got:
            assert_near(out[:, h:h + 1], want, tol, "out")
            assert_near(lse[h:h + 1], want_lse, ltol, "lse")


def test_wide_tiles_of_anything():
    """Ragged ranges, pages that are none, a scale that is NaN and lengths that are none, of tiles of 256 rows."""
    H, D, kvs, qs = 16, 128, [1300, 1100, 0], [1290, 1100, 700]
    c = Blocks(kvs, H, D, 16, seed=1, room=5200)
    c.table_cpu[0, 3], c.table_cpu[1, 60], c.table_cpu[0, 81] = -1, c.n_pages, 2**31 - 1
    c.page_table.copy_(c.table_cpu)
    c.scale["k"][c.table_cpu[1, 2], 5] = math.nan
    q = new_q(sum(qs) + 9, H, D)
    got = []
    for table in (c.page_table, c.page_table[:, :100].contiguous()):
        out, lse = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device="cuda"), torch.full((H, q.shape[0]), 5.0, device="cuda")
        heart.heart_cache_attn(q.cuda(), c.stored["k"], c.stored["v"], table, c.kv_len, cu_q=ends(qs), out=out, lse=lse, workspace=None, **c.scale_args())
        torch.cuda.synchronize()
        got.append((out, lse))
    assert torch.equal(got[0][0].view(torch.int16), got[1][0].view(torch.int16)) and torch.equal(got[0][1].view(torch.int32), got[1][1].view(torch.int32))
    out, lse = got[0]
    assert out[1290 + 40:2390, 5].isnan().all() and not out[:1290].isnan().any() and not out[:, :5].isnan().any()
    assert (out[2390:3090] == 0).all() and (lse[:, 2390:3090] == -math.inf).all() and (out[3090:] == 5.0).all()


def test_many_parts_and_tails():
    """Sizes at which the keys of tiles are divided in each way: few tiles, two rounds of parts, a divided last round."""
    for B, n, kv, H, G in ((1, 300, 9000, 2, 1), (3, 130, 5000, 4, 4), (70, 33, 300, 2, 4), (1, 1200, 6000, 60, 1), (1, 16, 20000, 1, 1)):
        c = Blocks([max(n, kv - 37 * b) for b in range(B)], H, 64, 64, seed=n)
        q = new_q(B * n, H * G, 64)
        a = heart.heart_cache_attn(q.cuda(), *c.args(), **c.scale_args())
        b = heart.heart_cache_attn(q.cuda(), *c.args(), workspace=None, **c.scale_args())
        torch.cuda.synchronize()
        assert (a.float() - b.float()).abs().max() <= 2.0**-7 * b.float().abs().max()
        if B * n * H * G * kv < 2e8:
            check(c, q, [n] * B, cu=False)

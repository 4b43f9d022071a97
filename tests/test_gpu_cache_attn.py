"""heart_cache_attn against attention in 64 bits: lengths, heads, pages, masks, layouts, divided keys."""
import math

import pytest
import torch

import paper_2605_14513_amd as heart
from cache_testlib import Cache, assert_near, attention, ends

pytestmark = pytest.mark.gpu


def run(cache, Hq, qs, causal=1, window=0, cu=True, workspace="auto", seed=1, scale=0.0, gain=1.0, what=""):
    T = sum(qs)
    q = (torch.randn((T, Hq, cache.D), generator=torch.Generator().manual_seed(seed)) * gain).bfloat16()
    print(f"cache_attn {what} kvs={cache.kvs} qs={qs} Hq={Hq} H={cache.H} D={cache.D} page={cache.page} {cache.kind} "
          f"causal={causal} window={window}", flush=True)
    out = torch.full((T, Hq, cache.D), math.nan, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((Hq, T), math.nan, device="cuda")
    if isinstance(workspace, str) and workspace == "garbage":
        need = heart.heart_cache_attn_workspace_bytes(q, cache.stored["k"], cache.page_table)
        workspace = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    heart.heart_cache_attn(q.cuda(), *cache.args(), cu_q=ends(qs) if cu else None, causal=causal, window=window, scale=scale,
                           out=out, lse=lse, workspace=workspace, **cache.exps())
    torch.cuda.synchronize()
    want, want_lse, tol, ltol = attention(cache, q, qs, causal, window, scale or None)
    assert_near(out, want, tol, "out")
    assert_near(lse, want_lse, ltol, "lse")
    return out, lse


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kv", [1, 15, 16, 31, 33, 63, 64, 65, 96, 127, 129, 200, 257, 1000])
def test_one_token(D, kv, kind):
    run(Cache([kv], 2, D, 16, kind, seed=kv), 2, [1], cu=False)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,kv", [(1, 64), (31, 31), (33, 100), (128, 128), (129, 131), (200, 500)])
def test_chunks(D, n, kv, kind):
    for causal in (1, 0, 7, 64):
        run(Cache([kv], 1, D, 32, kind, seed=n + kv), 1, [n], causal=causal, workspace=None)


@pytest.mark.parametrize("Hq,H", [(1, 1), (3, 1), (8, 1), (10, 2), (40, 1), (6, 3), (130, 1)])
def test_shared_key_heads(Hq, H):
    for D, kind in ((64, "e4m3"), (128, "bf16")):
        run(Cache([70, 200], H, D, 16, kind, seed=Hq), Hq, [5, 1])


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["head", "token", "joint"])
def test_pages_and_layouts(page, layout):
    for D, kind in ((64, "bf16"), (128, "e4m3"), (128, "bf16"), (64, "e4m3")):
        run(Cache([300, 77], 2, D, page, kind, layout, seed=page), 4, [20, 3])


@pytest.mark.parametrize("workspace", ["garbage", None])
@pytest.mark.parametrize("kvs,qs", [
    ([0], [1]), ([0, 5, 0], [1, 1, 0]), ([0, 0], [0, 3]), ([3, 700], [5, 2]), ([64, 1, 2000], [0, 1, 0]),
    ([100] * 70, [1] * 70), ([5, 1500, 33], [1, 150, 33]), ([2, 0, 9], [200, 4, 30])])
def test_ragged_batches(kvs, qs, workspace):
    """Empty sequences, sequences without new tokens, more new tokens than cached ones (those at positions below 0 see nothing)."""
    cache = Cache(kvs, 2, 128, 16, "bf16", seed=len(kvs))
    for causal, window in ((1, 0), (0, 0), (1, 20), (0, 100), (16, 40)):
        run(cache, 4, qs, causal=causal, window=window, workspace=workspace)


@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 300, 10**9])
@pytest.mark.parametrize("causal", [0, 1, 50])
def test_windows(causal, window):
    for D, kind in ((64, "bf16"), (128, "e4m3")):
        run(Cache([500], 1, D, 64, kind, seed=window % 97), 2, [140], causal=causal, window=window)


@pytest.mark.parametrize("causal", [2**31 - 1, 2**30])
def test_blocks_as_long_as_they_can_be(causal):
    run(Cache([90], 1, 64, 16, seed=3), 1, [10], causal=causal)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [64, 128])
def test_divided_keys(D, kind):
    """Long sequences of few queries: the same with and without division, and twice the same bits."""
    cache = Cache([5000, 4097, 130], 2, D, 32, kind, seed=D)
    for qs, causal in (([1, 1, 1], 1), ([40, 3, 130], 1), ([20, 1, 2], 0)):
        a, la = run(cache, 6, qs, causal=causal, workspace="garbage", what="divided")
        b, lb = run(cache, 6, qs, causal=causal, workspace="garbage", what="again")
        assert torch.equal(a, b) and torch.equal(la, lb)
        run(cache, 6, qs, causal=causal, workspace=None, what="undivided")


def test_page_ids_beyond_one_register():
    """More than 64 stages of 64 keys in one part: 9000 keys, undivided."""
    for kind, page in (("bf16", 16), ("e4m3", 128)):
        run(Cache([9000], 1, 64, page, kind, seed=5), 1, [2], workspace=None)


@pytest.mark.parametrize("gain", [0.0, 1e-3, 8.0, 60.0])
def test_scales_of_logits(gain):
    """Equal logits, small ones, and ones of which one key takes all: the running reference moves or does not."""
    for D in (64, 128):
        run(Cache([400], 1, D, 16, seed=11), 2, [37], gain=gain)
    run(Cache([400], 1, 64, 16, seed=11), 2, [37], scale=0.37)


def test_growing_logits():
    """Keys whose logits grow along the cache, so that the reference moves in nearly every slice."""
    cache = Cache([600], 1, 64, 16, seed=2)
    for n in ("k",):
        for p in range(38):
            i = cache.table_cpu[0, p].item()
            ramp = (torch.arange(16) + 16 * p).double()[None, :, None] / 20
            x = (0.1 * torch.nan_to_num(cache.value[n][i]) + ramp).bfloat16()
            cache.value[n][i] = x.double()
            cache.stored[n][i] = x.cuda()
    q = torch.full((3, 1, 64), 0.5).bfloat16()
    out = heart.heart_cache_attn(q.cuda(), *cache.args())
    want, _, tol, _ = attention(cache, q, [3], 1, 0)
    assert_near(out, want, tol, "out")


def test_pages_that_the_table_does_not_name_read_as_zeros():
    cache = Cache([200], 2, 64, 16, seed=8)
    for p, bad in ((1, -1), (4, cache.n_pages), (7, 2**31 - 1), (9, -2**31)):
        cache.table_cpu[0, p] = bad
    cache.page_table = cache.table_cpu.cuda()
    run(cache, 2, [20])


def test_lengths_beyond_the_page_table():
    """kv_len past the room of the table: keys up to there."""
    cache = Cache([64], 1, 64, 16, seed=9, spare=0)
    cache.page_table = cache.table_cpu[:, :4].contiguous().cuda()
    cache.kv_len.fill_(100)
    q = torch.randn((1, 1, 64), generator=torch.Generator().manual_seed(1)).bfloat16()
    out = heart.heart_cache_attn(q.cuda(), *cache.args())
    want, _, tol, _ = attention(cache, q, [1], 0, 0)
    assert_near(out, want, tol, "out")


def test_tokens_behind_the_last_sequence_and_strided_tensors():
    """A padded batch: rows behind cu_q[B] are left as they were; q and out are views of larger tensors."""
    cache = Cache([50, 300], 2, 128, 32, seed=4)
    big = torch.randn((14, 6, 128), generator=torch.Generator().manual_seed(2)).bfloat16()
    q = big[:, 1:5]
    qs = [4, 7]
    room = torch.full((14, 3, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    out = room[:, 1]
    lse = torch.full((4, 14), 5.0, device="cuda")
    heart.heart_cache_attn(big.cuda()[:, 1:5], *cache.args(), cu_q=ends(qs), out=out, lse=lse)
    torch.cuda.synchronize()
    want, want_lse, tol, ltol = attention(cache, q[:11], qs, 1, 0)
    assert_near(out[:11], want, tol, "out")
    assert_near(lse[:, :11], want_lse, ltol, "lse")
    assert (out[11:] == 7.0).all() and (lse[:, 11:] == 5.0).all()
    assert (room[:, 0] == 7.0).all() and (room[:, 2] == 7.0).all()


def test_no_tokens():
    cache = Cache([50], 2, 128, 32, seed=4)
    q = torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda")
    assert heart.heart_cache_attn(q, *cache.args()).shape == (0, 4, 128)


@pytest.mark.parametrize("kind,D", [("bf16", 128), ("e4m3", 64)])
@pytest.mark.parametrize("H,n,kv,causal", [
    (40, 1664, 2000, 1), (40, 1664, 1700, 0),      # a last round of few tiles: those are divided
    (43, 1500, 1555, 300),                         # (heads that no XCD has alone)
    (20, 1900, 2100, 0), (9, 3000, 3100, 0)])      # fewer tiles than places: parts in two rounds, in one
def test_many_tiles_with_divided_keys(kind, D, H, n, kv, causal):
    cache = Cache([kv], H, D, 64, kind, seed=H)
    a, la = run(cache, H, [n], causal=causal, workspace="garbage", what="divided")
    b, lb = run(cache, H, [n], causal=causal, workspace=None, what="whole")
    c, lc = run(cache, H, [n], causal=causal, workspace="garbage", what="again")
    assert torch.equal(a, c) and torch.equal(la, lc)


@pytest.mark.parametrize("kind,D", [("bf16", 64), ("bf16", 128), ("e4m3", 128)])
@pytest.mark.parametrize("n,Hq", [(1, 1), (1, 6), (8, 8), (5, 40)])
def test_many_parts(kind, D, n, Hq):
    """One long sequence of one key head: more than 64 parts a tile, of tiles of 16 rows and of 128."""
    cache = Cache([30011], 1, D, 256, kind, seed=Hq)
    a, la = run(cache, Hq, [n], workspace="garbage", what="divided")
    b, lb = run(cache, Hq, [n], workspace="garbage", what="again")
    assert torch.equal(a, b) and torch.equal(la, lb)

"""Caches in 8 bits with a scale for each page and head, and the plan, without a GPU: what the calls refuse, the definitions that the
GPU tests go by, what the compiler made of the kernels."""
import ctypes
import math

import pytest
import torch

from cache_blocks_reference import Blocks, block_scale, plan
from test_cache_calls import EINVAL, EUNSUPPORTED, F, bf, cache, calls, lib  # noqa: F401
from test_kernel_resources import scratch_of

INT8 = 3


@pytest.mark.parametrize("change,code,text", [
    (dict(), EINVAL, "NULL"), (dict(k_exp=F), EINVAL, "NULL"), (dict(v_exp=F), EINVAL, "NULL"),
    (dict(k_exp=F, v_exp=F + 4), EUNSUPPORTED, "aligned"), (dict(k_exp=F + 8, v_exp=F), EUNSUPPORTED, "aligned"),
    (dict(k_exp=F, v_exp=F, k_stride=(4096, 2048, 136)), EUNSUPPORTED, "strides"),
    (dict(k_exp=F, v_exp=F, v_stride=(4096, 2040, 128)), EUNSUPPORTED, "strides"),
    (dict(k_exp=F, v_exp=F, k_stride=(4096, 2048, 0)), EUNSUPPORTED, "strides"), (dict(k_exp=F, v_exp=F, page=8), EUNSUPPORTED, "page"),
    (dict(k_exp=F, v_exp=F, D=32), EUNSUPPORTED, "64 or 128")])
def test_int8_caches_that_every_call_refuses(lib, change, code, text):  # noqa: F811
    for name, call in calls(lib, cache(type=INT8, **change)).items():
        assert call() == code, name
        assert text in lib.heart_last_error().decode(), name


@pytest.mark.parametrize("type", [2, 4, -1, 255])
def test_types_that_are_none(lib, type):  # noqa: F811
    for call in calls(lib, cache(type=type, k_exp=F, v_exp=F)).values():
        assert call() == EINVAL and b"type" in lib.heart_last_error()


def test_no_tokens_launch_nothing(lib):  # noqa: F811
    for name, call in calls(lib, cache(type=INT8, k_exp=F, v_exp=F), T=0, q=None, N=0).items():
        assert call() == 0, name


def test_a_write_has_less_than_2_to_the_32_threads(lib):  # noqa: F811
    # (a job is a page, head and tensor; a workgroup has at most one)
    c = cache(type=INT8, k_exp=F, v_exp=F, B=1, H=1, max_pages=1 << 26)
    assert calls(lib, c, T=1 << 30)["write"]() == EUNSUPPORTED and b"too many rows" in lib.heart_last_error()
    c = cache(type=INT8, k_exp=F, v_exp=F, B=1 << 29, H=1)
    assert calls(lib, c, T=1 << 29)["write"]() == EUNSUPPORTED and b"too many rows" in lib.heart_last_error()


def test_workspace_of_attention(lib):  # noqa: F811
    """Where either kernel may be meant, of int8 caches, the size is enough for both; else it is that of other types."""
    size = lambda T, Hq, **kw: lib.heart_cache_attn_workspace_bytes(ctypes.byref(cache(**kw)), T, Hq)  # noqa: E731
    int8 = dict(type=INT8, k_exp=F, v_exp=F)
    assert size(3, 4, **int8) == size(3, 4) > 0 and size(3 * 33, 4, **int8) == size(3 * 33, 4) > 0
    for T, Hq, B in ((3 * 9, 4, 3), (3 * 32, 4, 3), (64 * 16, 2, 64)):
        few = size(B, 2, B=B)
        assert size(T, Hq, B=B, **int8) == max(few, size(T, Hq, B=B)) >= few > 0
    assert size(300 * 20, 2, B=300, **int8) == size(300 * 20, 2, B=300)  # (more sequences than are divided)
    # tiles of 128 rows, and of 256 whose last round is divided
    assert size(1024, 60, B=1, H=60, **int8) > size(1024, 60, B=1, H=60) and size(1024, 60, B=1, H=60, D=64, **int8) == size(1024, 60, B=1, H=60, D=64)
    assert size(4680, 12, B=1, H=12, **int8) == size(4680, 12, B=1, H=12)


def test_binding_asks_for_the_workspace_of_the_type(lib):  # noqa: F811
    import paper_2605_14513_amd as heart

    q, table = bf(16 * 3, 16, 64), torch.zeros((3, 4), dtype=torch.int32)
    size = lambda t: heart.heart_cache_attn_workspace_bytes(q, torch.zeros((9, 8, 16, 64), dtype=t), table)  # noqa: E731
    want = lambda t: lib.heart_cache_attn_workspace_bytes(ctypes.byref(cache(B=3, H=8, D=64, type=t, k_exp=F, v_exp=F)), 48, 16)  # noqa: E731
    assert size(torch.int8) == want(INT8) and size(torch.bfloat16) == want(0)


def test_binding_refuses_what_does_not_belong_together(lib):  # noqa: F811
    import paper_2605_14513_amd as heart

    i = torch.zeros(1, dtype=torch.int32)
    c8, c16, x, s, e = torch.zeros((4, 2, 16, 64), dtype=torch.int8), bf(4, 2, 16, 64), bf(1, 2, 64), torch.zeros((4, 2)), bf(1, 2, 5, 64)
    exp = torch.zeros((4, 2, 16), dtype=torch.uint8)
    for c, kw, text in ((c16, dict(k_scale=s, v_scale=s), "only an int8"), (c16, dict(v_scale=s), "only an int8"),
                        (c8, dict(k_scale=s, v_scale=s, k_exp=exp), "no exponents"), (c8, dict(k_scale=s, v_exp=exp), "no exponents")):
        with pytest.raises(ValueError, match=text):
            heart.heart_cache_write(x, x, c, c, i[None], i, **kw)
        with pytest.raises(ValueError, match=text):
            heart.heart_cache_read(c, c, i[None], i, k=e, v=e, **kw)
        with pytest.raises(ValueError, match=text):
            heart.heart_cache_attn(x, c, c, i[None], i, workspace=None, **kw)
    with pytest.raises(TypeError, match="GPU"):
        heart.binding._native().cache_write(x, x, c8, c8, i[None], i, None, s, s, 0, 0)


# ---- the plan -----------------------------------------------------------------------------------

def plan_call(lib, B=3, M=4, page=16, n_pages=9, T=5, keep=None, add=F, kv=F, table=F, free=F, n_free=F, cu=F, slots=F, pos=F, ws=None,  # noqa: F811
              ws_bytes=0):
    return lib.heart_cache_plan(B, M, page, n_pages, T, keep, add, kv, table, free, n_free, cu, slots, pos, ws, ws_bytes, None)


@pytest.mark.parametrize("change,code,text", [
    (dict(B=0), EINVAL, "positive"), (dict(M=0), EINVAL, "positive"), (dict(n_pages=-1), EINVAL, "positive"),
    (dict(page=8), EUNSUPPORTED, "page"), (dict(page=24), EUNSUPPORTED, "page"), (dict(page=512), EUNSUPPORTED, "page"),
    (dict(page=0), EUNSUPPORTED, "page"), (dict(page=-16), EUNSUPPORTED, "page"),
    (dict(M=1 << 27), EUNSUPPORTED, "2^31"), (dict(T=-1), EINVAL, "negative"), (dict(T=(1 << 30) + 1), EUNSUPPORTED, "2^30"),
    (dict(B=(1 << 30) + 1), EUNSUPPORTED, "2^30"),
    (dict(add=None), EINVAL, "NULL"), (dict(kv=None), EINVAL, "NULL"), (dict(table=None), EINVAL, "NULL"), (dict(free=None), EINVAL, "NULL"),
    (dict(n_free=None), EINVAL, "NULL"), (dict(cu=None), EINVAL, "NULL"),
    (dict(B=5000), EINVAL, "workspace"), (dict(B=5000, ws=F, ws_bytes=5000 * 16), EINVAL, "workspace"),
    (dict(B=5000, ws=F + 8, ws_bytes=1 << 20), EUNSUPPORTED, "aligned"), (dict(T=1 << 20), EINVAL, "workspace")])
def test_plans_that_are_refused(lib, change, code, text):  # noqa: F811
    assert plan_call(lib, **change) == code
    msg = lib.heart_last_error().decode()
    assert text in msg and "heart_cache_plan" in msg, msg


def test_workspace_of_a_plan(lib):  # noqa: F811
    size = lib.heart_cache_plan_workspace_bytes
    assert size(0, 4, 4) == size(4, 0, 4) == size(4, 4, -1) == 0
    assert size(3, 40, 5) == 0 and size(5000, 4, 5) == 5001 * 16 and size(3, 4, 1 << 20) > 0


def test_binding_of_the_plan_refuses(lib):  # noqa: F811
    import paper_2605_14513_amd as heart
    from paper_2605_14513_amd import binding

    i, table = torch.zeros(3, dtype=torch.int32), torch.zeros((3, 4), dtype=torch.int32)
    with pytest.raises(ValueError, match="must be given"):
        heart.heart_cache_plan(i, i, table, i, i[:1], 16)
    with pytest.raises(ValueError, match="max_pages"):
        heart.heart_cache_plan(i, i, i, i, i[:1], 16, n=4)
    with pytest.raises(ValueError, match="n tokens"):
        heart.heart_cache_plan(i, i, table, i, i[:1], 16, n=4, slots=torch.zeros(5, dtype=torch.int64))
    with pytest.raises(ValueError, match="n tokens"):
        heart.heart_cache_plan(i, i, table, i, i[:1], 16, positions=i, slots=torch.zeros(5, dtype=torch.int64))
    with pytest.raises(ValueError, match=r"\[n\]"):
        heart.heart_cache_plan(i, i, table, i, i[:1], 16, positions=table)
    with pytest.raises(ValueError, match="workspace"):
        heart.heart_cache_plan(i, i, table, i, i[:1], 16, n=4, workspace="none")
    with pytest.raises(TypeError, match="GPU"):
        binding._native().cache_plan(i, i, table, i, i[:1], 16, None, i, i, i, None, 0, 0)
    with pytest.raises(TypeError, match="number of arguments"):
        binding._native().cache_plan(i)


# ---- the definitions ------------------------------------------------------------------------------

def test_scales():
    for top, scale in ((127.0, 1.0), (128.0, 1.25), (254.0, 2.0), (158.0, 1.25), (159.0, 1.5), (1.0, 2.0**-7 * 1.25), (0.0, 0.0)):
        assert block_scale(top) == scale, top
    assert math.isnan(block_scale(math.inf)) and block_scale(2.0**-133) == 2.0**-126
    every = torch.arange(1, 0x7F80, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).double()
    for top in every[::7].tolist():
        s = block_scale(top)
        m = math.frexp(s)[0] * 8
        below = s * 7 / 8 if m == 4 else s * (m - 1) / m
        assert 127 * s >= top and m == int(m) and (127 * below < top or s == 2.0**-126)


def test_a_quotient_by_a_scale_is_a_half_or_far_from_one():
    """So a division that is right to the last bit of fp32 rounds to the whole number that the exact quotient rounds to."""
    x = torch.arange(128, 256, dtype=torch.float64)  # significands of bf16
    for m in (4, 5, 6, 7):
        for e in range(0, 12):
            q = x / (m * 2.0**e)
            for half in (torch.floor(q) - 0.5, torch.floor(q) + 0.5, torch.floor(q) + 1.5):
                off = ((q - half).abs() / q)[half > 0]
                assert ((off == 0) | (off >= 2.0**-12)).all()


def test_definition_of_a_plan_by_hand():
    # page 16: request 0 keeps 20 of 40 tokens (a page goes back) and gets 30; 1 has ended; 2 begins anew; 3 only needs room it has; 4 finds
    # too few pages; 5 needs none
    table = [[7, 3, 5, -1], [2, -1, -1, -1], [-1, -1, -1, -1], [4, -1, -1, -1], [6, -1, -1, -1], [1, -1, -1, -1]]
    got = plan([30, 0, 17, 5, 40, 1], [40, 9, 0, 3, 16, 15], [20, 0, 0, 3, 16, 15], table, [0, 8, 9, -1, -1, -1, -1, -1, -1, -1], 3, 16, 60)
    assert got["kv_len"] == [50, 0, 17, 8, 16, 16] and got["cu_q"] == [0, 30, 30, 47, 52, 52, 53]
    # (back: 5 of request 0, then 2 of request 1; taken in that order, then 9)
    assert got["page_table"] == [[7, 3, 5, 2], [-1, -1, -1, -1], [9, 8, -1, -1], [4, -1, -1, -1], [6, -1, -1, -1], [1, -1, -1, -1]]
    assert got["free_pages"] == [0] and got["n_free"] == [1]
    assert got["slots"][0] == 3 * 16 + 4 and got["slots"][12] == 5 * 16 and got["slots"][46] == 8 * 16 and got["slots"][52] == 16 + 15
    assert got["positions"][52] == 15 and got["slots"][53:] == [-1] * 7


@pytest.mark.parametrize("kvs,qs", [([40], [7]), ([5, 33, 16], [5, 1, 3])])
def test_definition_of_writing(kvs, qs):
    """Values after a write are within half a step of what was written, and old ones within half a step more than they were."""
    c = Blocks(kvs, 2, 64, 16, device="cpu", seed=len(kvs))
    before = {n: [c.sequence(n, b).clone() for b in range(len(kvs))] for n in "kv"}
    g = torch.Generator().manual_seed(1)
    k, v = (4 * torch.randn((sum(qs), 2, 64), generator=g).bfloat16() for _ in range(2))
    c.write(qs, k, v)
    at = 0
    for b, n in enumerate(qs):
        for name, x in (("k", k), ("v", v)):
            now = c.sequence(name, b)
            for j in range(kvs[b]):
                s = c.scales[name][c.table_cpu[b, j // 16]].double()[:, None]
                want = x[at + j - (kvs[b] - n)].double() if j >= kvs[b] - n else before[name][b][:, j]
                assert ((now[:, j] - want).abs() <= s / 2).all()
        at += n


@pytest.mark.parametrize("source", ["cache_int8.hip", "cache_plan.hip"])
def test_kernels_use_no_scratch_memory(source):
    sizes = scratch_of(source)
    assert not any(sizes.values()), sizes

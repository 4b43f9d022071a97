"""What the calls on the paged cache refuse, without a GPU: in the library (the pointers are never followed) and in the binding."""
import ctypes

import pytest
import torch

from test_kernel_resources import scratch_of


@pytest.fixture(scope="module")
def lib():
    from paper_2605_14513_amd import binding
    from paper_2605_14513_amd import build as hb

    if hb.is_stale():
        hb.build(force=True)
    return binding.load_library()


F = 0x10000  # an address that nothing follows


def cache(**kw):
    from paper_2605_14513_amd import HeartCache

    c = HeartCache(n_pages=9, page=16, H=2, D=128, type=0, B=3, max_pages=4, k=F, v=F, page_table=F, kv_len=F)
    for i, s in enumerate((2 * 16 * 128, 16 * 128, 128)):
        c.k_stride[i] = c.v_stride[i] = s
    for name, x in kw.items():
        if name.endswith("stride"):
            for i, s in enumerate(x):
                getattr(c, name)[i] = s
        else:
            setattr(c, name, x)
    return c


def strides(*s):
    return (ctypes.c_longlong * len(s))(*s)


def calls(lib, c, T=3, q=F, out=2 * F, qs=(512, 128), cu=None, Hq=4, causal=1, window=0, ws=None, ws_bytes=0, N=5, rs=(1024, 512, 128)):
    r = None if c is None else ctypes.byref(c)
    s2, s3 = (strides(*qs) if qs else None), (strides(*rs) if rs else None)
    return {"write": lambda: lib.heart_cache_write(r, T, q, s2, q, s2, cu, None),
            "read": lambda: lib.heart_cache_read(r, N, q, s3, q, s3, None),
            "attn": lambda: lib.heart_cache_attn(r, T, Hq, q, s2, cu, causal, window, 0.0, q if q != F else out, s2, None, ws, ws_bytes, None)}


def test_struct_layout_matches_the_header(lib):
    from paper_2605_14513_amd import HeartCache

    # 7 ints (28 bytes, padded to 32) + 2 * 3 long long + 6 pointers
    assert ctypes.sizeof(HeartCache) == 32 + 48 + 48
    assert HeartCache.k_stride.offset == 32 and HeartCache.k.offset == 80 and HeartCache.kv_len.offset == 120


EINVAL, EUNSUPPORTED = -1, -2


@pytest.mark.parametrize("change,code,text", [
    (dict(n_pages=0), EINVAL, "positive"), (dict(H=0), EINVAL, "positive"), (dict(B=0), EINVAL, "positive"),
    (dict(max_pages=-1), EINVAL, "positive"), (dict(D=96), EUNSUPPORTED, "64 or 128"), (dict(D=256), EUNSUPPORTED, "64 or 128"),
    (dict(page=8), EUNSUPPORTED, "page"), (dict(page=48), EUNSUPPORTED, "page"), (dict(page=512), EUNSUPPORTED, "page"),
    (dict(type=2), EINVAL, "type"), (dict(k=None), EINVAL, "NULL"), (dict(v=None), EINVAL, "NULL"),
    (dict(page_table=None), EINVAL, "NULL"), (dict(kv_len=None), EINVAL, "NULL"), (dict(type=1), EINVAL, "NULL"),
    (dict(type=1, k_exp=F), EINVAL, "NULL"), (dict(k_exp=F), EINVAL, "exponents"), (dict(v_exp=F), EINVAL, "exponents"),
    (dict(k=F + 8), EUNSUPPORTED, "aligned"), (dict(type=1, k_exp=F, v_exp=F + 4), EUNSUPPORTED, "aligned"),
    (dict(k_stride=(4096, 2048, 132)), EUNSUPPORTED, "strides"), (dict(v_stride=(4100, 2048, 128)), EUNSUPPORTED, "strides"),
    (dict(v_stride=(4096, 2048, 0)), EUNSUPPORTED, "strides"), (dict(k_stride=(4096, 2048, -128)), EUNSUPPORTED, "strides"),
    (dict(type=1, k_exp=F, v_exp=F, k_stride=(4096, 2048, 136)), EUNSUPPORTED, "strides"),
    (dict(k_stride=(4096, 2048, 2**22 + 8)), EUNSUPPORTED, "2^22"), (dict(max_pages=2**27), EUNSUPPORTED, "2^31")])
def test_caches_that_every_call_refuses(lib, change, code, text):
    for name, call in calls(lib, cache(**change)).items():
        assert call() == code, name
        msg = lib.heart_last_error().decode()
        assert text in msg and f"heart_cache_{name}" in msg, msg


def test_no_cache(lib):
    for call in calls(lib, None).values():
        assert call() == EINVAL
    assert lib.heart_cache_attn_workspace_bytes(None, 1, 1) == 0


@pytest.mark.parametrize("which,change,code", [
    ("write attn", dict(T=-1), EINVAL), ("write attn", dict(T=4), EINVAL), ("read", dict(N=-1), EINVAL),
    ("write read attn", dict(q=None), EINVAL), ("write read attn", dict(q=F + 8), EUNSUPPORTED),
    ("write attn", dict(qs=(512, 100)), EUNSUPPORTED), ("write attn", dict(qs=(516, 128)), EUNSUPPORTED),
    ("write attn", dict(qs=None), EINVAL), ("read", dict(rs=None), EINVAL), ("read", dict(rs=(1024, 512, 4)), EUNSUPPORTED),
    ("attn", dict(Hq=0), EINVAL), ("attn", dict(Hq=3), EINVAL), ("attn", dict(Hq=-2), EINVAL), ("attn", dict(causal=-1), EINVAL),
    ("attn", dict(window=-1), EINVAL), ("attn", dict(out=F), EINVAL), ("attn", dict(T=3 * 2**28, Hq=4), EUNSUPPORTED), ("write", dict(T=3 * 2**29), EUNSUPPORTED),
    ("attn", dict(ws=F + 8, ws_bytes=1 << 40), EUNSUPPORTED), ("attn", dict(ws=F, ws_bytes=100), EINVAL)])
def test_arguments_that_a_call_refuses(lib, which, change, code):
    for name in which.split():
        assert calls(lib, cache(), **change)[name]() == code, name
        assert f"heart_cache_{name}" in lib.heart_last_error().decode()


def test_no_tokens_launch_nothing(lib):
    for name, call in calls(lib, cache(), T=0, q=None, N=0).items():
        assert call() == 0, name


def test_workspace_sizes(lib):
    size = lambda T, Hq, **kw: lib.heart_cache_attn_workspace_bytes(ctypes.byref(cache(**kw)), T, Hq)  # noqa: E731
    # room for parts of the keys, of few rows a key head and of more; a function of B, H, D, T, Hq alone
    assert size(3, 4) > 0 and size(300, 4) > 0 and size(3, 4, D=64) < size(3, 4) and size(300, 4, D=64) < size(300, 4)
    assert size(3, 4) == size(3, 4, n_pages=1, page=64, max_pages=1000, type=1, k_exp=F, v_exp=F)
    assert size(300000, 4) == 0      # (enough queries without division)
    assert size(0, 4) == size(3, 3) == size(3, 0) == size(3, 4, D=96) == size(3, 4, B=0) == 0


def bf(*s):
    return torch.zeros(s, dtype=torch.bfloat16)


def test_binding_refuses_cpu_tensors(lib):
    import paper_2605_14513_amd as heart
    from paper_2605_14513_amd import binding

    native, i = binding._native(), torch.zeros(1, dtype=torch.int32)
    c, x = bf(4, 2, 16, 64), bf(1, 2, 64)
    with pytest.raises(TypeError, match="GPU"):
        native.cache_write(x, x, c, c, i[None], i, None, None, None, 0, 0)
    with pytest.raises(TypeError, match="GPU"):
        native.cache_read(c, c, i[None], i, None, None, x[None], x[None], 0, 0)
    with pytest.raises(TypeError, match="GPU"):
        native.cache_attn(x, c, c, i[None], i, None, None, None, 1, 0, 0.0, x, None, None, 0, 0)
    with pytest.raises(TypeError, match="number of arguments"):
        native.cache_attn(x)
    with pytest.raises(ValueError, match="workspace"):
        heart.heart_cache_attn(x, c, c, i[None], i, workspace="none")
    with pytest.raises(ValueError, match="n tokens"):
        heart.heart_cache_read(c, c, i[None], i, k=bf(1, 2, 5, 64), v=bf(1, 2, 5, 64), n=3)


def test_a_launch_has_less_than_2_to_the_32_threads(lib):
    # (a wavefront has 16 tokens of a head in writing; a workgroup 64 tokens in reading, 16 rows or more in attention)
    c = cache(B=1, H=1, max_pages=1 << 26)
    for name, call in calls(lib, c, T=1 << 30, Hq=1, N=1 << 30).items():
        if name != "attn":  # (2^23 tiles of 128 rows)
            assert call() == EUNSUPPORTED and b"too many rows" in lib.heart_last_error(), name
    assert calls(lib, cache(B=1 << 24, H=1), T=1 << 24, Hq=1)["attn"]() == EUNSUPPORTED
    assert b"grid too large" in lib.heart_last_error()


@pytest.mark.parametrize("source", ["cache.hip", "cache_attn.hip", "cache_attn_few.hip"])
def test_cache_kernels_use_no_scratch_memory(source):
    sizes = scratch_of(source)
    assert not any(sizes.values()), sizes

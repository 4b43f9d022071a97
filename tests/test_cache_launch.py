"""Of the cache's calls, without a GPU: what the library's symbols show of launches, shapes that the binding looks at."""
import re
import subprocess

import pytest
import torch

from test_cache_calls import lib  # noqa: F401  (builds the library if it is stale)


def test_every_attention_kernel_has_a_flag_of_its_own(lib):  # noqa: F811
    """The largest dynamic LDS is an attribute of a function: one flag "it is set" for several kernels leaves all but the first
    that is launched without it."""
    from paper_2605_14513_amd import build as hb

    names = subprocess.run(["nm", "-C", hb.LIB], stdout=subprocess.PIPE, check=True, text=True).stdout.splitlines()
    for kernel, launcher in (("cache_attn_kernel", "launch_t"), ("cache_attn_few_kernel", "launch_few_t")):
        kernels = [n for n in names if re.search(rf"__device_stub__{kernel}<", n)]
        flags = [n for n in names if re.search(rf"heart::{launcher}<.*::attr_set$", n)]
        assert len(kernels) >= 12 and len(flags) == len(kernels), (kernel, len(kernels), len(flags))


def test_shapes_are_looked_at_before_sizes_are_taken_of_them(lib):  # noqa: F811
    """Tensors of the wrong number of axes are refused as such, also where the binding makes the workspace or the outputs."""
    import paper_2605_14513_amd as heart

    i = torch.zeros(1, dtype=torch.int32)
    c, q = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((1, 2, 64), dtype=torch.bfloat16)
    for bad in ((q[0], c, i[None]), (q[0, 0], c, i[None]), (q, c[0], i[None]), (q, c, i)):
        with pytest.raises(ValueError, match="must be"):
            heart.heart_cache_attn_workspace_bytes(*bad)
        with pytest.raises(ValueError, match="must be"):
            heart.heart_cache_attn(bad[0], bad[1], bad[1], bad[2], i)
    for table, cache, k in ((i, c, None), (i[None], c[0], None), (i[None], c, q)):
        with pytest.raises(ValueError, match="must"):
            heart.heart_cache_read(cache, cache, table, i, k=k)

"""What the library's symbols show of the cache's launches, without a GPU."""
import re
import subprocess

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

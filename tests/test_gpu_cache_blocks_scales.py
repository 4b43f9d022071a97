"""heart_cache_attn over int8 caches whose scales another program wrote: any positive ones, of 24 significant bits."""
import pytest
import torch

from cache_blocks_reference import Blocks, tolerance
from cache_testlib import assert_near
from test_gpu_cache_blocks_attn import check, new_q

import paper_2605_14513_amd as heart

pytestmark = pytest.mark.gpu

# Tiles of 128 and 256 rows: a scale of v is rounded to f16 (2^-11), its product with a code again, and weights too, as everywhere:
# (1 + 2^-11)^3 - 1 < 3 (1 + 2^-9) 2^-11.
THREE = 3 * (1 + 2.0**-9) * 2.0**-11


def set_scales(c, how, seed=1):
    """Scales of 24 bits: random ones, or a largest magnitude over 127."""
    g = torch.Generator().manual_seed(seed)
    for w in ("k", "v"):
        shape = c.scales[w].shape
        if how == "random":
            s = (1 + torch.rand(shape, generator=g)) * 2.0**-6
        else:
            s = (3.9 + 2 * torch.rand(shape, generator=g)).bfloat16().float() / 127.0
        c.scales[w] = s
        c.scale[w].copy_(s)
    return c


@pytest.mark.parametrize("workspace", ["auto", None])
@pytest.mark.parametrize("how", ["random", "over 127"])
@pytest.mark.parametrize("D,page", [(64, 256), (128, 256), (128, 16), (64, 32)])
def test_scales_of_any_number_of_bits(D, page, how, workspace):
    """Rows that see few pages, so that what shifts all elements of a page alike is not lost among others; single tokens, tiles of 16
    rows, of 128."""
    for n, room in ((1, 0), (20, 0), (100, 5200), (300, 5200)):
        c = set_scales(Blocks([900, 700], 2, D, page, seed=n, room=room), how)
        for causal, window in ((1, 90), (1, 0)):
            check(c, new_q(2 * n, 4, D), [n, n], causal, window, workspace=workspace, weight=THREE, what=how)


@pytest.mark.parametrize("window", [90, 0])
@pytest.mark.parametrize("page", [16, 256])
def test_scales_of_any_number_of_bits_in_tiles_of_256_rows(page, window):
    H, n = 44, 1024
    c = set_scales(Blocks([1300], H, 128, page, seed=page, room=5200), "over 127")
    q = new_q(n, H, 128)
    print(f"cache_attn int8 wide, scales of 24 bits page={page} window={window}", flush=True)
    out = heart.heart_cache_attn(q.cuda(), *c.args(), window=window, workspace=None, **c.scale_args())
    torch.cuda.synchronize()
    one = Blocks([1300], 1, 128, page, seed=page, room=5200, device="cpu")
    one.table_cpu = c.table_cpu
    for h in (0, 17, H - 1):
        for w in ("k", "v"):
            one.codes[w], one.scales[w] = c.codes[w][:, h:h + 1], c.scales[w][:, h:h + 1]
        want, _, tol, _ = tolerance(one, q[:, h:h + 1], [n], 1, window, weight=THREE)
        assert_near(out[:, h:h + 1], want, tol, "out")


@pytest.mark.parametrize("bits", [0x7FC00000, -0x400000, 0x7F800001, -1])  # (quiet and signalling, of either sign)
@pytest.mark.parametrize("n,room", [(1, 0), (20, 0), (150, 5200)])
def test_a_scale_that_is_any_nan(n, room, bits):
    """Queries that see the page get NaN, whatever NaN it is: 0 / 0 has its sign bit set on some machines."""
    for D in (64, 128):
        for w in ("k", "v"):
            c = Blocks([600, 300], 2, D, 32, seed=n, room=room)
            page = c.table_cpu[0, 3].item()  # (positions 96 to 127: all queries see it)
            c.scale[w].view(torch.int32)[page, 1] = bits
            print(f"cache_attn int8 NaN {bits:x} of {w} n={n} D={D} room={room}", flush=True)
            lse = torch.zeros((4, 2 * n), device="cuda")
            out = heart.heart_cache_attn(new_q(2 * n, 4, D).cuda(), *c.args(), lse=lse, **c.scale_args())
            assert out[:n, 2:].isnan().all() and (w == "v" or lse[2:, :n].isnan().all())
            assert not out[n:].isnan().any() and not out[:, :2].isnan().any() and not lse[:, n:].isnan().any()


def test_a_scale_that_is_any_nan_in_tiles_of_256_rows():
    H, n = 44, 1024
    for bits in (0x7FC00000, -0x400000):
        for w in ("k", "v"):
            c = Blocks([1300], H, 128, 64, seed=1, room=5200)
            c.scale[w].view(torch.int32)[c.table_cpu[0, 3].item(), 5] = bits
            print(f"cache_attn int8 wide NaN {bits:x} of {w}", flush=True)
            out = heart.heart_cache_attn(new_q(n, H, 128).cuda(), *c.args(), workspace=None, **c.scale_args())
            assert out[:, 5].isnan().all() and not out[:, :5].isnan().any() and not out[:, 6:].isnan().any()

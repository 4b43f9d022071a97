"""How large the errors of an int8 cache are beside those of e4m3, by the definitions of both: what the documents say of it."""
import pytest
import torch

from cache_blocks_reference import Blocks
from cache_testlib import e4m3_values

N, H, D = 256, 16, 128


def rows(kind, seed):
    """Normal rows; channels (of a head) or rows of different sizes."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((N, H, D), generator=g)
    if kind == "channels":
        x = x * torch.exp(0.4 * torch.randn((H, D), generator=g))
    elif kind != "equal":
        x = x * torch.exp((0.25 if kind == "rows" else 1.0) * torch.randn((N, H, 1), generator=g))
    return x.bfloat16()


def written(x, page, chunk):
    """fp64 [N,H,D]: rows as the cache holds them after `chunk` at a time were written."""
    c = Blocks([N], H, D, page, device="cpu", seed=1)
    for i in range(0, N, chunk):
        c.lens[0] = i + chunk
        c.write([chunk], x[i:i + chunk], x[i:i + chunk])
    return c.sequence("k", 0).transpose(0, 1)


# Error in the 2-norm over that of e4m3: pages of 16, 64, 256 tokens, written at once and token by token.
STATED = {"equal": ((0.34, 0.38), (0.38, 0.42), (0.42, 0.47)), "channels": ((0.54, 0.62), (0.65, 0.73), (0.73, 0.82)),
          "rows": ((0.42, 0.47), (0.49, 0.57), (0.56, 0.63)), "very different rows": ((0.80, 0.85), (1.3, 1.4), (1.8, 2.1))}


@pytest.mark.parametrize("i,page", enumerate((16, 64, 256)))
@pytest.mark.parametrize("kind", sorted(STATED))
def test_error_beside_that_of_e4m3(kind, i, page):
    """Means over 16 blocks of 256 rows, 256 of 16: what varies is their scales, by a fifth (by half where rows differ by e), so the ratio
    by four times a quarter of that at most."""
    x = rows(kind, 100 + page)
    of = (e4m3_values(x)[0] - x.double()).norm().item()
    for stated, chunk in zip(STATED[kind][i], (N, 1)):
        ratio = (written(x, page, chunk) - x.double()).norm().item() / of
        assert abs(ratio / stated - 1) <= (0.5 if kind == "very different rows" else 0.2), (ratio, stated)

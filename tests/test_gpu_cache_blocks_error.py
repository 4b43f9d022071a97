"""What an int8 cache loses while its pages fill token by token: of the values, not by the recurrence of codes."""
import pytest
import torch

import paper_2605_14513_amd as heart
from cache_blocks_reference import Blocks

pytestmark = pytest.mark.gpu

# Scales of a block that grows are m 2^e with m = 4 .. 7.  Those that one can have had before it, all of them, add up to most of it where
# its m is 4: 7/2 + 6/2 + 5/2 + 4/2 = 11 in the octave below, half of that in the next, 22 in all beside its 4.  Half of each is an error.
MOST = (1 + 22 / 4) / 2


@pytest.mark.parametrize("gain", [0.0, 0.004, 0.03, -0.02])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 64), (128, 256), (64, 256)])
def test_errors_while_a_page_fills(D, page, gain):
    """A value is off by half of each scale that its page has had since it was written, at most, and by 3.25 times the last one, however often
    it was rounded again; tokens of one size, rising and falling ones."""
    H, n = 3, 2 * page
    c = Blocks([0], H, D, page, seed=page, room=n, spare=2)
    c.table_cpu[0, :2] = torch.tensor([1, 0], dtype=torch.int32)
    c.page_table.copy_(c.table_cpu)
    g = torch.Generator().manual_seed(D)
    x = torch.randn((n, H, D), generator=g) * torch.exp(gain * torch.arange(n))[:, None, None]
    k = x.bfloat16()
    v = (x.flip(2) * torch.exp(0.25 * torch.randn((n, H, 1), generator=g))).bfloat16()
    print(f"cache_write int8 token by token D={D} page={page} gain={gain}", flush=True)
    off = {w: torch.zeros((n, H, 1), dtype=torch.float64) for w in "kv"}  # the bound
    before = {w: torch.zeros((2, H), dtype=torch.float64) for w in "kv"}
    ck, cv = k.cuda(), v.cuda()
    for i in range(n):
        c.kv_len.fill_(i + 1)
        heart.heart_cache_write(ck[i:i + 1], cv[i:i + 1], *c.args(), **c.scale_args())
        for w in "kv":
            now = c.scale[w].cpu().double()[[1, 0]]  # [page of the sequence, H]
            p = i // page
            grew = (now[p] > before[w][p])[None, :, None]
            off[w][p * page:i] += torch.where(grew, now[p][None, :, None] / 2, 0.0)
            off[w][i] = now[p][:, None] / 2
            before[w][p] = now[p]
    got = heart.heart_cache_read(*c.args(), n=n, **c.scale_args())
    for w, x, y in (("k", k, got[0]), ("v", v, got[1])):
        last = before[w].repeat_interleave(page, 0)[:, :, None]
        assert (off[w] <= MOST * last).all()
        y = y[0].transpose(0, 1).double().cpu()
        # (a value that is read is rounded to bf16: half a step of 2^-8)
        assert ((y - x.double()).abs() <= off[w] + 2.0**-8 * (x.double().abs() + off[w])).all(), w
        if gain == 0.03:
            assert (off[w] > 1.4 * last).any()  # (some were rounded again, several times)

"""Drafts that are taken back from an int8 cache through the plan: what stays of them in the pages of the tokens that stay, and how
those are had back."""
import math

import pytest
import torch

import paper_2605_14513_amd as heart

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,page", [(64, 16), (128, 32), (128, 256)])
def test_drafts_that_are_taken_back_leave_their_scale(D, page):
    H, B, M, old = 3, 2, 4, page + page // 2
    n_pages = B * M + 3
    i32 = dict(dtype=torch.int32, device="cuda")
    kv, table = torch.zeros(B, **i32), torch.full((B, M), -1, **i32)
    free, n_free = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).int().cuda(), torch.tensor([n_pages], **i32)
    kc, vc = (torch.full((n_pages, H, page, D), 99, dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((n_pages, H), math.nan, device="cuda") for _ in range(2))
    cache, scales = (kc, vc, table, kv), dict(k_scale=ks, v_scale=vs)
    g = torch.Generator().manual_seed(D)

    def step(add, keep, gain=1.0, x=None):
        print(f"plan and write of an int8 cache add={add} keep={keep} D={D} page={page}", flush=True)
        cu, _, _ = heart.heart_cache_plan(torch.tensor(add, **i32), kv, table, free, n_free, page, n=sum(add), keep=torch.tensor(keep, **i32))
        assert cu.tolist() == [0, add[0], add[0] + add[1]]
        if x is None:
            x = (gain * torch.randn((sum(add), H, D), generator=g)).bfloat16()
        heart.heart_cache_write(x.cuda(), (-x).cuda(), *cache, cu_q=cu, **scales)
        return x.double()

    def scale_of(s, b, p):
        return s[table[b, p].long()].double().cpu()

    def read(b):
        k, v = heart.heart_cache_read(*cache, n=int(kv[b]), **scales)
        return k[b].transpose(0, 1).double().cpu(), v[b].transpose(0, 1).double().cpu()

    def near(got, want, scale):  # (half of each scale that the rows have had, and bf16 that is read)
        return ((got - want).abs() <= scale / 2 + 2.0**-8 * (want.abs() + scale)).all()

    x = step([old, 5], [0, 0])
    first = [scale_of(ks, 0, p) for p in range(2)]
    assert near(read(0)[0][page:old], x[page:old], first[1][:, None])

    # eight drafts, eight times as large; of head 1 the fifth is not finite
    y = (8 * torch.randn((9, H, D), generator=g)).bfloat16()
    y[4, 1, 7] = math.nan
    y = step([8, 1], [old, 5], x=y)
    second = scale_of(ks, 0, 1)
    assert second[1].isnan() and (second[[0, 2]] >= 4 * first[1][[0, 2]]).all()

    # three are accepted, and a token comes behind them: the page has the scale of all eight still, and is lost to head 1
    z = step([1, 1], [old + 3, 6])
    assert torch.equal(scale_of(ks, 0, 1)[[0, 2]], second[[0, 2]]) and scale_of(ks, 0, 1)[1].isnan() and scale_of(vs, 0, 1)[1].isnan()
    want = torch.cat([x[:old], y[:3], z[:1]])
    for got, sign in zip(read(0), (1, -1)):
        assert got.shape[0] == old + 4
        both = [0, 2]
        assert near(got[:page], sign * want[:page], first[0][:, None])                                # (another page: as it was)
        assert near(got[page:old][:, both], sign * want[page:old][:, both], (first[1] + second)[both][:, None])
        assert near(got[old:][:, both], sign * want[old:][:, both], second[both][:, None])
        assert got[page:, 1].isnan().all()
    assert read(1)[0].isfinite().all()

    # to have them back: take back what the page has, and write its tokens anew
    step([old - page + 4, 1], [page, 7], x=torch.cat([want[page:], z[1:]]).bfloat16())
    third = scale_of(ks, 0, 1)
    assert third.isfinite().all()
    for got, sign in zip(read(0), (1, -1)):
        assert near(got[:page], sign * want[:page], first[0][:, None]) and near(got[page:], sign * want[page:], third[:, None])

"""Which scales of v a part of heart_cache_attn over an int8 cache looks at before it takes a unit for v's values in f16, in Python: all
of its pages; and that the GPU tests' caches have their largest scales where a wrong look would miss them."""
import pytest
import torch

import cache_rules as rules
from test_gpu_cache_blocks_units import LOOKED_AT, hot_pages


def looked_at(key0, end, page, rows, first=63, last=0):
    """Pages whose scales count in the part of keys key0 .. end - 1: those of its first 64 stages, which wavefronts of `rows` rows each
    have loaded (v's stages begin 32 keys before k's), and of longer parts all from stage `first` on."""
    n_stage = -(-(end - key0) // rules.STAGE)
    pages = set()
    for wave in range(rules.STAGE // rows):
        for lane in range(min(64, n_stage + 1)):
            key = key0 + lane * rules.STAGE - 32 + rows * wave
            if 0 <= key < end:
                pages.add(key // page)
    if n_stage > 63 and first is not None:
        pages |= set(range((key0 + first * rules.STAGE) // page, (end - 1) // page + 1 - last))
    return pages


@pytest.mark.parametrize("rows", [8, 16])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_every_page_of_a_part_is_looked_at(page, rows):
    for key0 in (0, 64, 1984, 4736):
        for n in [1, 15, 16, 31, 32, 33, 100] + list(range(LOOKED_AT - 70, LOOKED_AT + 140, 7)) + [6000, 9137, 10000]:
            assert looked_at(key0, key0 + n, page, rows) >= set(range(key0 // page, -(-(key0 + n) // page))), (key0, n)


@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("wrong", [dict(first=None), dict(last=1), dict(first=68), dict(first=69)])
def test_the_largest_scales_lie_where_a_wrong_look_misses_them(wrong, page):
    """No look, one that ends a page or begins some stages too late: one of the heads has its largest scale there alone."""
    missed = 0
    for kv, key0 in ((6000, 0), (9137, 0), (9300, 4160), (10000, 3840)):
        seen = looked_at(key0, kv, page, 16, **wrong)
        missed += any(h and not set(h) & seen for h in hot_pages(kv, page, key0))
    assert missed


@pytest.mark.parametrize("by", [10, 11, 12])
def test_f16_has_no_room_for_them_under_another_unit(by):
    """The largest of the first stages' scales is 2^4 units at least: one 2^by times any of them (which differ by 7/4 2^2) and more."""
    u = torch.tensor(2.0**(4 + by) * 4 / 7 / 4)
    assert (u.half() * torch.tensor(40, dtype=torch.float16)).isinf()

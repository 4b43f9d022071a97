"""The rules by which heart_cache_attn divides keys, on the CPU: no record is read that the call has not written, whatever token
ranges it is given; shares have every stage once."""
import random

import pytest

from cache_rules import FEW_PLACES, mode, records, shares_of


def ranges(rng, B, T):
    """Token ranges: rising ones, falling ones, some that leave [0, T]."""
    how = rng.choice(["rise", "any", "teeth", "out"])
    if how == "teeth":
        return [T * (i % 2) for i in range(B + 1)]
    cu = [rng.randint(0, T) for _ in range(B + 1)]
    if how == "rise":
        return sorted(cu)
    if how == "out":
        cu[rng.randrange(B + 1)] = rng.choice([-5, T + 1, 2**31 - 1, -2**31])
        if rng.random() < 0.5:
            cu = sorted(cu)
    return cu


@pytest.mark.parametrize("cu,T,H,G", [([0, 800, 0, 800, 0], 800, 8, 8), ([0, 5000] * 20 + [0], 5000, 1, 1)])
def test_records_of_ranges_that_fall(cu, T, H, G):
    """More tiles than places: without a look at the ranges the second launch reads records that nobody wrote."""
    kv = [4000] * (len(cu) - 1)
    written, read = records(cu, kv, T, H, G, 4096, looks=False)
    assert read - written
    written, read = records(cu, kv, T, H, G, 4096)
    assert not read - written


def test_records_of_any_ranges():
    rng = random.Random(5)
    seen = 0
    for _ in range(600):
        B, H, G = rng.randint(2, 40), rng.choice([1, 2, 3, 8]), rng.choice([1, 4, 8])
        T = rng.randint(1, 4000)
        cap = rng.choice([2000, 6144, 40000])
        if mode(B, H, T, H * G, cap)[0] != "parts":
            continue
        seen += 1
        cu = ranges(rng, B, T)
        written, read = records(cu, [rng.randint(0, cap + 50) for _ in range(B)], T, H, G, cap, rng.choice([0, 1, 100]), rng.choice([0, 500]))
        assert not read - written, cu
    assert seen > 100


def test_parts_of_few_rows_are_whole_tiles():
    """Every stage of every tile is in one part, parts of one tile in neighbouring shares, no two of them in one place."""
    rng = random.Random(6)
    modes = []
    for i in range(120):
        B, H, G = rng.randint(1, 70), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 5])
        top = rng.choice([300, 4000, 60000])
        kvs = [rng.choice([0, 1, rng.randint(1, top), rng.randint(1, top), top]) for _ in range(B)]
        qs = [rng.choice([0, 1, 1, 1, 2]) for _ in range(B)]
        if sum(qs) == 0:
            continue
        s = shares_of(qs, kvs, H, G, top + 100, rng.choice([0, 1, 64]), rng.choice([0, 0, 700]), rng.choice([64, 128]), rng.choice(["bf16", "e4m3"]))
        modes.append(s.mode)
        assert len(s.tiles) == H * sum(-(-n * G // 16) for n in qs)
        for _, _, stages, parts in s.tiles:
            assert [a for _, a, _ in parts] == [0] + [e for _, _, e in parts[:-1]] and parts[-1][2] == stages
            assert [x for x, _, _ in parts] == list(range(parts[0][0], parts[0][0] + len(parts)))
            assert 0 <= parts[0][0] and parts[-1][0] < FEW_PLACES
        slots = s.slots()
        assert len(slots) == len(set(slots)) and all(0 <= x < 2 * FEW_PLACES for x in slots)
    assert modes.count("parts") > 20 and modes.count("shares") > 20, modes

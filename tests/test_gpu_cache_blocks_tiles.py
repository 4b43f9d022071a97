"""That calls of heart_cache_attn over int8 caches have tiles of 256 rows where they are meant to, by what they leave in the workspace."""
import pytest
import torch

import cache_rules as rules
import paper_2605_14513_amd as heart
from cache_blocks_reference import Blocks
from cache_reference import FILL
from test_gpu_cache_blocks_attn import new_q
from test_gpu_cache_blocks_units import WIDE, attend, near_definition, wide
from test_gpu_cache_division import parts_written, records_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,n,kvs", [(2, 24, 1100, [1500, 1111]), (3, 16, 1100, [1100, 5000, 2000]), (2, 20, 1300, [1300, 4001])])
def test_tiles_of_256_rows_that_are_not_divided(B, H, n, kvs):
    """These leave the workspace as it was; tiles of 128 rows, which the same call has under a table without that room, are divided and
    leave records.  The results have the same bits without a workspace, and are those of the definition."""
    c = Blocks(kvs, H, 128, 32, seed=n, room=5200, spread=4)
    q = new_q(B * n, H, 128)
    assert wide(B, H, 128, B * n, H, c.table_cpu.shape[1] * 32)[0] == "whole"
    ws = torch.full((heart.heart_cache_attn_workspace_bytes(q, c.stored["k"], c.page_table),), FILL, dtype=torch.uint8, device="cuda")
    out, lse = attend(c, q, n, B=B, workspace=ws, what="wide, whole")
    assert ws.numel() and (ws == FILL).all()
    near_definition(c, q, [n] * B, out, lse, (0, H - 1))
    out2, lse2 = attend(c, q, n, B=B, workspace=None, what="wide, whole")
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    c.page_table = c.page_table[:, :160].contiguous()  # (room for 5120)
    assert wide(B, H, 128, B * n, H, 5120) is None and rules.mode(B, H, B * n, H, 5120)[0] == "parts"
    out2, lse2 = attend(c, q, n, B=B, workspace=ws, what="128 rows, parts")
    assert records_of(ws)
    near_definition(c, q, [n] * B, out2, lse2, (0, H - 1))
    out2, lse2 = attend(c, q, n, B=B, workspace=None, what="128 rows, whole")
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("H,n,kv,causal,window", [(60, 1100, 4200, 1, 0), (55, 1281, 2600, 0, 0), (72, 1060, 3000, 300, 2500)])
def test_tiles_of_256_rows_of_a_divided_round(H, n, kv, causal, window):
    """Records and parts in the workspace are those of the last round of tiles of 256 rows, eight wavefronts a part."""
    c = Blocks([kv], H, 128, 64, seed=n, room=5200, spread=5)
    q = new_q(n, H, 128)
    mode, whole, parts, tiles = wide(1, H, 128, n, H, c.table_cpu.shape[1] * 64)
    assert mode == "tail" and rules.mode(1, H, n, H, 5200)[2:] != (whole, parts)
    floats = 64 * 64 + 128
    need = rules.PLACES * 16 + (tiles - whole) * parts * (WIDE // 32) * floats * 4
    size = heart.heart_cache_attn_workspace_bytes(q, c.stored["k"], c.page_table)
    assert size >= need
    ws = torch.full((size,), FILL, dtype=torch.uint8, device="cuda")
    out, lse = attend(c, q, n, window=window, causal=causal, workspace=ws, what="wide, divided")
    records = records_of(ws)
    assert records and max(records) < tiles - whole and all(r[0] == i and r[2] == tiles - whole and 1 <= r[1] <= parts for i, r in records.items())
    divided = {i + p * r[2] for i, r in records.items() if r[1] > 1 for p in range(r[1])}
    assert divided
    # (a part of eight wavefronts is two of four)
    four = parts_written(ws[:rules.PLACES * 16 + (size - rules.PLACES * 16) // (16 * floats) * 16 * floats], 128)
    assert {i // 2 for i in four} == divided
    near_definition(c, q, [n], out, lse, (0, H // 2, H - 1), causal=causal, window=window)


def test_tiles_of_128_rows_where_256_would_not_fill_the_chip():
    """30 heads of 1024 rows (150 tiles of 256), sequences of less than four tiles each, D = 64: parts or tiles of 128 rows, as of e4m3."""
    for B, H, D, n, kv in ((1, 30, 128, 1024, 2000), (2, 20, 128, 900, 2000), (1, 48, 64, 1024, 1500)):
        c = Blocks([kv] * B, H, D, 64, seed=n, room=5200)
        q = new_q(B * n, H, D)
        room = c.table_cpu.shape[1] * 64
        assert wide(B, H, D, B * n, H, room) is None
        ws = torch.full((heart.heart_cache_attn_workspace_bytes(q, c.stored["k"], c.page_table),), FILL, dtype=torch.uint8, device="cuda")
        out, lse = attend(c, q, n, B=B, workspace=ws, what="128 rows")
        assert bool(ws.numel() and records_of(ws)) == (rules.mode(B, H, B * n, H, room)[0] != "whole")
        near_definition(c, q, [n] * B, out, lse, (0, H - 1))

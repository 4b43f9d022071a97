"""How heart_cache_attn divides the keys of a call, in Python: the host's choice of a kernel and a mode, the parts of tiles of 128 rows and
the records of them that the second launch reads, the shares of tiles of 16 rows.  The tests on the GPU compare these with
what a call leaves in its workspace, so that a changed rule cannot leave a mode untested."""
import math
from dataclasses import dataclass

TILE, STAGE, PLACES, MIN_STAGES, PART_COST, BRIEF, TAIL_ROUNDS = 128, 64, 512, 4, 8, 80 * 64, 8
FEW_TILE, FEW_STAGE, FEW_PLACES, FEW_MIN, FEW_CUT, FEW_ITEMS, SPLIT_SEQS = 16, 128, 512, 2, 1, 8192, 256


def few(B, H, T, Hq):
    return T * (Hq // H) <= FEW_TILE * B


def most_items(tile, B, H, T, Hq):
    return (T * (Hq // H) // tile + B) * H


def divide(B, n_items):
    """(mode, rounds, tiles that are not divided, parts of the others)."""
    if n_items < PLACES and B <= SPLIT_SEQS and (B > 1 or 3 * n_items <= 2 * PLACES):
        return "parts", 2 if 3 * n_items > PLACES else 1, 0, 1
    r = n_items % PLACES
    if n_items < PLACES or n_items > TAIL_ROUNDS * PLACES or r == 0:
        return "whole", 1, 0, 1
    best, least, p = 1, 1e9, 1
    while p <= 8 and r * p <= 2 * PLACES:
        cost = -(-r * p // PLACES) / p + (0.03 * p * r / PLACES + 0.02 if p > 1 else 0.0)
        if cost < least:
            least, best = cost, p
        p += 1
    return ("whole", 1, 0, 1) if best == 1 else ("tail", 1, n_items - r, best)


def mode(B, H, T, Hq, cap):
    """What a call with a workspace does (128-row tiles)."""
    items = most_items(TILE, B, H, T, Hq)
    m, rounds, whole, tail = divide(B, items)
    if cap <= BRIEF:
        if m == "tail" or (B == 1 and 2 * items > PLACES):
            m, rounds, whole, tail = "whole", 1, 0, 1
        rounds = 1
    return m, rounds, whole, tail


@dataclass
class Seq:
    first: int
    n: int
    len: int
    pos0: int


def sequences(cu, kv, T, cap):
    out = []
    for b in range(len(kv)):
        first, end = cu[b], cu[b + 1]
        n = end - first if first >= 0 and end > first and end <= T else 0
        k = max(kv[b], 0)
        out.append(Seq(first, n, min(k, cap), k - n))
    return out


def tiles_of(tile, G, s):
    return -(-s.n * G // tile)


def stages_of(tile, stage, G, causal, window, s):
    st = -(-s.len // stage)
    if window:
        st = min(st, (window + tile // G + max(causal, 1)) // stage + 2)
    return max(st, 1)


def tile_start(tile, G, cu, b):
    return max(cu[b], 0) * G % 2**32 // tile + b


def find_parts(seqs, H, G, causal, window, rounds):
    """Tiles of 128 rows whose keys are divided: (parts of a tile of each sequence, parts in all, places)."""
    wgs = [tiles_of(TILE, G, s) * H for s in seqs]
    st = [stages_of(TILE, STAGE, G, causal, window, s) for s in seqs]
    most = max([x for x, w in zip(st, wgs) if w], default=1)
    tiles, total = sum(wgs), sum(w * x for w, x in zip(wgs, st))
    parts = lambda L: [1 + (x - 1) // L for x in st]  # noqa: E731
    count = lambda L: sum(w * p for w, p in zip(wgs, parts(L)))  # noqa: E731

    def least(places):
        lo = min(max(total // places, MIN_STAGES), most)
        room = places - tiles
        hi = max(min(total // room + 2, most) if room > 0 else most, lo)
        while lo < hi:
            mid = (lo + hi) // 2
            lo, hi = (lo, mid) if count(mid) <= places else (mid + 1, hi)
        return lo

    L, room = least(PLACES), PLACES
    if rounds > 1 and L > PART_COST:
        two = least(2 * PLACES)
        if 2 * two + PART_COST < L:
            L, room = two, 2 * PLACES
    if count(L) > room:
        L = 2**30 - 1
    return parts(L), count(L), room


def records(cu, kv, T, H, G, cap, causal=1, window=0, looks=True):
    """A call of 128-row tiles in parts: the records that its workgroups write, and those that the second launch reads.
    looks: as the kernel does it, token ranges that fall anywhere are no work and leave records of no parts everywhere."""
    B = len(kv)
    n_items = most_items(TILE, B, H, T, H * G)
    m, rounds, _, _ = mode(B, H, T, H * G, cap)
    assert m == "parts"
    grid = rounds * PLACES
    falls = any(cu[b + 1] < cu[b] for b in range(B))
    if looks and falls:
        return set(range(min(grid, PLACES))), set(range(n_items))
    seqs = sequences(cu, kv, T, cap)
    parts, total, _ = find_parts(seqs, H, G, causal, window, rounds)
    written, start = set(), 0
    for b, s in enumerate(seqs):
        tiles = tiles_of(TILE, G, s)
        for h in range(H):
            for x in range(tiles):  # part 0 of head h, tile x: the number of its workgroup
                w = start + h * parts[b] * tiles + x
                xcd = next(i for i in range(8) if i * total // 8 <= w < (i + 1) * total // 8)
                if w - xcd * total // 8 < grid // 8:
                    written.add((tile_start(TILE, G, cu, b) + x) * H + h)
        start += H * parts[b] * tiles
    read = set()
    starts = [tile_start(TILE, G, cu, b) for b in range(B)]
    for item in range(n_items):
        tile, lo, n = item // H, 0, B
        while n > 1:
            step = -(-n // 64)
            k = max(sum(1 for i in range(64) if i * step < n and starts[lo + i * step] <= tile) - 1, 0)
            lo, n = lo + k * step, min(step, n - k * step)
        x = tile - starts[lo]
        if 0 <= x < tiles_of(TILE, G, seqs[lo]):
            read.add(item)
    return written, read


class Shares:
    """Tiles of 16 rows: the parts of the tiles of every sequence and key head, in order, as (share, first stage, end)."""

    def __init__(self, seqs, H, G, cap, causal, window, row_bytes, items):
        cost = 512 // row_bytes
        places = min(items * -(-(-(-cap // FEW_STAGE)) // FEW_MIN), FEW_PLACES)
        tiles = [tiles_of(FEW_TILE, G, s) for s in seqs]
        st = [stages_of(FEW_TILE, FEW_STAGE, G, causal, window, s) for s in seqs]
        self.total = sum(t * H * (2 * x + cost) for t, x in zip(tiles, st))
        self.tiles = []  # (sequence, number in it, stages, parts)
        for log in (1, 2, 3):
            if sum(t * H * -(-x >> log) for t, x in zip(tiles, st)) <= places:
                share = 0
                for b, (t, x) in enumerate(zip(tiles, st)):
                    n = -(-x >> log)
                    for i in range(t * H):
                        self.tiles.append((b, i, x, [(share + p, p * x // n, (p + 1) * x // n) for p in range(n)]))
                        share += n
                self.mode = "parts"
                return
        self.mode = "shares"
        n = min(places, max(self.total // (2 * FEW_MIN + cost), 1))
        self.step, self.rest = divmod(self.total, n)
        at = 0
        for b, (t, x) in enumerate(zip(tiles, st)):
            for i in range(t * H):
                mine = []
                for share in range(n):
                    a, e = self.cut(share) - at, self.cut(share + 1) - at
                    if e <= 0 or a >= 2 * x + cost:
                        continue
                    p = (share, self.inside(a, x, cost), self.inside(e, x, cost))
                    if p[1] < p[2]:
                        mine.append(p)
                first = self.last_cut(at + 2 * FEW_CUT + cost - 2)
                parts = self.last_cut(at + 2 * (x - FEW_CUT) + cost) + 1 - first
                self.tiles.append((b, i, x, mine))
                if len(mine) > 1:  # what the workgroup that adds them up goes by
                    assert (first, parts) == (mine[0][0], len(mine))
                at += 2 * x + cost

    def cut(self, k):
        return k * self.step + min(k, self.rest)

    def last_cut(self, v):
        longer = self.rest * (self.step + 1)
        return v // (self.step + 1) if v < longer else self.rest + (v - longer) // self.step

    @staticmethod
    def inside(d, n, cost):
        x = (d - cost + 1) >> 1
        return n if x >= n else 0 if x < FEW_CUT else n if n - x < FEW_CUT else x

    def slots(self):
        """Slots of the parts of divided tiles: a share's first is of a tile that began before it, its second of one that begins in it."""
        out = []
        for _, _, n, parts in self.tiles:
            if len(parts) > 1:
                out += [2 * share + (a == 0) for share, a, _ in parts]
        return out

    def longest(self):
        """(most stages of a part, most parts of a tile)"""
        return (max((e - a for t in self.tiles for _, a, e in t[3]), default=0), max((len(t[3]) for t in self.tiles), default=0))


def shares_of(qs, kvs, H, G, cap, causal, window, D, kind):
    cu = [sum(qs[:b]) for b in range(len(qs) + 1)]
    T = cu[-1]
    assert few(len(kvs), H, T, H * G) and len(kvs) <= SPLIT_SEQS
    items = most_items(FEW_TILE, len(kvs), H, T, H * G)
    assert items <= FEW_ITEMS and math.ceil(cap / FEW_STAGE) <= 2**27 // items
    return Shares(sequences(cu, kvs, T, cap), H, G, cap, causal, window, D * (1 if kind == "e4m3" else 2), items)

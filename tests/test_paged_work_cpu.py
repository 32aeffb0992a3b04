"""How the paged attention shares its work, restated on the CPU: units on one
line, cut into equal pieces; every unit has one worker, a shared item's workers
are neighbours, and the first and last of them are what the item's record says."""
import random

import pytest


def row_tiles(n, length, TP, window, n_top):
    """(first unit, units, pages) of every row tile of a sequence (csrc/paged/work.cuh: row_tile)."""
    out = []
    for j in range(-(-n // TP)):
        first, last = length - n + j * TP, length - n + min(n, (j + 1) * TP) - 1
        if n_top:
            kept = 0 if last < 0 else min(n_top, last // 64 + 1)
            out.append((0, max(1, (kept + 1) // 2), max(1, kept)))
            continue
        hi = max(0, last + 1)
        lo = min(hi, max(0, first - window + 1)) if window else 0
        t0 = lo // 128
        pages = max(1, -(-hi // 64) - 2 * t0)
        out.append((t0, (pages + 1) // 2, pages))
    return out


@pytest.mark.parametrize("seed", range(30))
def test_pieces_cover_every_unit_once(seed):
    r = random.Random(seed)
    n_kv, TP = r.choice([1, 2, 8]), r.choice([1, 8, 18, 64])
    n_top = r.choice([0, 0, 5]) if TP == 1 else 0
    window = r.choice([0, 0, 100])
    items = []
    for _ in range(r.randint(1, 9)):
        length = r.randint(0, 900)
        n = r.choice([0, 1, min(length, r.randint(0, 300)), length + 2])
        items += [t for t in row_tiles(n, length, TP, window, n_top) for _ in range(n_kv)]
    COST = 2  # places of the line before an item's first unit (kItemCost)
    line = [(i, u - COST) for i, (_, nt, _) in enumerate(items) for u in range(nt + COST)]
    total = len(line)
    S = min(r.choice([1, 7, 152, 304]), total)
    owner = {}
    for w in range(S):
        a, b = w * total // S, (w + 1) * total // S
        assert b > a
        # the walk of one worker (find_pieces and ItemWalk): the item at its start, what is left of its piece
        i, off = line[a]
        kv0, left = max(0, off), max(0, b - a + min(0, off))
        while left > 0:
            nt = items[i][1]
            kv1 = min(nt, kv0 + left)
            if kv0 == 0:  # the record of an item that starts here
                at = b - left
                assert line[at] == (i, 0)
                last = ((at + nt - 1 + 1) * S - 1) // total
                owner[i, "first"], owner[i, "last"] = w, last
            for u in range(kv0, kv1):
                assert (i, u) not in owner
                owner[i, u] = w
            left = max(0, left - (kv1 - kv0) - COST)
            i, kv0 = i + 1, 0
    for i, (_, nt, pages) in enumerate(items):
        mine = [owner[i, u] for u in range(nt)]  # every unit has a worker
        assert mine == sorted(mine) and set(mine) == set(range(mine[0], mine[-1] + 1))
        assert (mine[0], mine[-1]) == (owner[i, "first"], owner[i, "last"])
        assert 2 * nt - 1 <= pages <= 2 * nt
    for w in range(S):  # a worker leaves at most one part of an item that it began, and one of an item that it did not
        began = [i for i in range(len(items)) if owner[i, 0] == w and owner[i, items[i][1] - 1] != w]
        joined = [i for i in range(len(items)) if owner[i, 0] != w and w in {owner[i, u] for u in range(items[i][1])}]
        assert len(began) <= 1 and len(joined) <= 1


def test_rows_to_tokens():
    """x / G by a multiplication and a shift, for every row of a tile and every group."""
    for G in range(1, 17):
        magic = (65536 + G - 1) // G
        assert all((x * magic) >> 16 == x // G for x in range(256))


def test_partials_are_aligned():
    """Every partial, output group and (maximum, sum) pair lies on its load's boundary."""
    for dh in (64, 128):
        for rows in range(2, 258, 2):
            assert rows * (dh + 2) * 4 % 16 == 0 and rows * dh * 4 % 8 == 0

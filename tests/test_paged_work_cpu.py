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
    total = sum(t[1] for t in items)
    S = min(r.choice([1, 7, 152, 304]), total)
    owner = [None] * total
    for w in range(S):
        a, b = w * total // S, (w + 1) * total // S
        assert b > a  # a worker that is named has units
        for u in range(a, b):
            assert owner[u] is None
            owner[u] = w
            assert ((u + 1) * S - 1) // total == w  # worker_of
    assert None not in owner
    at = 0
    for t0, nt, pages in items:
        mine = owner[at:at + nt]
        assert mine == sorted(mine) and set(mine) == set(range(mine[0], mine[-1] + 1))
        assert 2 * nt - 1 <= pages <= 2 * nt
        # a worker begins at most one item that it does not end, and ends at most one that it did not begin
        at += nt
    for w in range(S):
        a, b = w * total // S, (w + 1) * total // S
        starts, at = 0, 0
        for _, nt, _ in items:
            begins, ends = a <= at < b, a < at + nt <= b
            starts += begins and not ends
            at += nt
        assert starts <= 1


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

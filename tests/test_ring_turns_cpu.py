"""Rings whose pages several warps take in turn (csrc/copy_ring.cuh: ring_turns_ok, ring_fillers_ok), modelled with
barriers that know a parity only: every order in which copies arrive and warps go on is tried, and no wait may pass
before what it waits for has happened."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def passes(phase, n):
    """A wait for phase n of a barrier whose present phase is `phase`: it sees parities."""
    return (phase & 1) != (n & 1)


def turns_hold(S, W, pages):
    """Copies into S stages in order, arriving in any; W consumers, page i the consumer i % W, which frees its stage."""
    start = (0, (0,) * S, (0,) * S, (-1,) * S, tuple(range(W)))
    seen, todo = {start}, [start]
    while todo:
        issued, full, freed, flying, at = todo.pop()  # per stage: phases of full and of free, the page on its way
        nxt = []
        st = issued % S
        # a copy goes out once the page before has been taken (a wait in order, for every page); one at a time a stage
        if issued < pages and flying[st] < 0 and (issued < S or passes(freed[st], issued // S - 1)):
            if freed[st] < issued // S:
                return False
            nxt.append((issued + 1, full, freed, flying[:st] + (issued,) + flying[st + 1:], at))
        for s in range(S):
            if flying[s] >= 0:
                nxt.append((issued, full[:s] + (full[s] + 1,) + full[s + 1:], freed, flying[:s] + (-1,) + flying[s + 1:], at))
        for w in range(W):
            i = at[w]
            s = i % S
            if i < pages and passes(full[s], i // S):
                if full[s] <= i // S:  # page i has not arrived
                    return False
                nxt.append((issued, full, freed[:s] + (freed[s] + 1,) + freed[s + 1:], flying, at[:w] + (i + W,) + at[w + 1:]))
        for x in nxt:
            if x not in seen:
                seen.add(x)
                todo.append(x)
    return True


def fillers_hold(S, W, pages):
    """W producers, page i the producer i % W, into S slots which one consumer frees in order."""
    start = ((0,) * S, (0,) * S, 0, tuple(range(W)))
    seen, todo = {start}, [start]
    while todo:
        full, freed, taken, at = todo.pop()
        nxt = []
        for w in range(W):
            i = at[w]
            s = i % S
            if i < pages and (i < S or passes(freed[s], i // S - 1)):
                if freed[s] < i // S:  # the page before is still in the slot
                    return False
                nxt.append((full[:s] + (full[s] + 1,) + full[s + 1:], freed, taken, at[:w] + (i + W,) + at[w + 1:]))
        s = taken % S
        if taken < pages and passes(full[s], taken // S):
            if full[s] <= taken // S:
                return False
            nxt.append((full, freed[:s] + (freed[s] + 1,) + freed[s + 1:], taken + 1, at))
        for x in nxt:
            if x not in seen:
                seen.add(x)
                todo.append(x)
    return True


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("ring")
    src, exe = d / "rules.cpp", d / "rules"
    src.write_text('#include "copy_ring.cuh"\n#include <cstdio>\nint main() { for (int s = 1; s < 8; ++s) for (int w = 1; w < 5; ++w)'
                   ' std::printf("%d %d %d %d\\n", s, w, (int)pipo::ring_turns_ok(s, w), (int)pipo::ring_fillers_ok(s, w)); }\n')
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2605_27255_gb300", "csrc"),
                           str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    return {(int(s), int(w)): (bool(int(a)), bool(int(b))) for s, w, a, b in map(str.split, out.splitlines())}


@pytest.mark.parametrize("S,W", [(s, w) for s in range(1, 7) for w in range(1, 4)])
def test_turns(rules, S, W):
    assert turns_hold(S, W, 2 * S + W + 1) == rules[S, W][0]


@pytest.mark.parametrize("S,W", [(s, w) for s in range(1, 6) for w in range(1, 5)])
def test_fillers(rules, S, W):
    assert fillers_hold(S, W, 3 * S + W) or not rules[S, W][1]

// Bookkeeping of copy rings whose waits are bounded: what a thread has to wait
// for before its kernel ends.  A copy must not land in the shared memory of a
// CTA that has left, whatever wait gave up before.
//
// Plain C++, so that the host compiles it too: a CPU test lets the waits give
// up at every point.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define PIPO_RING_FN __device__ __forceinline__
#define PIPO_RING_RULE __host__ __device__ constexpr
#else
#define PIPO_RING_FN inline
#define PIPO_RING_RULE constexpr
#endif

namespace pipo {

// The last uses, at most one per stage, of the n that a ring of ST stages has
// seen: wait(stage, parity, use) for each, also after one has given up.
template <int ST, class Wait>
PIPO_RING_FN void ring_drain(int n, Wait wait) {
    for (int i = n > ST ? n - ST : 0; i < n; ++i) wait(i % ST, (uint32_t)((i / ST) & 1), i);
}

// One thread fills two rings of ST stages (tensor 0 and tensor 1) with the tiles
// 0 .. nt - 1 in turn: empty(tensor, stage, parity, tile) waits until the tile
// before has left the stage (false: given up), load(tensor, stage, tile) issues
// the copy, full(tensor, stage, parity, tile) waits for it.  At the end no copy
// is in flight, also when an `empty` gave up with only tensor 0 of its tile
// issued.
template <int ST, class Empty, class Load, class Full>
PIPO_RING_FN void ring_fill_pair(int nt, Empty empty, Load load, Full full) {
    int n0 = 0, n1 = 0;  // copies issued
    for (int t = 0; t < nt; ++t) {
        const int st = t % ST;
        const uint32_t ph = (uint32_t)(((t / ST) & 1) ^ 1);
        if (t >= ST && !empty(0, st, ph, t)) break;
        load(0, st, t);
        n0 = t + 1;
        if (t >= ST && !empty(1, st, ph, t)) break;
        load(1, st, t);
        n1 = t + 1;
    }
    ring_drain<ST>(n0, [&](int st, uint32_t ph, int t) { full(0, st, ph, t); });
    ring_drain<ST>(n1, [&](int st, uint32_t ph, int t) { full(1, st, ph, t); });
}

// The end of a CTA pair's copying threads after n stages each: the leader waits
// for every copy (both CTAs' arrive on its barriers), whatever gave up before;
// then each CTA for the commits that freed its stages, which come in order, so
// that after one that never came there are none.
template <int ST, class Full, class Empty>
PIPO_RING_FN void pair_drain(int n, bool leader, Full full, Empty empty) {
    if (leader) ring_drain<ST>(n, full);
    bool ok = true;
    ring_drain<ST>(n, [&](int st, uint32_t ph, int i) { ok = ok && empty(st, ph, i); });
}

// Consumers that take the pages of a ring in turn, page i the consumer i % W, and wait for their own alone: a barrier's
// parity tells its present phase from the one before, so a wait that comes while the fill BEFORE the wanted one is still
// under way passes at once.  (Copies may arrive in any order, and a page without a copy arrives at once.)  The
// fill before is known to be over where the same consumer took it: stages must be a multiple of consumers.
PIPO_RING_RULE bool ring_turns_ok(int stages, int consumers) { return stages % consumers == 0; }
// Producers that fill the slots of a ring in turn, each after a wait for its own slot to be free, where slots are freed in
// order: a producer's page before, W back, was free to be filled, so that all pages up to W + S back have left
// their slots; that must reach the one that was two laps ago in this page's slot.
PIPO_RING_RULE bool ring_fillers_ok(int slots, int producers) { return producers <= slots; }

}  // namespace pipo

// A ring of slots that two matrices' tiles go through in turn, side 0 then side 1 of tile 0, 1, ... (device code; plain C++ for tests on the
// host).
#pragma once

#include "window.h"

namespace e2egrec {

constexpr int kWordRing = 8;                         // tiles whose visibility words are kept

// Copy g is side g & 1 of tile g / 2.  It lies in slot(g), which was used use(g) times before, and lands at barrier full(side, tile), one of
// kWordRing per side that go by the tile's number.  A wait names the parity of a phase, so whoever waits has to see every phase of a barrier: one that
// waits for one side's copies alone does so here, but not with a barrier per slot where the sides take turns in a slot (with an odd
// number of slots they do): there the phase before last passed for the one that was waited for, now and then, and the warp that
// zeroes hidden rows of one side did so in a tile of the other.  No barrier has two copies under way: kSlots <= 2 kWordRing.
template <int SLOTS> struct TileRing {
    static constexpr int kSlots = SLOTS, kBarriers = 2 * kWordRing;
    static_assert(SLOTS <= 2 * kWordRing, "a barrier per copy under way");
    E2EGREC_HD static uint32_t slot(uint32_t g) { return g % SLOTS; }
    E2EGREC_HD static uint32_t use(uint32_t g) { return g / SLOTS; }
    E2EGREC_HD static uint32_t full(uint32_t side, uint32_t tile) { return side * kWordRing + tile % kWordRing; }
    E2EGREC_HD static uint32_t parity(uint32_t tile) { return tile / kWordRing & 1u; }
};

}  // namespace e2egrec

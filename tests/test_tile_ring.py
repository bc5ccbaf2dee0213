"""The ring that tiles of two matrices go through in turn, compiled from its header with the host compiler: one that waits for one side's
copies alone never takes a slot's earlier phase for the one it waits for, in whatever order copies land and products follow."""
from test_host_logic import run_cpp

MODEL = """
// A barrier per slot, as a mistake that the model has to see
template <int SLOTS> struct BySlot {
    static constexpr int kSlots = SLOTS;
    static uint32_t slot(uint32_t g) { return g % SLOTS; }
    static uint32_t use(uint32_t g) { return g / SLOTS; }
    static uint32_t full(uint32_t side, uint32_t tile) { return slot(2 * tile + side); }
    static uint32_t parity(uint32_t) { return 0; }
};
// the barrier of copy g and the parity that is waited for
template <typename R> uint32_t full(uint32_t g) { return R::full(g & 1u, g >> 1); }
template <int S> uint32_t parity(TileRing<S>, uint32_t g) { return TileRing<S>::parity(g >> 1); }
template <int S> uint32_t parity(BySlot<S>, uint32_t g) { return BySlot<S>::use(g) & 1u; }

// `tiles` tiles through ring R, steps in random order.  Copies are started in order, each once its slot's last use was consumed, and land in
// any order.  Products: a tile's side is consumed once it landed, side `side` only after the waiter of that side, too; side 1 of a tile after
// its side 0, and side 0 of a tile not before side 1 of the last but one.  Returns the tile at which the waiter's parity passed while its copy had
// not landed; -1: never, -2: nothing could go on, -3: two copies under way at one barrier.
template <typename R> int walk(int tiles, int side, unsigned seed)
{
    srand(seed);
    static int phases[64], consumed[64], under_way[64];  // completed phases and copies under way per barrier, uses consumed per slot
    static bool in_flight[4096], done[4096];
    for (int s = 0; s < 64; ++s) phases[s] = consumed[s] = under_way[s] = 0;
    for (int g = 0; g < 4096; ++g) in_flight[g] = done[g] = false;
    int next = 0, waiter = 0, eaten[2] = {0, 0};         // the next copy, the waiter's tile, tiles consumed per side
    for (int idle = 0; idle < 100000; ++idle) {
        if (eaten[0] == tiles && eaten[1] == tiles) return -1;
        switch (rand() % 4) {
        case 0:                                          // start a copy
            if (next < 2 * tiles && consumed[R::slot(next)] == (int)R::use(next)) {
                if (under_way[full<R>(next)]++) return -3;
                in_flight[next++] = true, idle = 0;
            }
            break;
        case 1: {                                        // one of those on their way lands
            const int g = next - 1 - rand() % 16;
            if (g >= 0 && in_flight[g]) in_flight[g] = false, done[g] = true, ++phases[full<R>(g)], --under_way[full<R>(g)], idle = 0;
            break;
        }
        case 2: {                                        // the waiter of one side
            const uint32_t g = 2 * waiter + side;
            if (waiter < tiles && (uint32_t)(phases[full<R>(g)] & 1) != parity(R(), g)) {
                if (!done[g]) return waiter;
                ++waiter, idle = 0;
            }
            break;
        }
        case 3: {                                        // products
            const int s = rand() % 2, j = eaten[s];
            const uint32_t g = 2 * j + s;
            if (j == tiles || !done[g] || (s == side && waiter <= j) || (s == 1 && eaten[0] <= j) || (s == 0 && eaten[1] + 1 < j)) break;
            ++consumed[R::slot(g)], ++eaten[s], idle = 0;
            break;
        }
        }
    }
    return -2;
}
template <typename R> int worst(int side)
{
    for (unsigned seed = 0; seed < 300; ++seed)
        if (const int bad = walk<R>(200, side, seed); bad != -1) return bad;
    return -1;
}
"""


def test_waiting_for_one_side(tmp_path):
    model = tmp_path / "model.h"
    model.write_text('#include "tile_ring.h"\nnamespace e2egrec {\n' + MODEL + "}\n")
    run_cpp(tmp_path, """
// the rings of the forward kernel (zeros go to the values, side 1) and of the dQ kernel (to the keys, side 0)
if (worst<TileRing<2>>(1) != -1 || worst<TileRing<5>>(1) != -1 || worst<TileRing<8>>(1) != -1) return 1;
if (worst<TileRing<5>>(0) != -1 || worst<TileRing<8>>(0) != -1) return 2;
if (worst<BySlot<5>>(1) < 0 || worst<BySlot<5>>(0) < 0) return 3;
""", "cstdlib", str(model))


def test_every_phase_of_a_barrier_is_one_side_in_turn(tmp_path):
    run_cpp(tmp_path, """
using R = TileRing<5>;
int phases[R::kBarriers] = {}, uses[R::kSlots] = {};
for (uint32_t g = 0; g < 1000; ++g) {
    const uint32_t f = R::full(g & 1u, g >> 1);
    if (f >= R::kBarriers || (g & 1u) != (f >= kWordRing)) return 1;           // a side's own barriers
    if (R::parity(g >> 1) != (uint32_t)(phases[f]++ & 1)) return 2;
    if (R::use(g) != (uint32_t)uses[R::slot(g)]++) return 3;
}
""", "tile_ring.h")

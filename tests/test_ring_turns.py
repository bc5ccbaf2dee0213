"""The book of the ring of copies of the streaming attention kernels, compiled from its header with the host compiler: whatever wait
is given up, every copy that was started is waited for and none is started afterwards."""
from test_host_logic import run_cpp

WALK = """
// Walks of `lengths` turns one after the other, the wait for turn `fails` of walk `walk` given up; counts of copies per use
// number, and of waits for them.
struct Walks {
    int started[256] = {}, awaited[256] = {}, after = 0;
    bool ok = true;
    void run(const int *lengths, int walks, int walk, int fails)
    {
        int used = 0;
        for (int w = 0; w < walks; ++w) {
            const int turns = lengths[w];
            auto fill = [&](int t) {
                ++started[used + t];
                if (!ok) ++after;
            };
            for (int t = 0; t < ring_first(turns, ok); ++t) fill(t);
            for (int t = 0; t < turns && ok; ++t) {
                if (w == walk && t == fails) {
                    ok = false;
                    for (int i = t; i < ring_pending(t, turns); ++i) ++awaited[used + i];
                    break;
                }
                ++awaited[used + t];
                if (ring_next(t, turns, ok) >= 0) fill(ring_next(t, turns, ok));
            }
            used += turns;
        }
    }
};
"""


def test_every_copy_is_waited_for_once(tmp_path):
    run_cpp(tmp_path, WALK + """
const int lengths[] = {1, 0, 2, 3, 4, 9, 5};
int total = 0;
for (int n : lengths) total += n;
for (int walk = -1; walk < 7; ++walk)
    for (int fails = 0; fails < (walk < 0 ? 1 : lengths[walk]); ++fails) {
        Walks w;
        w.run(lengths, 7, walk, fails);
        if (w.ok != (walk < 0)) return 1;
        if (w.after) return 2;
        int started = 0;
        for (int u = 0; u < 256; ++u) {
            if (w.started[u] != w.awaited[u] || w.started[u] > 1) return 3;
            started += w.started[u];
        }
        if (walk < 0 && started != total) return 4;
    }
""", "ring_turns.h")


def test_a_stage_is_filled_again_only_after_it_was_read(tmp_path):
    run_cpp(tmp_path, """
for (int turns = 0; turns < 20; ++turns) {
    int started = ring_first(turns, true);
    if (started > kRingStages) return 1;
    for (int t = 0; t < turns; ++t) {
        if (t >= started) return 2;              // waited for before it was started
        const int next = ring_next(t, turns, true);
        if (next >= 0) {
            if (next != started || next % kRingStages != t % kRingStages) return 3;
            ++started;
        }
    }
    if (started != turns) return 4;
}
""", "ring_turns.h")

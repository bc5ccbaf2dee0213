// Turns of a ring of kRingStages stages: which copies are started, and which are on their way when a wait is given up (device code;
// plain C++ for tests on the host).
#pragma once

#include "window.h"

namespace e2egrec {

constexpr int kRingStages = 3;

// How many turns a walk over `turns` starts with; none once a wait was given up: the stages' phases are not known any more, and
// nobody would wait for the copies.
E2EGREC_HD int ring_first(int turns, bool ok) { return !ok ? 0 : (turns < kRingStages ? turns : kRingStages); }
// The turn whose copies go out when turn t has been read, or -1.
E2EGREC_HD int ring_next(int t, int turns, bool ok) { return ok && t + kRingStages < turns ? t + kRingStages : -1; }
// Where the wait for turn t is given up, turns t .. ring_pending(t, turns) - 1 are on their way, turn t itself among them.
E2EGREC_HD int ring_pending(int t, int turns) { return t + kRingStages < turns ? t + kRingStages : turns; }

}  // namespace e2egrec

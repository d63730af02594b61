// The tiles that are still on their way when the shared-prefix kernel unwinds: random runs of the two loaders, the copies and
// the consumer, stopped anywhere, against ring_last_tile().
#include "hg_ring.h"

#include <cstdio>
#include <random>
#include <vector>

static int fail(const char* what, int slots, int k, int v) {
    std::fprintf(stderr, "%s: %d slots, %d K tiles, %d V tiles\n", what, slots, k, v);
    return 1;
}

int main() {
    std::mt19937 rng(7);
    long in_flight = 0, revisited = 0;
    for (int run = 0; run < 60000; ++run) {
        const int slots = run & 1 ? 5 : 10;
        int issued[2] = {0, 0};                                        // K tiles, V tiles
        std::vector<int> state;                                        // per tile number: 0 none, 1 on its way, 2 landed, 3 consumed
        std::vector<int> filled(slots, 0), latest(slots, -1);          // per slot: completed phases, last tile requested
        for (int steps = (int)(rng() % 120); steps > 0; --steps) {
            const unsigned op = rng() % 6;
            if (op < 2) {
                const int n = 2 * issued[op] + (int)op;
                if ((int)state.size() <= n + 1) state.resize(n + 2, 0);
                if (n >= slots && state[n - slots] != 3) continue;     // the loader waits for the slot
                state[n] = 1;
                latest[n % slots] = n;
                ++issued[op];
            } else {                                                   // one of the tiles lands, or is consumed
                std::vector<int> can;
                for (int n = 0; n < (int)state.size(); ++n)
                    if (state[n] == (op < 4 ? 1 : 2)) can.push_back(n);
                if (can.empty()) continue;
                const int n = can[rng() % can.size()];
                if (state[n]++ == 1) ++filled[n % slots];
            }
        }
        std::vector<int> waited(state.size(), 0);
        for (int s = 0; s < slots; ++s) {
            const int n = hg::ring_last_tile(s, slots, issued[0], issued[1]);
            if (n != latest[s]) return fail("not the slot's last tile", slots, issued[0], issued[1]);
            if (n < 0) continue;
            waited[n] = 1;
            revisited += n >= slots;
            // a wait on parity p ends when the phase in progress has the other one
            const bool ends = (filled[s] & 1) != ((n / slots) & 1);
            if (ends != (state[n] >= 2)) return fail("a wait that does not follow the tile", slots, issued[0], issued[1]);
        }
        for (int n = 0; n < (int)state.size(); ++n)
            if (state[n] == 1) {
                ++in_flight;
                if (!waited[n]) return fail("a tile on its way that nobody waits for", slots, issued[0], issued[1]);
            }
    }
    if (in_flight < 1000 || revisited < 1000) return fail("the runs reach too little", 0, (int)in_flight, (int)revisited);
    std::puts("ring OK");
    return 0;
}

// Every piece of every moved row is one thread's, once, at any number of moves, in 32 bits: on the host.
#include <climits>
#include <cstdio>
#include <vector>

#include "row_moves.h"

using namespace audiokv;

static int g_failed = 0;
#define CHECK(cond)                                                                                  \
    do {                                                                                             \
        if (!(cond) && ++g_failed < 20) std::fprintf(stderr, "FAILED line %d: %s\n", __LINE__, #cond); \
    } while (0)

int main() {
    for (int d : {64, 128, 256}) {
        const int per = d / 4;
        for (int parts : {1, 3, 64, 4096}) {
            // all of them
            for (int moves : {0, 1, 31, 500, 5000}) {
                std::vector<int> seen((size_t)moves * per, 0);
                for (int t = 0; t < parts * 256; ++t) {
                    const MoveWalk w = move_walk(t, parts * 256, per);
                    for (int i = w.first; i < moves; i += w.step) ++seen[(size_t)i * per + w.piece];
                }
                for (int n : seen) CHECK(n == 1);
            }
            // the last ones of very many, and no thread's next move beyond them leaves the type
            for (int moves : {(1 << 25) + 3, (1 << 26) + 1, (1 << 30) - 1}) {
                for (int i = moves - 3; i < moves; ++i)
                    for (int p = 0; p < per; ++p) {
                        const int t = (int)(((long long)i * per + p) % (parts * 256));
                        const MoveWalk w = move_walk(t, parts * 256, per);
                        CHECK(w.piece == p && w.first < w.step && (i - w.first) % w.step == 0);
                    }
                const MoveWalk w = move_walk(parts * 256 - 1, parts * 256, per);
                CHECK((long long)moves + 4LL * w.step <= INT_MAX);
            }
        }
    }
    std::printf(g_failed ? "%d failures\n" : "ok\n", g_failed);
    return g_failed != 0;
}

// Where the workgroups of accumulate.hip put what they find for blocks that several share, on the host: no two parts have one slot,
// and the kernels that join a block's parts look for them where they are.
#include <cstdio>
#include <map>
#include <utility>
#include <vector>

#include "accumulate_plan.h"

using namespace audiokv;

static int g_failed = 0;
#define CHECK(cond)                                                                                  \
    do {                                                                                             \
        if (!(cond) && ++g_failed < 20) std::fprintf(stderr, "FAILED line %d: %s\n", __LINE__, #cond); \
    } while (0)

static void check(bool cols, int size, const std::vector<AccumItem>& items, int heads, int least) {
    const AccumSweep s = plan_sweep(cols, size, (int)items.size(), heads, least, [&](int i) { return items[i]; });
    const AccumSpans& sp = s.spans;
    // as the sweeps walk through their spans: block -> (workgroup, slot) of its parts in order, where it has several
    std::map<std::pair<int, int>, std::vector<std::pair<int, int>>> parts;
    std::vector<int> used(part_slots(sp.n), 0);
    for (int w = 0; w < sp.n; ++w) {
        const SpanStart end = sp.at[w + 1];
        int head = sp.at[w].head, block = sp.at[w].block, tile = sp.at[w].tile;
        while (head < end.head || (head == end.head && (block < end.block || (block == end.block && tile < end.tile)))) {
            const AccumItem& it = items[head / heads];
            if (block >= it.blocks(cols, size)) { ++head; block = tile = 0; continue; }
            const int tiles = it.tiles(cols, block, size), stop = head == end.head && block == end.block ? end.tile : tiles;
            if (stop - tile < tiles) {
                const int slot = part_slot(w, tile > 0);
                CHECK(slot >= 0 && slot < part_slots(sp.n));
                if (slot >= 0 && slot < part_slots(sp.n)) CHECK(++used[slot] == 1);
                parts[{head, block}].push_back({w, slot});
            }
            ++block;
            tile = 0;
        }
    }
    CHECK(parts.empty() || s.max_parts > 1);                  // (otherwise there are no slots)
    // as the joins look for them: from a block's first workgroup on
    for (const auto& [at, found] : parts) {
        CHECK(found.size() > 1);
        for (int c = 0; c < (int)found.size(); ++c) CHECK(found[c].second == part_slot_of(found[0].first, c));
    }
}

int main() {
    unsigned seed = 7;
    auto rnd = [&](int lo, int hi) { seed = seed * 1664525u + 1013904223u; return lo + (int)((seed >> 8) % (unsigned)(hi - lo + 1)); };
    for (int trial = 0; trial < 2000; ++trial) {
        std::vector<AccumItem> items;
        const int n = rnd(1, 6), G = rnd(1, 3) == 1 ? 1 : rnd(2, 17), causal = rnd(0, 3) != 0, top = rnd(0, 2) == 0 ? 9000 : 300;
        for (int i = 0; i < n; ++i) {
            const int L = rnd(1, top);
            items.push_back(AccumItem{L, rnd(0, 3) == 0 ? L : rnd(0, L), G, causal});
        }
        for (int size : {224, 448})
            for (int cols = 0; cols < 2; ++cols) check(cols, size, items, rnd(1, 8), rnd(1, 4));
    }
    std::vector<AccumItem> one_long(64, AccumItem{500, 500, 4, 1});
    one_long[0] = AccumItem{131072, 131072, 4, 1};
    for (int cols = 0; cols < 2; ++cols) check(cols, 448, one_long, 8, 1);
    std::printf(g_failed ? "%d failures\n" : "ok\n", g_failed);
    return g_failed != 0;
}

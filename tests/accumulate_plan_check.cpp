// The division of the sweeps of accumulate.hip into spans, on the host: every tile of every block is some workgroup's, once, in
// order; spans cost about the same; first_of and parts_of name a block's workgroups; max_parts bounds them.
#include <cstdio>
#include <vector>

#include "accumulate_plan.h"

using namespace audiokv;

static int g_failed = 0;
#define CHECK(cond)                                                                        \
    do {                                                                                   \
        if (!(cond) && ++g_failed < 20) std::fprintf(stderr, "FAILED line %d: %s (%s)\n", __LINE__, #cond, what); \
    } while (0)

static void check(bool cols, int size, const std::vector<AccumItem>& items, int heads, int least) {
    char what[200];
    std::snprintf(what, sizeof(what), "cols %d size %d items %zu first L %d Q %d G %d causal %d heads %d", cols, size, items.size(),
                  items[0].L, items[0].Q, items[0].G, items[0].causal, heads);
    const AccumSweep s = plan_sweep(cols, size, (int)items.size(), heads, least, [&](int i) { return items[i]; });
    const AccumSpans& sp = s.spans;
    CHECK(sp.n <= kSpans);
    // workgroups beyond the last span find nothing to do
    if (sp.n > 0)
        for (int w = sp.n; w <= kSpans; ++w) CHECK(sp.at[w].head == (int)items.size() * heads && sp.at[w].block == 0 && sp.at[w].tile == 0);
    // what the workgroups do, as the kernels walk through it
    long long lo = 1LL << 60, hi = 0;
    std::vector<std::vector<std::vector<int>>> by(items.size() * heads);      // head, block: workgroups in order
    std::vector<std::vector<int>> next(items.size() * heads);                 // the next tile of each block
    for (size_t g = 0; g < by.size(); ++g) {
        by[g].resize(items[g / heads].blocks(cols, size));
        next[g].assign(by[g].size(), 0);
        CHECK((int)by[g].size() <= s.max_blocks);
    }
    for (int w = 0; w < sp.n; ++w) {
        const SpanStart end = sp.at[w + 1];
        int head = sp.at[w].head, block = sp.at[w].block, tile = sp.at[w].tile;
        long long cost = 0;
        while (head < end.head || (head == end.head && (block < end.block || (block == end.block && tile < end.tile)))) {
            const AccumItem& it = items[head / heads];
            if (block >= it.blocks(cols, size)) { ++head; block = tile = 0; continue; }
            const int tiles = it.tiles(cols, block, size), stop = head == end.head && block == end.block ? end.tile : tiles;
            CHECK(stop <= tiles && tile < stop && next[head][block] == tile);
            next[head][block] = stop;
            by[head][block].push_back(w);
            cost += stop - tile + kBlockCost;
            ++block;
            tile = 0;
        }
        CHECK(cost > 0);
        if (w < sp.n - 1) lo = cost < lo ? cost : lo;
        hi = cost > hi ? cost : hi;
    }
    if (sp.n > 1) CHECK(hi - lo <= 2 * kBlockCost);
    for (size_t g = 0; g < by.size(); ++g)
        for (int b = 0; b < (int)by[g].size(); ++b) {
            const AccumItem& it = items[g / heads];
            const int tiles = it.tiles(cols, b, size);
            CHECK(tiles > 0 && next[g][b] == tiles);
            // the pairs of the block lie within its tiles
            if (cols) {
                const int from = it.key_tiles_from(b, size);
                CHECK(from >= 0 && from <= it.first_row(b * size) && from + tiles * kStream >= it.rows());
                CHECK(from + (tiles - 1) * kStream < it.rows());
            } else {
                CHECK((tiles - 1) * kStream < it.L);
            }
            const std::vector<int>& ws = by[g][b];
            CHECK((int)ws.size() <= s.max_parts);
            // (what parts_of counts)
            int before = 0, until = 0;
            for (int w = 0; w < sp.n; ++w) {
                before += !sp.at[w].after((int)g, b);
                until += sp.at[w].head < (int)g || (sp.at[w].head == (int)g && sp.at[w].block <= b);
            }
            CHECK(before - 1 == ws[0] && until - before + 1 == (int)ws.size());
            for (size_t i = 0; i < ws.size(); ++i) CHECK(ws[i] == ws[0] + (int)i && sp.first_of((int)g, b, ws[i]) == ws[0]);
        }
}

int main() {
    unsigned seed = 1;
    auto rnd = [&](int lo, int hi) { seed = seed * 1664525u + 1013904223u; return lo + (int)((seed >> 8) % (unsigned)(hi - lo + 1)); };
    for (int trial = 0; trial < 3000; ++trial) {
        std::vector<AccumItem> items;
        const int n = rnd(1, 6), G = rnd(1, 3) == 1 ? 1 : rnd(2, 17), causal = rnd(0, 3) != 0, top = rnd(0, 2) == 0 ? 9000 : 300;
        for (int i = 0; i < n; ++i) {
            const int L = rnd(1, top);
            items.push_back(AccumItem{L, rnd(0, 3) == 0 ? L : rnd(0, L), G, causal});
            if (rnd(0, 2) == 0) items.push_back(items.back());
        }
        for (int size : {224, 448})
            for (int cols = 0; cols < 2; ++cols) check(cols, size, items, rnd(1, 8), rnd(1, 4));
    }
    check(false, 448, {AccumItem{131072, 131072, 8, 1}}, 8, 2);
    check(true, 448, {AccumItem{131072, 131072, 8, 1}}, 8, 2);
    std::printf(g_failed ? "%d failures\n" : "ok\n", g_failed);
    return g_failed != 0;
}

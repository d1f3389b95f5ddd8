// fork_give (pages.h), what a thread of fork's second launch does, on the host: threads of a workgroup run in any order, heads too, and
// table, lengths, counts and the number of free pages are what the definition says.
#include <algorithm>
#include <cstdio>
#include <numeric>
#include <random>
#include <vector>

#include "pages.h"

using namespace audiokv;

static int g_failed = 0;
#define CHECK(cond)                                                                                                          \
    do {                                                                                                                     \
        if (!(cond) && ++g_failed < 20) std::fprintf(stderr, "FAILED line %d (turn %d, order %d): %s\n", __LINE__, turn, order, #cond); \
    } while (0)

int main() {
    constexpr int kThreads = 256, kHeads = 2;           // of a workgroup; of a sequence
    std::mt19937 r(1);
    for (int turn = 0; turn < 200; ++turn) {
        const int n = 1 + (int)(r() % 6), heads = n * kHeads, width = 1 + (int)(r() % (turn % 2 ? 900 : 70)), P = 32;
        // a cache, some of whose sequences have another's pages
        std::vector<int32_t> table((size_t)heads * width), lengths(heads), refs((size_t)heads * width + 9, 0);
        std::vector<int32_t> pages(refs.size());
        std::iota(pages.begin(), pages.end(), 0);
        std::shuffle(pages.begin(), pages.end(), r);
        size_t next = 0;
        for (int h = 0; h < heads; ++h) {
            const bool shares = h >= kHeads && (h / kHeads) % 3 == 2;
            lengths[h] = shares ? lengths[h - kHeads] : (int)(r() % (unsigned)(width * P + 1));
            for (int j = 0; j < width; ++j) {
                const bool there = j < (lengths[h] + P - 1) / P;
                table[(size_t)h * width + j] = !there ? (int)(r() % refs.size()) : shares ? table[(size_t)(h - kHeads) * width + j] : pages[next++];
                if (there) ++refs[table[(size_t)h * width + j]];
            }
        }
        std::vector<int32_t> parents(n), drop(n);
        for (int x = 0; x < n; ++x) {
            parents[x] = r() % 3 == 0 ? x : (int)(r() % (unsigned)(n + 2)) - 1;
            drop[x] = r() % 2 ? 0 : (int)(r() % (unsigned)(width * P));
        }
        // what the definition says, and what the first launch leaves
        std::vector<int32_t> table_then = table, lengths_then = lengths, refs_then = refs, taken = refs, entries((size_t)heads * width, -7);
        std::vector<int2> rows(heads);
        for (int h = 0; h < heads; ++h) {
            const int parent = parents[h / kHeads], from = parent * kHeads + h % kHeads, had = (lengths[h] + P - 1) / P;
            const bool is = parent >= 0 && parent < n;
            rows[h].x = lengths[h];
            rows[h].y = lengths_then[h] = is ? std::max(lengths[from] - drop[h / kHeads], 0) : 0;
            for (int j = 0; j < had; ++j) --refs_then[table[(size_t)h * width + j]];
            for (int j = 0; j < (rows[h].y + P - 1) / P; ++j) {
                const int page = table[(size_t)from * width + j];
                ++refs_then[page];
                table_then[(size_t)h * width + j] = page;
                if (from == h) continue;
                entries[(size_t)h * width + j] = page;
                if (j >= had || table[(size_t)h * width + j] != page) ++taken[page];
            }
        }
        const auto free_pages = [](const std::vector<int32_t>& counts) { return (int)std::count(counts.begin(), counts.end(), 0); };
        for (int order = 0; order < 3; ++order) {       // ascending, descending, none
            std::vector<int32_t> t = table, l = lengths, c = taken;
            PageView pv{};
            pv.table = t.data();
            pv.lengths = l.data();
            pv.refs = c.data();
            pv.n_pages = (int)refs.size();
            pv.width = width;
            pv.log_p = 5;
            pv.n_heads = heads;
            pv.H = kHeads;
            const ForkSpace f{rows.data(), entries.data()};
            std::vector<int> who((size_t)heads * kThreads);
            std::iota(who.begin(), who.end(), 0);
            if (order == 1) std::reverse(who.begin(), who.end());
            if (order == 2) std::shuffle(who.begin(), who.end(), r);
            int freed = 0;
            for (int w : who)
                freed += fork_give(pv, f, parents.data(), n, w / kThreads, w % kThreads, kThreads, [&](int page) { return --c[page] == 0; });
            CHECK(l == lengths_then);
            CHECK(c == refs_then);
            CHECK(free_pages(refs) + freed == free_pages(refs_then));
            for (int h = 0; h < heads; ++h)
                for (int j = 0; j < (l[h] + P - 1) / P; ++j) CHECK(t[(size_t)h * width + j] == table_then[(size_t)h * width + j]);
        }
    }
    return g_failed != 0;
}

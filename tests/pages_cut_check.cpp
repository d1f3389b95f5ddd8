// How attend cuts heads into parts where shares end with the heads: as attend_kernel decides and walks, and as join_kernel looks for the
// parts. Every unit goes to one workgroup, no workgroup has two heads, and all of them exist. (pages_check.cpp has the even cut.)
#include <climits>
#include <cstdio>
#include <random>
#include <vector>

#include "pages.h"

using namespace audiokv;

static int g_failed = 0, g_aligned = 0, g_even = 0;
#define CHECK(cond)                                                                                  \
    do {                                                                                             \
        if (!(cond) && ++g_failed < 20) std::fprintf(stderr, "FAILED line %d: %s\n", __LINE__, #cond); \
    } while (0)

static void cut(const std::vector<int>& units, int wgs, int waves) {
    const int n = (int)units.size();
    long long sum = 0;
    for (int u : units) sum += u;
    if (sum == 0 || sum > INT_MAX) return;
    const int total = (int)sum;
    const int share = 2 * n <= wgs ? std::max((int)(((unsigned)total + wgs - n - 1) / (wgs - n)), waves) : INT_MAX;
    if (share - 4 > total / wgs) {
        // the even cut: no share is empty
        const int W = std::min(wgs, total / waves + 1);
        const Shares all{total, W};
        for (int w : {0, W / 3, W - 1}) CHECK(all.begin(w) < all.begin(w + 1));
        ++g_even;
        return;
    }
    ++g_aligned;
    long long W = 0;
    for (int u : units) W += (u + share - 1) / share;
    CHECK(W <= wgs && n <= wgs);
    int b = 0;
    for (int u : units) {
        const int parts = (u + share - 1) / share;
        const Shares of_head{u, parts};
        int next = 0;
        for (int p = 0; p < parts; ++p, ++b) {
            const int u0 = of_head.begin(p), u1 = of_head.begin(p + 1);
            CHECK(u0 == next && u1 > u0 && u1 - u0 <= share);
            CHECK(part_slot(2 * (b - p), p) == 2 * b && 2 * b + 1 < 2 * wgs);
            next = u1;
        }
        CHECK(next == u && parts <= wgs);
    }
    CHECK(b == W);
}

int main() {
    std::mt19937 r(1);
    for (int wgs : {1024, 768, 512, 193, 8, 3, 2, 1})
        for (int i = 0; i < 4000; ++i) {
            std::vector<int> units(1 + r() % (unsigned)(i % 3 == 0 ? 4 : 1 + wgs / (i % 2 + 1)));
            const int most = i % 5 == 0 ? 3 : i % 5 == 1 ? 4000 : 90;
            for (int& u : units) u = r() % 4 == 0 ? 0 : (int)(r() % most);
            if (i % 7 == 0) std::fill(units.begin(), units.end(), 1 + (int)(r() % most));          // equal heads
            cut(units, wgs, 4);
        }
    for (int k : {1, 2, 3}) cut(std::vector<int>(k, INT_MAX / k), 1024, 4);                        // the most units there are
    cut({INT_MAX - 500, 0, 0, 1, 499}, 768, 4);
    CHECK(g_aligned > 1000 && g_even > 1000);
    return g_failed != 0;
}

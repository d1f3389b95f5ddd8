// pages.h on the host: the scale of every block, where a page's sections lie, and how attend shares units out: every unit to one
// workgroup, every part of a head where the join looks for it.
#include <cmath>
#include <cstdio>
#include <map>
#include <random>
#include <vector>

#include "pages.h"

using namespace audiokv;

static int g_failed = 0;
#define CHECK(cond)                                                                                  \
    do {                                                                                             \
        if (!(cond) && ++g_failed < 20) std::fprintf(stderr, "FAILED line %d: %s\n", __LINE__, #cond); \
    } while (0)

static void shares(int n, int k) {
    const Shares s{n, k};
    CHECK(s.begin(0) == 0 && s.begin(k) == n);
    for (int w : {0, 1, k / 3, k / 2, k - 2, k - 1}) {
        if (w < 0 || w >= k) continue;
        const int a = s.begin(w), b = s.begin(w + 1);
        CHECK(a <= b && b - a <= (long long)n / k + 1);
        for (int u : {a, a + 1, b - 1})
            if (u >= a && u < b) CHECK(s.of(u) == w);
    }
}

// as attend_kernel walks over its share, and as join_kernel looks for the parts
static void parts(const std::vector<int>& units, int W) {
    int total = 0;
    for (int n : units) total += n;
    if (total == 0) return;
    W = W < total ? W : total;
    const Shares all{total, W};
    std::map<int, std::vector<int>> written;           // head -> slots in order
    std::map<int, std::pair<int, int>> noted;          // head -> first slot, parts
    std::vector<int> used(2 * W, 0);
    for (int w = 0; w < W; ++w) {
        const int u0 = all.begin(w), u1 = all.begin(w + 1);
        int head = 0, start = 0;
        while (u0 >= start + units[head]) start += units[head++];
        for (int u = u0; u < u1;) {
            const int from = u - start, to = units[head] < u1 - start ? units[head] : u1 - start, slot = 2 * w + (u != u0);
            if (from != 0 || to != units[head]) {
                CHECK(slot < 2 * W && used[slot]++ == 0);
                written[head].push_back(slot);
                if (from == 0) noted[head] = {slot, all.of(start + units[head] - 1) - w + 1};
            }
            u = start + to;
            start += units[head++];
            while (u < u1 && units[head] == 0) ++head;
        }
    }
    CHECK(written.size() == noted.size() && (int)written.size() < (W < (int)units.size() + 1 ? W + 1 : (int)units.size() + 1));
    for (const auto& [head, slots] : written) {
        CHECK((int)slots.size() == noted[head].second);
        for (size_t p = 0; p < slots.size(); ++p) CHECK(slots[p] == part_slot(noted[head].first, (int)p));
    }
}

int main() {
    for (unsigned bits = 0; bits < 0x8000; ++bits) {
        const float top = [&] { const unsigned u = bits << 16; float f; __builtin_memcpy(&f, &u, 4); return f; }();
        const int e = scale_of(bits);
        if (!std::isfinite(top)) { CHECK(e == 255); continue; }
        CHECK(e >= 2 && e <= 252);
        CHECK(e == 252 || (double)top <= 7 * std::ldexp(1.0, e - 127));
        CHECK(e == 2 || (double)top > 7 * std::ldexp(1.0, e - 128));
    }
    for (int D : {64, 128, 256})
        for (int log_p = 5; log_p <= 8; ++log_p) {
            PageView pv{};
            pv.log_p = log_p;
            pv.D = D;
            pv.n_pages = 3;
            const int P = pv.rows();
            const size_t at[] = {pv.k_codes(0), pv.v_codes(0), pv.k_scales(0), pv.v_scales(0), pv.page_bytes()}, row[] = {(size_t)D / 2, (size_t)D / 2, (size_t)D / 32, (size_t)D / 32};
            for (int i = 0; i < 4; ++i) CHECK(at[i] + P * row[i] == at[i + 1] && at[i] % 16 == 0);
            CHECK(pv.k_codes(P - 1) + row[0] == pv.v_codes(0) && pv.v_scales(P - 1) + row[3] == pv.page_bytes() && pv.page_bytes() == (size_t)P * D * 17 / 16);
            CHECK(pv.pages_of(0) == 0 && pv.pages_of(1) == 1 && pv.pages_of(P) == 1 && pv.pages_of(P + 1) == 2 && pv.pages_of(INT_MAX) == (int)((INT_MAX + (long long)P - 1) / P));
            CHECK(pv.is_page(0) && pv.is_page(2) && !pv.is_page(3) && !pv.is_page(-1) && !pv.is_page(INT_MIN));
        }
    std::mt19937 r(1);
    for (int n : {1, 2, 7, 1000, 65537, 1 << 30, INT_MAX - 1, INT_MAX})
        for (int k : {1, 2, 3, 7, 255, 256, 511, 512, 767, 768, 1023, 1024}) shares(n, k);
    for (int i = 0; i < 20000; ++i) shares((int)(r() % INT_MAX) + 1, (int)(r() % 1024) + 1);
    for (int i = 0; i < 3000; ++i) {
        std::vector<int> units(1 + r() % (i % 3 == 0 ? 5 : 300));
        for (int& n : units) n = r() % 3 == 0 ? 0 : (int)(r() % (i % 2 ? 4 : 200));
        parts(units, 1 + (int)(r() % 64));
    }
    return g_failed != 0;
}

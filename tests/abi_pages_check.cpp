// Host-side exercise of the entry points around the cache in pages for a sanitizer build (AddressSanitizer + UndefinedBehaviorSanitizer
// on the host code of the library): validation, size queries and planning, up to the largest sizes. No kernel is launched and no
// device memory is touched: every call either runs on the host only or is refused before its first HIP call.
// Built and run by tests/test_host_sanitizers_pages.py; exits 0 when every check holds.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <vector>

#include "audiokv.h"

static int g_failed = 0;
#define CHECK(cond)                                                          \
    do {                                                                     \
        if (!(cond)) {                                                       \
            std::fprintf(stderr, "FAILED %s:%d: %s (last error: %s)\n", __FILE__, __LINE__, #cond, audiokv_last_error()); \
            ++g_failed;                                                      \
        }                                                                    \
    } while (0)

static audiokv_params make(int hq, int hkv, int d) {
    audiokv_params p;
    std::memset(&p, 0, sizeof(p));
    p.size = sizeof(p);
    p.n_q_heads = hq; p.n_kv_heads = hkv; p.head_dim = d;
    p.pool_kernel = 1; p.causal = 1;
    return p;
}

int main() {
    const int geoms[][3] = {{28, 4, 128}, {16, 1, 256}, {8, 2, 64}, {1, 1, 64}};
    void* const ptr = reinterpret_cast<void*>(4096);       // never read
    int32_t* const ints = static_cast<int32_t*>(ptr);
    int accepted = 0, refused = 0;
    for (const auto& gm : geoms) {
        const audiokv_params p = make(gm[0], gm[1], gm[2]);
        for (int rows : {32, 64, 128, 256, 16, 0, -64, 2147483647}) {
            size_t page = 0;
            const bool good = rows == 32 || rows == 64 || rows == 128 || rows == 256;
            CHECK((audiokv_page_bytes(&p, rows, &page) == AUDIOKV_OK) == good);
            CHECK(!good || page == (size_t)rows * gm[2] / 16 * 17);
            for (int pages_of_pool : {1, 1000, 2147483647})
                for (int width : {1, 7, 512, 65535, 67108863, 2147483647})
                    for (int seqs : {1, 64, 262144, 1 << 20, 2147483647}) {
                        audiokv_pages c{sizeof(c), rows, pages_of_pool, width, ptr, ints, ints, ints, ints};
                        size_t a = 0, f = 0, k = 0, s = 0;
                        const int32_t rc = audiokv_pages_attend_workspace_bytes(&p, &c, seqs, &a);
                        CHECK(rc == audiokv_pages_fork_workspace_bytes(&p, &c, seqs, &f));
                        CHECK(rc == audiokv_pages_keep_workspace_bytes(&p, &c, seqs, 2147483647, &k));
                        CHECK(rc == audiokv_pages_append_workspace_bytes(&p, &c, seqs, 3, 2147483647, &s));
                        const long long heads = (long long)seqs * gm[1];
                        const bool fits = good && heads <= (1 << 20) && (long long)width * rows <= 2147483647LL && heads * width <= 2147483647LL / (rows / 32);
                        CHECK((rc == AUDIOKV_OK) == fits);
                        (fits ? accepted : refused) += 1;
                        if (!fits) continue;
                        CHECK(f >= (size_t)heads * (1 + (size_t)width) * 4 && a > 0 && k > 0 && s > 0);
                        CHECK(audiokv_pages_attend(&p, &c, seqs, ptr, ptr, nullptr, ptr, a - 1, nullptr) == AUDIOKV_E_WORKSPACE_TOO_SMALL);
                        CHECK(audiokv_pages_fork(&p, &c, seqs, ints, nullptr, ptr, f - 1, nullptr) == AUDIOKV_E_WORKSPACE_TOO_SMALL);
                        CHECK(audiokv_pages_keep(&p, &c, seqs, ints, ints, 2147483647, nullptr, ptr, k - 1, nullptr) == AUDIOKV_E_WORKSPACE_TOO_SMALL);
                        const std::vector<int32_t> lens = {5, 1, 70};
                        CHECK(audiokv_pages_append_workspace_bytes(&p, &c, seqs, 3, 76LL * gm[1], &s) == AUDIOKV_OK);
                        CHECK(audiokv_pages_append(&p, &c, seqs, ptr, ptr, nullptr, nullptr, 0, ints, lens.data(), 3, ints, nullptr, ptr, s - 1, nullptr) ==
                              AUDIOKV_E_WORKSPACE_TOO_SMALL);
                    }
        }
        // never shrinking
        audiokv_pages c{sizeof(c), 64, 100000, 300, ptr, ints, ints, ints, ints};
        size_t before = 0, now = 0;
        for (int64_t n = 0; n < 3000000; n += 9973) {
            CHECK(audiokv_pages_append_workspace_bytes(&p, &c, 40, 30, n, &now) == AUDIOKV_OK && now >= before);
            before = now;
        }
    }
    CHECK(accepted > 0 && refused > 0);
    if (g_failed) return 1;
    std::puts("all checks passed");
    return 0;
}

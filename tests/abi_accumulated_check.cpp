// Host-side exercise of the entry points around accumulated weights for a sanitizer build (AddressSanitizer +
// UndefinedBehaviorSanitizer on the host code of the library): validation, size queries and planning. No kernel is launched and
// no device memory is touched: every call either runs on the host only or is refused before its first HIP call.
// Built and run by tests/test_host_sanitizers_accumulated.py; exits 0 when every check holds.
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
    const int geoms[][3] = {{28, 4, 128}, {32, 4, 128}, {8, 2, 256}, {8, 2, 64}, {1, 1, 64}, {32, 1, 64}, {17, 1, 128}};
    void* const ptr = reinterpret_cast<void*>(4096);       // never read
    for (const auto& gm : geoms) {
        audiokv_params p = make(gm[0], gm[1], gm[2]);
        for (int causal = 0; causal < 2; ++causal) {
            p.causal = causal;
            // plans over many batches, the longest ones included
            for (int n = 1; n <= 40; n += 13)
                for (int top : {1, 90, 4000, 131072}) {
                    std::vector<int32_t> lens(n), queries(n);
                    for (int i = 0; i < n; ++i) {
                        lens[i] = i == 0 ? top : 1 + (i * 7919 + n * 104729) % top;
                        queries[i] = i % 3 == 0 ? lens[i] : i % 3 == 1 ? 0 : (i * 31) % (lens[i] + 1);
                    }
                    size_t bytes = 1;
                    CHECK(audiokv_accumulate_workspace_bytes(&p, n, lens.data(), queries.data(), &bytes) == AUDIOKV_OK && bytes > 0);
                    // refused behind the plan, in front of the launch
                    CHECK(audiokv_accumulate(&p, ptr, ptr, nullptr, static_cast<int32_t*>(ptr), lens.data(), static_cast<int32_t*>(ptr),
                                             queries.data(), n, static_cast<float*>(ptr), 0, ptr, bytes - 1, nullptr) == AUDIOKV_E_WORKSPACE_TOO_SMALL);
                    queries[0] = lens[0] + 1;
                    CHECK(audiokv_accumulate_workspace_bytes(&p, n, lens.data(), queries.data(), &bytes) == AUDIOKV_E_INVALID_ARG);
                }
        }
        for (int64_t rows : {0LL, 1LL, 127LL, 128LL, 100000LL, 2147483647LL})
            for (int seqs : {1, 3, 64, 700})
                for (int own : {0, 1, 64, 65, 5000, 2000000}) {
                    size_t bytes = 0;
                    const int32_t rc = audiokv_decode_shared_workspace_bytes(&p, rows > 0 ? 3 : 0, rows, seqs, seqs, own, &bytes);
                    CHECK(rc == AUDIOKV_OK && bytes > 0);
                    audiokv_slots s;
                    std::memset(&s, 0, sizeof(s));
                    s.size = sizeof(s);
                    s.capacity = own > 0 ? own : 1;
                    s.k = s.v = ptr;
                    s.lengths = static_cast<int32_t*>(ptr);
                    s.weights = static_cast<float*>(ptr);
                    CHECK(audiokv_decode_shared(&p, ptr, ptr, ptr, static_cast<int32_t*>(ptr), rows > 0 ? 3 : 0, rows, static_cast<int32_t*>(ptr), seqs,
                                                seqs, &s, own, nullptr, nullptr, nullptr, ptr, ptr, bytes - 1, nullptr) == AUDIOKV_E_WORKSPACE_TOO_SMALL);
                    size_t moves = 0;
                    CHECK(audiokv_evict_accumulated_workspace_bytes(&p, seqs, own, own / 2, &moves) == AUDIOKV_OK);
                    if (moves > 0)
                        CHECK(audiokv_evict_accumulated(&p, &s, seqs, own / 2, nullptr, 0, own, ptr, moves - 1, nullptr) == AUDIOKV_E_WORKSPACE_TOO_SMALL);
                    CHECK(audiokv_evict_accumulated(&p, &s, seqs, own / 2, nullptr, 1, own, ptr, moves, nullptr) == AUDIOKV_E_INVALID_ARG);   // no positions
                }
    }
    // sizes at which sums leave 32 bits, and counts that no launch holds
    audiokv_params p = make(8, 1, 64);
    size_t bytes = 0;
    const int32_t huge[2] = {INT32_MAX, INT32_MAX}, half[1] = {INT32_MAX / 2};
    CHECK(audiokv_accumulate_workspace_bytes(&p, 2, huge, huge, &bytes) == AUDIOKV_E_UNSUPPORTED);
    CHECK(audiokv_accumulate_workspace_bytes(&p, 1, half, half, &bytes) == AUDIOKV_E_UNSUPPORTED);
    CHECK(audiokv_decode_shared_workspace_bytes(&p, INT32_MAX, 5, 5, 5, 0, &bytes) == AUDIOKV_E_UNSUPPORTED);
    CHECK(audiokv_decode_shared_workspace_bytes(&p, 1, INT32_MAX, INT32_MAX, INT32_MAX, INT32_MAX, &bytes) == AUDIOKV_E_UNSUPPORTED);
    CHECK(audiokv_decode_shared_workspace_bytes(&p, 1, 1LL << 31, 5, 5, 0, &bytes) == AUDIOKV_E_INVALID_ARG);
    CHECK(audiokv_decode_shared_workspace_bytes(&p, 1, 100, 5, INT32_MAX, 0, &bytes) == AUDIOKV_OK);        // no more than there are
    CHECK(audiokv_evict_accumulated_workspace_bytes(&p, INT32_MAX, 5, 5, &bytes) == AUDIOKV_E_UNSUPPORTED);
    CHECK(audiokv_evict_accumulated_workspace_bytes(&p, 1, INT32_MAX, 0, &bytes) == AUDIOKV_OK);
    for (const audiokv_params* q : {static_cast<const audiokv_params*>(nullptr)}) {
        CHECK(audiokv_accumulate_workspace_bytes(q, 1, half, half, &bytes) == AUDIOKV_E_INVALID_ARG);
        CHECK(audiokv_decode_shared_workspace_bytes(q, 1, 1, 1, 1, 1, &bytes) == AUDIOKV_E_INVALID_ARG);
        CHECK(audiokv_evict_accumulated_workspace_bytes(q, 1, 1, 1, &bytes) == AUDIOKV_E_INVALID_ARG);
    }
    CHECK(audiokv_accumulate_workspace_bytes(&p, 1, half, half, nullptr) == AUDIOKV_E_INVALID_ARG);
    CHECK(audiokv_decode_shared_workspace_bytes(&p, 1, 1, 1, 1, 1, nullptr) == AUDIOKV_E_INVALID_ARG);
    CHECK(audiokv_evict_accumulated_workspace_bytes(&p, 1, 1, 1, nullptr) == AUDIOKV_E_INVALID_ARG);
    std::printf(g_failed ? "%d checks failed\n" : "all checks passed\n", g_failed);
    return g_failed ? 1 : 0;
}

// The largest numbers that the entry points around accumulated weights can be given, for a sanitizer build as in
// abi_accumulated_check.cpp: sizes are right or the call is refused, and no sum leaves its type on the way. No kernel is launched.
// Built and run by tests/test_accumulated_limits.py; exits 0 when every check holds.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <initializer_list>

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
    for (int d : {64, 128, 256}) {
        const audiokv_params p = make(8, 2, d);
        // own rows: a logit per query head and row is the least that a step needs, and more rows never need less
        for (int seqs : {1, 5, 1023, 1024, 1025, 5000}) {
            size_t before = 0;
            for (int64_t own = 1; own <= INT32_MAX; own += 1 + own / 3) {
                size_t bytes = 0;
                const int32_t rc = audiokv_decode_shared_workspace_bytes(&p, 0, 0, seqs, 0, (int32_t)own, &bytes);
                // (refused as well where a launch would have too many workgroups: 8388608, a thousand rows each)
                const bool many = (double)seqs * 2 * (own / 1024 + 1) >= 8000000.;
                CHECK(rc == AUDIOKV_OK ? own < (1 << 30) : rc == AUDIOKV_E_UNSUPPORTED && (many || own >= (1 << 30)));
                if (rc != AUDIOKV_OK) continue;
                CHECK(bytes >= (size_t)seqs * 8 * own * sizeof(float) && bytes >= before);
                before = bytes;
            }
            for (int64_t own : {(1LL << 30) - 1, 1LL << 30, (1LL << 31) - 64, (1LL << 31) - 1}) {
                size_t bytes = 0;
                const int32_t rc = audiokv_decode_shared_workspace_bytes(&p, 0, 0, seqs, 0, (int32_t)own, &bytes);
                CHECK(rc == AUDIOKV_OK ? own < (1 << 30) : rc == AUDIOKV_E_UNSUPPORTED);
                CHECK(rc == AUDIOKV_OK || own >= (1 << 30) || seqs > 1);
                if (rc == AUDIOKV_OK) CHECK(bytes >= (size_t)seqs * 8 * own * sizeof(float) && bytes >= before);
            }
        }
    }
    std::printf(g_failed ? "%d checks failed\n" : "all checks passed\n", g_failed);
    return g_failed ? 1 : 0;
}

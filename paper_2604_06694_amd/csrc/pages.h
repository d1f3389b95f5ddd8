// The cache in 4 bits and in pages (audiokv_pages): where things lie, and how rows are rounded and read. A header of its own
// because the limits, the walk over segments and fork's second launch are checked on the host as well (tests/pages_check.cpp,
// tests/pages_fork_check.cpp).
//
// A page holds P rows of one KV head: K's codes [P][D / 2], V's codes, K's scales [P][D / 32], V's scales. Rows of codes are 32 to
// 128 bytes, so that sections begin at multiples of 16 bytes whatever P (a multiple of 32) is.
#pragma once

#include "common.h"

namespace audiokv {

struct PageView {
    char* pool;
    int32_t *table, *lengths, *refs, *state;
    int n_pages, width, log_p;      // pages of the pool; entries of a head's table row; log2 of a page's rows
    int n_heads, H, D;

    __host__ __device__ int rows() const { return 1 << log_p; }
    __host__ __device__ size_t page_bytes() const { return (size_t)(D + D / 16) << log_p; }
    __host__ __device__ int pages_of(int n) const { return (int)(((long long)n + rows() - 1) >> log_p); }
    // Sections of a page, from its first byte
    __host__ __device__ size_t k_codes(int row) const { return (size_t)row * (D / 2); }
    __host__ __device__ size_t v_codes(int row) const { return ((size_t)(D / 2) << log_p) + (size_t)row * (D / 2); }
    __host__ __device__ size_t k_scales(int row) const { return ((size_t)D << log_p) + (size_t)row * (D / 32); }
    __host__ __device__ size_t v_scales(int row) const { return ((size_t)(D + D / 32) << log_p) + (size_t)row * (D / 32); }
    __host__ __device__ char* page(int p) const { return pool + (size_t)p * page_bytes(); }
    __host__ __device__ bool is_page(int p) const { return (unsigned)p < (unsigned)n_pages; }
    // Rows of a head. A length that its table row cannot hold is a caller's error; cut so that nothing is read past the row
    __device__ __forceinline__ int length(int head) const { return min(max(lengths[head], 0), width << log_p); }
};

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// The scale byte of a block whose largest magnitude has the bits `top` (bf16 without the sign): the smallest power of two s with
// top <= 7 s. 7 is in the middle of 6 and 8 and goes to 6, so that no value is further off than half a step of its neighbours.
// Added 0x1f carries into the exponent where the mantissa is beyond 1.75 = 7 / 4. Within 2 and 252, so that every value that codes
// stand for is a normal number of bf16 or zero; 255 with an infinity or NaN in the block.
__host__ __device__ __forceinline__ int scale_of(unsigned top) {
    const int e = (int)((top + 0x1f) >> 7) - 2;
    return top >= 0x7f80 ? 255 : e < 2 ? 2 : e > 252 ? 252 : e;
}

// How the units of attend are shared out (pages_attend.hip).
// n units in k shares: where share w begins, and which one has unit u. Spread evenly, so that equal heads and a multiple of their number of
// shares end together. In float64, where both are exact: numerators are below 2^42, and a quotient that is no whole number is at least
// 2^-31 away from one. (Divisions of 64-bit integers took 130 instructions each.)
struct Shares {
    int n, k;
    __host__ __device__ __forceinline__ int begin(int w) const { return (int)((double)n * w / k); }
    __host__ __device__ __forceinline__ int of(int u) const { return (int)((((double)u + 1) * k - 1) / n); }
};

// A workgroup has the parts of two heads at most, and a slot for each: 2 w for the one with which its share begins, 2 w + 1 for another.
// Part p of a head whose first part is in slot `first`: the others are the first of the workgroups behind.
__host__ __device__ __forceinline__ int part_slot(int first, int p) { return p == 0 ? first : (first & ~1) + 2 * p; }

// Largest g with cu[g] * times <= p (cu is a non-decreasing exclusive scan; p uniform). Every round probes 64 entries
// at equal distances, one per lane: one load latency for up to 64 of them, two up to 4096.
__device__ __forceinline__ int owner_of_row(const int32_t* __restrict__ cu, int n, int times, long long p) {
    int head = 0;
    for (int span = n; span > 1;) {
        const int step = (span + 63) >> 6;
        const int probe = head + (int)(threadIdx.x & 63) * step;
        const bool at_or_before = probe < head + span && (long long)cu[min(probe, n - 1)] * times <= p;
        const int k = __builtin_popcountll(__builtin_amdgcn_ballot_w64(at_or_before));   // a prefix of the lanes
        const int skip = k > 0 ? (k - 1) * step : 0;
        head += skip;
        span = min(step, span - skip);
    }
    return __builtin_amdgcn_readfirstlane(head);
}

// Sum over the threads before this one and, in `total`, over the workgroup, whose waves' sums go through `sums` (_once: LDS that nobody
// uses before or after).
template <int THREADS>
__device__ __forceinline__ int exclusive_sum_once(int x, int* sums, int& total) {
    const int incl = wave_incl(x), wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 63) sums[wave] = incl;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const int s = sums[w];
        before += w < wave ? s : 0;
        total += s;
    }
    return before + incl - x;
}
template <int THREADS>
__device__ __forceinline__ int exclusive_sum(int x, int* sums, int& total) {
    __syncthreads();
    return exclusive_sum_once<THREADS>(x, sums, total);
}

// What append and keep plan on the device, by one workgroup: which pages the heads get.
//
// A round of the search for pages with refs 0 looks at U * THREADS of them, a wave at U * 64 in a row, and begins at state[1]. The first
// round's counts are loaded ahead (PageSearch), since where it begins is known before how many are wanted.
template <int THREADS, int U>
struct PageSearch {
    int begin, page[U], refs[U];

    __device__ __forceinline__ void load(const PageView& pv, int base) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned n = pv.n_pages, i = base + ((threadIdx.x >> 6) * U + u) * 64 + (threadIdx.x & 63);      // (below 2^31 + THREADS * U)
            const bool there = i < n;
            unsigned p = begin + i;
            p -= p >= n ? n : 0;
            page[u] = there ? p : 0;
            refs[u] = pv.refs[page[u]];
            refs[u] = there ? refs[u] : 1;
        }
    }
    __device__ __forceinline__ PageSearch(const PageView& pv, int from) : begin(min(max(from, 0), pv.n_pages - 1)) { load(pv, 0); }

    // The first `want` free pages, in the order in which they are looked at, to found[]. Returns how many there were, `want` at most, and
    // in `next` where the following search begins. Fewer than `want`: the state said that there were more; the caller wants that many
    // then, and calls again. sums: THREADS / 64 + 1 ints of LDS. (A barrier before the first and after the last use of LDS.)
    __device__ int find(const PageView& pv, int want, int32_t* __restrict__ found, int* sums, int& next) {
        constexpr int WAVES = THREADS / 64;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        int have = 0;
        for (int base = 0; have < want; ) {
            unsigned long long free_in[U];
            int mine = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                free_in[u] = __builtin_amdgcn_ballot_w64(refs[u] == 0);
                mine += __builtin_popcountll(free_in[u]);
            }
            __syncthreads();
            if (lane == 0) sums[wave] = mine;
            __syncthreads();
            int at = have, total = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const int n = sums[w];
                at += w < wave ? n : 0;
                total += n;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int to = __builtin_amdgcn_mbcnt_hi((unsigned)(free_in[u] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)free_in[u], at));
                if (refs[u] == 0 && to < want) {
                    found[to] = page[u];
                    if (to == want - 1) sums[WAVES] = page[u];
                }
                at += __builtin_popcountll(free_in[u]);
            }
            have += total;
            if (pv.n_pages - base <= THREADS * U) break;
            base += THREADS * U;
            if (have < want) load(pv, base);
        }
        __syncthreads();
        next = begin;
        if (want > 0 && have >= want) next = sums[WAVES] + 1 == pv.n_pages ? 0 : sums[WAVES] + 1;
        if (have < want) load(pv, 0);
        return min(have, want);
    }
};

// Pages of a thread in a round: rounds come one after the other, and what a round does for its pages is vector work of one CU. Kernel times
// with 1, 2, 4 and 8 pages a thread of 256: 192 heads that get three pages 4.0, 4.0, 4.2, 4.4 us, the same in a pool of 8000 with 100 free
// ones behind the rest 17.3, 12.1, 8.9, 7.3, a keep of 112 heads 7.9, 6.7, 6.2, 6.4. With 4, 8 and 16 a thread of 1024: 64 heads that get
// 4300 pages 10.0, 8.9, 9.6, 112 heads that get 5800 7.3, 7.1, 9.1.
template <int THREADS> constexpr int kLooked = THREADS == 256 ? 4 : 8;

// What fork's first launch leaves for its second, in the workspace.
struct ForkSpace {
    int2* rows;             // [heads]: length before and after the call
    int32_t* entries;       // [heads][width]: table after the call, as far as it is not what it was
};

// What one of a head's threads does in fork's second launch. On the host as well, because threads run in any order and one of them writes
// the length (tests/pages_fork_check.cpp): the length before the call comes from the workspace. owner_goes(page): is the page free now?
// Returns how many are.
template <class OwnerGoes>
__host__ __device__ __forceinline__ int fork_give(const PageView& pv, const ForkSpace& f, const int32_t* parents, int n_seqs, int head,
                                                  int thread, int threads, OwnerGoes owner_goes) {
    const int x = head / pv.H, parent = parents ? parents[x] : x;
    const bool same = parent == x || (unsigned)parent >= (unsigned)n_seqs;      // no entry changes, some may go
    const int was = f.rows[head].x, rows = f.rows[head].y;
    const int had = pv.pages_of(was), has = pv.pages_of(rows), last = had > has ? had : has;
    int32_t* mine = pv.table + (size_t)head * pv.width;
    int freed = 0;
    for (int j = thread; j < last; j += threads) {
        const int now = j < has ? same ? mine[j] : f.entries[(size_t)head * pv.width + j] : -1;
        if (j < had) {
            const int page = mine[j];
            if (page != now && pv.is_page(page)) freed += owner_goes(page);
        }
        if (j < has && !same) mine[j] = now;
    }
    if (rows != was && thread == 0) pv.lengths[head] = rows;
    return freed;
}

inline size_t up256(size_t bytes) { return (bytes + 255) & ~(size_t)255; }    // parts of a workspace begin at multiples of 256 bytes

// Part of a workspace; without one (a size is asked for) there is no address.
template <class T> T* part_at(void* workspace, size_t offset) {
    return workspace ? reinterpret_cast<T*>(static_cast<char*>(workspace) + offset) : nullptr;
}

// CALL with kD, the head's channels, a constant
#define AUDIOKV_FOR_DIM(D, CALL)                                 \
    switch (D) {                                                 \
        case 64: { constexpr int kD = 64; CALL; break; }         \
        case 128: { constexpr int kD = 128; CALL; break; }       \
        case 256: { constexpr int kD = 256; CALL; break; }       \
        default: return hipErrorInvalidValue;                    \
    }

// ---- launchers ---------------------------------------------------------------------------------------------------------------------

struct AppendCall {
    const void *k, *v;
    const int32_t *indices, *cu_budgets, *cu_seqlens, *seqs;
    int n_items, n_seqs, same_length;       // same_length: tokens of every item, 0: they differ
    long long total_rows;
    int32_t* refused;
};
size_t pages_append_bytes(const PageView& pv, int n_seqs, int n_items, long long total_rows);
hipError_t launch_pages_append(const Geom& g, const PageView& pv, const AppendCall& c, void* workspace, hipStream_t s);
hipError_t launch_pages_read(const PageView& pv, const int32_t* first, const int32_t* cu_rows, long long total_rows, void* k_out,
                             void* v_out, hipStream_t s);
size_t pages_fork_bytes(const PageView& pv);
hipError_t launch_pages_fork(const PageView& pv, const int32_t* parents, const int32_t* drop, void* workspace, hipStream_t s);
size_t pages_keep_bytes(const PageView& pv, long long total_rows);
hipError_t launch_pages_keep(const PageView& pv, const int32_t* indices, const int32_t* cu_budgets, long long total_rows,
                             int32_t* refused, void* workspace, hipStream_t s);
size_t pages_attend_bytes(const Geom& g, const PageView& pv);
hipError_t launch_pages_attend(const Geom& g, const PageView& pv, const void* q, void* out, float* lse, void* workspace, hipStream_t s);

}  // namespace audiokv

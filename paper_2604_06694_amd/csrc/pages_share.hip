// Pages that sequences take over, share and give back (audiokv_pages_fork), and heads cut to given rows (audiokv_pages_keep).
// No arithmetic: table entries and counts, and for keep the kept rows' bytes.
//
// fork is two launches over the table, because a sequence may take over pages of one whose own entries change in the same call: the
// first lists every new entry and every length in the workspace and counts the pages' new owners, the second takes away the old owners and
// writes table and lengths (fork_give in pages.h). A page is free when its last owner goes, which only the second launch can bring about, once for every page: what it adds to
// state[0] does not depend on the order. Entries that stay as they are touch no count (after a reorder of beams that share their
// prompt nearly all do), which spares the atomics on pages that many sequences have.
//
// keep is three launches: one workgroup decides who gets which pages; the kept rows are copied into them, the table still as it was;
// the table and the counts change. Whole pages whose rows are all kept, from the first on, stay (and stay shared).
#include "pages.h"

namespace audiokv {

namespace {

constexpr int kThreads = 256, kPlanThreads = 1024;

// ---- fork --------------------------------------------------------------------------------------------------------------------------

ForkSpace fork_space(const PageView& pv, void* workspace, size_t* bytes) {
    ForkSpace f;
    f.rows = static_cast<int2*>(workspace);
    const size_t at = up256((size_t)pv.n_heads * sizeof(int2));
    f.entries = part_at<int32_t>(workspace, at);
    if (bytes) *bytes = at + up256((size_t)pv.n_heads * pv.width * 4);
    return f;
}

// One workgroup per head, in both launches.
__global__ __launch_bounds__(kThreads) void fork_take_kernel(PageView pv, const int32_t* __restrict__ parents,
                                                             const int32_t* __restrict__ drop, int n_seqs, ForkSpace f)
{
    const int head = blockIdx.x, x = head / pv.H, h = head - x * pv.H;
    const int parent = parents ? parents[x] : x;
    const bool taken = (unsigned)parent < (unsigned)n_seqs;
    const int from = taken ? parent * pv.H + h : head;
    const int was = pv.length(head), rows = taken ? max(pv.length(from) - (drop ? max(drop[x], 0) : 0), 0) : 0;
    if (threadIdx.x == 0) f.rows[head] = int2{was, rows};
    if (from == head) return;                              // its own pages, or none
    const int had = pv.pages_of(was), has = pv.pages_of(rows);
    const int32_t *mine = pv.table + (size_t)head * pv.width, *theirs = pv.table + (size_t)from * pv.width;
    for (int j = threadIdx.x; j < has; j += kThreads) {
        const int page = theirs[j];
        f.entries[(size_t)head * pv.width + j] = page;
        if (pv.is_page(page) && (j >= had || mine[j] != page)) atomicAdd(&pv.refs[page], 1);
    }
}

__global__ __launch_bounds__(kThreads) void fork_give_kernel(PageView pv, const int32_t* __restrict__ parents, int n_seqs, ForkSpace f)
{
    int freed = fork_give(pv, f, parents, n_seqs, blockIdx.x, threadIdx.x, kThreads, [&](int page) { return atomicSub(&pv.refs[page], 1) == 1; });
    freed = wave_incl(freed);
    if ((threadIdx.x & 63) == 63 && freed > 0) atomicAdd(&pv.state[0], freed);
}

// Both for small tables, U entries a thread of one workgroup: what the first launch lists is in registers here. (Entries of tables, us by
// the two kernels and by this one: 272 3.4 + 3.2, 2.8; 1024 3.4 + 3.2, 3.9; 2048 3.7 + 3.2, 6.5, and a launch less; 4096 3.6 + 3.3, 14.)
constexpr int kForkEntries = 2;

template <int U>
__global__ __launch_bounds__(kPlanThreads) void fork_small_kernel(PageView pv, const int32_t* __restrict__ parents,
                                                                  const int32_t* __restrict__ drop, int n_seqs)
{
    const int entries = pv.n_heads * pv.width;
    int rows[U], was[U], mine[U], theirs[U];
    bool goes[U], comes[U];          // its owner before the call, after it
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int e = min((int)threadIdx.x + u * kPlanThreads, entries - 1), head = e / pv.width, j = e - head * pv.width;
        const int x = head / pv.H, h = head - x * pv.H;
        const int parent = parents ? parents[x] : x;
        const bool taken = (unsigned)parent < (unsigned)n_seqs;
        const int from = taken ? parent * pv.H + h : head;
        was[u] = pv.length(head);
        rows[u] = taken ? max(pv.length(from) - (drop ? max(drop[x], 0) : 0), 0) : 0;
        mine[u] = pv.table[e];
        theirs[u] = pv.table[(size_t)from * pv.width + j];
        const bool had = j < pv.pages_of(was[u]), has = j < pv.pages_of(rows[u]), stays = had && has && mine[u] == theirs[u];
        goes[u] = had && !stays && pv.is_page(mine[u]);
        comes[u] = has && !stays;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
        if ((int)threadIdx.x + u * kPlanThreads < entries && comes[u] && pv.is_page(theirs[u])) atomicAdd(&pv.refs[theirs[u]], 1);
    __syncthreads();          // all new owners are counted, and all of the table is read
    int freed = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int e = threadIdx.x + u * kPlanThreads;
        if (e >= entries) break;
        if (goes[u]) freed += atomicSub(&pv.refs[mine[u]], 1) == 1;
        if (comes[u]) pv.table[e] = theirs[u];
        const int head = e / pv.width;
        if (e == head * pv.width && rows[u] != was[u]) pv.lengths[head] = rows[u];
    }
    freed = wave_incl(freed);
    if ((threadIdx.x & 63) == 63 && freed > 0) atomicAdd(&pv.state[0], freed);
}

// ---- keep --------------------------------------------------------------------------------------------------------------------------

struct KeepJob {
    int rows;               // kept: the length after the call; -1: the head stays as it is
    int same;               // whole pages that stay
    int first;              // where its new pages begin in the list
    int had;                // rows before
};
struct KeepSpace {
    KeepJob* jobs;
    int32_t* found;
    int most;
};
KeepSpace keep_space(const PageView& pv, long long total_rows, void* workspace, size_t* bytes) {
    KeepSpace a;
    a.jobs = static_cast<KeepJob*>(workspace);
    const size_t at = up256((size_t)pv.n_heads * sizeof(KeepJob));
    a.found = part_at<int32_t>(workspace, at);
    const long long n = (total_rows >> pv.log_p) + pv.n_heads;       // a head's last page may be begun
    a.most = (int)(n < pv.n_pages ? n : pv.n_pages);
    if (bytes) *bytes = at + up256((size_t)a.most * 4);
    return a;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void keep_plan_kernel(PageView pv, const int32_t* __restrict__ indices,
                                                                 const int32_t* __restrict__ cu_b, int total_rows, KeepSpace a,
                                                                 int32_t* __restrict__ refused)
{
    __shared__ int sums[THREADS / 64 + 1];
    __shared__ int served_pages, lost;
    const int tid = threadIdx.x, P = pv.rows();
    PageSearch<THREADS, kLooked<THREADS>> search(pv, pv.state[1]);
    if (tid == 0) served_pages = lost = 0;
    const int n_free = min(max(pv.state[0], 0), a.most);
    int running = 0;
    for (int base = 0; base < pv.n_heads; base += THREADS) {
        const int head = base + tid;
        KeepJob job{-1, 0, 0, 0};
        int need = 0;
        if (head < pv.n_heads) {
            const int begin = min(max(cu_b[head], 0), total_rows), rows = max(min(cu_b[head + 1], total_rows) - begin, 0);
            job.had = pv.length(head);
            if (rows < job.had) {
                job.rows = rows;
                // Rows come in order, none twice: where row r is index r, the ones before are theirs, too. The first page and the
                // last are asked together, for heads that keep a choice of their rows have no whole page, and heads that lose the
                // last ones only such (64 heads of 8000 rows 9.6 -> 8.2 us).
                const int32_t* mine = indices + begin;
                const auto whole = [&](int pages) { return mine[pages * P - 1] == pages * P - 1; };
                int lo = 0, hi = rows >> pv.log_p;
                if (hi > 0) {
                    const bool first = whole(1), all = whole(hi);
                    lo = all ? hi : first;
                    hi = all || !first ? lo : hi - 1;
                }
                while (lo < hi) {
                    const int mid = (lo + hi + 1) >> 1;
                    if (whole(mid)) lo = mid;
                    else hi = mid - 1;
                }
                job.same = lo;
                need = pv.pages_of(rows) - lo;
            }
        }
        int total;
        job.first = running + exclusive_sum<THREADS>(need, sums, total);
        running += total;
        // Heads are served while the free pages last.
        if (job.first + need <= n_free) {
            if (need > 0) atomicMax(&served_pages, job.first + need);
        } else if (need > 0) {
            job.rows = -1;
            atomicAdd(&lost, 1);
        }
        if (head < pv.n_heads) a.jobs[head] = job;
    }
    __syncthreads();
    int next, have;
    for (;;) {
        const int want = served_pages;
        have = search.find(pv, want, a.found, sums, next);
        if (have == want) break;
        if (tid == 0) served_pages = 0;      // (the state promised more)
        __syncthreads();
        for (int head = tid; head < pv.n_heads; head += THREADS) {
            const KeepJob job = a.jobs[head];
            const int end = job.first + (job.rows < 0 ? 0 : pv.pages_of(job.rows) - job.same);
            if (job.rows < 0 || end == job.first) continue;
            if (end <= have) {
                atomicMax(&served_pages, end);
            } else {
                a.jobs[head].rows = -1;
                atomicAdd(&lost, 1);
            }
        }
        __syncthreads();
    }
    __syncthreads();
    if (tid == 0) {
        pv.state[0] -= have;
        pv.state[1] = next;
        if (refused) *refused = lost;
    }
}

// A row as it is held, D / 32 lanes to it: a block's codes and scale of K and V each. Rows are numbered within their head.
template <int D>
struct HeldRow {
    u32x4 k, v;
    char ks, vs;
    __device__ __forceinline__ void load(const PageView& pv, int page, int row, int lane) {
        const char* s = pv.page(pv.is_page(page) ? page : 0);
        row &= pv.rows() - 1;
        k = *reinterpret_cast<const u32x4*>(s + pv.k_codes(row) + lane * 16);
        v = *reinterpret_cast<const u32x4*>(s + pv.v_codes(row) + lane * 16);
        ks = s[pv.k_scales(row) + lane];
        vs = s[pv.v_scales(row) + lane];
    }
    __device__ __forceinline__ void store(const PageView& pv, int page, int row, int lane) const {
        char* d = pv.page(page);
        row &= pv.rows() - 1;
        *reinterpret_cast<u32x4*>(d + pv.k_codes(row) + lane * 16) = k;
        *reinterpret_cast<u32x4*>(d + pv.v_codes(row) + lane * 16) = v;
        d[pv.k_scales(row) + lane] = ks;
        d[pv.v_scales(row) + lane] = vs;
    }
};

// The kept rows into the new pages, consecutive rows to a workgroup. (A row in a page that stays has nothing to do.)
template <int D>
__global__ __launch_bounds__(kThreads) void keep_move_kernel(PageView pv, const int32_t* __restrict__ indices,
                                                             const int32_t* __restrict__ cu_b, long long first_row,
                                                             long long total_rows, KeepSpace a)
{
    constexpr int LANES = D / 32, ROWS = kThreads / LANES;
    const int lane = threadIdx.x % LANES;
    const long long row0 = first_row + (long long)blockIdx.x * ROWS;
    const long long r = row0 + threadIdx.x / LANES;
    int head = owner_of_row(cu_b, pv.n_heads, 1, row0);
    const long long rc = min(r, total_rows - 1);
    while (head + 1 < pv.n_heads && cu_b[head + 1] <= rc) ++head;
    const KeepJob job = a.jobs[head];
    const int t = (int)(rc - cu_b[head]), slot = t >> pv.log_p;
    if (r >= total_rows || t < 0 || t >= job.rows || slot < job.same) return;
    const int at = min(max(indices[rc], 0), job.had - 1);              // an index outside is a caller error; cut
    const int from = pv.table[(size_t)head * pv.width + (at >> pv.log_p)], to = a.found[job.first + slot - job.same];
    if (!pv.is_page(from) || !pv.is_page(to)) return;
    HeldRow<D> row;
    row.load(pv, from, at, lane);
    row.store(pv, to, t, lane);
}

// The table's new entries, refs and length of a head; `before` its entries until then.
__device__ __forceinline__ void commit_head(const PageView& pv, const KeepSpace& a, const KeepJob& job, int head, const int32_t* before) {
    int32_t* mine = pv.table + (size_t)head * pv.width;
    const int had = pv.pages_of(job.had), has = pv.pages_of(job.rows);
    int freed = 0;
    for (int j = job.same + threadIdx.x; j < had; j += blockDim.x) {
        const int page = before[j];
        if (pv.is_page(page)) freed += atomicSub(&pv.refs[page], 1) == 1;
        if (j < has) {
            const int now = a.found[job.first + j - job.same];
            mine[j] = now;
            if (pv.is_page(now)) pv.refs[now] = 1;
        }
    }
    if (threadIdx.x == 0) pv.lengths[head] = job.rows;
    freed = wave_incl(freed);
    if ((threadIdx.x & 63) == 63 && freed > 0) atomicAdd(&pv.state[0], freed);
}

__global__ __launch_bounds__(kThreads) void keep_table_kernel(PageView pv, KeepSpace a)
{
    const KeepJob job = a.jobs[blockIdx.x];
    if (job.rows >= 0) commit_head(pv, a, job, blockIdx.x, pv.table + (size_t)blockIdx.x * pv.width);
}

// Both for heads whose tables hold kWholeRows rows at most, a workgroup each: the old entries wait in LDS, and no other workgroup reads
// them. (16 heads of 1100 rows: 3.5 + 3.2 us by the two kernels, 6.2 by this one, 256 of 2000 16.8 + 5.0 and 17.0.)
constexpr long long kWholeRows = 2048;
constexpr int kWholeThreads = 512;

template <int D>
__global__ __launch_bounds__(kWholeThreads) void keep_whole_kernel(PageView pv, const int32_t* __restrict__ indices,
                                                                   const int32_t* __restrict__ cu_b, KeepSpace a)
{
    constexpr int LANES = D / 32;
    __shared__ int32_t before[kWholeRows / 32];
    const int head = blockIdx.x, lane = threadIdx.x % LANES;
    const KeepJob job = a.jobs[head];
    const int begin = max(cu_b[head], 0);
    if (job.rows < 0) return;
    for (int j = threadIdx.x; j < pv.pages_of(job.had); j += kWholeThreads) before[j] = pv.table[(size_t)head * pv.width + j];
    __syncthreads();
    constexpr int U = 4, STEP = kWholeThreads / LANES;                   // rows of a thread on their way
    for (int t0 = (job.same << pv.log_p) + threadIdx.x / LANES; t0 < job.rows; t0 += U * STEP) {
        int at[U], to[U];
        HeldRow<D> row[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = min(t0 + u * STEP, job.rows - 1);
            at[u] = min(max(indices[begin + t], 0), job.had - 1);
            to[u] = a.found[job.first + (t >> pv.log_p) - job.same];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) row[u].load(pv, before[at[u] >> pv.log_p], at[u], lane);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t0 + u * STEP < job.rows && pv.is_page(before[at[u] >> pv.log_p]) && pv.is_page(to[u])) row[u].store(pv, to[u], t0 + u * STEP, lane);
    }
    commit_head(pv, a, job, head, before);
}

}  // namespace

size_t pages_fork_bytes(const PageView& pv) {
    size_t bytes;
    fork_space(pv, nullptr, &bytes);
    return bytes;
}

hipError_t launch_pages_fork(const PageView& pv, const int32_t* parents, const int32_t* drop, void* workspace, hipStream_t s)
{
    const ForkSpace f = fork_space(pv, workspace, nullptr);
    const int n_seqs = pv.n_heads / pv.H;
    const long long entries = (long long)pv.n_heads * pv.width;
    if (entries <= kForkEntries * kPlanThreads) {
        if (entries <= kPlanThreads) hipLaunchKernelGGL(fork_small_kernel<1>, dim3(1), dim3(kPlanThreads), 0, s, pv, parents, drop, n_seqs);
        else hipLaunchKernelGGL(fork_small_kernel<kForkEntries>, dim3(1), dim3(kPlanThreads), 0, s, pv, parents, drop, n_seqs);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(fork_take_kernel, dim3(pv.n_heads), dim3(kThreads), 0, s, pv, parents, drop, n_seqs, f);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(fork_give_kernel, dim3(pv.n_heads), dim3(kThreads), 0, s, pv, parents, n_seqs, f);
    return hipGetLastError();
}

size_t pages_keep_bytes(const PageView& pv, long long total_rows) {
    size_t bytes;
    keep_space(pv, total_rows, nullptr, &bytes);
    return bytes;
}

hipError_t launch_pages_keep(const PageView& pv, const int32_t* indices, const int32_t* cu_budgets, long long total_rows,
                             int32_t* refused, void* workspace, hipStream_t s)
{
    const KeepSpace a = keep_space(pv, total_rows, workspace, nullptr);
    // (fewer waves meet sooner at the barriers: 16 heads of 1100 rows 3.5 us by 256 threads, 4.6 by 1024, 64 of 500 5.2, 6.2)
    if (pv.n_heads <= 256 && a.most <= 2048)
        hipLaunchKernelGGL(keep_plan_kernel<256>, dim3(1), dim3(256), 0, s, pv, indices, cu_budgets, (int)total_rows, a, refused);
    else
        hipLaunchKernelGGL(keep_plan_kernel<kPlanThreads>, dim3(1), dim3(kPlanThreads), 0, s, pv, indices, cu_budgets, (int)total_rows, a, refused);
    hipError_t e = hipGetLastError();
    if ((long long)pv.width << pv.log_p <= kWholeRows) {
        if (e != hipSuccess) return e;
        AUDIOKV_FOR_DIM(pv.D, hipLaunchKernelGGL(keep_whole_kernel<kD>, dim3(pv.n_heads), dim3(kWholeThreads), 0, s, pv, indices, cu_budgets, a))
        return hipGetLastError();
    }
    const int rows_per_block = kThreads / (pv.D / 32);
    const long long slab = (long long)rows_per_block << 22;
    for (long long first = 0; first < total_rows && e == hipSuccess; first += slab) {
        const long long rows = total_rows - first < slab ? total_rows - first : slab;
        const dim3 grid((unsigned)((rows + rows_per_block - 1) / rows_per_block));
        AUDIOKV_FOR_DIM(pv.D, hipLaunchKernelGGL(keep_move_kernel<kD>, grid, dim3(kThreads), 0, s, pv, indices, cu_budgets, first,
                                                 total_rows, a))
        e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(keep_table_kernel, dim3(pv.n_heads), dim3(kThreads), 0, s, pv, a);
    return hipGetLastError();
}

}  // namespace audiokv

// Rows into the cache in 4 bits and back (audiokv_pages_append, audiokv_pages_read).
//
// append is two launches. The first, one workgroup, decides: which items take part (a sequence named twice: the first), how many
// pages every head needs, which items the pool has pages for, and which pages those are; it counts lengths, shared pages and free ones.
// The second writes: rows, rounded to 4 bits, the table's new entries and the rows of shared pages that are copied. What the first
// reads of table and lengths and the second needs goes through a job per head, so that no launch reads what it writes.
//
// Bound: the rows' bytes (bf16 in, 17/16 byte a channel of K and V out), below some thousand rows the first launch's chain of loads
// (lengths -> table -> refs -> refs of the pool) and barriers. A row is D / 8 lanes, 8 channels of K and of V each: whole cache lines
// as they come, and the largest of a block of 32 is two exchanges between neighbouring lanes. Conversions are the hardware's, which
// round as the format says (nearest, in the middle to the even code, beyond 6 to 6; all bf16 values compared at eight scales).
#include "pages.h"

namespace audiokv {

namespace {

constexpr int kThreads = 256, kPlanThreads = 1024;

struct AppendJob {
    int start, rows;        // where the head's new rows begin, how many (0: nothing to do)
    int copy_from;          // the page to copy rows from, -1: none
    int first;              // where its new pages begin in the list
};

struct AppendSpace {
    AppendJob* jobs;        // [heads of items]
    int32_t *bad, *owner;   // [items]: does not fit its table rows; [sequences]: the item that it belongs to
    int32_t* found;         // pages
    int most;               // of them
};

// New pages of a call at most: a head has one begun page and a copied one beside those that its rows fill.
__host__ long long most_pages(const PageView& pv, long long heads, long long total_rows) {
    const long long n = (total_rows >> pv.log_p) + 2 * heads;
    return n < pv.n_pages ? n : pv.n_pages;
}

AppendSpace append_space(const PageView& pv, int n_seqs, int n_items, long long total_rows, void* workspace, size_t* bytes) {
    AppendSpace a{};
    const long long heads = (long long)n_items * pv.H;
    a.most = (int)most_pages(pv, heads, total_rows);
    char* at = static_cast<char*>(workspace);
    a.jobs = reinterpret_cast<AppendJob*>(at);
    size_t off = up256((size_t)heads * sizeof(AppendJob));
    a.bad = reinterpret_cast<int32_t*>(at + off);
    off += up256((size_t)n_items * 4);
    a.owner = reinterpret_cast<int32_t*>(at + off);
    off += up256((size_t)n_seqs * 4);
    a.found = reinterpret_cast<int32_t*>(at + off);
    off += up256((size_t)a.most * 4);
    if (bytes) *bytes = off;
    return a;
}

// Rows that head g (of items) gets.
__device__ __forceinline__ int rows_of(const int32_t* __restrict__ cu_b, const int32_t* __restrict__ cu_seq, int H, int g, int total_rows) {
    if (cu_b) return max(min(cu_b[g + 1], total_rows) - min(max(cu_b[g], 0), total_rows), 0);
    const int i = g / H;
    return max(cu_seq[i + 1] - cu_seq[i], 0);
}

__global__ __launch_bounds__(kPlanThreads) void append_plan_kernel(
    PageView pv, const int32_t* __restrict__ cu_b, const int32_t* __restrict__ cu_seq, const int32_t* __restrict__ seqs, int n_items,
    int n_seqs, int total_rows, AppendSpace a, int32_t* __restrict__ refused)
{
    __shared__ int sums[4 * kPlanThreads / 64];
    __shared__ int served_pages, lost, freed;
    const int tid = threadIdx.x, H = pv.H, heads = n_items * H;
    if (tid == 0) served_pages = lost = freed = 0;
    for (int i = tid; i < n_items; i += kPlanThreads) a.bad[i] = 0;
    if (seqs) {
        for (int x = tid; x < n_seqs; x += kPlanThreads) a.owner[x] = INT_MAX;
        __syncthreads();
        for (int i = tid; i < n_items; i += kPlanThreads)
            if ((unsigned)seqs[i] < (unsigned)n_seqs) atomicMin(&a.owner[seqs[i]], i);
    }
    __syncthreads();
    auto sequence = [&](int item) {          // of an item that takes part, or -1
        if (!seqs) return item;
        const int x = seqs[item];
        return (unsigned)x < (unsigned)n_seqs && a.owner[x] == item ? x : -1;
    };
    // what every head needs; `first` holds the number of pages until they are numbered
    for (int g = tid; g < heads; g += kPlanThreads) {
        const int item = g / H, x = sequence(item);
        AppendJob job{0, 0, -1, 0};
        const int rows = rows_of(cu_b, cu_seq, H, g, total_rows);
        if (x >= 0 && rows > 0) {
            const int head = x * H + g - item * H;
            const int start = pv.length(head);
            const long long end = (long long)start + rows;
            if (end > (long long)pv.width << pv.log_p) {
                a.bad[item] = 1;
            } else {
                int first = pv.pages_of(start);
                if (start & (pv.rows() - 1)) {
                    const int page = pv.table[(size_t)head * pv.width + (start >> pv.log_p)];
                    if (pv.is_page(page) && pv.refs[page] > 1) {
                        job.copy_from = page;
                        --first;
                    }
                }
                job.start = start;
                job.rows = rows;
                job.first = pv.pages_of((int)end) - first;
            }
        }
        a.jobs[g] = job;
    }
    __syncthreads();
    // pages numbered in the order of the heads
    int running = 0;
    for (int base = 0; base < heads; base += kPlanThreads) {
        const int g = base + tid;
        const int need = g < heads && !a.bad[g / H] ? a.jobs[g].first : 0;
        int total;
        const int before = exclusive_sum<kPlanThreads>(need, sums, total);
        if (g < heads) a.jobs[g].first = running + before;
        running += total;
    }
    __syncthreads();
    // Items are served while the free pages last: the ends of their pages do not fall.
    const int n_free = min(max(pv.state[0], 0), a.most);
    const int really_free = max(pv.state[0], 0);
    auto end_of = [&](int item) { return item + 1 < n_items ? a.jobs[(item + 1) * H].first : running; };
    auto served = [&](int item) {
        const int end = end_of(item);
        return !a.bad[item] && (end <= n_free || end == a.jobs[item * H].first);
    };
    for (int i = tid; i < n_items; i += kPlanThreads)
        if (end_of(i) <= n_free) atomicMax(&served_pages, end_of(i));
    __syncthreads();
    const int want = served_pages;
    int next;
    const int have = find_pages<kPlanThreads>(pv, want, a.found, sums, next);
    // lengths, and what shared pages lose: after the search, so that a page which is still to be copied is not handed out
    __syncthreads();
    for (int g = tid; g < heads; g += kPlanThreads) {
        const int item = g / H, x = sequence(item);
        AppendJob job = a.jobs[g];
        if (!served(item)) {
            if (x >= 0 && rows_of(cu_b, cu_seq, H, g, total_rows) > 0) atomicAdd(&lost, 1);
            a.bad[item] = 1;      // (for the loop below)
        } else if (job.rows > 0) {
            pv.lengths[x * H + g - item * H] = job.start + job.rows;
            if (job.copy_from >= 0 && atomicSub(&pv.refs[job.copy_from], 1) == 1) atomicAdd(&freed, 1);
        }
    }
    __syncthreads();
    for (int g = tid; g < heads; g += kPlanThreads)
        if (a.bad[g / H]) a.jobs[g].rows = 0;
    if (tid == 0) {
        pv.state[0] = really_free - have + freed;
        pv.state[1] = next;
        if (refused) *refused = lost;
    }
}

// What 8 channels of a lane become: four bytes of codes, and the scale byte of the block, the same in the four lanes that hold it.
__device__ __forceinline__ unsigned round_to_4(u32x4 x, int& scale) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        top = max(top, x[i] & 0x7fff);
        top = max(top, (x[i] >> 16) & 0x7fff);
    }
    top = max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0xb1, 0xf, 0xf, false));      // lanes 1 0 3 2 of a quad
    top = max(top, (unsigned)__builtin_amdgcn_update_dpp(0, (int)top, 0x4e, 0xf, 0xf, false));      // lanes 2 3 0 1
    scale = scale_of(top);
    const float s = __uint_as_float((unsigned)scale << 23);
    unsigned codes = 0;
#if defined(__HIP_DEVICE_COMPILE__)
    const auto pair = [](unsigned w) { return __builtin_bit_cast(bf16x2, w); };      // (of a vector's element itself, it takes the first)
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, pair(x[0]), s, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, pair(x[1]), s, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, pair(x[2]), s, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, pair(x[3]), s, 3);
#endif
    return scale == 255 ? 0 : codes;
}

// Workgroups up to `copies_at` take consecutive rows, D / 8 lanes a row; those behind copy the shared page of a head each.
template <int D>
__global__ __launch_bounds__(kThreads) void append_rows_kernel(
    Geom g, PageView pv, const __bf16* __restrict__ k, const __bf16* __restrict__ v, const int32_t* __restrict__ indices,
    const int32_t* __restrict__ cu_b, const int32_t* __restrict__ cu_seq, const int32_t* __restrict__ seqs, int same_length,
    AppendSpace a, long long first_row, long long total_rows, int copies_at)
{
    constexpr int LANES = D / 8, ROWS = kThreads / LANES;
    const int H = pv.H, tid = threadIdx.x;
    if ((int)blockIdx.x >= copies_at) {
        const int head = blockIdx.x - copies_at;
        const AppendJob job = a.jobs[head];
        if (job.rows == 0 || job.copy_from < 0) return;
        const int to = a.found[job.first];
        if (!pv.is_page(to)) return;
        const int n = job.start & (pv.rows() - 1);
        const char *src = pv.page(job.copy_from);
        char* dst = pv.page(to);
        for (int i = tid; i < n * (D / 32); i += kThreads) {             // 16-byte pieces of codes, single scales
            reinterpret_cast<u32x4*>(dst)[i] = reinterpret_cast<const u32x4*>(src)[i];
            reinterpret_cast<u32x4*>(dst + pv.v_codes(0))[i] = reinterpret_cast<const u32x4*>(src + pv.v_codes(0))[i];
            dst[pv.k_scales(0) + i] = src[pv.k_scales(0) + i];
            dst[pv.v_scales(0) + i] = src[pv.v_scales(0) + i];
        }
        return;
    }
    const int n_heads = g.n_items * H;
    const int lane = tid % LANES;
    const long long row0 = first_row + (long long)blockIdx.x * ROWS;
    const long long r = row0 + tid / LANES;
    const long long rc = min(r, total_rows - 1);            // a row past the end is the last one again, and not stored
    int head, t;                                            // head (of items) and its row
    if (cu_b) {
        head = owner_of_row(cu_b, n_heads, 1, row0);
        while (head + 1 < n_heads && cu_b[head + 1] <= rc) ++head;
        t = (int)(rc - cu_b[head]);
    } else if (same_length > 0) {
        head = (int)((unsigned)rc / (unsigned)same_length);                  // (rows are fewer than 2^31)
        t = (int)((unsigned)rc % (unsigned)same_length);
    } else {
        int item = owner_of_row(cu_seq, g.n_items, H, row0);
        while (item + 1 < g.n_items && (long long)cu_seq[item + 1] * H <= rc) ++item;
        const int L = max(cu_seq[item + 1] - cu_seq[item], 1);
        const unsigned in_item = (unsigned)(rc - (long long)cu_seq[item] * H);
        head = item * H + min((int)(in_item / (unsigned)L), H - 1);
        t = (int)(in_item % (unsigned)L);
    }
    const int item = head / H, h = head - item * H;
    const int tok0 = cu_seq[item], L = cu_seq[item + 1] - tok0;
    const AppendJob job = a.jobs[head];
    const int token = indices ? indices[rc] : t;
    if (t < 0 || t >= job.rows || L <= 0) return;           // (whole groups of lanes)
    const int x = seqs ? seqs[item] : item;
    // an index outside the item is a caller error; cut so that it can never fault
    const int64_t src = kv_row_offset(g, item, tok0, L, h, min(max(token, 0), L - 1)) + lane * 8;
    const u32x4 kk = *reinterpret_cast<const u32x4*>(k + src), vv = *reinterpret_cast<const u32x4*>(v + src);
    const int at = job.start + t, slot = at >> pv.log_p, row = at & (pv.rows() - 1);
    const int first_new = pv.pages_of(job.start) - (job.copy_from >= 0);
    const size_t entry = (size_t)(x * H + h) * pv.width + slot;
    const int page = slot >= first_new ? a.found[job.first + slot - first_new] : pv.table[entry];
    int ks, vs;
    const unsigned kc = round_to_4(kk, ks), vc = round_to_4(vv, vs);
    if (r >= total_rows || !pv.is_page(page)) return;
    char* to = pv.page(page);
    *reinterpret_cast<unsigned*>(to + pv.k_codes(row) + lane * 4) = kc;
    *reinterpret_cast<unsigned*>(to + pv.v_codes(row) + lane * 4) = vc;
    if ((lane & 3) == 0) {
        to[pv.k_scales(row) + lane / 4] = (char)ks;
        to[pv.v_scales(row) + lane / 4] = (char)vs;
    }
    if (lane == 0 && slot >= first_new && (row == 0 || t == 0)) {        // the first row that the page gets
        pv.table[entry] = page;
        pv.refs[page] = 1;
    }
}

// Eight channels of a lane from 4 bits.
__device__ __forceinline__ u32x4 values_of(unsigned codes, unsigned scale) {
    u32x4 x = {0, 0, 0, 0};
    const float s = __uint_as_float(scale << 23);
#if defined(__HIP_DEVICE_COMPILE__)
    x[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0));
    x[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1));
    x[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2));
    x[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
#endif
    return x;
}

// read: as many lanes to a row. Bound by the bf16 rows that it writes.
template <int D>
__global__ __launch_bounds__(kThreads) void read_kernel(
    PageView pv, const int32_t* __restrict__ first, const int32_t* __restrict__ cu, long long first_row, long long total_rows,
    u32x4* __restrict__ k_out, u32x4* __restrict__ v_out)
{
    constexpr int LANES = D / 8, ROWS = kThreads / LANES;
    const int lane = threadIdx.x % LANES;
    const long long row0 = first_row + (long long)blockIdx.x * ROWS;
    const long long r = row0 + threadIdx.x / LANES;
    int head = owner_of_row(cu, pv.n_heads, 1, row0);
    const long long rc = min(r, total_rows - 1);
    while (head + 1 < pv.n_heads && cu[head + 1] <= rc) ++head;
    const long long at = rc - cu[head] + (first ? first[head] : 0);
    const u32x4 zero = {0, 0, 0, 0};
    u32x4 kk = zero, vv = zero;
    if (at >= 0 && at < pv.length(head)) {
        const int page = pv.table[(size_t)head * pv.width + (at >> pv.log_p)];
        if (pv.is_page(page)) {
            const int row = (int)at & (pv.rows() - 1);
            const char* from = pv.page(page);
            kk = values_of(*reinterpret_cast<const unsigned*>(from + pv.k_codes(row) + lane * 4), (unsigned char)from[pv.k_scales(row) + lane / 4]);
            vv = values_of(*reinterpret_cast<const unsigned*>(from + pv.v_codes(row) + lane * 4), (unsigned char)from[pv.v_scales(row) + lane / 4]);
        }
    }
    if (r < total_rows) {
        k_out[r * LANES + lane] = kk;
        v_out[r * LANES + lane] = vv;
    }
}

}  // namespace

size_t pages_append_bytes(const PageView& pv, int n_seqs, int n_items, long long total_rows) {
    size_t bytes;
    append_space(pv, n_seqs, n_items, total_rows, nullptr, &bytes);
    return bytes;
}

hipError_t launch_pages_append(const Geom& g, const PageView& pv, const AppendCall& c, void* workspace, hipStream_t s)
{
    const AppendSpace a = append_space(pv, c.n_seqs, c.n_items, c.total_rows, workspace, nullptr);
    hipLaunchKernelGGL(append_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, pv, c.cu_budgets, c.cu_seqlens, c.seqs, c.n_items,
                       c.n_seqs, (int)c.total_rows, a, c.refused);
    hipError_t e = hipGetLastError();
    // a launch holds fewer than 2^32 threads: rows beyond that take further ones. Copies go along with the first
    const int rows_per_block = kThreads / (g.D / 8);
    const long long slab = (long long)rows_per_block << 22;
    for (long long first = 0; first < c.total_rows && e == hipSuccess; first += slab) {
        const long long rows = c.total_rows - first < slab ? c.total_rows - first : slab;
        const int blocks = (int)((rows + rows_per_block - 1) / rows_per_block);
        const int copies = first == 0 ? c.n_items * pv.H : 0;
        AUDIOKV_FOR_DIM(g.D, hipLaunchKernelGGL(append_rows_kernel<kD>, dim3(blocks + copies), dim3(kThreads), 0, s, g, pv,
                                                (const __bf16*)c.k, (const __bf16*)c.v, c.indices, c.cu_budgets, c.cu_seqlens, c.seqs,
                                                c.same_length, a, first, c.total_rows, blocks))
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_pages_read(const PageView& pv, const int32_t* first_dev, const int32_t* cu_rows, long long total_rows, void* k_out,
                             void* v_out, hipStream_t s)
{
    const int rows_per_block = kThreads / (pv.D / 8);
    const long long slab = (long long)rows_per_block << 22;
    hipError_t e = hipSuccess;
    for (long long first = 0; first < total_rows && e == hipSuccess; first += slab) {
        const long long rows = total_rows - first < slab ? total_rows - first : slab;
        AUDIOKV_FOR_DIM(pv.D, hipLaunchKernelGGL(read_kernel<kD>, dim3((unsigned)((rows + rows_per_block - 1) / rows_per_block)),
                                                 dim3(kThreads), 0, s, pv, first_dev, cu_rows, first, total_rows, (u32x4*)k_out,
                                                 (u32x4*)v_out))
        e = hipGetLastError();
    }
    return e;
}

}  // namespace audiokv

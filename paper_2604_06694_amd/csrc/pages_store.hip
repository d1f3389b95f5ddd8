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
// Bytes of bf16 rows, K and V, from which they pass the caches by. append (the rows written just before, or 2 sets in turn; us with and
// without): 97 MB 23.2, 23.6 or 28.3, 23.3, 117 MB 26.9, 27.5 or 32.2, 31.8, 156 MB 34.9, 35.2 or 40.8, 44.6. read and a decoding step on
// what it wrote: 4 MB 16.3, 15.8, 8 MB 17.4, 17.6, 16 MB 19.8, 20.7, 32 MB 24.9, 25.9, 62 MB 36.8, 37.8.
constexpr long long kAppendStream = 128LL << 20, kReadStream = 8LL << 20;

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
    size_t off = 0;
    a.jobs = part_at<AppendJob>(workspace, off);
    off += up256((size_t)heads * sizeof(AppendJob));
    a.bad = part_at<int32_t>(workspace, off);
    off += up256((size_t)n_items * 4);
    a.owner = part_at<int32_t>(workspace, off);
    off += up256((size_t)n_seqs * 4);
    a.found = part_at<int32_t>(workspace, off);
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
    __shared__ int sums[kPlanThreads / 64 + 1];
    __shared__ int served_pages, lost, freed;
    const int tid = threadIdx.x, H = pv.H, heads = n_items * H;
    PageSearch<kPlanThreads, kLooked<kPlanThreads>> search(pv, pv.state[1]);
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
    int n_free = min(max(pv.state[0], 0), a.most);
    auto end_of = [&](int item) { return item + 1 < n_items ? a.jobs[(item + 1) * H].first : running; };
    auto served = [&](int item) {
        const int end = end_of(item);
        return !a.bad[item] && (end <= n_free || end == a.jobs[item * H].first);
    };
    int next, have;
    for (;;) {
        for (int i = tid; i < n_items; i += kPlanThreads)
            if (end_of(i) <= n_free) atomicMax(&served_pages, end_of(i));
        __syncthreads();
        const int want = served_pages;
        have = search.find(pv, want, a.found, sums, next);
        if (have == want) break;
        n_free = have;                       // (the state promised more)
        if (tid == 0) served_pages = 0;
        __syncthreads();
    }
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
        pv.state[0] += freed - have;
        pv.state[1] = next;
        if (refused) *refused = lost;
    }
}

// The same for up to THREADS heads, one a thread, and up to kSmallSeqs sequences: what is a pass over the workspace there is a register
// or LDS here, and the counts of the first pages that the search looks at are loaded beside the rest. What is left is the chain item ->
// sequence -> length -> table -> refs and the barriers. (192 heads by the kernel above and so: 7.4 and 3.2 us where none needs a page, 8.9 and
// 6.3 where many do and some copy; 1000 heads 9.5 and 5.5 where none needs one, 9.5 and 8.8 where each does.)
constexpr int kSmallSeqs = 4096;

template <int THREADS>
__global__ __launch_bounds__(THREADS) void append_plan_small_kernel(
    PageView pv, const int32_t* __restrict__ cu_b, const int32_t* __restrict__ cu_seq, const int32_t* __restrict__ seqs, int n_items,
    int n_seqs, int total_rows, AppendSpace a, int32_t* __restrict__ refused)
{
    __shared__ int sums[THREADS / 64 + 1], begins[THREADS], bad[THREADS], owner[kSmallSeqs];
    __shared__ int want, lost;
    const int tid = threadIdx.x, H = pv.H, heads = n_items * H;
    const bool mine = tid < heads;
    const int item = mine ? tid / H : 0, h = tid - item * H;
    const int state = pv.state[0];
    int x = mine ? (seqs ? seqs[item] : item) : -1;
    const int rows = mine ? rows_of(cu_b, cu_seq, H, tid, total_rows) : 0;
    PageSearch<THREADS, kLooked<THREADS>> search(pv, pv.state[1]);
    if (tid == 0) want = lost = 0;
    if (mine) bad[item] = 0;
    if (seqs) {
        for (int i = tid; i < n_seqs; i += THREADS) owner[i] = INT_MAX;
        __syncthreads();
        const bool is_sequence = (unsigned)x < (unsigned)n_seqs;
        if (is_sequence && h == 0) atomicMin(&owner[x], item);
        __syncthreads();
        x = is_sequence && owner[x] == item ? x : -1;
    } else {
        __syncthreads();
    }
    const int head = x * H + h;
    const bool asks = x >= 0 && rows > 0;
    AppendJob job{0, 0, -1, 0};
    int need = 0;
    if (asks) {
        const int start = pv.length(head);
        const long long end = (long long)start + rows;
        if (end > (long long)pv.width << pv.log_p) {
            bad[item] = 1;
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
            need = pv.pages_of((int)end) - first;
        }
    }
    __syncthreads();
    const bool fits = mine && !bad[item];
    int total;
    job.first = exclusive_sum<THREADS>(fits ? need : 0, sums, total);
    begins[tid] = job.first;
    __syncthreads();
    // Items are served while the free pages last: the ends of their pages do not fall.
    int n_free = min(max(state, 0), a.most), next, have;
    const int last = (item + 1) * H, end = last < THREADS ? begins[last] : total;
    bool served;
    for (;;) {
        served = fits && (end <= n_free || end == begins[item * H]);
        if (served && need > 0) atomicMax(&want, end);
        if (asks && !served) atomicAdd(&lost, 1);
        __syncthreads();
        const int wanted = want;
        have = search.find(pv, wanted, a.found, sums, next);
        if (have == wanted) break;
        n_free = have;                       // (the state promised more)
        if (tid == 0) want = lost = 0;
        __syncthreads();
    }
    if (asks && served) {
        job.rows = rows;
        pv.lengths[head] = job.start + rows;
        // after the search, so that a page which is still to be copied is not handed out
        if (job.copy_from >= 0 && atomicSub(&pv.refs[job.copy_from], 1) == 1) atomicAdd(&pv.state[0], 1);
    }
    if (mine) a.jobs[tid] = job;
    if (tid == 0) {
        if (have > 0) atomicSub(&pv.state[0], have);
        pv.state[1] = next;
        if (refused) *refused = lost;
    }
}

// What 8 channels of a lane become: four bytes of codes, and the scale byte of the block, the same in the four lanes that hold it.
__device__ __forceinline__ unsigned round_to_4(u32x4 x, int& scale) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    const auto magnitudes = [](unsigned w) { return __builtin_bit_cast(u16x2, w & 0x7fff7fffu); };
    const u16x2 tops = __builtin_elementwise_max(__builtin_elementwise_max(magnitudes(x[0]), magnitudes(x[1])),
                                                 __builtin_elementwise_max(magnitudes(x[2]), magnitudes(x[3])));
    unsigned top = max(tops[0], tops[1]);
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

constexpr int kStreamRows = 2;        // rows of a thread then: 367 thousand rows with one 66 us, two 55, four 59

// What a call reads or writes once, 16 bytes of it. STREAM: more than the memory-side cache should keep.
template <bool STREAM> __device__ __forceinline__ u32x4 row_piece(const __bf16* p) {
    return STREAM ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)) : *reinterpret_cast<const u32x4*>(p);
}

// The scale bytes of 16 lanes' blocks (8 lanes': D = 64) in one word, the first block lowest, in all of them.
template <int D> __device__ __forceinline__ unsigned scales_of_row(int scale, int lane) {
    int w = scale << (lane / 4 % (D == 64 ? 2 : 4) * 8);
    w |= __builtin_amdgcn_update_dpp(0, w, 0x141, 0xf, 0xf, false);                                  // lane 7 - i of eight
    if constexpr (D > 64) w |= __builtin_amdgcn_update_dpp(0, w, 0x140, 0xf, 0xf, false);            // lane 15 - i of sixteen
    return (unsigned)w;
}

// Workgroups up to `copies_at` take consecutive rows, D / 8 lanes a row; those behind copy the shared page of a head each.
template <int D, int R, bool STREAM>
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
    const long long row0 = first_row + (long long)blockIdx.x * (ROWS * R);
    // The head of the workgroup's first row, or its item, is found once; later rows walk forward from there. (Begin and end of the head's
    // rows, or of the item's, are held, and looked up again only where a row is behind them.)
    int walk = 0;
    long long begin = 0, end = 0;
    if (cu_b) {
        walk = owner_of_row(cu_b, n_heads, 1, row0);
        begin = cu_b[walk], end = cu_b[walk + 1];
    } else if (same_length <= 0) {
        walk = owner_of_row(cu_seq, g.n_items, H, row0);
        begin = (long long)cu_seq[walk] * H, end = (long long)cu_seq[walk + 1] * H;
    }
    u32x4 kk[R], vv[R];
    int head = -1, ts[R], entry_row[R];                      // row of the head, -1: none; row of the table
    int64_t base = 0;                                       // where the head's first token lies in K and V, and tokens of it
    int L = 0, table_row = 0;
    const int64_t stride = kv_tok_stride(g);
    AppendJob job{}, jobs[R];
#pragma unroll
    for (int u = 0; u < R; ++u) {
        const long long r = row0 + u * ROWS + tid / LANES;
        const long long rc = min(r, total_rows - 1);        // a row past the end is the last one again, and not stored
        int its, t;
        if (cu_b) {
            while (walk + 1 < n_heads && end <= rc) begin = end, end = cu_b[++walk + 1];
            its = walk;
            t = (int)(rc - begin);
        } else if (same_length > 0) {
            its = (int)((unsigned)rc / (unsigned)same_length);                   // (rows are fewer than 2^31)
            t = (int)((unsigned)rc % (unsigned)same_length);
        } else {
            while (walk + 1 < g.n_items && end <= rc) begin = end, end = (long long)cu_seq[++walk + 1] * H;
            const int of_head = max((int)(end - begin) / H, 1);
            its = walk * H + min((int)((unsigned)(rc - begin) / (unsigned)of_head), H - 1);
            t = (int)((unsigned)(rc - begin) % (unsigned)of_head);
        }
        if (its != head) {
            head = its;
            const int item = head / H, h = head - item * H, tok0 = cu_seq[item];
            L = cu_seq[item + 1] - tok0;
            base = kv_row_offset(g, item, tok0, L, h, 0);
            job = a.jobs[head];
            table_row = (seqs ? seqs[item] : item) * H + h;
        }
        const int token = indices ? indices[rc] : t;
        // an index outside the item is a caller error; cut so that it can never fault. (Loaded before it is known whether the head gets
        // rows: a load latency less on the way of those that do)
        const int64_t src = L > 0 ? base + max(min(token, L - 1), 0) * stride + lane * 8 : 0;
        kk[u] = row_piece<STREAM>(k + src);
        vv[u] = row_piece<STREAM>(v + src);
        jobs[u] = job;
        entry_row[u] = table_row;
        ts[u] = r < total_rows && L > 0 ? t : -1;
    }
#pragma unroll
    for (int u = 0; u < R; ++u) {
        const AppendJob to = jobs[u];
        const int t = ts[u];
        int ks, vs;
        const unsigned kc = round_to_4(kk[u], ks), vc = round_to_4(vv[u], vs);
        const unsigned k_scales = scales_of_row<D>(ks, lane), v_scales = scales_of_row<D>(vs, lane);
        if (t < 0 || t >= to.rows) continue;                // (whole groups of lanes)
        const int at = to.start + t, slot = at >> pv.log_p, row = at & (pv.rows() - 1);
        const int first_new = pv.pages_of(to.start) - (to.copy_from >= 0);
        const bool fresh = slot >= first_new;
        int32_t* entry = pv.table + (size_t)entry_row[u] * pv.width + slot;
        const int page = fresh ? a.found[to.first + slot - first_new] : *entry;
        if (!pv.is_page(page)) continue;
        char* bytes = pv.page(page);
        *reinterpret_cast<unsigned*>(bytes + pv.k_codes(row) + lane * 4) = kc;
        *reinterpret_cast<unsigned*>(bytes + pv.v_codes(row) + lane * 4) = vc;
        if (lane % 16 == 0) {
            if constexpr (D == 64) {
                *reinterpret_cast<unsigned short*>(bytes + pv.k_scales(row)) = (unsigned short)k_scales;
                *reinterpret_cast<unsigned short*>(bytes + pv.v_scales(row)) = (unsigned short)v_scales;
            } else {
                *reinterpret_cast<unsigned*>(bytes + pv.k_scales(row) + lane / 4) = k_scales;
                *reinterpret_cast<unsigned*>(bytes + pv.v_scales(row) + lane / 4) = v_scales;
            }
        }
        if (lane == 0 && fresh && (row == 0 || t == 0)) {                    // the first row that the page gets
            *entry = page;
            pv.refs[page] = 1;
        }
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
template <int D, bool STREAM>
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
    // (loads without branches around them: a row that is not there reads some page's, and is zero in the end)
    const long long at = rc - cu[head] + (first ? first[head] : 0);
    const int most = (pv.width << pv.log_p) - 1, in = (int)min(max(at, 0ll), (long long)most);
    const int page = pv.table[(size_t)head * pv.width + (in >> pv.log_p)];
    const bool there = at >= 0 && at < pv.length(head) && pv.is_page(page);
    const int row = in & (pv.rows() - 1);
    const char* from = pv.page(pv.is_page(page) ? page : 0);
    const unsigned kc = *reinterpret_cast<const unsigned*>(from + pv.k_codes(row) + lane * 4);
    const unsigned vc = *reinterpret_cast<const unsigned*>(from + pv.v_codes(row) + lane * 4);
    const unsigned char ks = from[pv.k_scales(row) + lane / 4], vs = from[pv.v_scales(row) + lane / 4];
    const u32x4 zero = {0, 0, 0, 0};
    const u32x4 kk = there ? values_of(kc, ks) : zero, vv = there ? values_of(vc, vs) : zero;
    if (r < total_rows) {
        if constexpr (STREAM) {
            __builtin_nontemporal_store(kk, k_out + r * LANES + lane);
            __builtin_nontemporal_store(vv, v_out + r * LANES + lane);
        } else {
            k_out[r * LANES + lane] = kk;
            v_out[r * LANES + lane] = vv;
        }
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
    const int heads = c.n_items * pv.H;
#define AUDIOKV_PLAN(KERNEL, THREADS)                                                                                                    \
    hipLaunchKernelGGL(KERNEL, dim3(1), dim3(THREADS), 0, s, pv, c.cu_budgets, c.cu_seqlens, c.seqs, c.n_items, c.n_seqs,                \
                       (int)c.total_rows, a, c.refused)
    if (heads <= 256 && a.most <= 2048 && c.n_seqs <= kSmallSeqs) AUDIOKV_PLAN(append_plan_small_kernel<256>, 256);
    else if (heads <= 1024 && c.n_seqs <= kSmallSeqs) AUDIOKV_PLAN(append_plan_small_kernel<1024>, 1024);
    else AUDIOKV_PLAN(append_plan_kernel, kPlanThreads);
#undef AUDIOKV_PLAN
    hipError_t e = hipGetLastError();
    // a launch holds fewer than 2^32 threads: rows beyond that take further ones. Copies go along with the first
    const int rows_per_block = kThreads / (g.D / 8);
    const long long slab = (long long)rows_per_block << 22;
    const bool stream = c.total_rows * g.D * 4 > kAppendStream;
    for (long long first = 0; first < c.total_rows && e == hipSuccess; first += slab) {
        const long long rows = c.total_rows - first < slab ? c.total_rows - first : slab;
        const int per_block = rows_per_block * (stream ? kStreamRows : 1), blocks = (int)((rows + per_block - 1) / per_block);
        const int copies = first == 0 ? c.n_items * pv.H : 0;
#define AUDIOKV_ROWS(STREAM)                                                                                                             \
    AUDIOKV_FOR_DIM(g.D, hipLaunchKernelGGL((append_rows_kernel<kD, (STREAM) ? kStreamRows : 1, STREAM>), dim3(blocks + copies), dim3(kThreads), 0, s, g, pv,        \
                                            (const __bf16*)c.k, (const __bf16*)c.v, c.indices, c.cu_budgets, c.cu_seqlens, c.seqs,       \
                                            c.same_length, a, first, c.total_rows, blocks))
        if (stream) AUDIOKV_ROWS(true) else AUDIOKV_ROWS(false)
#undef AUDIOKV_ROWS
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
        const dim3 grid((unsigned)((rows + rows_per_block - 1) / rows_per_block));
#define AUDIOKV_READ(STREAM)                                                                                                             \
    AUDIOKV_FOR_DIM(pv.D, hipLaunchKernelGGL((read_kernel<kD, STREAM>), grid, dim3(kThreads), 0, s, pv, first_dev, cu_rows, first,        \
                                             total_rows, (u32x4*)k_out, (u32x4*)v_out))
        if (total_rows * pv.D * 4 > kReadStream) AUDIOKV_READ(true) else AUDIOKV_READ(false)
#undef AUDIOKV_READ
        e = hipGetLastError();
    }
    return e;
}

}  // namespace audiokv

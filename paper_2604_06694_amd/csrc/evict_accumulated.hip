// Rows of growing caches cut to a budget by recency and accumulated weight, in place.
//
// A head with n rows and budget b < n keeps the first b in this order: rows at positions above newest - recent; then by
// weight, the largest first, NaN last; equal ones by slot. The rows that stay in slots below b do not move: the slots of the
// others there ("holes") take, in order, the kept rows of slots b .. n - 1 ("movers"). Sources and destinations are disjoint,
// and no more than min(b, n - b) rows move however long the cache is: one, where a step's new row is the only one too many.
//
// Ranks are integers (an order-preserving map of the weights), so the result is exact. A workgroup per head: few rows too
// many are found one by one, as the next larger minimum of (rank, slot) each; otherwise the rank of the last one to go is
// found digit by digit from histograms in LDS, and two scans over the slots number holes and movers.
// Bound: latency of a chain of barriers. The rows themselves are moved by the same workgroup where they are few, otherwise by
// a second launch with several workgroups per head.
#include "mfma_tile.h"

namespace audiokv {

namespace {

constexpr int kLdsRanks = 8192;       // rows whose ranks are kept in LDS (of more, they are worked out again where needed)
constexpr int kOneByOne = 8;          // rows too many that are found one by one
constexpr int kFewMoves = 256;        // moves that the ranking workgroup makes itself
constexpr int kDigit = 11, kBins = 1 << kDigit;

struct EvictAccum {
    Geom g;
    __bf16 *k, *v;
    int32_t* lengths;
    float* weights;
    int32_t* positions;
    const int32_t* budgets;
    int capacity, max_own, budget, recent;
    int32_t* moves;                   // [head][1 + 2 * max_moves]: how many, then (hole, mover); nullptr: kept in LDS
    int max_moves;
};

__device__ __forceinline__ unsigned rank_of(float w) {
    const unsigned bits = __float_as_uint(w + 0.f);               // -0 = +0
    const unsigned r = bits >> 31 ? ~bits : bits | 0x80000000u;
    return w != w ? 0u : r;                                       // -inf is above NaN, +inf below the recent ones
}

template <int THREADS>
struct Scan {
    int wave_total[2][THREADS / 64];
};
// exclusive sums of x and y over the threads, and their totals
template <int THREADS>
__device__ __forceinline__ void scan2(Scan<THREADS>& s, int& x, int& y, int& total_x, int& total_y) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int ix = wave_incl(x), iy = wave_incl(y);
    __syncthreads();                                              // (the array may still be read from before)
    if (lane == 63) {
        s.wave_total[0][wave] = ix;
        s.wave_total[1][wave] = iy;
    }
    __syncthreads();
    int bx = 0, by = 0, tx = 0, ty = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        bx += w < wave ? s.wave_total[0][w] : 0;
        by += w < wave ? s.wave_total[1][w] : 0;
        tx += s.wave_total[0][w];
        ty += s.wave_total[1][w];
    }
    x = bx + ix - x;
    y = by + iy - y;
    total_x = tx;
    total_y = ty;
}

// one 16-byte piece of a moved row: piece p of 2 * (D / 8) of move (hole, mover)
__device__ __forceinline__ void move_piece(const EvictAccum& a, int x, int h, int hole, int mover, int p) {
    const int per = a.g.D >> 3, c = (p < per ? p : p - per) * 8;
    __bf16* cache = p < per ? a.k : a.v;
    const int64_t from = kv_row_offset(a.g, x, (int64_t)x * a.capacity, a.capacity, h, mover) + c;
    const int64_t to = kv_row_offset(a.g, x, (int64_t)x * a.capacity, a.capacity, h, hole) + c;
    *reinterpret_cast<u32x4*>(cache + to) = *reinterpret_cast<const u32x4*>(cache + from);
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void evict_rank_kernel(EvictAccum a)
{
    constexpr int WAVES = THREADS / 64;
    __shared__ unsigned ranks[kLdsRanks];
    __shared__ int bins[kBins];
    __shared__ int2 few[kFewMoves];
    __shared__ Scan<THREADS> scan;
    __shared__ int wave_top[WAVES];
    __shared__ unsigned long long wave_min[2][WAVES];
    __shared__ int found[2];
    const int head = blockIdx.x, x = head / a.g.H_kv, h = head - x * a.g.H_kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = a.lengths[head], b = a.budgets ? max(a.budget, a.budgets[head]) : a.budget;
    int32_t* listed = a.moves ? a.moves + (int64_t)head * (1 + 2 * a.max_moves) : nullptr;
    if (n <= b || n > a.max_own) {
        if (listed && tid == 0) listed[0] = 0;
        return;
    }
    float* w = a.weights + (int64_t)head * a.capacity;
    int32_t* pos = a.positions ? a.positions + (int64_t)head * a.capacity : nullptr;

    // positions above `old` are recent (64 bits: newest - recent may pass the smallest int)
    int64_t old = INT64_MAX;
    if (a.recent > 0) {
        int top = INT_MIN;
        for (int t = tid; t < n; t += THREADS) top = max(top, pos[t]);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = max(top, __shfl_xor(top, o, 64));
        if (lane == 0) wave_top[wave] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) top = max(top, wave_top[i]);
        old = (int64_t)top - a.recent;
    }
    const bool kept_ranks = n <= kLdsRanks;
    auto fresh_rank = [&](int t) { return a.recent > 0 && (int64_t)pos[t] > old ? 0xffffffffu : rank_of(w[t]); };
    if (kept_ranks) {
        for (int t = tid; t < n; t += THREADS) ranks[t] = fresh_rank(t);
        __syncthreads();
    }
    auto rank = [&](int t) { return kept_ranks ? ranks[t] : fresh_rank(t); };

    const int gone = n - b;
    int moves = 0;
    if (gone <= kOneByOne) {
        // the next one to go: the smallest (rank, slots from the end) above the one before
        unsigned long long last = 0;
        unsigned out[kOneByOne];
        for (int e = 0; e < gone; ++e) {
            unsigned long long least = ~0ull;
            for (int t = tid; t < n; t += THREADS) {
                const unsigned long long v = ((unsigned long long)rank(t) << 32) | (unsigned)(INT_MAX - t);
                least = (e == 0 || v > last) && v < least ? v : least;
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                const unsigned long long v = __shfl_xor(least, o, 64);
                least = v < least ? v : least;
            }
            if (lane == 0) wave_min[e & 1][wave] = least;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < WAVES; ++i) least = wave_min[e & 1][i] < least ? wave_min[e & 1][i] : least;
            last = least;
#pragma unroll
            for (int i = 0; i < kOneByOne; ++i)
                if (i == e) out[i] = (unsigned)(INT_MAX - (int)(unsigned)least);
        }
        // holes below b in order, and the slots from b on that are none of those that go
        if (tid == 0) {
            int hole = -1, mover = b;
            for (;;) {
                int next = INT_MAX;
#pragma unroll
                for (int i = 0; i < kOneByOne; ++i)
                    if (i < gone && (int)out[i] > hole && (int)out[i] < next) next = (int)out[i];
                if (next >= b) break;
                for (bool goes = true; goes; mover += goes) {
                    goes = false;
#pragma unroll
                    for (int i = 0; i < kOneByOne; ++i) goes |= i < gone && (int)out[i] == mover;
                }
                if (listed) {
                    listed[1 + 2 * moves] = next;
                    listed[2 + 2 * moves] = mover;
                }
                few[moves++] = make_int2(next, mover);
                hole = next;
                ++mover;
            }
            found[0] = moves;
        }
        __syncthreads();
        moves = found[0];
        if (tid < moves) {
            w[few[tid].x] = w[few[tid].y];
            if (pos) pos[few[tid].x] = pos[few[tid].y];
        }
    } else {
        // T: the rank of the last one to go; `left`: how many of that rank go
        unsigned T = 0;
        int left = gone;
        for (int shift = 32 - kDigit, bits = kDigit; bits > 0;) {
            for (int i = tid; i < (1 << bits); i += THREADS) bins[i] = 0;
            __syncthreads();
            const unsigned mask = (1u << bits) - 1;
            for (int t = tid; t < n; t += THREADS) {
                const unsigned r = rank(t);
                if (shift + bits == 32 || (r >> (shift + bits)) == (T >> (shift + bits))) atomicAdd(&bins[(r >> shift) & mask], 1);
            }
            __syncthreads();
            // the bin in which the `left`-th lies: threads on runs of bins
            const int run = (1 << bits) / THREADS > 0 ? (1 << bits) / THREADS : 1;
            int sum = 0, none = 0, total, total2;
            if (tid * run < (1 << bits))
                for (int i = 0; i < run; ++i) sum += bins[tid * run + i];
            int before = sum;
            scan2<THREADS>(scan, before, none, total, total2);
            if (before < left && left <= before + sum) {
                int i = tid * run;
                while (before + bins[i] < left) before += bins[i++];
                found[0] = i;
                found[1] = left - before;
            }
            __syncthreads();
            T |= (unsigned)found[0] << shift;
            left = found[1];
            bits = shift < kDigit ? shift : kDigit;
            shift -= bits;
        }
        // a thread takes a run of slots: how many of rank T before it, then how many holes and movers
        const int run = (n + THREADS - 1) / THREADS, t0 = min(tid * run, n), t1 = min(t0 + run, n);
        int equal = 0, none = 0, equals, total2;
        for (int t = t0; t < t1; ++t) equal += rank(t) == T;
        scan2<THREADS>(scan, equal, none, equals, total2);
        const int stay = equals - left;                           // of rank T, the first ones
        int holes = 0, movers = 0, at = equal;
        for (int t = t0; t < t1; ++t) {
            const unsigned r = rank(t);
            const bool goes = r < T || (r == T && at >= stay);
            at += r == T;
            holes += goes && t < b;
            movers += !goes && t >= b;
        }
        int all_movers;
        scan2<THREADS>(scan, holes, movers, moves, all_movers);   // (as many of the one as of the other)
        at = equal;
        for (int t = t0; t < t1; ++t) {
            const unsigned r = rank(t);
            const bool goes = r < T || (r == T && at >= stay);
            at += r == T;
            if (goes && t < b) {
                if (listed) listed[1 + 2 * holes] = t; else few[holes].x = t;
                ++holes;
            }
            if (!goes && t >= b) {
                if (listed) listed[2 + 2 * movers] = t; else few[movers].y = t;
                ++movers;
            }
        }
        __syncthreads();                                          // (also: every rank has been read)
        for (int i = tid; i < moves; i += THREADS) {
            const int hole = listed ? listed[1 + 2 * i] : few[i].x, mover = listed ? listed[2 + 2 * i] : few[i].y;
            w[hole] = w[mover];
            if (pos) pos[hole] = pos[mover];
        }
    }
    if (tid == 0) {
        a.lengths[head] = b;
        if (listed) listed[0] = moves;
    }
    if (!listed) {
        const int per = a.g.D >> 2;                               // pieces of a move, of K and V
        for (int i = tid; i < moves * per; i += THREADS) move_piece(a, x, h, few[i / per].x, few[i / per].y, i % per);
    }
}

__global__ __launch_bounds__(256) void evict_move_kernel(EvictAccum a, int parts)
{
    const int head = blockIdx.x / parts, part = blockIdx.x - head * parts, x = head / a.g.H_kv, h = head - x * a.g.H_kv;
    const int32_t* listed = a.moves + (int64_t)head * (1 + 2 * a.max_moves);
    const int per = a.g.D >> 2, n = listed[0] * per;
#pragma unroll 4
    for (int i = part * 256 + threadIdx.x; i < n; i += parts * 256)
        move_piece(a, x, h, listed[1 + 2 * (i / per)], listed[2 + 2 * (i / per)], i % per);
}

// no head moves more rows than this
int most_moves(int max_own, int budget) { return max_own - budget < max_own / 2 ? max_own - budget : max_own / 2; }

}  // namespace

size_t evict_accumulated_bytes(const Geom& g, int max_own, int budget)
{
    const int moves = most_moves(max_own, budget);
    return moves <= kFewMoves ? 0 : (size_t)g.n_items * g.H_kv * (1 + 2 * (size_t)moves) * sizeof(int32_t);
}

hipError_t launch_evict_accumulated(const Geom& g, const EvictAccumCall& c, void* workspace, hipStream_t s)
{
    EvictAccum a{};
    a.g = g;
    a.k = static_cast<__bf16*>(c.k);
    a.v = static_cast<__bf16*>(c.v);
    a.lengths = c.lengths;
    a.weights = c.weights;
    a.positions = c.positions;
    a.budgets = c.budgets;
    a.capacity = c.capacity;
    a.max_own = c.max_own;
    a.budget = c.budget;
    a.recent = c.recent;
    a.max_moves = most_moves(c.max_own, c.budget);
    const bool few = a.max_moves <= kFewMoves;
    a.moves = few ? nullptr : static_cast<int32_t*>(workspace);
    const int heads = g.n_items * g.H_kv;
    if (c.max_own <= 2048) hipLaunchKernelGGL(evict_rank_kernel<256>, dim3((unsigned)heads), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(evict_rank_kernel<1024>, dim3((unsigned)heads), dim3(1024), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || few) return e;
    // workgroups per head: 32 rows of K and V each, as long as there are fewer than eight per CU
    int parts = (a.max_moves + 31) / 32;
    const int most = (2048 + heads - 1) / heads;
    if (parts > most) parts = most;
    hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(heads * parts)), dim3(256), 0, s, a, parts);
    return hipGetLastError();
}

}  // namespace audiokv

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
#include "row_moves.h"

namespace audiokv {

namespace {

constexpr int kRun = 8;               // slots that a thread keeps in registers
constexpr int kLdsMoves = 1024 * kRun / 2;    // moves that are paired up in LDS: all of a head's whose slots are in registers
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

// REGS: max_own <= THREADS * kRun, slots in registers; otherwise they are read again where needed
template <int THREADS, bool REGS>
__global__ __launch_bounds__(THREADS) void evict_rank_kernel(EvictAccum a)
{
    constexpr int WAVES = THREADS / 64, MOVES = REGS ? THREADS * kRun / 2 : kFewMoves;
    static_assert(MOVES <= kLdsMoves);
    __shared__ int bins[2][kBins];
    __shared__ int digit_total[2][WAVES], wave_count[2][REGS ? kRun * WAVES : 1];
    __shared__ int holes_at[MOVES], movers_at[MOVES];
    __shared__ Scan<THREADS> scan;
    __shared__ int wave_top[WAVES];
    __shared__ unsigned long long wave_min[2][WAVES];
    __shared__ int found[2];
    const int head = blockIdx.x, x = head / a.g.H_kv, h = head - x * a.g.H_kv;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    float* w = a.weights + (int64_t)head * a.capacity;
    int32_t* pos = a.positions ? a.positions + (int64_t)head * a.capacity : nullptr;
    const int n = a.lengths[head], b = a.budgets ? max(a.budget, a.budgets[head]) : a.budget;
    float wv[REGS ? kRun : 1];
    int pv[REGS ? kRun : 1];
    if constexpr (REGS) {                                         // (slots up to max_own, whatever the length turns out to be)
#pragma unroll
        for (int e = 0; e < kRun; ++e) wv[e] = w[min(e * THREADS + tid, a.max_own - 1)];
#pragma unroll
        for (int e = 0; e < kRun; ++e) pv[e] = a.recent > 0 ? pos[min(e * THREADS + tid, a.max_own - 1)] : 0;
    }
    int32_t* listed = a.moves ? a.moves + (int64_t)head * (1 + 2 * a.max_moves) : nullptr;
    if (n <= b || n > a.max_own) {
        if (listed && tid == 0) listed[0] = 0;
        return;
    }
    // slots in registers: every THREADS-th; otherwise a run of them
    const int run = (n + THREADS - 1) / THREADS, t0 = min(tid * run, n), t1 = min(t0 + run, n);

    // positions above `old` are recent (64 bits: newest - recent may pass the smallest int)
    int64_t old = INT64_MAX;
    if (a.recent > 0) {
        int top = INT_MIN;
        if constexpr (REGS) {
#pragma unroll
            for (int e = 0; e < kRun; ++e) top = e * THREADS + tid < n ? max(top, pv[e]) : top;
        } else {
            for (int t = t0; t < t1; ++t) top = max(top, pos[t]);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = max(top, __shfl_xor(top, o, 64));
        if (lane == 0) wave_top[wave] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) top = max(top, wave_top[i]);
        old = (int64_t)top - a.recent;
    }
    unsigned ranks[REGS ? kRun : 1];
    if constexpr (REGS) {
#pragma unroll
        for (int e = 0; e < kRun; ++e) ranks[e] = a.recent > 0 && (int64_t)pv[e] > old ? 0xffffffffu : rank_of(wv[e]);
    }
    // f(slot, rank) for the thread's slots in order
    auto each = [&](auto f) {
        if constexpr (REGS) {
#pragma unroll
            for (int e = 0; e < kRun; ++e)
                if (e * THREADS + tid < n) f(e * THREADS + tid, ranks[e]);
        } else {
            for (int t = t0; t < t1; ++t) f(t, a.recent > 0 && (int64_t)pos[t] > old ? 0xffffffffu : rank_of(w[t]));
        }
    };

    const int gone = n - b;
    int moves = 0;
    if (gone <= kOneByOne) {
        // the next one to go: the smallest (rank, slots from the end) above the one before
        unsigned long long last = 0;
        int out[kOneByOne];
        for (int e = 0; e < gone; ++e) {
            unsigned long long least = ~0ull;
            each([&](int t, unsigned r) {
                const unsigned long long v = ((unsigned long long)r << 32) | (unsigned)(INT_MAX - t);
                least = (e == 0 || v > last) && v < least ? v : least;
            });
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
                if (i == e) out[i] = INT_MAX - (int)(unsigned)least;
        }
        // holes below b in order, and the slots from b on that are none of those that go
        if (tid == 0) {
            int hole = -1, mover = b;
            for (;;) {
                int next = INT_MAX;
#pragma unroll
                for (int i = 0; i < kOneByOne; ++i)
                    if (i < gone && out[i] > hole && out[i] < next) next = out[i];
                if (next >= b) break;
                for (bool goes = true; goes; mover += goes) {
                    goes = false;
#pragma unroll
                    for (int i = 0; i < kOneByOne; ++i) goes |= i < gone && out[i] == mover;
                }
                holes_at[moves] = next;
                movers_at[moves++] = mover++;
                hole = next;
            }
            found[0] = moves;
        }
        __syncthreads();
        moves = found[0];
    } else {
        // T: the rank of the last one to go; `left`: how many of that rank go
        unsigned T = 0;
        int left = gone;
        for (int i = tid; i < kBins; i += THREADS) bins[0][i] = 0;
        __syncthreads();
        for (int shift = 32 - kDigit, bits = kDigit, pass = 0; bits > 0; pass ^= 1) {
            const unsigned mask = (1u << bits) - 1;
            int* count = bins[pass];
            each([&](int, unsigned r) {
                if (shift + bits == 32 || (r >> (shift + bits)) == (T >> (shift + bits))) atomicAdd(&count[(r >> shift) & mask], 1);
            });
            for (int i = tid; i < kBins; i += THREADS) bins[pass ^ 1][i] = 0;        // the next pass's
            __syncthreads();
            // the bin in which the `left`-th lies: threads on runs of bins
            constexpr int per = kBins / THREADS;
            int sum = 0;
#pragma unroll
            for (int i = 0; i < per; ++i) sum += count[tid * per + i];               // (the last digit's unused bins are 0)
            const int upto = wave_incl(sum);
            if (lane == 63) digit_total[pass][wave] = upto;
            __syncthreads();
            int before = upto - sum;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) before += i < wave ? digit_total[pass][i] : 0;
            if (before < left && left <= before + sum) {
                int i = tid * per;
                while (before + count[i] < left) before += count[i++];
                found[0] = i;
                found[1] = left - before;
            }
            __syncthreads();
            T |= (unsigned)found[0] << shift;
            left = found[1];
            bits = shift < kDigit ? shift : kDigit;
            shift -= bits;
        }
        if constexpr (REGS) {
            // Slots of a wave are consecutive in every e: a lane mask counts them, and every wave scans the counts of all for itself,
            // (e, wave) in order, two to a lane.
            static_assert(kRun * WAVES <= 128);
            auto before_waves = [&](int which, const int (&mine)[kRun], int (&before)[kRun], int* total) {
#pragma unroll
                for (int e = 0; e < kRun; ++e)
                    if (lane == 0) wave_count[which][e * WAVES + wave] = mine[e];
                __syncthreads();
                const int c0 = 2 * lane < kRun * WAVES ? wave_count[which][2 * lane] : 0, c1 = 2 * lane < kRun * WAVES ? wave_count[which][2 * lane + 1] : 0;
                const int upto = wave_incl(c0 + c1);
                *total = __builtin_amdgcn_readlane(upto, 63);
#pragma unroll
                for (int e = 0; e < kRun; ++e) {
                    const int i = e * WAVES + wave, l = i >> 1;
                    before[e] = __builtin_amdgcn_readlane(upto - c0 - c1, l) + (i & 1 ? __builtin_amdgcn_readlane(c0, l) : 0);
                }
            };
            const unsigned long long below = (1ull << lane) - 1;
            unsigned long long same[kRun], hole[kRun], mover[kRun];
            int mine[kRun], before[kRun], equals, both;
#pragma unroll
            for (int e = 0; e < kRun; ++e) {
                same[e] = __builtin_amdgcn_ballot_w64(e * THREADS + tid < n && ranks[e] == T);
                mine[e] = __builtin_popcountll(same[e]);
            }
            before_waves(0, mine, before, &equals);
            const int stay = equals - left;                       // of rank T, the first ones
#pragma unroll
            for (int e = 0; e < kRun; ++e) {
                const int t = e * THREADS + tid;
                const bool goes = ranks[e] < T || (ranks[e] == T && before[e] + __builtin_popcountll(same[e] & below) >= stay);
                hole[e] = __builtin_amdgcn_ballot_w64(t < b && goes);
                mover[e] = __builtin_amdgcn_ballot_w64(t >= b && t < n && !goes);
                mine[e] = __builtin_popcountll(hole[e]) | __builtin_popcountll(mover[e]) << 16;
            }
            before_waves(1, mine, before, &both);                 // (as many of the one as of the other)
            moves = both & 0xffff;
#pragma unroll
            for (int e = 0; e < kRun; ++e) {
                const int t = e * THREADS + tid;
                if (hole[e] >> lane & 1) holes_at[(before[e] & 0xffff) + __builtin_popcountll(hole[e] & below)] = t;
                if (mover[e] >> lane & 1) movers_at[(before[e] >> 16) + __builtin_popcountll(mover[e] & below)] = t;
            }
        } else {
            // how many of rank T lie before a thread's slots, then how many holes and movers
            int equal = 0, none = 0, equals, total2;
            each([&](int, unsigned r) { equal += r == T; });
            scan2<THREADS>(scan, equal, none, equals, total2);
            const int stay = equals - left;
            int holes = 0, movers = 0, at = equal, all_movers;
            auto goes = [&](unsigned r) {
                const bool g = r < T || (r == T && at >= stay);
                at += r == T;
                return g;
            };
            each([&](int t, unsigned r) {
                const bool g = goes(r);
                holes += g && t < b;
                movers += !g && t >= b;
            });
            scan2<THREADS>(scan, holes, movers, moves, all_movers);
            at = equal;
            each([&](int t, unsigned r) {
                const bool g = goes(r), hole = g && t < b, mover = !g && t >= b;
                if (hole || mover) {
                    const int i = hole ? holes : movers;
                    if (listed) listed[(hole ? 1 : 2) + 2 * i] = t;
                    else (hole ? holes_at : movers_at)[i] = t;
                }
                holes += hole;
                movers += mover;
            });
        }
        __syncthreads();                                          // (also: every rank has been read)
    }
    const bool in_lds = REGS || !listed || gone <= kOneByOne;
    for (int i = tid; i < moves; i += THREADS) {
        const int hole = in_lds ? holes_at[i] : listed[1 + 2 * i], mover = in_lds ? movers_at[i] : listed[2 + 2 * i];
        if (listed && in_lds) {
            listed[1 + 2 * i] = hole;
            listed[2 + 2 * i] = mover;
        }
        w[hole] = w[mover];
        if (pos) pos[hole] = pos[mover];
    }
    if (tid == 0) {
        a.lengths[head] = b;
        if (listed) listed[0] = moves;
    }
    if (!listed) {
        const int per = a.g.D >> 2;                               // pieces of a move, of K and V
        for (int i = tid; i < moves * per; i += THREADS) move_piece(a, x, h, holes_at[i / per], movers_at[i / per], i % per);
    }
}

__global__ __launch_bounds__(256) void evict_move_kernel(EvictAccum a, int parts)
{
    const int head = blockIdx.x / parts, part = blockIdx.x - head * parts, x = head / a.g.H_kv, h = head - x * a.g.H_kv;
    const int32_t* listed = a.moves + (int64_t)head * (1 + 2 * a.max_moves);
    const int n = listed[0];
    const MoveWalk walk = move_walk(part * 256 + threadIdx.x, parts * 256, a.g.D >> 2);
#pragma unroll 4
    for (int i = walk.first; i < n; i += walk.step) move_piece(a, x, h, listed[1 + 2 * i], listed[2 + 2 * i], walk.piece);
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
    const dim3 grid((unsigned)heads);
    if (c.max_own <= 256 * kRun) hipLaunchKernelGGL((evict_rank_kernel<256, true>), grid, dim3(256), 0, s, a);
    else if (c.max_own <= 1024 * kRun) hipLaunchKernelGGL((evict_rank_kernel<1024, true>), grid, dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((evict_rank_kernel<1024, false>), grid, dim3(1024), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || few) return e;
    // workgroups per head: 32 rows of K and V each, as long as there are fewer than sixteen per CU
    int parts = (a.max_moves + 31) / 32;
    const int most = (4096 + heads - 1) / heads;
    if (parts > most) parts = most;
    hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(heads * parts)), dim3(256), 0, s, a, parts);
    return hipGetLastError();
}

}  // namespace audiokv

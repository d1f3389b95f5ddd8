// Accumulated attention weight: what every cached token has received from ALL queries of a prompt, or of a chunk of it.
//
//   weights[h, j] += sum over rows r = (query i, query head of the group) that see j of
//                    softmax_j(scale * <q_r, k_j>),      row r sees keys j <= L - Q + i (causal)
//
// score (score_impl.h) does this for a window of a few dozen queries that stays in registers; here both sides are long, so
// the work is a triangle of (row, key) pairs, 2 d flops and one exponential each, twice: a softmax row needs its sum before a
// column sum exists.
//   rows   row blocks stay in registers as MFMA operands, keys stream through LDS: per row and key range (reference, sum)
//   cols   key blocks stay in registers, rows stream through LDS: exp2(z - max - log2 sum) summed per key
// Both compute C = K Q^T (a lane owns a row). rows: the row's sum stays in the lane. cols: a lane adds up its sixteen keys over
// all row tiles and the lanes are joined once, at the end, so that a logit costs fma, exp2 and add in both.
// Rows are numbered r = i * G + (head of the group): what a key block sees is then a contiguous tail of the rows, whatever G.
//
// Work is cut into spans of equal numbers of tiles, one workgroup per CU, across blocks and heads (accumulate_plan.h): the
// triangle leaves blocks of very different lengths, and a workgroup costs as much to start as three tiles. A grid of (block,
// range of 13 to 32 tiles) took 350 + 340 us for one layer of 8192 tokens where this took 262 + 274 on the same card. What the parts of a block that several
// workgroups share have found is joined by two small kernels in fixed order (row statistics; column sums). No atomics.
//
// References of a row are not maxima (see score_impl.h): the first logits set one, and only a tile whose sum leaves the safe
// range is redone against a new one. Everything is in base-2 units: z = <q,k> * scale * log2(e).
#include "accumulate_plan.h"
#include "mfma_tile.h"

namespace audiokv {

namespace {

using namespace mfma_tile;

struct Accum {
    Geom g;
    const __bf16* q;
    const __bf16* k;
    const int32_t* cu_seq;
    const int32_t* cu_q;
    const float* lse;          // given, or nullptr
    float* norms;              // [row of all items]: log2 of the row's sum of exp2
    float2* stats;             // [part_slot][row of the block] (reference, sum), of blocks that have several parts
    float* parts;              // [part_slot][key of the block] column sums, of blocks that have several
    float* weights;
    int64_t pitch;             // between heads of weights; 0: packed like scores
    unsigned div_g;            // r / G = umulhi(r, div_g), G > 1
    int block;                 // rows (keys) of a block of the sweep
    AccumSpans spans;          // of the sweep (a kernel's arguments hold no more than 4 KB)
};
static_assert(sizeof(Accum) < 4000);

struct Place {
    int item, h, L, Q, R;
    int64_t tok0, q0;          // first token and first query of the item
    AccumItem item_of;
};
__device__ __forceinline__ Place place_of(const Accum& a, int head) {
    Place p;
    p.item = head / a.g.H_kv;
    p.h = head - p.item * a.g.H_kv;
    p.tok0 = a.cu_seq[p.item];
    p.L = a.cu_seq[p.item + 1] - (int)p.tok0;
    p.q0 = a.cu_q[p.item];
    p.Q = min(a.cu_q[p.item + 1] - (int)p.q0, p.L);
    p.R = p.Q * a.g.G;
    p.item_of = AccumItem{p.L, p.Q, a.g.G, a.g.causal};
    return p;
}
__device__ __forceinline__ int query_of(const Accum& a, int r) { return a.g.G == 1 ? r : (int)__umulhi((unsigned)r, a.div_g); }
// where row r of an item's KV head starts in q: [H_q][Q][d] or [Q][H_q][d]
__device__ __forceinline__ int64_t q_offset(const Accum& a, const Place& p, int r) {
    const int i = query_of(a, r), hq = p.h * a.g.G + (r - i * a.g.G);
    const int64_t row = a.g.layout == AUDIOKV_LAYOUT_HEAD_MAJOR ? (int64_t)hq * p.Q + i : (int64_t)i * a.g.H_q + hq;
    return (p.q0 * a.g.H_q + row) * a.g.D;
}
// last key that row r sees (-1: no such row)
__device__ __forceinline__ int last_key(const Accum& a, const Place& p, int r) {
    return r >= p.R ? -1 : a.g.causal ? p.L - p.Q + query_of(a, r) : p.L - 1;
}
// what a row's exponents are taken against: log2 of its sum of exp2. Nothing but -inf: the row gives nothing.
__device__ __forceinline__ float norm_from(float M, float Z) { return Z == 0.f ? INFINITY : M + __log2f(Z); }
__device__ __forceinline__ int64_t stat_row(const Accum& a, const Place& p, int r) { return p.q0 * a.g.H_q + (int64_t)p.h * p.R + r; }

// Compute waves of a workgroup; one more wave loads. The waves of a workgroup hold kComputeWaves * NB tiles of 32 rows (or keys) as
// stationary operands, tiles of kStream keys (or rows) come through a ring of LDS buffers that the loader fills straight from HBM
// or L2, one barrier per tile.
constexpr int kLeastTiles = 1;           // 700 tokens, four heads: two 10.2 + 13.2 us on 160 + 144 CUs, one 9.6 + 13.1 on 200 + 176
constexpr int kComputeWaves = 7, kSweepThreads = 64 * (kComputeWaves + 1), kStages = 4;
constexpr int stationary(int NB) { return kComputeWaves * NB * 32; }

typedef __attribute__((address_space(3))) void* lds_void_ptr;
typedef const __attribute__((address_space(1))) void* global_void_ptr;

// LDS traffic only: the waves exchange nothing else
__device__ __forceinline__ void sweep_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The loader wave: begin(r) sets out at row r of the stream (the lane's first), next() is where the row that it has come to begins,
// and goes on by the rows of an instruction. Rows past the end read the last one.
// more(t): what else a tile brings.
template <int D, class Walk, class More>
__device__ __forceinline__ void load_stream(unsigned char* ring, int n_tiles, Walk walk, More more)
{
    constexpr int CPR = D / 8, RPI = 64 / CPR, CH = kStream / RPI;       // chunks of a row, rows and instructions of a tile
    const int lane = threadIdx.x & 63, row = lane / CPR, slot = lane % CPR;
    int from[8 / RPI];                                                   // the slots' rotation repeats after eight rows
#pragma unroll
    for (int v = 0; v < 8 / RPI; ++v) from[v] = ((slot & ~7) | ((slot - (v * RPI + row)) & 7)) * 8;
    walk.begin(row, RPI);
    auto issue = [&](int t) {
        unsigned char* dst = ring + (t % kStages) * (kStream * D * 2);
#pragma unroll
        for (int it = 0; it < CH; ++it)
            // a wave-wide instruction fills consecutive LDS: the lane fetches the chunk that belongs in its slot (slot_of)
            __builtin_amdgcn_global_load_lds((global_void_ptr)(walk.next() + from[it % (8 / RPI)]), (lds_void_ptr)(dst + it * 1024), 16, 0, 0);
        more(t);
    };
    // Compute waves reduce tile t and begin with the next one between the barrier that opens iteration t and the one that ends it: at the
    // first, tiles up to t + 1 have landed. More of them requested ahead only put off the first barrier (a request takes some
    // 70 cycles to issue). Tile t + 2 goes where tile t - 2 was, which every wave has left.
    int t = 0;
    for (; t < 2 && t < n_tiles; ++t) issue(t);
    for (int ended = 0;; ++ended) {
        __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (15 << 8));             // vmcnt(0): all that was requested is there
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        if (ended == n_tiles) break;
        if (t < n_tiles) issue(t++);
    }
}
// Keys of a head from j0 on
struct KeyWalk {
    const __bf16 *at, *last;
    int64_t stride;
    int left;                  // rows up to the last
    int step;
    int64_t on;
    __device__ __forceinline__ KeyWalk(const Accum& a, const Place& p, int j0) {
        stride = kv_tok_stride(a.g);
        at = a.k + kv_row_offset(a.g, p.item, p.tok0, p.L, p.h, j0);
        left = p.L - 1 - j0;
        last = at + left * stride;
    }
    __device__ __forceinline__ void begin(int row, int rows) {
        at += row * stride;
        left -= row;
        step = rows;
        on = rows * stride;
    }
    __device__ __forceinline__ const __bf16* next() {
        const __bf16* here = left >= 0 ? at : last;
        at += on;
        left -= step;
        return here;
    }
};
// Query rows of a KV head from r0 on: a step is some queries and some heads, with a carry
struct RowWalk {
    const __bf16 *at, *last;
    const Accum& a;
    int64_t per_query, per_head, on, carry;
    int left, step, heads_on, in_group, r0;
    __device__ __forceinline__ RowWalk(const Accum& accum, const Place& p, int r) : a(accum) {
        const bool head_major = a.g.layout == AUDIOKV_LAYOUT_HEAD_MAJOR;
        per_query = head_major ? a.g.D : (int64_t)a.g.H_q * a.g.D;
        per_head = head_major ? (int64_t)p.Q * a.g.D : a.g.D;
        at = a.q + q_offset(a, p, 0);
        last = a.q + q_offset(a, p, p.R - 1);
        r0 = r;
        left = p.R - 1;
    }
    __device__ __forceinline__ void begin(int row, int rows) {
        const int r = r0 + row, i = query_of(a, r);
        in_group = r - i * a.g.G;
        at += i * per_query + in_group * per_head;
        left -= r;
        step = rows;
        const int queries = query_of(a, rows);
        heads_on = rows - queries * a.g.G;
        on = queries * per_query + heads_on * per_head;
        carry = per_query - a.g.G * per_head;
    }
    __device__ __forceinline__ const __bf16* next() {
        const __bf16* here = left >= 0 ? at : last;
        left -= step;
        in_group += heads_on;
        const bool wraps = in_group >= a.g.G;
        in_group -= wraps ? a.g.G : 0;
        at += on + (wraps ? carry : 0);
        return here;
    }
};

// A compute wave's blocks: its NB stationary tiles times 32 rows of the stream, NB * KK MFMAs, then per logit fma, exp2, add.
// Both take about as long, so (score_impl.h) while the MFMAs of one block accumulate into one register set the logits of the block
// before are reduced from the other, a slice after each MFMA; an empty asm statement that takes accumulator, sums and scale in and
// out keeps the compiler from gathering the MFMAs. PIPE false: one register set, a block after the other.
template <int D, int NB, bool COLS, bool PIPE>
struct Wave {
    static constexpr int KK = D / 16, SLICE = 16 / KK, PF = 2, RING = 4;
    static_assert(KK % RING == 0 && SLICE * KK == 16);
    bf16x8 still[NB][KK];
    f32x16 acc[PIPE ? 2 : 1][NB];
    bf16x8 frag[RING];
    int frag_at[4];
    float c;                                  // scale * log2(e)
    float m[NB], l[NB], red[NB];              // rows: reference, sum, and the sum of a block
    float sum[NB][16];                        // cols: a lane's share of its sixteen keys' sums
    float norm;                               // cols: of the lane's row of the block that is reduced
    const unsigned char* ring;
    int hf, col;

    __device__ __forceinline__ void begin(const unsigned char* r, float scale) {
        const int lane = threadIdx.x & 63;
        hf = lane >> 5;
        col = lane & 31;
        ring = r;
        c = scale;
#pragma unroll
        for (int v = 0; v < 4; ++v) frag_at[v] = (col * D + slot_of((2 * v) | hf, col) * 8) * 2;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            m[b] = -INFINITY;
            l[b] = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[b][i] = 0.f;
        }
    }
    // (a block is numbered from the first tile, two to a tile)
    __device__ __forceinline__ void load(int block, int kk, int to) {
        frag[to] = *reinterpret_cast<const bf16x8*>(ring + ((block >> 1) % kStages) * (kStream * D * 2) + (block & 1) * (32 * D * 2) +
                                                    frag_at[kk & 3] + (kk >> 2) * 128);
    }
    __device__ __forceinline__ void reduce_part(f32x16 (&z)[NB], int kk, int b) {
#pragma unroll
        for (int e = 0; e < SLICE; ++e) {
            const int i = kk * SLICE + e;
            if (COLS) sum[b][i] += fast_exp2(__builtin_fmaf(z[b][i], c, -norm));
            else red[b] += fast_exp2(__builtin_fmaf(z[b][i], c, -m[b]));
        }
    }
    // MFMAs of block `next` into zm (the first PF fragments are in the ring already if STREAM, and those of the block after it are
    // fetched at the end), reduction of zr
    template <bool MFMA, bool REDUCE, bool STREAM>
    __device__ __forceinline__ void run(f32x16 (&zm)[NB], int next, f32x16 (&zr)[NB]) {
        if (MFMA && !STREAM) {
#pragma unroll
            for (int kk = 0; kk < PF; ++kk) load(next, kk, kk);
        }
        if (REDUCE && !COLS) {
#pragma unroll
            for (int b = 0; b < NB; ++b) red[b] = 0.f;
        }
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (MFMA) {
                if (kk + PF < KK) load(next, kk + PF, (kk + PF) % RING);
                else if (STREAM) load(next + 1, kk + PF - KK, (kk + PF) % RING);
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (MFMA) {
                    const f32x16 zero = {};
                    const f32x16 in = kk == 0 ? zero : zm[b];
                    // C[key][row]
                    zm[b] = COLS ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(still[b][kk], frag[kk % RING], in, 0, 0, 0)
                                 : __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[kk % RING], still[b][kk], in, 0, 0, 0);
                }
                if (REDUCE) reduce_part(zr, kk, b);
#if defined(__HIP_DEVICE_COMPILE__)
                if (MFMA && REDUCE) {
                    if constexpr (!COLS) asm volatile("" : "+v"(c), "+v"(zm[b]), "+v"(red[b]));
                    else if constexpr (SLICE == 1) asm volatile("" : "+v"(c), "+v"(zm[b]), "+v"(sum[b][kk]));
                    else if constexpr (SLICE == 2) asm volatile("" : "+v"(c), "+v"(zm[b]), "+v"(sum[b][2 * kk]), "+v"(sum[b][2 * kk + 1]));
                    else asm volatile("" : "+v"(c), "+v"(zm[b]), "+v"(sum[b][4 * kk]), "+v"(sum[b][4 * kk + 1]), "+v"(sum[b][4 * kk + 2]), "+v"(sum[b][4 * kk + 3]));
                }
#endif
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // rows: a block's sums join the rows'; where one has left the safe range (the first logits of a lane, whose reference is -inf;
    // logits far above the reference; NaN), the block is summed again against a new reference
    __device__ __forceinline__ void finish(f32x16 (&z)[NB]) {
        if constexpr (!COLS) {
            float worst = red[0];
#pragma unroll
            for (int b = 1; b < NB; ++b) worst = red[b] < 0x1p64f ? worst : red[b];
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(worst < 0x1p64f)) != 0, 0)) {
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    float top = z[b][0];
#pragma unroll
                    for (int i = 1; i < 16; ++i) top = fmaxf(top, z[b][i]);
                    const bool redo = !(red[b] < 0x1p64f);
                    const float ref = redo ? fmaxf(m[b], top * c) : m[b], ref0 = ref == -INFINITY ? 0.f : ref;
                    float again = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) again += fast_exp2(__builtin_fmaf(z[b][i], c, -ref0));
                    l[b] = redo ? l[b] * fast_exp2(m[b] - ref0) : l[b];
                    red[b] = redo ? again : red[b];
                    m[b] = ref;
                }
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) l[b] += red[b];
        }
    }
    // Tiles t0 to t1, all of whose pairs count. norm_of(block): the lane's row's norm in that block.
    template <class Norm>
    __device__ __forceinline__ void plain(int t0, int t1, Norm norm_of) {
        if (t0 >= t1) return;
        if constexpr (PIPE) {
            float next_norm = COLS ? norm_of(2 * t0) : 0.f;
            run<true, false, false>(acc[0], 2 * t0, acc[1]);
            load(2 * t0 + 1, 0, 0);
            load(2 * t0 + 1, 1, 1);
            for (int t = t0; t < t1; ++t) {
                norm = next_norm;
                if (COLS) next_norm = norm_of(2 * t + 1);
                run<true, true, true>(acc[1], 2 * t + 1, acc[0]);
                finish(acc[0]);
                norm = next_norm;
                if (t + 1 < t1) {
                    if (COLS) next_norm = norm_of(2 * t + 2);
                    run<true, true, true>(acc[0], 2 * t + 2, acc[1]);
                } else {
                    run<false, true, false>(acc[0], 0, acc[1]);
                }
                finish(acc[1]);
                sweep_barrier();
            }
        } else {
            for (int t = t0; t < t1; ++t) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    if (COLS) norm = norm_of(2 * t + s);
                    run<true, false, false>(acc[0], 2 * t + s, acc[0]);
                    run<false, true, false>(acc[0], 0, acc[0]);
                    finish(acc[0]);
                }
                sweep_barrier();
            }
        }
    }
    // Tiles t0 to t1 with pairs that do not: most_of(block, b) is the last key of the block's 32, as the lane's half counts them,
    // that counts for the lane's row and stationary tile b.
    template <class Norm, class Most>
    __device__ __forceinline__ void masked(int t0, int t1, Norm norm_of, Most most_of) {
        for (int t = t0; t < t1; ++t) {
#pragma unroll 1
            for (int s = 0; s < 2; ++s) {
                run<true, false, false>(acc[0], 2 * t + s, acc[0]);
                if (COLS) norm = norm_of(2 * t + s);
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const int most = most_of(2 * t + s, b) - 4 * hf;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if (COLS) {                           // (a row's NaN is none of the keys' that it does not see)
                            const float e = fast_exp2(__builtin_fmaf(acc[0][b][i], c, -norm));
                            sum[b][i] += key_of(i, 0) <= most ? e : 0.f;
                        } else {
                            acc[0][b][i] = key_of(i, 0) <= most ? acc[0][b][i] : -INFINITY;
                        }
                    }
                }
                if (!COLS) {
                    run<false, true, false>(acc[0], 0, acc[0]);
                    finish(acc[0]);
                }
            }
            sweep_barrier();
        }
    }
};

// The parts of blocks in a workgroup's span: body(place, head, block, first tile, tiles, the part's slot, whether the block has others).
// Neighbouring spans go to one XCD, whose L2 then holds the head that they are about.
template <bool COLS, int SIZE, class Body>
__device__ __forceinline__ void for_parts(const Accum& a, Body body)
{
    const AccumSpans& s = a.spans;
    const int w = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
    const SpanStart begin = s.at[w], end = s.at[w + 1];           // (the same behind the last span)
    int head = begin.head, block = begin.block, tile = begin.tile;
    while (head < end.head || (head == end.head && (block < end.block || (block == end.block && tile < end.tile)))) {
        const Place p = place_of(a, head);
        if (block >= p.item_of.blocks(COLS, SIZE)) {
            ++head;
            block = tile = 0;
            continue;
        }
        const int tiles = p.item_of.tiles(COLS, block, SIZE), stop = head == end.head && block == end.block ? min(tiles, end.tile) : tiles;
        if (tile < stop) body(p, head, block, tile, stop - tile, part_slot(w, tile > 0), stop - tile < tiles);
        ++block;
        tile = 0;
    }
}

// ---- rows: statistics of blocks of stationary(NB) rows ----
template <int D, int NB>
__global__ __launch_bounds__(kSweepThreads, 2) void accumulate_rows_kernel(Accum a)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    for_parts<false, stationary(NB)>(a, [&](const Place& p, int, int block, int tile0, int n_tiles, int slot, bool shared) {
        const int j0 = tile0 * kStream;
        if (wave == kComputeWaves) {
            load_stream<D>(lds, n_tiles, KeyWalk(a, p, j0), [](int) {});
            return;
        }
        Wave<D, NB, false, true> w;
        w.begin(lds, a.g.c_log2);
        const int r_wave = block * stationary(NB) + wave * NB * 32;
        int vis[NB];                           // last key that the lane's row sees, from the part's first
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            load_fragments<D, NB>(w.still[b], [&](int i) { return a.q + q_offset(a, p, min(r_wave + b * 32 + i, p.R - 1)); });
            vis[b] = last_key(a, p, min(r_wave + b * 32 + w.col, p.R - 1)) - j0;
        }
        // tiles that every row of the wave sees, and that some row does
        int all = 0, some = 0;
        if (r_wave < p.R) {
            all = min(max(0, last_key(a, p, r_wave) + 1 - j0) / kStream, n_tiles);
            some = min((max(0, last_key(a, p, min(r_wave + NB * 32, p.R) - 1) + 1 - j0) + kStream - 1) / kStream, n_tiles);
        }
        all = __builtin_amdgcn_readfirstlane(all);
        some = __builtin_amdgcn_readfirstlane(some);
        auto none = [](int) { return 0.f; };
        sweep_barrier();                       // the first tiles are in the ring
        w.plain(0, all, none);
        w.masked(all, some, none, [&](int blk, int b) { return vis[b] - blk * 32; });
        for (int t = some; t < n_tiles; ++t) sweep_barrier();
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            // the two halves of the wave hold different keys of the same row
            const float m2 = __shfl_xor(w.m[b], 32, 64), l2 = __shfl_xor(w.l[b], 32, 64);
            const float M = fmaxf(w.m[b], m2), ref = M == -INFINITY ? 0.f : M;
            const float sum = w.l[b] * fast_exp2(w.m[b] - ref) + l2 * fast_exp2(m2 - ref);
            const int r = r_wave + b * 32 + w.col;
            if (w.hf == 0 && r < p.R) {
                if (shared) a.stats[slot * stationary(NB) + wave * NB * 32 + b * 32 + w.col] = make_float2(M, sum);
                else a.norms[stat_row(a, p, r)] = norm_from(M, sum);
            }
        }
    });
}

// The statistics of rows whose block has several parts, joined to one norm each. A workgroup per block.
__global__ __launch_bounds__(kThreads) void accumulate_norm_kernel(Accum a, int max_blocks)
{
    const int head = blockIdx.x / max_blocks, block = blockIdx.x - head * max_blocks;
    const Place p = place_of(a, head);
    if (block >= p.item_of.row_blocks(a.block)) return;
    int first, n;
    parts_of(a.spans, head, block, &first, &n);
    if (n == 1) return;
    const int end = min((block + 1) * a.block, p.R);
    for (int r = block * a.block + threadIdx.x; r < end; r += kThreads) {
        const float2* st = a.stats + (r - block * a.block);
        float M = -INFINITY, Z = 0.f;
        for (int c0 = 0; c0 < n; c0 += 8) {
            float2 s[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) s[c] = st[part_slot_of(first, min(c0 + c, n - 1)) * a.block];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                if (c0 + c >= n) continue;
                const float M2 = fmaxf(M, s[c].x), ref = M2 == -INFINITY ? 0.f : M2;
                Z = Z * fast_exp2(M - ref) + s[c].y * fast_exp2(s[c].x - ref);
                M = M2;
            }
        }
        a.norms[stat_row(a, p, r)] = norm_from(M, Z);
    }
}

// ---- cols: column sums of blocks of stationary(NB) keys ----
template <int D, int NB, bool PIPE>
__global__ __launch_bounds__(kSweepThreads, 2) void accumulate_cols_kernel(Accum a)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    float* norm = reinterpret_cast<float*>(lds + kStages * kStream * D * 2);      // of a tile's rows, beside the tile in the ring
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    for_parts<true, stationary(NB)>(a, [&](const Place& p, int head, int block, int tile0, int n_tiles, int slot, bool shared) {
        const int r0 = p.item_of.key_tiles_from(block, stationary(NB)) + tile0 * kStream;
        if (wave == kComputeWaves) {
            load_stream<D>(lds, n_tiles, RowWalk(a, p, r0), [&](int t) {
                const int r = min(r0 + t * kStream + lane, p.R - 1);
                const float* src;
                if (a.lse) {
                    const int i = query_of(a, r), hq = p.h * a.g.G + (r - i * a.g.G);
                    src = a.lse + p.q0 * a.g.H_q + (int64_t)hq * p.Q + i;
                } else {
                    src = a.norms + stat_row(a, p, r);
                }
                __builtin_amdgcn_global_load_lds((global_void_ptr)src, (lds_void_ptr)(norm + (t % kStages) * kStream), 4, 0, 0);
            });
            return;
        }
        Wave<D, NB, true, PIPE> w;
        w.begin(lds, a.g.c_log2);
        const int key0 = block * stationary(NB) + wave * NB * 32;
#pragma unroll
        for (int b = 0; b < NB; ++b)
            load_fragments<D, NB>(w.still[b], [&](int i) {
                return a.k + kv_row_offset(a.g, p.item, p.tok0, p.L, p.h, min(key0 + b * 32 + i, p.L - 1));
            });
        // tiles that see none of the wave's keys, and the first that sees them all
        int none = n_tiles, all = n_tiles;
        if (key0 < p.L) {
            none = min(max(0, p.item_of.first_row(key0) - r0) / kStream, n_tiles);
            all = min((max(0, p.item_of.first_row(min(key0 + NB * 32, p.L) - 1) - r0) + kStream - 1) / kStream, n_tiles);
        }
        none = __builtin_amdgcn_readfirstlane(none);
        all = __builtin_amdgcn_readfirstlane(all);
        const bool given = a.lse != nullptr;
        const int end = p.R - r0 - w.col;      // the lane's row of a block 32 * blk rows on is there below it
        auto norm_of = [&](int blk) {
            float v = norm[((blk >> 1) % kStages) * kStream + (blk & 1) * 32 + w.col];
            if (given) v = v == -INFINITY ? INFINITY : v * 1.44269504088896340736f;      // (-inf: the row saw nothing, and gives nothing)
            return blk * 32 < end ? v : INFINITY;                                        // no such row: exp2(z - inf) = 0
        };
        sweep_barrier();                       // the first tiles are in the ring
        for (int t = 0; t < none; ++t) sweep_barrier();
        w.masked(none, all, norm_of, [&](int blk, int b) { return last_key(a, p, min(r0 + blk * 32 + w.col, p.R - 1)) - key0 - b * 32; });
        w.plain(all, n_tiles, norm_of);
        // The lanes of a half hold the same sixteen keys of different rows: with every exchange a lane keeps half of its keys, until
        // it has one, that of its number mod 16, and so has the lane sixteen on.
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int o = 8, n = 16; o > 0; o >>= 1, n >>= 1) {
                const bool upper = lane & o;
#pragma unroll
                for (int i = 0; i < n / 2; ++i) {
                    const float keep = upper ? w.sum[b][i + n / 2] : w.sum[b][i], give = upper ? w.sum[b][i] : w.sum[b][i + n / 2];
                    w.sum[b][i] = keep + __shfl_xor(give, o, 64);
                }
            }
            const float mine = w.sum[b][0] + __shfl_xor(w.sum[b][0], 16, 64);
            const int j = key0 + b * 32 + key_of(lane & 15, w.hf);
            if (w.col < 16 && j < p.L) {
                if (shared) {
                    a.parts[slot * stationary(NB) + wave * NB * 32 + b * 32 + key_of(lane & 15, w.hf)] = mine;
                } else {
                    float* to = a.weights + (a.pitch ? head * a.pitch : p.tok0 * a.g.H_kv + (int64_t)p.h * p.L);
                    to[j] += mine;
                }
            }
        }
    });
}

// weights += the column sums of keys whose block has several parts. A workgroup per block.
__global__ __launch_bounds__(kThreads) void accumulate_join_kernel(Accum a, int max_blocks)
{
    const int head = blockIdx.x / max_blocks, block = blockIdx.x - head * max_blocks;
    const Place p = place_of(a, head);
    if (block >= p.item_of.key_blocks(a.block)) return;
    int first, n;
    parts_of(a.spans, head, block, &first, &n);
    if (n == 1) return;
    const int end = min((block + 1) * a.block, p.L);
    for (int j = block * a.block + threadIdx.x; j < end; j += kThreads) {
        const float* src = a.parts + (j - block * a.block);
        float v = 0.f;
#pragma unroll 8
        for (int c = 0; c < n; ++c) v += src[part_slot_of(first, c) * a.block];
        a.weights[(a.pitch ? head * a.pitch : p.tok0 * a.g.H_kv + (int64_t)p.h * p.L) + j] += v;
    }
}

}  // namespace

// Pure function of the batch, so that the workspace query and the launch agree.
AccumPlan accumulate_plan(const Geom& g, const int32_t* seqlens, const int32_t* queries, int n_items)
{
    AccumPlan p;
    double pairs = 0.;
    for (int i = 0; i < n_items; ++i) {
        const double L = seqlens[i], Q = queries[i];
        p.max_L = seqlens[i] > p.max_L ? seqlens[i] : p.max_L;
        p.max_Q = queries[i] > p.max_Q ? queries[i] : p.max_Q;
        p.rows_total += (long long)queries[i] * g.H_q;
        pairs += (g.causal ? Q * (L - Q) + Q * (Q + 1.) / 2. : Q * L) * g.H_q;
    }
    // two tiles per wave where they still make eight tiles of work for every CU
    p.tiles_per_wave = pairs / (stationary(2) * (double)kStream) >= 8. * kSpans ? 2 : 1;
    // launches stay below 2^32 threads, tiles below 2^31, and a row's number below what query_of divides exactly
    const double rows = (double)p.max_Q * g.G, blocks = (rows > p.max_L ? rows : p.max_L) / stationary(1) + 1.;
    p.too_large = (double)n_items * g.H_kv * blocks >= 8388608. || rows * g.G >= 2147483648. ||
                  pairs / (stationary(1) * (double)kStream) + (double)n_items * g.H_kv * blocks * (g.G + 2.) >= 2e9;
    if (p.too_large) return p;
    auto item = [&](int i) { return AccumItem{seqlens[i], queries[i], g.G, g.causal}; };
    p.rows = plan_sweep(false, stationary(p.tiles_per_wave), n_items, g.H_kv, kLeastTiles, item);
    p.cols = plan_sweep(true, stationary(p.tiles_per_wave), n_items, g.H_kv, kLeastTiles, item);
    return p;
}

namespace {
inline size_t up(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
// entries for the parts of blocks that have several
inline size_t part_entries(const AccumSweep& s) { return s.max_parts > 1 ? (size_t)part_slots(s.spans.n) * s.size : 0; }
}  // namespace

size_t accumulate_stats_bytes(const AccumPlan& p) {
    return up((size_t)p.rows_total * sizeof(float)) + up(part_entries(p.rows) * sizeof(float2));
}
size_t accumulate_parts_bytes(const AccumPlan& p) { return part_entries(p.cols) * sizeof(float); }
namespace {
// more than 64 KB of LDS have to be asked for, once per device and kernel
template <class Kernel>
hipError_t launch_sweep(Kernel kernel, unsigned lds, const AccumSweep& sweep, Accum& a, hipStream_t s)
{
    a.spans = sweep.spans;
    a.block = sweep.size;
    if (sweep.spans.n == 0) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((sweep.spans.n + 7) / 8 * 8)), dim3(kSweepThreads), lds, s, a);
    return hipGetLastError();
}
template <int D>
hipError_t launch_sweeps(const Geom& g, const AccumPlan& p, Accum& a, hipStream_t s)
{
    constexpr unsigned ring = kStages * kStream * D * 2;
    const int heads = g.n_items * g.H_kv;
    const bool two = p.tiles_per_wave == 2;
    hipError_t e = hipSuccess;
    if (!a.lse) {
        e = two ? launch_sweep(accumulate_rows_kernel<D, 2>, ring, p.rows, a, s) : launch_sweep(accumulate_rows_kernel<D, 1>, ring, p.rows, a, s);
        if (e == hipSuccess && p.rows.max_parts > 1) {
            hipLaunchKernelGGL(accumulate_norm_kernel, dim3((unsigned)(heads * p.rows.max_blocks)), dim3(kThreads), 0, s, a, p.rows.max_blocks);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
    }
    constexpr unsigned norms = kStages * kStream * sizeof(float);
    e = two ? launch_sweep(accumulate_cols_kernel<D, 2, D != 256>, ring + norms, p.cols, a, s)
            : launch_sweep(accumulate_cols_kernel<D, 1, true>, ring + norms, p.cols, a, s);
    if (e != hipSuccess || p.cols.max_parts == 1) return e;
    hipLaunchKernelGGL(accumulate_join_kernel, dim3((unsigned)(heads * p.cols.max_blocks)), dim3(kThreads), 0, s, a, p.cols.max_blocks);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_accumulate(const Geom& g, const AccumPlan& p, const void* q, const void* k, const int32_t* cu_seqlens,
                             const int32_t* cu_queries, const float* lse, float* weights, int64_t pitch, void* workspace, hipStream_t s)
{
    Accum a{};
    char* ws = static_cast<char*>(workspace);
    a.g = g;
    a.q = static_cast<const __bf16*>(q);
    a.k = static_cast<const __bf16*>(k);
    a.cu_seq = cu_seqlens;
    a.cu_q = cu_queries;
    a.lse = lse;
    if (!lse) {                                // (otherwise there may be no workspace at all)
        a.norms = reinterpret_cast<float*>(ws);
        a.stats = reinterpret_cast<float2*>(ws + up((size_t)p.rows_total * sizeof(float)));
        ws += accumulate_stats_bytes(p);
    }
    a.parts = reinterpret_cast<float*>(ws);
    a.weights = weights;
    a.pitch = pitch;
    a.div_g = g.G > 1 ? (unsigned)((0x100000000ULL + g.G - 1) / g.G) : 0;
    switch (g.D) {
        case 64:  return launch_sweeps<64>(g, p, a, s);
        case 128: return launch_sweeps<128>(g, p, a, s);
        case 256: return launch_sweeps<256>(g, p, a, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace audiokv

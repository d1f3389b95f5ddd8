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
// The long side is cut into ranges of equal size (rows: of keys, cols: of rows), a workgroup per (block, range) that has a
// visible pair: all workgroups cost the same but those on the diagonal. Column sums of several ranges are joined by a third
// kernel in fixed order; row statistics by the workgroups of cols, for their rows, before they start. No atomics.
//
// References of a row are not maxima (see score_impl.h): the first logits set one, and only a tile whose sum leaves the safe
// range is redone against a new one. Everything is in base-2 units: z = <q,k> * scale * log2(e).
#include "mfma_tile.h"

namespace audiokv {

namespace {

using namespace mfma_tile;

constexpr int kStream = 64;               // rows of a tile that streams through LDS
constexpr int kMaxRowsPerRange = 2048;    // cols: rows whose log-sum-exp a workgroup keeps in LDS

struct Accum {
    Geom g;
    const __bf16* q;
    const __bf16* k;
    const int32_t* cu_seq;
    const int32_t* cu_q;
    const float* lse;          // given, or nullptr
    float2* stats;             // [key range][row of all items] (reference, sum)
    float* parts;              // [row range][head][longest item, padded]
    float* weights;
    int64_t pitch;             // between heads of weights; 0: packed like scores
    int64_t rows_total;        // of all items
    unsigned div_g;            // r / G = umulhi(r, div_g), G > 1
    int key_range, row_range;  // keys, rows of a range
    int n_key_ranges, n_row_ranges, n_row_blocks, n_key_blocks;
    int part_pitch;
};

struct Place {
    int item, h, L, Q, R;
    int64_t tok0, q0;          // first token and first query of the item
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
// first row that sees key j
__device__ __forceinline__ int first_row(const Accum& a, const Place& p, int j) {
    return a.g.causal ? max(0, j - (p.L - p.Q)) * a.g.G : 0;
}
__device__ __forceinline__ int64_t stat_row(const Accum& a, const Place& p, int r) { return p.q0 * a.g.H_q + (int64_t)p.h * p.R + r; }

// ---- rows: statistics of NB * 128 rows over a range of keys ----
template <int D, int NB>
__global__ __launch_bounds__(kThreads, 2) void accumulate_rows_kernel(Accum a)
{
    constexpr int KK = D / 16, N = kPieces<D, kStream>;
    __shared__ __attribute__((aligned(16))) __bf16 tile[2][kStream * D];
    const int range = blockIdx.x % a.n_key_ranges, rest = blockIdx.x / a.n_key_ranges;
    const int block = rest % a.n_row_blocks;
    const Place p = place_of(a, rest / a.n_row_blocks);
    const int r_first = block * (NB * 32 * kWaves);
    if (r_first >= p.R) return;
    const int j0 = range * a.key_range;
    const int seen = last_key(a, p, min(r_first + NB * 32 * kWaves, p.R) - 1);       // by the last row of the block
    const int j1 = min(j0 + a.key_range, seen + 1);
    if (j0 >= j1) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5, col = lane & 31;

    bf16x8 qf[NB][KK];
    int vis[NB], least[NB];            // last key that the lane's row sees, and the first row of the tile
    float m[NB], l[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int r = r_first + (wave * NB + b) * 32 + col;
        const __bf16* src = a.q + q_offset(a, p, min(r, p.R - 1)) + hf * 8;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) qf[b][kk] = *reinterpret_cast<const bf16x8*>(src + kk * 16);
        vis[b] = last_key(a, p, r);
        least[b] = __builtin_amdgcn_readfirstlane(min(last_key(a, p, r_first + (wave * NB + b) * 32),
                                                      last_key(a, p, r_first + (wave * NB + b) * 32 + 31)));   // -1: some are no rows
        m[b] = -INFINITY;
        l[b] = 0.f;
    }
    const int chunk = piece_chunk<D>() * 8;
    u32x4 piece[N];
    auto fetch = [&](int j) {
#pragma unroll
        for (int u = 0; u < N; ++u)
            piece[u] = *reinterpret_cast<const u32x4*>(
                a.k + kv_row_offset(a.g, p.item, p.tok0, p.L, p.h, min(j + piece_row<D>(u), p.L - 1)) + chunk);
    };
    fetch(j0);
    put_tile<D>(tile[0], piece);
    __syncthreads();
    for (int j = j0, at = 0; j < j1; j += kStream, at ^= 1) {
        if (j + kStream < j1) fetch(j + kStream);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < kStream / 32; ++s) {
            const int key0 = j + s * 32;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                f32x16 z = {};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
                    z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fragment<D>(tile[at], s * 32 + col, kk, hf), qf[b][kk], z, 0, 0, 0);
                // keys past the range belong to another workgroup's
                const int most = min(vis[b], j1 - 1);
                if (key0 + 31 > min(least[b], j1 - 1)) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[i] = key0 + key_of(i, hf) <= most ? z[i] : -INFINITY;
                }
                float sum = 0.f;
                const float mc = m[b];
#pragma unroll
                for (int i = 0; i < 16; ++i) sum += fast_exp2(__builtin_fmaf(z[i], a.g.c_log2, -mc));
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum < 0x1p64f)) != 0, 0)) {
                    // the first logits of a lane (its reference is -inf), or far above its reference, or NaN
                    float top = z[0];
#pragma unroll
                    for (int i = 1; i < 16; ++i) top = fmaxf(top, z[i]);
                    const bool redo = !(sum < 0x1p64f);
                    const float ref = redo ? fmaxf(mc, top * a.g.c_log2) : mc, ref0 = ref == -INFINITY ? 0.f : ref;
                    float again = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) again += fast_exp2(__builtin_fmaf(z[i], a.g.c_log2, -ref0));
                    l[b] = redo ? l[b] * fast_exp2(mc - ref0) : l[b];
                    sum = redo ? again : sum;
                    m[b] = ref;
                }
                l[b] += sum;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (j + kStream < j1) put_tile<D>(tile[at ^ 1], piece);
        __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        // the two halves of the wave hold different keys of the same row
        const float m2 = __shfl_xor(m[b], 32, 64), l2 = __shfl_xor(l[b], 32, 64);
        const float M = fmaxf(m[b], m2), ref = M == -INFINITY ? 0.f : M;
        const float sum = l[b] * fast_exp2(m[b] - ref) + l2 * fast_exp2(m2 - ref);
        const int r = r_first + (wave * NB + b) * 32 + col;
        if (hf == 0 && r < p.R) a.stats[(int64_t)range * a.rows_total + stat_row(a, p, r)] = make_float2(M, sum);
    }
}

// ---- cols: column sums of 256 keys over a range of rows ----
constexpr int kKeyTiles = 2, kKeyBlock = kKeyTiles * 32 * kWaves;

template <int D>
__global__ __launch_bounds__(kThreads, 2) void accumulate_cols_kernel(Accum a)
{
    constexpr int KK = D / 16, N = kPieces<D, kStream>;
    __shared__ __attribute__((aligned(16))) __bf16 tile[2][kStream * D];
    __shared__ float norm[kMaxRowsPerRange + kStream];        // log2 of a row's sum of exp2, by row of the range
    const int range = blockIdx.x % a.n_row_ranges, rest = blockIdx.x / a.n_row_ranges;
    const int block = rest % a.n_key_blocks, head = rest / a.n_key_blocks;
    const Place p = place_of(a, head);
    const int k_first = block * kKeyBlock;
    if (k_first >= p.L) return;
    const int r1 = min((range + 1) * a.row_range, p.R);
    const int r0 = max(range * a.row_range, first_row(a, p, k_first) & ~31);
    if (r0 >= r1) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5, col = lane & 31;

    // key tiles, the stationary operand
    bf16x8 kf[kKeyTiles][KK];
    const int key0 = k_first + wave * (kKeyTiles * 32);
#pragma unroll
    for (int b = 0; b < kKeyTiles; ++b) {
        const __bf16* src = a.k + kv_row_offset(a.g, p.item, p.tok0, p.L, p.h, min(key0 + b * 32 + col, p.L - 1)) + hf * 8;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) kf[b][kk] = *reinterpret_cast<const bf16x8*>(src + kk * 16);
    }
    const int chunk = piece_chunk<D>() * 8;
    u32x4 piece[N];
    auto fetch = [&](int r) {
#pragma unroll
        for (int u = 0; u < N; ++u)
            piece[u] = *reinterpret_cast<const u32x4*>(a.q + q_offset(a, p, min(r + piece_row<D>(u), p.R - 1)) + chunk);
    };
    fetch(r0);
    for (int r = r0 + tid; r < r1 + kStream; r += kThreads) {
        float v = INFINITY;                                   // no such row: exp2(z - inf) = 0
        if (r < r1) {
            if (a.lse) {
                const int i = query_of(a, r), hq = p.h * a.g.G + (r - i * a.g.G);
                const float given = a.lse[p.q0 * a.g.H_q + (int64_t)hq * p.Q + i];
                v = given == -INFINITY ? INFINITY : given * 1.44269504088896340736f;
            } else {
                const int n = last_key(a, p, r) / a.key_range + 1;
                const float2* st = a.stats + stat_row(a, p, r);
                float M = -INFINITY, Z = 0.f;
                for (int c = 0; c < n; ++c) {
                    const float2 s = st[(int64_t)c * a.rows_total];
                    const float M2 = fmaxf(M, s.x), ref = M2 == -INFINITY ? 0.f : M2;
                    Z = Z * fast_exp2(M - ref) + s.y * fast_exp2(s.x - ref);
                    M = M2;
                }
                v = Z == 0.f ? INFINITY : M + __log2f(Z);     // nothing but -inf: the row gives nothing
            }
        }
        norm[r - r0] = v;
    }
    put_tile<D>(tile[0], piece);
    __syncthreads();

    float sum[kKeyTiles][16];
#pragma unroll
    for (int b = 0; b < kKeyTiles; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[b][i] = 0.f;
    for (int r = r0, at = 0; r < r1; r += kStream, at ^= 1) {
        if (r + kStream < r1) fetch(r + kStream);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < kStream / 32; ++s) {
            const int row0 = r + s * 32;
            const float c = norm[row0 + col - r0];
            const int vis = row0 + col < r1 ? last_key(a, p, row0 + col) : -1;
            const int least = __builtin_amdgcn_readfirstlane(row0 + 31 < r1 ? last_key(a, p, row0) : -1);
#pragma unroll
            for (int b = 0; b < kKeyTiles; ++b) {
                f32x16 z = {};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
                    z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[b][kk], fragment<D>(tile[at], s * 32 + col, kk, hf), z, 0, 0, 0);
                if (key0 + b * 32 + 31 <= least) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) sum[b][i] += fast_exp2(__builtin_fmaf(z[i], a.g.c_log2, -c));
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float e = fast_exp2(__builtin_fmaf(z[i], a.g.c_log2, -c));
                        sum[b][i] += key0 + b * 32 + key_of(i, hf) <= vis ? e : 0.f;
                    }
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (r + kStream < r1) put_tile<D>(tile[at ^ 1], piece);
        __syncthreads();
    }
    // the lanes of a half hold the same keys of different rows
#pragma unroll
    for (int b = 0; b < kKeyTiles; ++b) {
        float mine = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float v = sum[b][i];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
            mine = (lane & 15) == i ? v : mine;
        }
        const int j = key0 + b * 32 + key_of(lane & 15, hf);
        if (col < 16 && j < p.L) {
            if (a.n_row_ranges > 1) {
                a.parts[((int64_t)range * a.g.n_items * a.g.H_kv + head) * a.part_pitch + j] = mine;
            } else {
                float* w = a.weights + (a.pitch ? head * a.pitch : p.tok0 * a.g.H_kv + (int64_t)p.h * p.L);
                w[j] += mine;
            }
        }
    }
}

// weights += the column sums of the row ranges that see the key's block
__global__ __launch_bounds__(kThreads) void accumulate_join_kernel(Accum a, int blocks)
{
    const int head = blockIdx.x / blocks;
    const Place p = place_of(a, head);
    const int j = (blockIdx.x - head * blocks) * kThreads + threadIdx.x;
    if (j >= p.L) return;
    const int first = (first_row(a, p, j / kKeyBlock * kKeyBlock) & ~31) / a.row_range, n = (p.R + a.row_range - 1) / a.row_range;
    if (first >= n) return;
    const int64_t step = (int64_t)a.g.n_items * a.g.H_kv * a.part_pitch;
    const float* src = a.parts + (int64_t)head * a.part_pitch + j;
    float v = 0.f;
#pragma unroll 8
    for (int c = first; c < n; ++c) v += src[c * step];
    a.weights[(a.pitch ? head * a.pitch : p.tok0 * a.g.H_kv + (int64_t)p.h * p.L) + j] += v;
}

}  // namespace

// How a call is cut. Pure function of the batch, so that the workspace query and the launch agree.
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
    const long long R = (long long)p.max_Q * g.G;
    constexpr double kWorkgroups = 1024.;                 // two rounds of two per CU
    auto round_up = [](double x, int to, long long least, long long most) {
        long long v = ((long long)x / to + 1) * to;
        return v < least ? least : v > most ? most : v;
    };
    p.row_tiles = pairs / (256. * 64.) >= 65536. ? 2 : 1;
    const int row_block = p.row_tiles * 32 * kWaves;
    const long long least = ((long long)p.max_L + 15) / 16;               // sixteen key ranges at most
    p.key_range = (int)round_up(pairs / (kWorkgroups * row_block), kStream, (least + kStream - 1) / kStream * kStream, 1LL << 30);
    if (p.key_range < 256) p.key_range = 256;
    p.n_key_ranges = (p.max_L + p.key_range - 1) / p.key_range;
    p.row_range = (int)round_up(pairs / (kWorkgroups * kKeyBlock), kStream, 256, kMaxRowsPerRange);
    p.n_row_ranges = (int)((R + p.row_range - 1) / p.row_range);
    p.n_row_blocks = (int)((R + row_block - 1) / row_block);
    p.n_key_blocks = (p.max_L + kKeyBlock - 1) / kKeyBlock;
    p.part_pitch = p.n_key_blocks * kKeyBlock;
    return p;
}

size_t accumulate_stats_bytes(const AccumPlan& p) {
    return ((size_t)p.n_key_ranges * (size_t)p.rows_total * sizeof(float2) + 255) & ~(size_t)255;
}
size_t accumulate_parts_bytes(const Geom& g, const AccumPlan& p) {
    return p.n_row_ranges > 1 ? (size_t)p.n_row_ranges * g.n_items * g.H_kv * p.part_pitch * sizeof(float) : 0;
}
// launches stay below 2^32 threads, and a row's number below what query_of divides exactly
bool accumulate_supported(const Geom& g, const AccumPlan& p) {
    const double heads = (double)g.n_items * g.H_kv, most = 8388608.;
    return heads * p.n_key_ranges * p.n_row_blocks < most && heads * p.n_row_ranges * p.n_key_blocks < most &&
           (double)p.max_Q * g.G * g.G < 4294967296.;
}

hipError_t launch_accumulate(const Geom& g, const AccumPlan& p, const void* q, const void* k, const int32_t* cu_seqlens,
                             const int32_t* cu_queries, const float* lse, float* weights, int64_t pitch, void* workspace, hipStream_t s)
{
    Accum a{};
    a.g = g;
    a.q = static_cast<const __bf16*>(q);
    a.k = static_cast<const __bf16*>(k);
    a.cu_seq = cu_seqlens;
    a.cu_q = cu_queries;
    a.lse = lse;
    a.stats = static_cast<float2*>(workspace);
    a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + (lse ? 0 : accumulate_stats_bytes(p)));
    a.weights = weights;
    a.pitch = pitch;
    a.rows_total = p.rows_total;
    a.div_g = g.G > 1 ? (unsigned)((0x100000000ULL + g.G - 1) / g.G) : 0;
    a.key_range = p.key_range;
    a.row_range = p.row_range;
    a.n_key_ranges = p.n_key_ranges;
    a.n_row_ranges = p.n_row_ranges;
    a.n_row_blocks = p.n_row_blocks;
    a.n_key_blocks = p.n_key_blocks;
    a.part_pitch = p.part_pitch;
    const int heads = g.n_items * g.H_kv;
    const dim3 rows((unsigned)(heads * p.n_row_blocks * p.n_key_ranges)), cols((unsigned)(heads * p.n_key_blocks * p.n_row_ranges));
    const dim3 threads(kThreads);
#define AUDIOKV_ACCUMULATE(DD)                                                                                       \
    do {                                                                                                             \
        if (!lse) {                                                                                                  \
            if (p.row_tiles == 2) hipLaunchKernelGGL((accumulate_rows_kernel<DD, 2>), rows, threads, 0, s, a);       \
            else hipLaunchKernelGGL((accumulate_rows_kernel<DD, 1>), rows, threads, 0, s, a);                        \
        }                                                                                                            \
        hipLaunchKernelGGL((accumulate_cols_kernel<DD>), cols, threads, 0, s, a);                                    \
    } while (0)
    switch (g.D) {
        case 64:  AUDIOKV_ACCUMULATE(64);  break;
        case 128: AUDIOKV_ACCUMULATE(128); break;
        case 256: AUDIOKV_ACCUMULATE(256); break;
        default: return hipErrorInvalidValue;
    }
#undef AUDIOKV_ACCUMULATE
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.n_row_ranges == 1) return e;
    const int blocks = (p.max_L + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(accumulate_join_kernel, dim3((unsigned)(heads * blocks)), threads, 0, s, a, blocks);
    return hipGetLastError();
}

}  // namespace audiokv

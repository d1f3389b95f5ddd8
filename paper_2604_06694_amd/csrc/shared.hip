// One decoding step of sequences that share compacted caches: sequence x continues item i, attends to the rows that the
// eviction kept of i's prompt (packed, read once for all sequences of the item) and to rows of its own (slots of a growing
// cache, to which the step appends one).
//
//   out[x, q] = softmax over both sets of rows (scale * <q, K>) V          weights[own row] += sum over the group's q of p
//
// The queries of an item's sequences that read one KV head, S * G of them, are the rows of a product with the prompt's keys; a
// sequence's own rows meet its G queries only. Both are the same work for a workgroup of four waves: up to 128 query rows
// against a chunk of rows of K and V. C = K Q^T on v_mfma_f32_32x32x16_bf16 leaves a lane with one query row (mfma_tile.h):
// exponentials and their sum stay in the lane, and four keys at a time its weights, as bf16, are already the operand of
// O^T = V^T P^T, whose other operand the transposing LDS read fetches from V as it lies. A weight is the sum of two bf16 values, good
// to 2^-15, and the product with V is taken twice: rounded to one, weights add as much error as the bf16 output's own rounding
// (against 64 bits 1.7e-3 -> 1.9e-3 to 2.5e-3 of the output). The second product costs 32 sequences on 13107 rows a head 29.2 -> 32.3 us
// a pass, 24 on eight prompts at d = 256 36.6 -> 38.0, and nothing where HBM or latency bounds. The sums that divide are of fp32 weights.
// 32 query rows a wave. Up to 64 rows the tile's keys are split over two (groups of) waves, joined at the end through LDS.
// A row's exponentials are taken against a reference, the maximum of the first tile: where a later sum leaves the safe range,
// accumulators and sum are rescaled (see score_impl.h; here the two halves of a wave share their row's reference, since the
// product joins their keys).
//
// Up to a few dozen query rows the bound is HBM, above it the matrix pipe. What a workgroup costs beside that is latency: the
// next tile is in flight, in registers, while one is worked on.
//
// Budgets, lengths and the sequences of an item are known on the device only. A chunk of prompt rows finds its head as in
// decode.hip: chunk c of head g has slot floor(cu_b[g] / R) + g + c. A second kernel joins the chunks of a query in fixed order
// and adds the own rows' weights from the logits that the first one left. No atomics.
#include "mfma_tile.h"

namespace audiokv {

namespace {

using namespace mfma_tile;

// At d = 256 tiles are half as long and a wave's accumulators half the channels (two waves then share their rows): so that two
// workgroups share a CU there, too.
template <int D> struct Shape {
    static constexpr int kTile = D == 256 ? 32 : 64;              // keys of a tile
    static constexpr int kSplit = D == 256 ? 2 : 1;               // waves that share 32 rows, each its part of the channels
    static constexpr int kRowWaves = kWaves / kSplit;             // 32 rows each
};
int max_row_block(int D) { return D == 256 ? 64 : 128; }          // query rows of a workgroup

struct Shared {
    Geom g;
    const __bf16* q;
    const __bf16 *kp, *vp;                    // prompts' rows
    const int32_t* cu_b;
    const int32_t* cu_seqs;
    int n_items, total_rows, n_seqs, max_seqs;
    int log_r, slots, slots_pad, row_block, row_blocks;  // prompt chunks; slots_pad: a multiple of 8, so that a chunk stays on one XCD
    __bf16 *ko, *vo;                          // own rows
    int32_t* lengths;
    int32_t* positions;
    float* weights;
    int capacity, max_own, own_chunk, own_chunks;
    const __bf16 *k_new, *v_new;
    const int32_t* pos_new;
    // What the chunks have found, by query: [D] sums and (reference, sum). A head's first chunk has a place per sequence, [KV head][seq][G];
    // later ones begin in the row block (of a chunk's length, from the prompts' first row on) that no other chunk begins in, and have
    // [row block - 1][max_seqs][G]; own rows' [own head][chunk][G]. So all of it follows the sequences that there are, not the widest
    // item times the heads.
    float* part;
    float2* stats;
    int64_t later_at, own_at;                 // where the second and third begin
    float* logits;                            // [own head][G][logit_pitch], base 2
    int logit_pitch;
    int32_t* after;                           // [own head]: 2 * rows after the step + whether one was appended
    __bf16* out;
};

__device__ __forceinline__ int head_start(const Shared& a, int g) { return min(max(a.cu_b[g], 0), a.total_rows); }
__device__ __forceinline__ int first_slot(const Shared& a, int g) { return (head_start(a, g) >> a.log_r) + g; }

// The last of n entries of a rising table of n + 1 whose value is not past v; the first is not. Tables of up to 63 entries are
// loaded at once, an entry per lane, and what follows is read from the lanes: one latency. Of longer ones 64 entries are probed at
// a time.
struct Entry {
    int at, value, next;       // the entry, its value and that of the one behind
};
template <typename Value>
__device__ __forceinline__ Entry last_at_or_before(int n, int v, Value value) {
    const int lane = threadIdx.x & 63;
    if (n < 64) {
        const int mine = value(min(lane, n));
        const int at = max(__builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < n && mine <= v)) - 1, 0);
        return Entry{at, __builtin_amdgcn_readlane(mine, at), __builtin_amdgcn_readlane(mine, at + 1)};
    }
    int at = 0;
    for (int span = n; span > 1;) {
        const int step = (span + 63) >> 6, probe = at + lane * step;
        const bool before = probe < at + span && value(min(probe, n - 1)) <= v;
        const int found = __builtin_popcountll(__builtin_amdgcn_ballot_w64(before));
        const int skip = found > 0 ? (found - 1) * step : 0;
        at += skip;
        span = min(step, span - skip);
    }
    at = __builtin_amdgcn_readfirstlane(at);
    return Entry{at, value(at), value(at + 1)};
}

// The item that sequence x continues and its first sequence; item -1: x takes no part. (Without prompts all take part, as item 0.)
struct ItemOf {
    int item, first;
};
__device__ __forceinline__ ItemOf item_of(const Shared& a, int x) {
    if (!a.cu_seqs) return ItemOf{0, 0};
    const Entry e = last_at_or_before(a.n_items, x, [&](int i) { return a.cu_seqs[i]; });
    return ItemOf{x >= e.value && x < e.next && x - e.value < a.max_seqs ? e.at : -1, e.value};
}

// What a workgroup attends to
struct Rows {
    const __bf16 *k, *v;       // first row of the chunk
    int64_t stride;            // elements between rows
    int n;                     // rows of the chunk
    int fresh;                 // row that is read from k_new / v_new and stored into k_dst / v_dst (-1: none)
    const __bf16 *k_new, *v_new;
    __bf16 *k_dst, *v_dst;
    float* logits;             // of the chunk's first row and the group's first query, or nullptr
};

// The upper part of a weight: itself with the lower half of its bits cleared, a bf16 value, and below the weight also where that half
// is clear (unless the weight is zero). The rest is then above zero: times an infinity both parts have its sign.
__device__ __forceinline__ float upper_part(float x) {
    return __uint_as_float(__builtin_elementwise_sub_sat(__float_as_uint(x), 1u) & 0xffff0000u);
}

template <int D>
__device__ __forceinline__ void attend(const Shared& a, const Rows& rows, int first_seq, int h, int r_first, int r_end, float* part, float2* stats)
{
    typedef Shape<D> W;
    constexpr int KK = D / 16, CT = D / 32 / W::kSplit, kTile = W::kTile, N = kPieces<D, kTile>;
    __shared__ __attribute__((aligned(16))) __bf16 tile[2][2][kTile * D];     // [buffer][K, V]
    __shared__ float2 joint[kWaves][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5, col = lane & 31;
    const int G = a.g.G;
    // waves over query rows, and, where these leave some and a tile has two, over its halves
    const int left = r_end - r_first, wq_n = left <= 32 ? 1 : left <= 64 || W::kRowWaves == 2 ? 2 : 4;
    const int part_of = wave % W::kSplit, wq = __builtin_amdgcn_readfirstlane(wave / W::kSplit % wq_n), wk = wave / W::kSplit / wq_n;
    const bool halves = kTile > 32 && wq_n < 4, works = wk < (halves ? 2 : 1);
    const int sub0 = halves ? wk : 0, sub1 = halves ? wk + 1 : kTile / 32;
    const int r_wave = r_first + wq * 32;

    // A tile's first row is uniform, and so is the distance to the rows of a thread's next piece.
    const int chunk = piece_chunk<D>() * 8;
    const int64_t apart = piece_row<D>(0) * rows.stride + chunk;
    constexpr int kStep = kThreads / (D / 8);
    // What only few tiles need is computed where they need it: kept from the start, addresses of the new row and the like took more
    // registers than d = 256 has left (ten spilled, some in every tile: 24 sequences on eight prompts 47 us a pass instead of 37).
    auto once = [](int x) {
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" : "+v"(x));
#endif
        return x;
    };
    auto other_half = [&](int x) { return __builtin_amdgcn_ds_bpermute((once(lane) ^ 32) * 4, x); };
    u32x4 kpiece[N], vpiece[N];
    auto plain = [&](int t) { return t + kTile <= rows.n && (rows.fresh < t || rows.fresh >= t + kTile); };
    auto fetch = [&](int t) {
        if (plain(t)) {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int64_t first = (t + u * kStep) * rows.stride;
                kpiece[u] = *reinterpret_cast<const u32x4*>(rows.k + first + apart);
                vpiece[u] = *reinterpret_cast<const u32x4*>(rows.v + first + apart);
            }
        } else {
            const int here = once(chunk);
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int j = t + piece_row<D>(u);
                const int64_t at = min(j, rows.n - 1) * rows.stride + here;
                kpiece[u] = *reinterpret_cast<const u32x4*>(j == rows.fresh ? rows.k_new + here : rows.k + at);
                vpiece[u] = *reinterpret_cast<const u32x4*>(j == rows.fresh ? rows.v_new + here : rows.v + at);
            }
        }
    };
    auto put = [&](int t, int buffer) {
        if (!plain(t)) {
            const int here = once(chunk);
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int j = t + piece_row<D>(u);
                if (j == rows.fresh) {                        // the new row takes its slot
                    *reinterpret_cast<u32x4*>(rows.k_dst + here) = kpiece[u];
                    *reinterpret_cast<u32x4*>(rows.v_dst + here) = vpiece[u];
                }
                // rows past the end have weight 0, but 0 times an infinity is NaN
                vpiece[u] = j < rows.n ? vpiece[u] : u32x4{0, 0, 0, 0};
            }
        }
        put_tile<D>(tile[buffer][0], kpiece);
        put_tile<D>(tile[buffer][1], vpiece);
    };

    fetch(0);
    bf16x8 qf[KK];
    load_fragments<D, 1>(qf, [&](int i) {
        const int rc = min(r_wave + i, r_end - 1);
        return a.q + ((int64_t)(first_seq + rc / G) * a.g.H_q + h * G + rc % G) * D;
    });
    f32x16 acc[CT] = {};
    float m = -INFINITY, l = 0.f;
    // the transposing read: sixteen lanes take four keys x sixteen channels, each lane then holds a channel's four keys
    const int tr_key = 4 * hf + ((lane & 15) >> 2), tr_chunk = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), tr_low = (lane & 1) * 4;
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    auto values = [&](const __bf16* v, int key0, int ct) {       // sixteen keys of 32 channels
        s16x4 four[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int row = key0 + e * 8 + tr_key;
            const __bf16* at = v + row * D + slot_of((part_of * CT + ct) * 4 + tr_chunk, row) * 8 + tr_low;
            typedef __attribute__((address_space(3))) s16x4* lds_ptr;
            four[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)const_cast<__bf16*>(at));
        }
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(four[0], four[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };

    put(0, 0);
    __syncthreads();
    for (int t = 0, at = 0; t < rows.n; t += kTile, at ^= 1) {
        if (t + kTile < rows.n) fetch(t + kTile);
        __builtin_amdgcn_sched_barrier(0);
        for (int s = sub0; works && s < sub1 && t + s * 32 < rows.n; ++s) {
            const int key0 = t + s * 32;
            // Fragments are requested four k-steps ahead of their MFMA, those of V for the first sixteen keys in front of the
            // exponentials: left alone the compiler waits for each in turn.
            const __bf16 *kt = tile[at][0] + s * 32 * D, *vt = tile[at][1] + s * 32 * D;
            f32x16 z = {};
            bf16x8 kf[4];
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) kf[kk] = fragment<D>(kt, col, kk, hf);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk % 4], qf[kk], z, 0, 0, 0);
                if (kk + 4 < KK) kf[kk % 4] = fragment<D>(kt, col, kk + 4, hf);
                __builtin_amdgcn_sched_barrier(0);
            }
            bf16x8 vf[CT];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) vf[ct] = values(vt, 0, ct);
            __builtin_amdgcn_sched_barrier(0);
            if (key0 + 32 > rows.n) {
                const int most = rows.n - key0 - 4 * once(hf);
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] = key_of(i, 0) < most ? z[i] : -INFINITY;
            }
            if (rows.logits && col < G && part_of == 0) {
                float* dst = rows.logits + (int64_t)col * a.logit_pitch + key0 + 4 * hf;
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<f32x4*>(dst + 2 * i) =
                        f32x4{z[i] * a.g.c_log2, z[i + 1] * a.g.c_log2, z[i + 2] * a.g.c_log2, z[i + 3] * a.g.c_log2};
            }
            float p[16], sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[i] = fast_exp2(__builtin_fmaf(z[i], a.g.c_log2, -m));
                sum += p[i];
            }
            const bool far = !(sum < 0x1p10f);
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(far) != 0, 0)) {
                float top = z[0];
#pragma unroll
                for (int i = 1; i < 16; ++i) top = fmaxf(top, z[i]);
                top = fmaxf(top, __int_as_float(other_half(__float_as_int(top))));
                const int theirs = other_half((int)far);       // (in front of the test: all lanes take part)
                const bool redo = far | (theirs != 0);
                const float ref = redo ? fmaxf(m, top * a.g.c_log2) : m, ref0 = ref == -INFINITY ? 0.f : ref;
                const float by = redo ? fast_exp2(m - ref0) : 1.f;
                sum = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    p[i] = fast_exp2(__builtin_fmaf(z[i], a.g.c_log2, -ref0));
                    sum += p[i];
                }
                l *= by;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[ct][i] *= by;
                m = ref;
            }
            l += sum;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                bf16x8 low;
                u32x4 pairs;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float p0 = p[kb * 8 + e], p1 = p[kb * 8 + e + 1], top0 = upper_part(p0), top1 = upper_part(p1);
                    pairs[e / 2] = __builtin_amdgcn_perm(__float_as_uint(top1), __float_as_uint(top0), 0x07060302);
                    low[e] = (__bf16)(p0 - top0);
                    low[e + 1] = (__bf16)(p1 - top1);
                }
                const bf16x8 high = __builtin_bit_cast(bf16x8, pairs);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) acc[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[ct], low, acc[ct], 0, 0, 0);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    acc[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[ct], high, acc[ct], 0, 0, 0);
                    if (kb == 0) vf[ct] = values(vt, 16, ct);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (t + kTile < rows.n) put(t + kTile, at ^ 1);
        __syncthreads();
    }

    // A lane has every second group of four channels of one row: rows are put together in LDS (where the tiles were), so that whole
    // ones are stored, and where a second wave had the other half of the keys it hands its share over there. Groups of four are
    // rotated by the row.
    constexpr int kGroups = CT * 8;
    f32x4* const all = reinterpret_cast<f32x4*>(&tile[0][0][0]);
    f32x4* mine = all + (wq * W::kSplit + part_of) * (32 * kGroups);
    auto group = [&](int ct, int i) { return col * kGroups + ((ct * 8 + i / 2 + hf) ^ (col & 15)); };
    l += __shfl_xor(l, 32, 64);
    // At d = 128 both waves' shares go there and all threads join and store them: one wave took 5000 cycles for it, a third of a short
    // workgroup's time (48 caches of up to 4096 rows 39.5 -> 36.4 us). Not at d = 64: 1024 sequences
    // with few rows 24.5 -> 23.8 us, but 48 caches of up to 4096 31.6 -> 33.1.
    if constexpr (D == 128) {
        if (halves) {                                         // uniform
            if (works) {
                mine = all + wave * (32 * kGroups);
                if (hf == 0) joint[wave][col] = make_float2(m, l);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) mine[group(ct, i)] = f32x4{acc[ct][i], acc[ct][i + 1], acc[ct][i + 2], acc[ct][i + 3]};
            }
            __syncthreads();
            f32x4* dst = reinterpret_cast<f32x4*>(part + (int64_t)r_first * D);
#pragma unroll 2
            for (int u = tid; u < left * kGroups; u += kThreads) {
                const int row = u / kGroups, c = u % kGroups, w = row >> 5, r = row & 31;
                const f32x4* at = all + (w * 32 + r) * kGroups + (c ^ (r & 15));
                const float2 s0 = joint[w][r], s1 = joint[w + wq_n][r];
                const float M = fmaxf(s0.x, s1.x), ref = M == -INFINITY ? 0.f : M, by = fast_exp2(s0.x - ref), other = fast_exp2(s1.x - ref);
                dst[u] = at[0] * by + at[wq_n * 32 * kGroups] * other;
                if (c == 0) stats[r_first + row] = make_float2(M, s0.y * by + s1.y * other);
            }
            return;
        }
    }
    if (halves) {                                             // uniform
        if (wk == 1) {
            joint[wq][lane] = make_float2(m, l);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int i = 0; i < 16; i += 4) mine[group(ct, i)] = f32x4{acc[ct][i], acc[ct][i + 1], acc[ct][i + 2], acc[ct][i + 3]};
        }
        __syncthreads();
    }
    if (wk != 0) return;
    float by = 1.f;
    if (halves) {
        const float2 o = joint[wq][lane];
        const float M2 = fmaxf(m, o.x), ref = M2 == -INFINITY ? 0.f : M2;
        by = fast_exp2(m - ref);
        const float other = fast_exp2(o.x - ref);
        l = l * by + o.y * other;
        m = M2;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const f32x4 v = mine[group(ct, i)];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[ct][i + e] = acc[ct][i + e] * by + v[e] * other;
            }
    }
    if (hf == 0 && part_of == 0 && r_wave + col < r_end) stats[r_wave + col] = make_float2(m, l);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int i = 0; i < 16; i += 4) mine[group(ct, i)] = f32x4{acc[ct][i], acc[ct][i + 1], acc[ct][i + 2], acc[ct][i + 3]};
    f32x4* dst = reinterpret_cast<f32x4*>(part + (int64_t)r_wave * D) + part_of * kGroups;
    const int n_rows = min(32, r_end - r_wave);
#pragma unroll
    for (int e = 0; e < 32 * kGroups; e += 64) {
        const int row = (e + lane) / kGroups, c = (e + lane) % kGroups;
        if (row < n_rows) dst[row * (D / 4) + c] = mine[row * kGroups + (c ^ (row & 15))];
    }
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void shared_partial_kernel(Shared a)
{
    const int prompt_blocks = a.slots_pad * a.row_blocks;
    Rows rows{};
    rows.fresh = -1;
    int first_seq, h, M, r_first = 0, r_end;
    float* part;
    float2* stats;
    if ((int)blockIdx.x < prompt_blocks) {
        const int block = blockIdx.x / a.slots_pad, slot = blockIdx.x - block * a.slots_pad;
        if (slot >= a.slots) return;
        const int n_heads = a.n_items * a.g.H_kv;
        const Entry e = last_at_or_before(n_heads, slot, [&](int g) { return first_slot(a, g); });
        const int head = e.at, item = head / a.g.H_kv;
        h = head - item * a.g.H_kv;
        const int c = slot - e.value, begin = head_start(a, head);
        const int64_t row0 = begin + ((int64_t)c << a.log_r);
        rows.n = (int)min((int64_t)1 << a.log_r, head_start(a, head + 1) - row0);
        first_seq = max(0, a.cu_seqs[item]);
        M = min(min(a.cu_seqs[item + 1], a.n_seqs) - first_seq, a.max_seqs) * a.g.G;
        r_first = block * a.row_block;
        r_end = min(M, r_first + a.row_block);
        if (c < 0 || rows.n <= 0 || r_first >= M) return;
        rows.k = a.kp + row0 * D;
        rows.v = a.vp + row0 * D;
        rows.stride = D;
        const int64_t base = c == 0 ? ((int64_t)h * a.n_seqs + first_seq) * a.g.G : a.later_at + ((row0 >> a.log_r) - 1) * a.max_seqs * a.g.G;
        part = a.part + base * D;
        stats = a.stats + base;
    } else {
        const int id = blockIdx.x - prompt_blocks, own = id / a.own_chunks, c = id - own * a.own_chunks;
        const int x = own / a.g.H_kv;
        h = own - x * a.g.H_kv;
        const int length = a.lengths[own];
        if (item_of(a, x).item < 0) return;
        const int before = max(0, min(length, a.max_own));
        const bool appends = a.k_new != nullptr && before < a.max_own;
        const int n = before + appends, j0 = c * a.own_chunk;
        if (c == 0 && threadIdx.x == 0) a.after[own] = 2 * n + appends;
        rows.n = min(a.own_chunk, n - j0);
        if (rows.n <= 0) return;
        first_seq = x;
        M = r_end = a.g.G;
        const int64_t at = kv_row_offset(a.g, x, (int64_t)x * a.capacity, a.capacity, h, j0);
        rows.k = a.ko + at;
        rows.v = a.vo + at;
        rows.stride = kv_tok_stride(a.g);
        if (appends && before >= j0 && before < j0 + a.own_chunk) {
            rows.fresh = before - j0;
            rows.k_new = a.k_new + (int64_t)own * D;
            rows.v_new = a.v_new + (int64_t)own * D;
            rows.k_dst = a.ko + at + rows.fresh * rows.stride;
            rows.v_dst = a.vo + at + rows.fresh * rows.stride;
        }
        const int64_t base = a.own_at + ((int64_t)own * a.own_chunks + c) * a.g.G;
        part = a.part + base * D;
        stats = a.stats + base;
        if (a.weights) rows.logits = a.logits + (int64_t)own * a.g.G * a.logit_pitch + j0;
    }
    attend<D>(a, rows, first_seq, h, r_first, r_end, part, stats);
}

// The chunks that a query of sequence x has rows in, first those of the prompt, then its own: where each has its result
struct Chunks {
    int64_t first, later, own; // of the prompt's chunk 0, of its chunk c less c steps, of the first own one
    int64_t step;
    int np, no, G;
    __device__ __forceinline__ int64_t at(int c) const { return c >= np ? own + (int64_t)(c - np) * G : c == 0 ? first : later + c * step; }
};
// after: of the sequence's own head h
__device__ __forceinline__ Chunks chunks_of(const Shared& a, int x, ItemOf it, int h, int gq, int after) {
    Chunks t{0, 0, 0, 0, 0, 0, a.g.G};
    if (a.cu_seqs) {
        const int head = it.item * a.g.H_kv + h, begin = head_start(a, head), n = head_start(a, head + 1) - begin;
        t.np = n > 0 ? (n + (1 << a.log_r) - 1) >> a.log_r : 0;
        t.step = (int64_t)a.max_seqs * a.g.G;
        t.first = ((int64_t)h * a.n_seqs + x) * a.g.G + gq;
        t.later = a.later_at + ((begin >> a.log_r) - 1) * t.step + (int64_t)(x - it.first) * a.g.G + gq;
    }
    if (a.own_chunks > 0) {
        t.no = ((after >> 1) + a.own_chunk - 1) / a.own_chunk;
        t.own = a.own_at + (int64_t)(x * a.g.H_kv + h) * a.own_chunks * a.g.G + gq;
    }
    return t;
}

// The weights of kWeightRows own rows of a head
constexpr int kWeightRows = 4 * kThreads;

__device__ __forceinline__ void add_weights(const Shared& a, int own, int j0)
{
    __shared__ float norm[32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, G = a.g.G;
    const int x = own / a.g.H_kv, h = own - x * a.g.H_kv, after = a.after[own], n = after >> 1;
    const ItemOf it = item_of(a, x);
    if (it.item < 0 || j0 >= n) return;
    // the logits of the first heads are on their way while the statistics are joined
    constexpr int kRows = kWeightRows / kThreads, kEarly = 8;
    const float* z = a.logits + (int64_t)own * G * a.logit_pitch;
    float early[kEarly][kRows];
#pragma unroll
    for (int gq = 0; gq < kEarly; ++gq)
#pragma unroll
        for (int u = 0; u < kRows; ++u) early[gq][u] = z[(int64_t)min(gq, G - 1) * a.logit_pitch + min(j0 + u * kThreads + tid, n - 1)];
    // max + log2(sum) of the group's queries, a wave on every fourth
    for (int gq = wave; gq < G; gq += kWaves) {
        const Chunks t = chunks_of(a, x, it, h, gq, after);
        float m = -INFINITY, l = 0.f;
        for (int c = lane; c < t.np + t.no; c += 64) {
            const float2 s = a.stats[t.at(c)];
            const float m2 = fmaxf(m, s.x), ref = m2 == -INFINITY ? 0.f : m2;
            l = l * fast_exp2(m - ref) + s.y * fast_exp2(s.x - ref);
            m = m2;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const float mo = __shfl_xor(m, o, 64), lo = __shfl_xor(l, o, 64);
            const float m2 = fmaxf(m, mo), ref = m2 == -INFINITY ? 0.f : m2;
            l = l * fast_exp2(m - ref) + lo * fast_exp2(mo - ref);
            m = m2;
        }
        if (lane == 0) norm[gq] = l == 0.f ? INFINITY : m + __log2f(l);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int j = j0 + u * kThreads + tid;
        if (j >= n) break;
        float w = 0.f;
#pragma unroll
        for (int gq = 0; gq < kEarly; ++gq)
            if (gq < G) w += fast_exp2(early[gq][u] - norm[gq]);
        for (int gq = kEarly; gq < G; ++gq) w += fast_exp2(z[(int64_t)gq * a.logit_pitch + j] - norm[gq]);
        float* dst = a.weights + (int64_t)own * a.capacity + j;
        *dst = (after & 1) && j == n - 1 ? w : *dst + w;      // the appended row begins at nothing
    }
}

// Workgroups of kWeightRows own rows each add the rows' weights; behind those, THREADS threads per query join its chunks: a wave,
// four queries to a workgroup, or a whole workgroup where heads have many chunks (launch_shared).
template <int THREADS>
__global__ __launch_bounds__(kThreads) void shared_join_kernel(Shared a, int weight_blocks)
{
    constexpr int WAVES = THREADS / 64;
    __shared__ float wave_m[kWaves], wave_l[kWaves];
    __shared__ __attribute__((aligned(16))) f32x4 red[kThreads];
    if ((int)blockIdx.x < a.n_seqs * a.g.H_kv * weight_blocks) {
        const int own = blockIdx.x / weight_blocks;
        add_weights(a, own, (blockIdx.x - own * weight_blocks) * kWeightRows);
        return;
    }
    const int tid = threadIdx.x % THREADS, lane = threadIdx.x & 63, wave = tid >> 6, G = a.g.G, D = a.g.D;
    const int query = (blockIdx.x - a.n_seqs * a.g.H_kv * weight_blocks) * (kThreads / THREADS) +
                      __builtin_amdgcn_readfirstlane((int)threadIdx.x / THREADS);
    if (query >= a.n_seqs * a.g.H_q) return;                  // (a whole wave, or workgroup)
    const int x = query / a.g.H_q, hq = query - x * a.g.H_q, h = hq / G, gq = hq - h * G;
    const int after = a.own_chunks > 0 ? a.after[x * a.g.H_kv + h] : 0;      // (of a sequence that takes no part: anything)
    const ItemOf it = item_of(a, x);
    if (it.item < 0) return;
    const Chunks t = chunks_of(a, x, it, h, gq, after);
    if (gq == 0 && tid == 0 && (after & 1)) {
        const int own = x * a.g.H_kv + h;
        a.lengths[own] = after >> 1;
        if (a.positions) a.positions[(int64_t)own * a.capacity + (after >> 1) - 1] = a.pos_new[x];
    }
    const int nc = t.np + t.no;
    float m = -INFINITY, l = 0.f;
    for (int c = tid; c < nc; c += THREADS) {
        const float2 s = a.stats[t.at(c)];
        const float m2 = fmaxf(m, s.x), ref = m2 == -INFINITY ? 0.f : m2;
        l = l * fast_exp2(m - ref) + s.y * fast_exp2(s.x - ref);
        m = m2;
    }
    float M = m;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
    if constexpr (WAVES > 1) {
        if (lane == 0) wave_m[wave] = M;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) M = fmaxf(M, wave_m[w]);
    }
    const float ref = M == -INFINITY ? 0.f : M;
    l *= fast_exp2(m - ref);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
    float den = l;
    if constexpr (WAVES > 1) {
        if (lane == 0) wave_l[wave] = l;
        __syncthreads();
        den = ((wave_l[0] + wave_l[1]) + wave_l[2]) + wave_l[3];
    }
    // a thread has four channels of every (THREADS / (D / 4))-th chunk
    const int log_quads = 29 - __builtin_clz(D), quads = 1 << log_quads, groups = THREADS >> log_quads, ch = tid & (quads - 1), grp = tid >> log_quads;
    const f32x4* part = reinterpret_cast<const f32x4*>(a.part) + ch;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int c = grp; c < nc; c += groups) {
        const int64_t at = t.at(c);
        acc += part[at * quads] * fast_exp2(a.stats[at].x - ref);
    }
    if constexpr (WAVES > 1) {
        red[tid] = acc;
        __syncthreads();
        if (grp == 0)
            for (int k = 1; k < groups; ++k) acc += red[k * quads + ch];
    } else {
        for (int o = quads; o < 64; o <<= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += __shfl_xor(acc[i], o, 64);
    }
    if (grp == 0) {
        const float by = 1.f / den;
        bf16x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = (__bf16)(den == 0.f ? 0.f : acc[i] * by);      // no row, or nothing but -inf: zeros
        *reinterpret_cast<bf16x4*>(a.out + ((int64_t)x * a.g.H_q + hq) * D + ch * 4) = o;
    }
}

inline size_t up(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

}  // namespace

// Workgroups that a call's prompts, and own rows, are cut for at least, where they are long enough. A prompt's chunk costs a result per
// query, 512 bytes written and read at d = 128: few, long ones. Both kernels, us: 32 sequences on 13107 rows, 4 heads, 42 with 96
// workgroups, 30.3 with 192. At d = 128, from three blocks of query rows on, the products are most of it and two workgroups share a CU:
// 64 sequences on the same rows 43.9 with 192, 39.4 with 384, 47.9 with 768; 512 on eight prompts 82 and 85 (at d = 64 55 and 56,
// at d = 256 56 and 65: not there). Own rows: 48 caches of up to 4096 rows, 4 heads, 1024 workgroups 53.6, 2048 50.5.
constexpr int kPromptBlocks = 192, kOwnBlocks = 2048;
// What one wave joins per query: four channels to a lane, 256 floats at a time. Both kernels: 48 caches of 11 chunks at d = 128 50.5 us
// by a wave and 51.2 by a workgroup per query, 512 sequences on 9 chunks of eight prompts 85 and 101; at d = 256 32 sequences on 13107
// rows with caches of up to 4096 67.9 and 59.5.
constexpr int kWaveFloats = 4096;

// How a call is cut. Pure function of its sizes, so that the workspace query and the launch agree. The workspace never shrinks as
// total_rows or max_own grow: one that is sized for the largest step serves the smaller ones.
SharedPlan shared_plan(const Geom& g, int n_items, long long total_rows, int n_seqs, int max_seqs, int max_own)
{
    SharedPlan p;
    long long later = 0, chunks = 0;            // what the workspace is charged
    if (n_items > 0) {
        p.row_block = max_row_block(g.D);
        p.row_blocks = (int)(((long long)max_seqs * g.G + p.row_block - 1) / p.row_block);
        const int blocks = g.D == 128 && p.row_blocks > 2 ? 2 * kPromptBlocks : kPromptBlocks;
        const long long wanted = (blocks + p.row_blocks - 1) / p.row_blocks;
        p.log_r = 7;
        while (p.log_r < 16 && (total_rows >> (p.log_r + 1)) >= wanted) ++p.log_r;
        p.slots = (total_rows >> p.log_r) + (long long)n_items * g.H_kv;
        p.later_at = (long long)n_seqs * g.H_q;
        p.own_at = p.later_at + (total_rows >> p.log_r) * max_seqs * g.G;
        later = total_rows >> p.log_r;          // where the chunks double, their number halves
        if (p.log_r > 7 && later < 2 * wanted - 1) later = 2 * wanted - 1;
    }
    if (max_own > 0) {
        const long long heads = (long long)n_seqs * g.H_kv;
        chunks = (max_own + 127) / 128;
        const long long most = (kOwnBlocks + heads - 1) / heads;
        if (chunks > most) chunks = most;
        p.own_chunk = (int)(((max_own + chunks - 1) / chunks + 63) / 64 * 64);
        p.own_chunks = (max_own + p.own_chunk - 1) / p.own_chunk;
        p.logit_pitch = (max_own + 63) / 64 * 64;
    }
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += up(bytes); return here; };
    const size_t parts = (size_t)p.later_at + (size_t)later * max_seqs * g.G + (size_t)n_seqs * g.H_q * chunks;
    p.stats = take(parts * sizeof(float2));
    p.after = take((size_t)n_seqs * g.H_kv * sizeof(int32_t));
    p.part = take(parts * g.D * sizeof(float));
    p.logits = take((size_t)n_seqs * g.H_q * p.logit_pitch * sizeof(float));
    p.bytes = at;
    return p;
}
bool shared_supported(const Geom& g, const SharedPlan& p, int n_seqs)
{
    const double most = 8388608.;               // launches stay below 2^32 threads
    return g.G <= 32 && (double)(p.slots + 8) * p.row_blocks + (double)n_seqs * g.H_kv * p.own_chunks < most &&
           (double)n_seqs * g.H_q + (double)n_seqs * g.H_kv * (p.logit_pitch / kWeightRows + 1) < most;
}

hipError_t launch_shared(const Geom& g, const SharedPlan& p, const SharedCall& c, void* workspace, hipStream_t s)
{
    Shared a{};
    char* ws = static_cast<char*>(workspace);
    a.g = g;
    a.q = static_cast<const __bf16*>(c.q);
    a.kp = static_cast<const __bf16*>(c.k_prompt);
    a.vp = static_cast<const __bf16*>(c.v_prompt);
    a.cu_b = c.cu_budgets;
    a.cu_seqs = c.cu_seqs;
    a.n_items = c.n_items;
    a.total_rows = (int)c.total_rows;
    a.n_seqs = c.n_seqs;
    a.max_seqs = c.max_seqs;
    a.log_r = p.log_r;
    a.slots = (int)p.slots;
    a.slots_pad = (int)((p.slots + 7) / 8 * 8);
    a.row_block = p.row_block;
    a.row_blocks = p.row_blocks;
    a.ko = static_cast<__bf16*>(c.k_own);
    a.vo = static_cast<__bf16*>(c.v_own);
    a.lengths = c.lengths;
    a.positions = c.positions;
    a.weights = c.weights;
    a.capacity = c.capacity;
    a.max_own = c.max_own;
    a.own_chunk = p.own_chunk;
    a.own_chunks = p.own_chunks;
    a.k_new = static_cast<const __bf16*>(c.k_new);
    a.v_new = static_cast<const __bf16*>(c.v_new);
    a.pos_new = c.pos_new;
    a.stats = reinterpret_cast<float2*>(ws + p.stats);
    a.later_at = p.later_at;
    a.own_at = p.own_at;
    a.after = reinterpret_cast<int32_t*>(ws + p.after);
    a.part = reinterpret_cast<float*>(ws + p.part);
    a.logits = reinterpret_cast<float*>(ws + p.logits);
    a.logit_pitch = p.logit_pitch;
    a.out = static_cast<__bf16*>(c.out);
    const dim3 threads(kThreads);
    const unsigned blocks = (unsigned)(a.slots_pad * a.row_blocks + c.n_seqs * g.H_kv * p.own_chunks);
    if (blocks > 0) {
        switch (g.D) {
            case 64:  hipLaunchKernelGGL(shared_partial_kernel<64>, dim3(blocks), threads, 0, s, a); break;
            case 128: hipLaunchKernelGGL(shared_partial_kernel<128>, dim3(blocks), threads, 0, s, a); break;
            case 256: hipLaunchKernelGGL(shared_partial_kernel<256>, dim3(blocks), threads, 0, s, a); break;
            default: return hipErrorInvalidValue;
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int weight_blocks = c.weights ? (c.max_own + kWeightRows - 1) / kWeightRows : 0;
    const long long weights = (long long)c.n_seqs * g.H_kv * weight_blocks, queries = (long long)c.n_seqs * g.H_q;
    // chunks of an average head
    const long long chunks = (c.n_items > 0 ? p.slots / ((long long)c.n_items * g.H_kv) : 0) + p.own_chunks;
    if (chunks * g.D <= kWaveFloats)
        hipLaunchKernelGGL(shared_join_kernel<64>, dim3((unsigned)(weights + (queries + 3) / 4)), threads, 0, s, a, weight_blocks);
    else
        hipLaunchKernelGGL(shared_join_kernel<kThreads>, dim3((unsigned)(weights + queries)), threads, 0, s, a, weight_blocks);
    return hipGetLastError();
}

}  // namespace audiokv

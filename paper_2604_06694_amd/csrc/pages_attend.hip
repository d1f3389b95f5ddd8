// One decoding step on the cache in 4 bits and in pages (audiokv_pages_attend): every query head attends to its KV head's rows.
//
// Bound: the rows' bytes, 17/16 per channel of K and V together, each read once for all G query heads of the group. A row of D channels
// costs 2 G D products and G exponentials; on the vector units its conversion, about one instruction per channel of K and V and 64 rows.
//
// Heads have lengths of their own, known on the device only, so the work is cut there: the units of 32 rows of all heads one behind
// the other, and workgroup w of W takes units [T w / W, T (w + 1) / W), which may end one head, hold several and begin another. Every
// workgroup adds up the lengths for itself. A head that lies within one workgroup is finished there; what the others find for a part of
// a head goes to the workspace (at most two parts a workgroup, its first and its last) and a second launch joins it. No atomics;
// every sum has a fixed order.
//
// The waves of a workgroup take its units in turn. Both products are 16 x 16 x 32 on the matrix cores, with the query heads as columns, padded to 16:
//   C[key][query] = K Q^T       lane (c = lane & 15, r = lane >> 4) holds row c of K, channels of scale block r: its codes are one load,
//                               its scale one byte, and the conversion to bf16 is exact (a magnitude of e2m1 has two bits)
//   O[channel][query] += V^T P  the lane's C, keys 4 r .. 4 r + 3 of two tiles, is its column of P as it is: the product runs over keys in
//                               that order, and V's rows are loaded so
// The running reference of the softmax moves only where a logit exceeds it by 2^8, or V's scales say that a sum might overflow: a wave-wide
// test per unit instead of a maximum over lanes and a rescaling. P goes to the second product as two bf16 numbers (16 bits of it), V in
// bf16 is exact. Up to eight query heads (PAIRS) columns c and c + 8 hold the same query, and the two numbers of P are one in each: half
// the instructions of the second product, whose halves are added in the end. (The matrix cores' products of 4-bit keys as they are, with
// queries in 8 bits, are no choice: their sums are off by 2^-13 of the sum of magnitudes, those of bf16 by less than 2^-23.)
#include "pages.h"

#include <algorithm>

namespace audiokv {

namespace {

constexpr int kThreads = 256, kWaves = 4, kUnit = 32;       // of the kernels that share heads out
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4_t;

// Bytes of a pool: what the memory-side cache holds. How much of a larger pool is in use is not known here; where it is little and read again
// and again, streaming costs (a pool of 2 GB, with and without: 9 MB in use 11.8, 11.5 us, 35 MB 16.2, 15.5, 104 MB 26.9, 26.1, 226 MB 42.9, 41.8).
constexpr size_t kStreamBytes = 256u << 20;
constexpr float kSlack = 8.f;       // octaves that a logit may lie above the reference

// What the reference has to do with V. A head of 2^n rows or fewer sums up that many terms, a weight times a value of V each, which is
// 6 * 2^e at most at a scale 2^e. That stays below 0.75 * 2^128 where weights are 2^kSlack at most and e is up to 117 - n; beyond it the
// reference moves to the unit's largest logit, and to e + n - 125 octaves above it where that is positive (31 at most).
constexpr int kAnyWeight = 117;

struct AttendSpace {
    int4* joins;            // [the fewer of heads and workgroups]: head, slot of its first part, parts (0: nothing to join)
    float* stats;           // [slot][G][2]: reference in base-2 units, sum
    float* parts;           // [slot][G][D]
};

// how the channels of a row lie over the lanes: k-step `s` of lane group r begins at this channel
template <int D> __device__ __forceinline__ constexpr int channel_of(int s, int r) {
    return D == 64 ? r * 16 + s * 8 : (s >> 2) * 128 + r * 32 + (s & 3) * 8;
}

template <int D> struct Rows32 {         // one unit on its way: what a lane holds of it
    static constexpr int KW = D / 32;    // dwords of K's codes per tile of 16 rows
    static constexpr int VS = D == 64 ? 4 : 8;      // dwords with the scales of its eight rows of V (two rows in one at D = 64)
    unsigned k[2][KW], ks[2], v[8][(D + 127) / 128], vs[VS];
};

__device__ __forceinline__ float exponent_of(unsigned word, int byte) {     // 2^(e - 127) of a byte (the conversions read no other bits)
    return __uint_as_float(__builtin_amdgcn_alignbit(word, word, (9 + 8 * byte) & 31));
}

// Where a lane's share of a unit lies behind the unit's first row in each section: the same for all units, so that a load's address is
// a scalar (page, section, row) and one of these, with the tile and the row in the instruction.
template <int D> struct LaneOffsets {
    unsigned k, ks, v, vs;
    __device__ __forceinline__ LaneOffsets() {
        const unsigned lane = threadIdx.x & 63, c = lane & 15, r = lane >> 4;
        k = c * (D / 2) + r * (D == 64 ? 8 : 16);
        ks = c * (D / 32) + (D == 64 ? r >> 1 : r);
        v = r * 4 * (D / 2) + c * (D / 32);
        vs = r * 4 * (D / 32) + (D == 256 ? (c >> 3) * 4 : 0);
    }
};

template <class T, bool STREAM = false> __device__ __forceinline__ T at(const char* base, unsigned lane_offset, int offset) {
    const T* p = reinterpret_cast<const T*>(base + offset + lane_offset);
    return STREAM ? __builtin_nontemporal_load(p) : *p;
}

// STREAM: what takes whole cache lines with one instruction (K's codes up to D = 128, V's at 256) passes the caches by. The rest shares
// lines with the next instruction. For caches that the memory-side cache does not hold: 522 MB 98 -> 82 us, 1 GB at D = 128 190 -> 177, at
// 256 181 -> 170, while one of 261 MB took 43.8 instead of 42.8.
template <int D, bool STREAM>
__device__ __forceinline__ void load_unit(Rows32<D>& u, const PageView& pv, const LaneOffsets<D>& of, int page, int row0) {
    const char* base = pv.page(page);
    const char *k = base + pv.k_codes(row0), *v = base + pv.v_codes(row0), *ks = base + pv.k_scales(row0), *vs = base + pv.v_scales(row0);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if constexpr (D == 64) {
            const u32x2 w = at<u32x2, STREAM>(k, of.k, t * 16 * (D / 2));
            u.k[t][0] = w[0];
            u.k[t][1] = w[1];
        } else {
#pragma unroll
            for (int b = 0; b < D / 128; ++b) {
                const u32x4 w = at<u32x4, STREAM && D == 128>(k, of.k, t * 16 * (D / 2) + b * 64);
#pragma unroll
                for (int i = 0; i < 4; ++i) u.k[t][b * 4 + i] = w[i];
            }
        }
        u.ks[t] = at<unsigned char>(ks, of.ks, t * 16 * (D / 32));
        if constexpr (D == 256) u.ks[t] |= (unsigned)at<unsigned char>(ks, of.ks, t * 16 * (D / 32) + 4) << 8;
    }
    // V: rows 4 r + i of either tile, channels c * D / 16 ..
#pragma unroll
    for (int n = 0; n < 8; ++n) {
        const int row = (n >> 2) * 16 + (n & 3);
        if constexpr (D == 64) u.v[n][0] = at<unsigned short>(v, of.v, row * (D / 2));
        else if constexpr (D == 128) u.v[n][0] = at<unsigned>(v, of.v, row * (D / 2));
        else {
            const u32x2 w = at<u32x2, STREAM>(v, of.v, row * (D / 2));
            u.v[n][0] = w[0];
            u.v[n][1] = w[1];
        }
        if constexpr (D == 256) u.vs[n] = at<unsigned>(vs, of.vs, row * (D / 32));
    }
    if constexpr (D == 128) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const u32x4 w = at<u32x4>(vs, of.vs, t * 64);
#pragma unroll
            for (int i = 0; i < 4; ++i) u.vs[t * 4 + i] = w[i];
        }
    } else if constexpr (D == 64) {                                           // two rows to a dword
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const u32x2 w = at<u32x2>(vs, of.vs, t * 32);
            u.vs[t * 2] = w[0];
            u.vs[t * 2 + 1] = w[1];
        }
    }
}
// which byte of the dword is the scale of the lane's channels of V in its row n
template <int D> __device__ __forceinline__ int scale_byte(int n, int c) {
    return D == 64 ? (n & 1) * 2 + (c >> 3) : D == 128 ? c >> 2 : (c >> 1) & 3;
}

#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ unsigned pair_of(unsigned codes, float scale, int byte) {
    switch (byte) {
        case 0: return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
        case 1: return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
        case 2: return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
        default: return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    }
}
#else
__device__ __forceinline__ unsigned pair_of(unsigned, float, int) { return 0; }
#endif

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {             // nearest even
    bf16x2 x;
    x[0] = (__bf16)a;
    x[1] = (__bf16)b;
    return __builtin_bit_cast(unsigned, x);
}

// Of three scales as exponent_of leaves them. (In asm: fmaxf makes two instructions of one, to quiet a NaN first. A scale that says NaN hides
// the others of its lane here; the lane's channels are NaN whatever they are.)
__device__ __forceinline__ float max_magnitude(float a, float b, float c) {
    float m;
    asm("v_max3_f32 %0, |%1|, |%2|, |%3|" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}

// What a wave knows of a head so far. Column c = lane & 15 is a query; `sum` is the lane's share of it.
template <int D> struct Running {
    f32x4 out[D / 16];      // out[ct][i]: channel (4 r + i) * D / 16 + ct
    float ref, sum;
};

template <int D, bool PAIRS>
__device__ __forceinline__ void add_unit(Running<D>& o, const Rows32<D>& u, const bf16x8 (&q)[D / 32], float c_log2, int rows, int log_rows) {
    const int lane = threadIdx.x & 63, c = lane & 15, r = lane >> 4;
    f32x4 z[2];                                            // products, keys 4 r + i of either tile
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        z[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            const float scale = __uint_as_float(D == 256 && s >= 4 ? u.ks[t] << 15 : u.ks[t] << 23);
            u32x4_t f;
#pragma unroll
            for (int b = 0; b < 4; ++b) f[b] = pair_of(u.k[t][s], scale, b);
            z[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), q[s], z[t], 0, 0, 0);
        }
    }
    float vs[8];
#pragma unroll
    for (int n = 0; n < 8; ++n) vs[n] = exponent_of(u.vs[D == 64 ? n >> 1 : n], scale_byte<D>(n, c));
    if (rows < kUnit) {                                    // wave-uniform: a head's last unit
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const bool there = (n >> 2) * 16 + r * 4 + (n & 3) < rows;
            z[n >> 2][n & 3] = there ? z[n >> 2][n & 3] : -INFINITY;
            vs[n] = there ? vs[n] : 1.f;                   // what lies behind the last row may say NaN, which zero times is NaN
        }
    }
    float top = fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])), fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3]))) * c_log2;
    const float large = max_magnitude(max_magnitude(max_magnitude(max_magnitude(vs[0], vs[1], vs[2]), vs[3], vs[4]), vs[5], vs[6]), vs[7], vs[7]);
    const unsigned long long largest = __builtin_amdgcn_ballot_w64(large >= __uint_as_float((unsigned)(127 + kAnyWeight + 1 - log_rows) << 23));
    if ((__builtin_amdgcn_ballot_w64(top > o.ref + kSlack) | largest) != 0) {
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        if (largest != 0) {
            float all = large;
#pragma unroll
            for (int m = 32; m > 0; m >>= 1) all = fmaxf(all, __shfl_xor(all, m, 64));
            top += (float)max((int)(__float_as_uint(all) >> 23) - 127 + log_rows - (kAnyWeight + 8), 0);
        }
        const float ref = fmaxf(o.ref, top);
        const float shrink = o.ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(o.ref - ref);
        o.ref = ref;
        o.sum *= shrink;
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) o.out[ct] *= shrink;
    }
    const float ref = o.ref == -INFINITY ? 0.f : o.ref;
    u32x4_t hi, lo;            // PAIRS: hi is the column's own part, see above
    [[maybe_unused]] const unsigned minus = PAIRS && (c & 8) ? 0x80000000u : 0;
    [[maybe_unused]] const float whole = PAIRS && (c & 8) ? 1.f : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = __builtin_amdgcn_exp2f(fmaf(z[i >> 1][2 * i & 3], c_log2, -ref)), b = __builtin_amdgcn_exp2f(fmaf(z[i >> 1][(2 * i & 3) + 1], c_log2, -ref));
        o.sum += a + b;
        if constexpr (PAIRS) {         // the upper sixteen bits, or what they leave
            const float ta = __uint_as_float((__float_as_uint(a) & 0xffff0000u) ^ minus), tb = __uint_as_float((__float_as_uint(b) & 0xffff0000u) ^ minus);
            hi[i] = pack_bf16(fmaf(a, whole, ta), fmaf(b, whole, tb));
        } else {
            hi[i] = pack_bf16(a, b);
            lo[i] = pack_bf16(a - __uint_as_float(hi[i] << 16), b - __uint_as_float(hi[i] & 0xffff0000u));
        }
    }
#pragma unroll
    for (int w = 0; w < (D + 127) / 128; ++w)
#pragma unroll
        for (int b = 0; b < (D == 64 ? 2 : 4); ++b) {
            u32x4_t even, odd;                             // channels 8 w + 2 b and 2 b + 1 of the lane's, keys by twos
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned x = pair_of(u.v[2 * i][w], vs[2 * i], b), y = pair_of(u.v[2 * i + 1][w], vs[2 * i + 1], b);
                even[i] = __builtin_amdgcn_perm(y, x, 0x05040100);
                odd[i] = __builtin_amdgcn_perm(y, x, 0x07060302);
            }
            const int ct = w * 8 + b * 2;
            o.out[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), __builtin_bit_cast(bf16x8, hi), o.out[ct], 0, 0, 0);
            o.out[ct + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), __builtin_bit_cast(bf16x8, hi), o.out[ct + 1], 0, 0, 0);
            if constexpr (!PAIRS) {
                o.out[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), __builtin_bit_cast(bf16x8, lo), o.out[ct], 0, 0, 0);
                o.out[ct + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), __builtin_bit_cast(bf16x8, lo), o.out[ct + 1], 0, 0, 0);
            }
        }
}

// First of 64 heads or more, from `head` on, that has rows; n_heads if none has. (wave-uniform)
__device__ __forceinline__ int next_with_rows(const PageView& pv, int head) {
    for (; head < pv.n_heads; head += 64) {
        const int g = head + (int)(threadIdx.x & 63);
        const unsigned long long m = __builtin_amdgcn_ballot_w64(g < pv.n_heads && pv.length(min(g, pv.n_heads - 1)) > 0);
        if (m) return head + __builtin_ctzll(m);
    }
    return pv.n_heads;
}

__device__ __forceinline__ int units_of(int rows) { return (rows + kUnit - 1) / kUnit; }

// By how many units the largest share may grow so that shares end with heads: one for each wave. (64 ragged heads 16.3 -> 15.1 us, 12 at
// D = 256 16.6 -> 14.9; 64 equal heads, which end together anyway, 12.3 -> 13.4, for the sum over heads is formed twice.)
constexpr int kAlignedUnits = 4;

// waves of a SIMD: what two units on their way leave registers for
template <int D> constexpr int kResident = D == 64 ? 4 : D == 128 ? 3 : 2;

// WHOLE: workgroup x takes head x, whatever its length; nothing is left to join.
// dynamic LDS: [wave][G][D + 4]
template <int D, bool PAIRS, int WAVES, bool WHOLE, bool STREAM>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(kResident<D>, kResident<D>))) void attend_kernel(
    Geom g, PageView pv, const __bf16* __restrict__ q, __bf16* __restrict__ out, float* __restrict__ lse, AttendSpace a)
{
    constexpr int THREADS = 64 * WAVES;
    extern __shared__ __attribute__((aligned(16))) float merge[];
    __shared__ int sums[2 * WAVES];
    __shared__ float ref_of[WAVES][16], sum_of[WAVES][16];
    __shared__ int begin_head, begin_at, begin_rows, begin_parts;
    __shared__ int4 plan;        // for the end of a head, out of the way until then: all units, workgroups, parts of a head if aligned, by head
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, r = lane >> 4;
    const int G = g.G, PITCH = D + 4;
    const LaneOffsets<D> offsets;

    int head, start, rows, u0, u1;
    if constexpr (WHOLE) {
        head = blockIdx.x;
        start = u0 = 0;
        rows = __builtin_amdgcn_readfirstlane(pv.length(head));
        u1 = max(units_of(rows), 1);                                   // (a head without rows has one unit of none: zeros)
    } else {
        const int b = blockIdx.x, wgs = gridDim.x;
        const bool by_head = pv.n_heads <= wgs;                        // which entry of a.joins: a head's, or a workgroup's last head's
        int total, W;
        if (!by_head && tid == 0) a.joins[b] = int4{0, 0, 0, 0};
        // all units; and zeros for heads without rows, each by one workgroup
        const int each = (pv.n_heads + THREADS - 1) / THREADS, h0 = min(tid * each, pv.n_heads), h1 = min(h0 + each, pv.n_heads);
        int mine = 0;
        for (int h = h0; h < h1; ++h) {
            const int n = units_of(pv.length(h));
            mine += n;
            if (n == 0 && h % wgs == b) {
                for (int e = 0; e < G * D; e += 8) *reinterpret_cast<u32x4*>(out + (size_t)h * G * D + e) = u32x4{0, 0, 0, 0};
                for (int e = 0; lse && e < G; ++e) lse[(size_t)h * G + e] = -INFINITY;
                if (by_head) a.joins[h] = int4{0, 0, 0, 0};
            }
        }
        int before = exclusive_sum_once<THREADS>(mine, sums, total);
        if (total == 0) return;
        // Workgroups that have parts of two heads work on them one after the other, some 3 us. Where shares that end with the heads are
        // not much larger, there are those instead: of `share` units at most.
        const int share = 2 * pv.n_heads <= wgs ? max((int)(((unsigned)total + wgs - pv.n_heads - 1) / (wgs - pv.n_heads)), WAVES) : INT_MAX;
        const bool aligned = share - kAlignedUnits <= total / wgs;
        if (aligned) {
            mine = 0;
            for (int h = h0; h < h1; ++h) mine += (units_of(pv.length(h)) + share - 1) / share;
            before = exclusive_sum_once<THREADS>(mine, sums + WAVES, W);
        } else {
            W = min(wgs, total / WAVES + 1);
        }
        if (b >= W) return;
        // the head in which this workgroup's share begins: `at` units (or workgroups) are before it
        const Shares of_all{total, W};
        const int first = aligned ? b : of_all.begin(b);
        if (first >= before && first < before + mine) {
            int h = h0, at = before;
            for (;; ++h) {
                rows = pv.length(h);
                const int n = aligned ? (units_of(rows) + share - 1) / share : units_of(rows);
                if (first < at + n || h + 1 >= h1) {                   // (the second: lengths that change meanwhile lead nowhere else)
                    begin_parts = max(n, 1);
                    break;
                }
                at += n;
            }
            begin_head = h;
            begin_at = at;
            begin_rows = rows;
        }
        __syncthreads();
        head = __builtin_amdgcn_readfirstlane(begin_head);
        rows = __builtin_amdgcn_readfirstlane(begin_rows);
        start = __builtin_amdgcn_readfirstlane(begin_at);
        if (aligned) {
            const Shares of_head{units_of(rows), __builtin_amdgcn_readfirstlane(begin_parts)};
            u0 = __builtin_amdgcn_readfirstlane(of_head.begin(b - start));
            u1 = __builtin_amdgcn_readfirstlane(of_head.begin(b - start + 1));
            start = 0;
        } else {
            u0 = __builtin_amdgcn_readfirstlane(first);
            u1 = __builtin_amdgcn_readfirstlane(of_all.begin(b + 1));
        }
        if (tid == 0) plan = int4{total, W, aligned ? begin_parts : 0, by_head};
    }

    for (int u = u0; u < u1;) {
        const int units = units_of(rows), log_rows = rows > 1 ? 32 - __builtin_clz(rows - 1) : 0;
        const int from = u - start, to = min(units, u1 - start);           // units of this head
        const int x = head / g.H_kv, h = head - x * g.H_kv;
        const int32_t* table = pv.table + (size_t)head * pv.width;
        const int log_u = pv.log_p - 5;                                    // units to a page
        bf16x8 qf[D / 32];
        {
            const __bf16* src = q + ((size_t)x * g.H_q + (size_t)h * G + min(PAIRS ? c & 7 : c, G - 1)) * D;    // (columns from G on: copies, unused)
#pragma unroll
            for (int s = 0; s < D / 32; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(src + channel_of<D>(s, r));
        }
        Running<D> o;
#pragma unroll
        for (int ct = 0; ct < D / 16; ++ct) o.out[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
        o.ref = -INFINITY;
        o.sum = 0.f;
        // Two units on their way: while one is worked on, the next is loaded (the last one again behind it, so that every step waits
        // for as many loads), and the page of the one after that is looked up.
        if (from + wave < to) {
            const int last = from + wave + (to - 1 - from - wave) / WAVES * WAVES;
            auto page_of = [&](int i) { return __builtin_amdgcn_readfirstlane(table[min(i, last) >> log_u]); };
            auto load = [&](Rows32<D>& unit, int i, int page) {
                load_unit<D, STREAM>(unit, pv, offsets, pv.is_page(page) ? page : 0, (min(i, last) & ((1 << log_u) - 1)) * kUnit);
            };
            auto add = [&](const Rows32<D>& unit, int i, int page) {       // (rows of no page take no part)
                add_unit<D, PAIRS>(o, unit, qf, g.c_log2, pv.is_page(page) ? min(kUnit, rows - i * kUnit) : 0, log_rows);
            };
            Rows32<D> a0, a1;
            int i = from + wave, p0 = page_of(i), p1 = page_of(i + WAVES);
            load(a0, i, p0);
            for (;;) {
                int p2 = page_of(i + 2 * WAVES);
                load(a1, i + WAVES, p1);
                __builtin_amdgcn_sched_barrier(0);
                add(a0, i, p0);
                i += WAVES;
                if (i > last) break;
                p0 = page_of(i + 2 * WAVES);
                load(a0, i + WAVES, p2);
                __builtin_amdgcn_sched_barrier(0);
                add(a1, i, p1);
                i += WAVES;
                if (i > last) break;
                p1 = p0;
                p0 = p2;
            }
        }
        // The four waves' findings. (The thread's number goes through an asm, so that no address below is worked out ahead of the loop
        // and held in registers during it.)
        int me = tid;
        asm volatile("" : "+v"(me));
        const int c = me & 15, r = (me & 63) >> 4;
        float sum = o.sum;
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        if (r == 0) {
            ref_of[wave][c] = o.ref;
            sum_of[wave][c] = sum;
        }
        __syncthreads();
        float all = ref_of[0][c];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) all = fmaxf(all, ref_of[w][c]);
        const float shrink = o.ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(o.ref - all);
        if constexpr (PAIRS) {
#pragma unroll
            for (int ct = 0; ct < D / 16; ++ct)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    o.out[ct][i] += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(o.out[ct][i]), 0x128, 0xf, 0xf, false));   // lane 8 away of 16
        }
        if (c < G) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int ct = 0; ct < D / 16; ct += 4)
                    *reinterpret_cast<f32x4*>(&merge[(wave * G + c) * PITCH + (r * 4 + i) * (D / 16) + ct]) =
                        f32x4{o.out[ct][i], o.out[ct + 1][i], o.out[ct + 2][i], o.out[ct + 3][i]} * shrink;
        }
        __syncthreads();
        const bool whole = WHOLE || (from == 0 && to == units);
        const int slot = 2 * blockIdx.x + (u != u0);
        if (!WHOLE && me == 0) {
            const int4 all = plan;
            const int n = all.z > 0 ? all.z : Shares{all.x, all.y}.of(start + units - 1) - (int)blockIdx.x + 1;
            if (from == 0 && (all.w || !whole)) a.joins[all.w ? head : blockIdx.x] = int4{head, slot, whole ? 0 : n, 0};
        }
        auto sums_of = [&](int n, float& m) {
            m = ref_of[0][n];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) m = fmaxf(m, ref_of[w][n]);
            float l = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) l += sum_of[w][n] * (ref_of[w][n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref_of[w][n] - m));   // (NaN stays NaN)
            return l;
        };
        for (int e = me * 4; e < G * D; e += THREADS * 4) {
            const int n = e / D, ch = e % D;
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v += *reinterpret_cast<const f32x4*>(&merge[(w * G + n) * PITCH + ch]);
            if (whole) {
                float m;
                const float l = sums_of(n, m);
                if (l != 0.f) v /= l;                                     // (no weight at all: zeros)
                *reinterpret_cast<u32x2*>(out + ((size_t)x * g.H_q + (size_t)h * G + n) * D + ch) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            } else {
                *reinterpret_cast<f32x4*>(a.parts + ((size_t)slot * G + n) * D + ch) = v;
            }
        }
        if (me < G) {
            float m;
            const float l = sums_of(me, m);
            if (!whole) {
                a.stats[((size_t)slot * G + me) * 2] = m;
                a.stats[((size_t)slot * G + me) * 2 + 1] = l;
            } else if (lse) {
                lse[(size_t)x * g.H_q + (size_t)h * G + me] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
            }
        }
        if (WHOLE) return;
        u = start + to;
        start += units;
        if (u < u1) {
            head = next_with_rows(pv, head + 1);
            if (head >= pv.n_heads) return;
            rows = __builtin_amdgcn_readfirstlane(pv.length(head));
        }
        __syncthreads();                                                   // the LDS is free again
    }
}

// One workgroup per query head of a head in parts: the parts in order. A chain of loads from end to end: the first parts are on their way
// with the statistics.
constexpr int kMaxWorkgroups = 256 * 4, kEarly = 2;

template <int D>
__global__ __launch_bounds__(kThreads) void join_kernel(Geom g, __bf16* __restrict__ out, float* __restrict__ lse, AttendSpace a)
{
    constexpr int QUADS = D / 4, GROUPS = kThreads / QUADS, WAVES = kThreads / 64;     // threads on four channels each, parts at a time
    const int G = g.G, entry = blockIdx.x / G, n = blockIdx.x - entry * G, tid = threadIdx.x;
    const int4 from = a.joins[entry];
    const int parts = min(from.z, kMaxWorkgroups);
    if (parts == 0) return;
    const size_t row = (size_t)from.x * G + n;                              // (query heads of a KV head are neighbours)
    __shared__ float weight[kMaxWorkgroups], wave_m[WAVES], wave_l[WAVES];
    __shared__ __attribute__((aligned(16))) f32x4 red[kThreads];
    auto slot_of = [&](int p) { return part_slot(from.y, p); };
    const int ch = tid % QUADS * 4, grp = tid / QUADS;
    auto part = [&](int p) { return *reinterpret_cast<const f32x4*>(a.parts + ((size_t)slot_of(p) * G + n) * D + ch); };
    f32x4 early[kEarly];
#pragma unroll
    for (int u = 0; u < kEarly; ++u) early[u] = part(min(grp + u * GROUPS, parts - 1));
    float2 stat[kMaxWorkgroups / kThreads];
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < kMaxWorkgroups / kThreads; ++u) {
        stat[u] = float2{-INFINITY, 0.f};
        if (tid + u * kThreads < parts) stat[u] = *reinterpret_cast<const float2*>(&a.stats[((size_t)slot_of(tid + u * kThreads) * G + n) * 2]);
        m = fmaxf(m, stat[u].x);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    if ((tid & 63) == 0) wave_m[tid >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(wave_m[0], wave_m[1]), fmaxf(wave_m[2], wave_m[3]));
    float l = 0.f;
#pragma unroll
    for (int u = 0; u < kMaxWorkgroups / kThreads; ++u) {
        const float w = stat[u].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stat[u].x - m);
        if (tid + u * kThreads < parts) weight[tid + u * kThreads] = w;
        l += w * stat[u].y;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
    if ((tid & 63) == 0) wave_l[tid >> 6] = l;
    __syncthreads();
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < kEarly; ++u)
        if (grp + u * GROUPS < parts) acc += early[u] * weight[grp + u * GROUPS];
#pragma unroll 4
    for (int p = grp + kEarly * GROUPS; p < parts; p += GROUPS) acc += part(p) * weight[p];
    red[tid] = acc;
    __syncthreads();
    l = ((wave_l[0] + wave_l[1]) + wave_l[2]) + wave_l[3];
    if (grp == 0) {
        for (int k = 1; k < GROUPS; ++k) acc += red[k * QUADS + tid];
        if (l != 0.f) acc /= l;
        *reinterpret_cast<u32x2*>(out + row * D + ch) = u32x2{pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3])};
        if (lse && tid == 0) lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
    }
}

template <int D> constexpr int kWholeWaves = 4 * kResident<D>;
// Short heads go to a workgroup each, of as many waves as a CU holds, and there is no second launch. By what a table can hold, since
// lengths are not known here. Kernel times of whole heads, and in parts with the join: 4 heads of 500 rows 6.8, 9.3 us, of 2000 12.2, 11.5
// (and the host launches once, some 3 us less), 64 of 2000 13.2, 13.5, 256 of 500 8.1, 15.2, 256 of 2000 16.1, 22.3, 512 of 500 14.8, 20,
// 1792 of 500 47.7, 38 (so a head of 900 rows in a table for 32768 takes 11.7 us with the binding, in one for 1024 8.9); at D = 256, where a CU holds eight waves, 16 of 500 11.1, 10.6, of 1000 14.3, 11.5, but 256 of 1500 21.6, 26.3.
bool whole_heads(const PageView& pv) {
    const long long rows = (long long)pv.width << pv.log_p;
    return pv.n_heads <= 512 && rows <= (pv.D < 256 || pv.n_heads >= 128 ? 2048 : 512);
}

// Workgroups: as many as the registers let run at once, so that equal shares end together
int workgroups(const Geom& g, const PageView& pv) {
    const long long most = ((long long)pv.n_heads * pv.width << pv.log_p) / (kUnit * kWaves) + pv.n_heads;
    const int w = 256 * (g.D == 64 ? kResident<64> : g.D == 128 ? kResident<128> : kResident<256>);
    static_assert(256 * kResident<64> <= kMaxWorkgroups, "join_kernel holds the statistics of as many parts");
    return (int)(most < w ? most : w);
}

// heads in parts at most: every boundary between workgroups is within one head
int joins(const Geom& g, const PageView& pv) { return std::min(pv.n_heads, workgroups(g, pv)); }

AttendSpace attend_space(const Geom& g, const PageView& pv, void* workspace, size_t* bytes) {
    AttendSpace a;
    const size_t slots = 2 * (size_t)workgroups(g, pv);
    size_t off = 0;
    a.joins = part_at<int4>(workspace, off);
    off += up256((size_t)joins(g, pv) * sizeof(int4));
    a.stats = part_at<float>(workspace, off);
    off += up256(slots * g.G * 2 * sizeof(float));
    a.parts = part_at<float>(workspace, off);
    off += slots * g.G * g.D * sizeof(float);
    if (bytes) *bytes = off;
    return a;
}

}  // namespace

size_t pages_attend_bytes(const Geom& g, const PageView& pv) {
    size_t bytes;
    attend_space(g, pv, nullptr, &bytes);
    return bytes;
}

hipError_t launch_pages_attend(const Geom& g, const PageView& pv, const void* q, void* out, float* lse, void* workspace, hipStream_t s)
{
    const AttendSpace a = attend_space(g, pv, workspace, nullptr);
    const unsigned lds = (unsigned)sizeof(float) * g.G * (g.D + 4);
#define AUDIOKV_ATTEND(PAIRS, WAVES, WHOLE, STREAM)                                                                                      \
    AUDIOKV_FOR_DIM(g.D, hipLaunchKernelGGL((attend_kernel<kD, PAIRS, WAVES, WHOLE, STREAM>), grid, dim3(64 * (WAVES)), lds * (WAVES), s, g, \
                                            pv, (const __bf16*)q, (__bf16*)out, lse, a))
    if (whole_heads(pv)) {
        const dim3 grid((unsigned)pv.n_heads);
        if (g.G <= 8) AUDIOKV_ATTEND(true, kWholeWaves<kD>, true, false) else AUDIOKV_ATTEND(false, kWholeWaves<kD>, true, false)
        return hipGetLastError();
    }
    const dim3 grid((unsigned)workgroups(g, pv)), join((unsigned)(joins(g, pv) * g.G));
    if ((size_t)pv.n_pages * pv.page_bytes() <= kStreamBytes) {
        if (g.G <= 8) AUDIOKV_ATTEND(true, kWaves, false, false) else AUDIOKV_ATTEND(false, kWaves, false, false)
    } else {
        if (g.G <= 8) AUDIOKV_ATTEND(true, kWaves, false, true) else AUDIOKV_ATTEND(false, kWaves, false, true)
    }
#undef AUDIOKV_ATTEND
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    AUDIOKV_FOR_DIM(g.D, hipLaunchKernelGGL(join_kernel<kD>, join, dim3(kThreads), 0, s, g, (__bf16*)out, lse, a))
    return hipGetLastError();
}

}  // namespace audiokv

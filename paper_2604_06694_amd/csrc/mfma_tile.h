// What the kernels share that multiply tiles of queries and keys in the same orientation: C = K Q^T on
// v_mfma_f32_32x32x16_bf16, so that a lane owns one query row (column lane & 31 of C) and its sixteen accumulators are
// sixteen keys. Row statistics then stay in the lane, and a lane's exponentials are, four keys at a time, the operand of a
// second product over the keys.
#pragma once

#include "common.h"
#include "quad_transpose.h"

namespace audiokv {

typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

namespace mfma_tile {

constexpr int kThreads = 256, kWaves = 4;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// key of accumulator i in a 32 x 32 block, for lane half hf
__device__ __forceinline__ constexpr int key_of(int i, int hf) { return (i >> 2) * 8 + hf * 4 + (i & 3); }

// LDS rows are unpadded: the 16-byte chunk c of row r sits at chunk slot (c + r) mod 8 of its group of eight. The fragment reads
// (32 rows, the same chunk) and the transposing reads (eight rows, four neighbouring chunks) both spread evenly over the banks so.
__host__ __device__ constexpr int slot_of(int c, int r) { return (c & ~7) | ((c + r) & 7); }

// Sixteen-byte pieces per thread of a tile of ROWS rows
template <int D, int ROWS> constexpr int kPieces = ROWS * (D / 8) / kThreads;

// A tile on its way: this thread's pieces, row and chunk of each by piece number
template <int D> __device__ __forceinline__ int piece_row(int u) { return (int)threadIdx.x / (D / 8) + u * (kThreads / (D / 8)); }
template <int D> __device__ __forceinline__ int piece_chunk() { return (int)threadIdx.x % (D / 8); }

template <int D, int N>
__device__ __forceinline__ void put_tile(__bf16* tile, const u32x4 (&piece)[N]) {
    const int c = piece_chunk<D>();
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int r = piece_row<D>(u);
        *reinterpret_cast<u32x4*>(tile + r * D + slot_of(c, r) * 8) = piece[u];
    }
}

// Fragment kk (channels 16 kk + 8 hf ..) of row `row` of a tile: an A operand if the rows are keys, a B operand if queries
template <int D>
__device__ __forceinline__ bf16x8 fragment(const __bf16* tile, int row, int kk, int hf) {
    return *reinterpret_cast<const bf16x8*>(tile + row * D + slot_of(2 * kk + hf, row) * 8);
}

// The fragments of the lane's row of 32 (lane & 31), kk as above, straight from global memory: row(i) is where row i begins. Load
// i of a quad of lanes takes row i of its four rows, lane q of the quad the pieces of k-steps q, q + 4, ...: whole cache lines,
// where lanes that load their own rows touch a line for every 32 bytes. The quad then exchanges its pieces.
// (The exchange needs registers beside the fragments: where these are 128, NB = 2 sets of d = 256, lanes load their own rows.)
template <int D, int NB, class Row>
__device__ __forceinline__ void load_fragments(bf16x8 (&f)[D / 16], Row row) {
    const int lane = threadIdx.x & 63, hf = lane >> 5;
    if constexpr (D * NB > 256) {
        const __bf16* src = row(lane & 31) + hf * 8;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) f[kk] = *reinterpret_cast<const bf16x8*>(src + kk * 16);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __bf16* src = row((lane & 28) + i) + (lane & 3) * 16 + hf * 8;
#pragma unroll
        for (int kq = 0; kq < D / 16; kq += 4) f[kq + i] = *reinterpret_cast<const bf16x8*>(src + kq * 16);
    }
#pragma unroll
    for (int kq = 0; kq < D / 16; kq += 4) quad_transpose(f[kq], f[kq + 1], f[kq + 2], f[kq + 3], lane);
}

}  // namespace mfma_tile
}  // namespace audiokv

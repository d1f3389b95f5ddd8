// Four rows' pieces exchanged within quads of lanes: fragments of rows that lanes would otherwise load 16 bytes at a time from
// rows of their own come as whole cache lines so.
#pragma once

#include <hip/hip_runtime.h>

namespace audiokv {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

// Transpose four 16-byte pieces per lane over each quad of lanes: piece i of lane q becomes piece q of lane i.
__device__ __forceinline__ void quad_transpose(bf16x8& p0, bf16x8& p1, bf16x8& p2, bf16x8& p3, int lane) {
    typedef __attribute__((ext_vector_type(4))) int i32x4;
    i32x4 a = __builtin_bit_cast(i32x4, p0), b = __builtin_bit_cast(i32x4, p1);
    i32x4 c = __builtin_bit_cast(i32x4, p2), d = __builtin_bit_cast(i32x4, p3);
    const bool odd = lane & 1, high = lane & 2;
    // swap what differs in bit 0 of piece and lane (quad_perm 1,0,3,2), then in bit 1 (quad_perm 2,3,0,1)
    auto swap1 = [&](int& x, int& y) {
        const int xs = __builtin_amdgcn_mov_dpp(x, 0xb1, 0xf, 0xf, true), ys = __builtin_amdgcn_mov_dpp(y, 0xb1, 0xf, 0xf, true);
        x = odd ? ys : x;
        y = odd ? y : xs;
    };
    auto swap2 = [&](int& x, int& y) {
        const int xs = __builtin_amdgcn_mov_dpp(x, 0x4e, 0xf, 0xf, true), ys = __builtin_amdgcn_mov_dpp(y, 0x4e, 0xf, 0xf, true);
        x = high ? ys : x;
        y = high ? y : xs;
    };
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        int x0 = a[w], x1 = b[w], x2 = c[w], x3 = d[w];
        swap1(x0, x1);
        swap1(x2, x3);
        swap2(x0, x2);
        swap2(x1, x3);
        a[w] = x0; b[w] = x1; c[w] = x2; d[w] = x3;
    }
    p0 = __builtin_bit_cast(bf16x8, a);
    p1 = __builtin_bit_cast(bf16x8, b);
    p2 = __builtin_bit_cast(bf16x8, c);
    p3 = __builtin_bit_cast(bf16x8, d);
}

}  // namespace audiokv

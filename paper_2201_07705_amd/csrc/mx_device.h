// Pieces that the products of 4-bit matrices share.
#pragma once
#include <hip/hip_runtime.h>

#include "mx_args.h"
#include "op_moves.h"

namespace gemel {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float mx_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 mx_bf16x8 __attribute__((ext_vector_type(8)));

// 16 rows of a times 16 rows of b over 128 columns, a block of 32 of each row
// in a lane (row lane % 16, block lane / 16); its scales are byte S of the
// words. 4-bit operands take the first half of the registers.
template <int S>
__device__ __forceinline__ mx_f32x4 mx_mul(i32x4 a, i32x4 b, mx_f32x4 c, int scale_a, int scale_b) {
    const i32x8 x = __builtin_shufflevector(a, a, 0, 1, 2, 3, 0, 1, 2, 3), y = __builtin_shufflevector(b, b, 0, 1, 2, 3, 0, 1, 2, 3);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, S, scale_a, S, scale_b);
}

// 8 codes as the bf16 values they stand for.
__device__ __forceinline__ mx_bf16x8 mx_bf16(uint32_t codes, float scale) {
    union {
        mx_bf16x2 p[4];
        mx_bf16x8 v;
    } r;
    r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return r.v;
}
// A scale byte as a float (2^-127 is denormal; 255: NaN).
__device__ __forceinline__ float mx_scale(uint32_t byte) {
    return __uint_as_float(byte == 255 ? 0x7fc00000u : byte == 0 ? 0x00400000u : byte << 23);
}

// y[m][n .. n + 3] of the type that f32 says, n + i < N only.
__device__ __forceinline__ void mx_put(void *y, int64_t ldy, int f32, int m, int n, int N, mx_f32x4 v) {
    const int64_t at = (int64_t)m * ldy + n;
    if (f32) {
        float *p = (float *)y + at;
        if (n + 4 <= N) {
            put_f32x4(p, v);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i < N) p[i] = v[i];
        }
    } else {
        u16 *p = (u16 *)y + at;
        u16 h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __builtin_bit_cast(u16, (__bf16)v[i]);
        if (n + 4 <= N) {
            put_u16x4(p, make_ushort4(h[0], h[1], h[2], h[3]));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i < N) p[i] = h[i];
        }
    }
}
__device__ __forceinline__ mx_f32x4 mx_bias(const float *bias, int n, int N) {
    mx_f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (!bias) return v;
    if (n + 4 <= N) return get_f32x4<mx_f32x4>(bias + n);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < N) v[i] = bias[n + i];
    return v;
}

// 16 bytes of bf16 from element c of a row of `cols`, zeros from there on.
__device__ __forceinline__ uint4 mx_chunk(const u16 *row, int c, int cols) {
    const int there = mx_piece_cols(c, cols);
    if (there == 8) return get_16b(row + c);
    uint4 v = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < there) (&v.x)[j / 2] |= (uint32_t)row[c + j] << (j & 1) * 16;
    return v;
}

}  // namespace gemel

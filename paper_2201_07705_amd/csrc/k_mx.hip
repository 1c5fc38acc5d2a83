// Matrices in microscaled 4-bit floating point: blocks of 32 values of a row
// share a power of two 2^e, e = floor(log2 max|x|) - 2, held in a byte with a
// bias of 127, and each is the nearest of 0 .5 1 1.5 2 3 4 6 to |x| 2^-e with
// its sign (ties to the even code; 6 for all above). A block that holds a
// value that is not finite has the byte 255, and all its values are NaN.
//
// What bounds these kernels: memory. A wave takes 512 columns of 4 rows, 8
// columns to a lane, with all loads in flight before the first is used; the
// 4 lanes of a block agree on its scale by two lane moves, and the conversion
// to 4 bits is the hardware's (it divides by the scale and rounds as above).
// 4096 x 25088 float32 in 86 us (5.4 TB/s), its values again in 88 (116 for
// the first while the values of the call before are still written back);
// 16384 x 4096 bf16 in 34.
#include <hip/hip_runtime.h>

#include "mx_args.h"
#include "op_args.h"
#include "op_moves.h"

namespace gemel {

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int ROWS = 4;   // rows of a wave

// A scale byte as a float (2^-127 is denormal; 255: NaN).
__device__ __forceinline__ float scale_of(uint32_t byte) {
    return __uint_as_float(byte == 255 ? 0x7fc00000u : byte == 0 ? 0x00400000u : byte << 23);
}
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true));   // lanes 1 0 3 2
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xf, 0xf, true));   // lanes 2 3 0 1
}

// 8 elements of a row from column c on, zeros from `cols` on.
template <bool F32>
struct Eight {
    uint4 v[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const char *row, int c, int cols, bool whole) {
        if (whole || c + 8 <= cols) {
            v[0] = get_16b(row + (int64_t)c * (F32 ? 4 : 2));
            if constexpr (F32) v[1] = get_16b(row + (int64_t)c * 4 + 16);
            return;
        }
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) v[i] = uint4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (c + j >= cols) continue;
            if constexpr (F32)
                (&v[j / 4].x)[j % 4] = *(const uint32_t *)(row + (int64_t)(c + j) * 4);
            else
                (&v[0].x)[j / 2] |= (uint32_t) * (const u16 *)(row + (int64_t)(c + j) * 2) << (j & 1) * 16;
        }
    }
    // exponent field of the largest magnitude (255: some value is not finite)
    __device__ __forceinline__ uint32_t exponent() const {
        uint32_t m = 0;
        if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, (&v[j / 4].x)[j % 4] & 0x7fffffffu);
            return m >> 23;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t w = (&v[0].x)[j] & 0x7fff7fffu;
                m = max(m, max(w & 0xffffu, w >> 16));
            }
            return m >> 7;
        }
    }
    __device__ __forceinline__ uint32_t codes(float scale) const {
        uint32_t r = 0;
        if constexpr (F32) {
            const f32x4 a = __builtin_bit_cast(f32x4, v[0]), b = __builtin_bit_cast(f32x4, v[1]);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, a[0], a[1], scale, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, a[2], a[3], scale, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, b[0], b[1], scale, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, b[2], b[3], scale, 3);
        } else {
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v[0].x), scale, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v[0].y), scale, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v[0].z), scale, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v[0].w), scale, 3);
        }
        return r;
    }
};

// The rows and group of 512 columns of a wave.
struct Place {
    int row0, group, c;
    bool there;
};
__device__ __forceinline__ Place place(int rows, int groups) {
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    Place p;
    p.group = blockIdx.x * 4 + wave;
    p.row0 = blockIdx.y * ROWS;
    p.c = p.group * MX_GROUP + (threadIdx.x & 63) * 8;
    p.there = p.group < groups;
    return p;
}

template <bool F32>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const MxCast a) {
    const int groups = (a.q.cols + MX_GROUP - 1) / MX_GROUP, lane = threadIdx.x & 63;
    const int64_t pitch = mx_pitch(a.q.cols);
    for (int64_t y = blockIdx.y; y * ROWS < a.q.rows; y += gridDim.y) {
        Place p = place(a.q.rows, groups);
        p.row0 = (int)(y * ROWS);
        if (!p.there) return;
        const bool whole = (p.group + 1) * MX_GROUP <= a.q.cols;
        Eight<F32> v[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            v[r].load((const char *)a.x + (int64_t)min(p.row0 + r, a.q.rows - 1) * a.ld * (F32 ? 4 : 2), p.c, a.q.cols, whole);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int row = p.row0 + r;
            if (row >= a.q.rows) break;
            const uint32_t e = quad_max(v[r].exponent());
            const uint32_t byte = e == 255 ? 255u : max(e, 2u) - 2;
            const uint32_t codes = v[r].codes(e == 255 ? 1.f : scale_of(byte));
            *(uint32_t *)(a.q.codes + row * pitch + p.c / 2) = codes;
            const int q = lane >> 2;
            if ((lane & 3) == 0)
                a.q.scales[((int64_t)p.group * a.q.rows + row) * 16 + (q & 3) * 4 + (q >> 2)] = (uint8_t)byte;
        }
    }
}

template <bool F32>
__global__ __launch_bounds__(256) void mx_values_kernel(const MxCast a) {
    const int groups = (a.out_cols + MX_GROUP - 1) / MX_GROUP, lane = threadIdx.x & 63;
    const int64_t pitch = mx_pitch(a.q.cols);
    for (int64_t y = blockIdx.y; y * ROWS < a.q.rows; y += gridDim.y) {
        Place p = place(a.q.rows, groups);
        p.row0 = (int)(y * ROWS);
        if (!p.there) return;
        const bool inside = p.c < pitch * 2;   // (columns beyond the codes' padding are zeros)
        const int q = lane >> 2;
        uint32_t codes[ROWS], byte[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int row = min(p.row0 + r, a.q.rows - 1);
            codes[r] = inside ? *(const uint32_t *)(a.q.codes + row * pitch + p.c / 2) : 0u;
            byte[r] = inside ? a.q.scales[((int64_t)p.group * a.q.rows + row) * 16 + (q & 3) * 4 + (q >> 2)] : 0u;
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int row = p.row0 + r;
            if (row >= a.q.rows) break;
            const float s = scale_of(byte[r]);
            char *const out = (char *)a.out + (int64_t)row * a.ld * (F32 ? 4 : 2);
            const int n = min(8, a.out_cols - p.c), used = a.q.cols - p.c;
            if constexpr (F32) {
                f32x2 v[4];
                v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], s, 0);
                v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], s, 1);
                v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], s, 2);
                v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], s, 3);
                if (n == 8 && used >= 8) {
                    put_f32x4(out + (int64_t)p.c * 4, f32x4{v[0][0], v[0][1], v[1][0], v[1][1]});
                    put_f32x4(out + (int64_t)p.c * 4 + 16, f32x4{v[2][0], v[2][1], v[3][0], v[3][1]});
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < n) *(float *)(out + (int64_t)(p.c + j) * 4) = j < used ? v[j / 2][j % 2] : 0.f;
                }
            } else {
                uint32_t v[4];
                v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[r], s, 0));
                v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[r], s, 1));
                v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[r], s, 2));
                v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[r], s, 3));
                if (n == 8 && used >= 8) {
                    *(u32x4_any *)(out + (int64_t)p.c * 2) = u32x4_any{v[0], v[1], v[2], v[3]};
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < n) *(u16 *)(out + (int64_t)(p.c + j) * 2) = j < used ? (u16)(v[j / 2] >> (j & 1) * 16) : (u16)0;
                }
            }
        }
    }
}

// x = hi + mid + lo, each the leading 8 bits of what the ones before leave.
__global__ __launch_bounds__(256) void mx_planes_kernel(const MxPlanes a) {
    const int64_t per = a.ld / 8, n = a.rows * per, plane = (int64_t)a.rows * a.ld;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int row = (int)(i / per), c = (int)(i - row * per) * 8;
        Eight<true> v;
        v.load((const char *)(a.x + row * a.ldx), c, a.cols, false);
        uint4 out[3];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t b[2][3];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float f = __uint_as_float((&v.v[j / 2].x)[(2 * j + k) % 4]);
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    b[k][p] = __float_as_uint(f) & 0xffff0000u;
                    f -= __uint_as_float(b[k][p]);
                }
            }
#pragma unroll
            for (int p = 0; p < 3; ++p) (&out[p].x)[j] = b[0][p] >> 16 | b[1][p];
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) *(uint4 *)(a.out + p * plane + row * a.ld + c) = out[p];
    }
}

__global__ __launch_bounds__(256) void mx_sum_kernel(const MxSum a) {
    const int64_t per = a.ldp / 4, n = a.rows * per, step = (int64_t)a.rows * a.ldp;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int row = (int)(i / per), c = (int)(i - row * per) * 4;
        const float *p = a.part + row * a.ldp + c;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        int k = 0;
        for (; k + 4 <= a.parts; k += 4) {
            f32x4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = *(const f32x4 *)(p + (k + j) * step);
#pragma unroll
            for (int j = 0; j < 4; ++j) v += x[j];
        }
        for (; k < a.parts; ++k) v += *(const f32x4 *)(p + k * step);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (c + j >= a.cols) continue;
            const float y = v[j] + (a.bias ? a.bias[c + j] : 0.f);
            if (a.f32)
                ((float *)a.y)[row * a.ldy + c + j] = y;
            else
                ((u16 *)a.y)[row * a.ldy + c + j] = __builtin_bit_cast(u16, (__bf16)y);
        }
    }
}

template <typename A, typename K>
hipError_t go(K kernel, const A &a, dim3 grid, hipStream_t s) {
    void *p[] = {const_cast<A *>(&a)};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3(256), p, 0, s);
}
dim3 cast_grid(int rows, int cols) {
    const int64_t groups = mx_groups(cols);
    return dim3((unsigned)((groups + 3) / 4), (unsigned)((rows + ROWS - 1) / ROWS < 65535 ? (rows + ROWS - 1) / ROWS : 65535));
}
unsigned flat_grid(int64_t items) { return (unsigned)((items + 255) / 256 < 1 << 20 ? (items + 255) / 256 : 1 << 20); }

}  // namespace

hipError_t launch_mx_quantize(const MxCast &a, hipStream_t s) {
    if (!mx_cast_valid(a, false)) return hipErrorInvalidValue;
    return a.f32 ? go(&mx_quantize_kernel<true>, a, cast_grid(a.q.rows, a.q.cols), s)
                 : go(&mx_quantize_kernel<false>, a, cast_grid(a.q.rows, a.q.cols), s);
}
hipError_t launch_mx_values(const MxCast &a, hipStream_t s) {
    if (!mx_cast_valid(a, true)) return hipErrorInvalidValue;
    return a.f32 ? go(&mx_values_kernel<true>, a, cast_grid(a.q.rows, a.out_cols), s)
                 : go(&mx_values_kernel<false>, a, cast_grid(a.q.rows, a.out_cols), s);
}
hipError_t launch_mx_planes(const MxPlanes &a, hipStream_t s) {
    if (!mx_planes_valid(a)) return hipErrorInvalidValue;
    return go(&mx_planes_kernel, a, dim3(flat_grid(a.rows * a.ld / 8)), s);
}
hipError_t launch_mx_sum(const MxSum &a, hipStream_t s) {
    if (!mx_sum_valid(a)) return hipErrorInvalidValue;
    return go(&mx_sum_kernel, a, dim3(flat_grid(a.rows * a.ldp / 4)), s);
}

}  // namespace gemel

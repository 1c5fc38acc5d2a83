// Low-rank adapters of many requests beside a shared projection: the thin
// products and the layouts around the large ones (k_mm.hip).
#include <hip/hip_runtime.h>

#include "op_args.h"

namespace gemel {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf_up(u16 h) { return __uint_as_float((uint32_t)h << 16); }
__device__ __forceinline__ u16 bf_down(float f) { return __builtin_bit_cast(u16, (__bf16)f); }
__device__ __forceinline__ u16 half_down(float f) { return __builtin_bit_cast(u16, (_Float16)f); }
__device__ __forceinline__ float half_up(u16 h) { return (float)__builtin_bit_cast(_Float16, h); }

// 8 elements of a row from k on; elements at k_end and beyond are zeros.
__device__ __forceinline__ bf16x8 load8(const u16 *row, int k, int k_end, int whole) {
    union {
        u16 h[8];
        bf16x8 v;
        uint4 q;
    } r;
    if (whole && k + 8 <= k_end) {
        r.q = *(const uint4 *)(row + k);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.h[i] = k + i < k_end ? row[k + i] : (u16)0;
    }
    return r.v;
}
__device__ __forceinline__ f32x4 load4(const float *row, int k, int k_end, int whole) {
    f32x4 r;
    if (whole && k + 4 <= k_end) {
        r = *(const f32x4 *)(row + k);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = k + i < k_end ? row[k + i] : 0.f;
    }
    return r;
}

// t[p][r] = scale * sum_k x[row p][k] a[r][k] for 16 positions of one run and
// 16 rank indices. 8 waves share the depth, chunk by chunk, and add their
// sums in LDS in wave order. Sums are float32; float32 operands go through
// the float32 MFMA unrounded.
template <bool F32>
__global__ __launch_bounds__(512) void shrink_kernel(const ShrinkArgs a) {
    __shared__ f32x4 part[8][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, l16 = lane & 15;
    const int *it = a.b.items + 3 * blockIdx.x;
    const int u = it[0], p0 = it[1], n = it[2];
    const int rank = a.b.run_rank[u], r0 = blockIdx.y * 16;
    const int pos = p0 + min(l16, n - 1);
    const int64_t xrow = (int64_t)a.b.perm[pos] * a.ldx;
    const int r = r0 + l16;
    const bool used = r < rank;
    const int64_t arow = ((int64_t)(a.by_run ? u : a.b.run_id[u]) * (a.by_run ? a.rp : a.b.rank) + (used ? r : 0)) * a.lda;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (r0 < rank) {
        if constexpr (F32) {
            for (int k = wave * 16 + 4 * g; k - 4 * g < a.K; k += 128) {
                const f32x4 xv = load4((const float *)a.x + xrow, k, a.K, a.vx);
                f32x4 av = load4((const float *)a.a + arow, k, a.K, a.va);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(used ? av[e] : 0.f, xv[e], acc, 0, 0, 0);
            }
        } else {
            for (int k = wave * 32 + 8 * g; k - 8 * g < a.K; k += 256) {
                const bf16x8 xv = load8((const u16 *)a.x + xrow, k, a.K, a.vx);
                bf16x8 av = load8((const u16 *)a.a + arow, k, used ? a.K : 0, a.va);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, xv, acc, 0, 0, 0);
            }
        }
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
    for (int w = 1; w < 8; ++w) acc += part[w][lane];
    if (l16 >= n) return;
    const float scale = a.b.run_scale[u];
    const int64_t p = p0 + l16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int q = r0 + 4 * g + i;
        const float t = q < rank ? acc[i] * scale : 0.f;
        if (a.t) a.t[p * a.rp + q] = t;
        if (a.planes) {
            // bf16 pair: t to 16 bits, so that its product with B is as
            // exact as the main product's sums
            const u16 h = bf_down(t);
            a.planes[p * 2 * a.rp + q] = h;
            a.planes[p * 2 * a.rp + a.rp + q] = bf_down(t - bf_up(h));
        }
    }
}

__global__ __launch_bounds__(256) void pack_rank_kernel(const PackRankArgs a) {
    const int u = blockIdx.y;
    const int rank = a.b.run_rank[u];
    const int64_t id = a.b.run_id[u];
    const int64_t n = a.by_rank ? (int64_t)a.rp * a.ldc : (int64_t)a.C * a.rp;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int r = a.by_rank ? (int)(i / a.ldc) : (int)(i % a.rp);
        const int c = a.by_rank ? (int)(i - (int64_t)r * a.ldc) : (int)(i / a.rp);
        const bool in = r < rank && c < a.C;
        const int64_t at = id * a.C * a.R + (a.in_rc ? (int64_t)r * a.C + c : (int64_t)c * a.R + r);
        if (a.f32) {
            ((float *)a.out)[(int64_t)u * n + i] = in ? ((const float *)a.in)[at] : 0.f;
        } else {
            const u16 v = in ? ((const u16 *)a.in)[at] : (u16)0;
            u16 *out = (u16 *)a.out;
            if (a.by_rank) {
                out[(int64_t)u * n + i] = v;
            } else {
                out[((int64_t)u * a.C + c) * 2 * a.rp + r] = v;
                out[((int64_t)u * a.C + c) * 2 * a.rp + a.rp + r] = v;
            }
        }
    }
}

// part[r][c] = sum over the chunk's positions of p[pos][r] q[row][c], for 16
// rank indices and 64 columns: float32 MFMA on widened values.
template <bool F32>
__global__ __launch_bounds__(256) void outer_kernel(const OuterArgs a) {
    __shared__ float qs[16][68], ps[16][17];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, l16 = lane & 15;
    const int *ch = a.b.chunks + 3 * blockIdx.z;
    const int p0 = ch[1], n = ch[2];
    const int c0 = blockIdx.x * 64, r0 = blockIdx.y * 16;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < n; s += 16) {
        __syncthreads();
        {
            const int row = tid >> 4, col = tid & 15;
            const bool in = s + row < n;
            ps[row][col] = in ? a.p[(int64_t)(p0 + s + row) * a.rp + r0 + col] : 0.f;
            const int64_t at = (int64_t)a.b.perm[in ? p0 + s + row : p0] * a.ldq;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = c0 + col + 16 * i;
                float v = 0.f;
                if (in && c < a.C) v = F32 ? ((const float *)a.q)[at + c] : bf_up(((const u16 *)a.q)[at + c]);
                qs[row][col + 16 * i] = v;
            }
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e)
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(ps[4 * e + g][l16], qs[4 * e + g][wave * 16 + l16], acc, 0, 0, 0);
    }
    const int c = c0 + wave * 16 + l16;
    if (c >= a.C) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        a.part[((int64_t)blockIdx.z * a.rp + r0 + 4 * g + i) * a.C + c] = acc[i];
}

// Chunks of an adapter added in order; adapters without rows and rank
// indices beyond the adapter's own give zeros.
__global__ __launch_bounds__(256) void outer_sum_kernel(const OuterArgs a) {
    const int ad = blockIdx.y, u = a.b.run_of[ad], R = a.b.rank;
    const int64_t n = (int64_t)R * a.C;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int r = a.transposed ? (int)(i % R) : (int)(i / a.C);
        const int c = a.transposed ? (int)(i / R) : (int)(i - (int64_t)r * a.C);
        float v = 0.f;
        if (u >= 0 && r < a.b.run_rank[u])
            for (int k = a.b.chunk_first[u]; k < a.b.chunk_first[u + 1]; ++k)
                v += a.part[((int64_t)k * a.rp + r) * a.C + c];
        a.out[ad * n + i] = v;
    }
}

__global__ __launch_bounds__(256) void colsum_kernel(const ColsumArgs a) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    const int r0 = (int)((int64_t)a.rows * blockIdx.y / a.parts), r1 = (int)((int64_t)a.rows * (blockIdx.y + 1) / a.parts);
    float v = 0.f;
    for (int r = r0; r < r1; ++r)
        v += a.f32 ? ((const float *)a.in)[r * a.ld + c] : bf_up(((const u16 *)a.in)[r * a.ld + c]);
    a.part[(int64_t)blockIdx.y * a.cols + c] = v;
}
__global__ __launch_bounds__(256) void colsum_sum_kernel(const ColsumArgs a) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float v = 0.f;
    for (int p = 0; p < a.parts; ++p) v += a.part[(int64_t)p * a.cols + c];
    a.out[c] = v;
}

template <typename E>
__global__ __launch_bounds__(256) void pad_kernel(const PadArgs a) {
    const int64_t n = (int64_t)a.rows * a.ldo;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / a.ldo, c = i - r * a.ldo;
        ((E *)a.out)[i] = c < a.cols ? ((const E *)a.in)[(a.perm ? a.perm[r] : r) * a.ldi + c] : (E)0;
    }
}

// 64 x 64 tiles through LDS; out[c][r], zeros for r in [rows, ldo).
__global__ __launch_bounds__(256) void pad_t_kernel(const PadArgs a) {
    __shared__ u16 tile[64][66];
    const u16 *in = (const u16 *)a.in;
    u16 *out = (u16 *)a.out;
    const int r0 = blockIdx.x * 64, c0 = blockIdx.y * 64, x = threadIdx.x & 63, y = threadIdx.x >> 6;
    for (int i = y; i < 64; i += 4)
        tile[i][x] = r0 + i < a.rows && c0 + x < a.cols ? in[(int64_t)(r0 + i) * a.ldi + c0 + x] : (u16)0;
    __syncthreads();
    for (int i = y; i < 64; i += 4)
        if (c0 + i < a.cols && r0 + x < a.ldo) out[(int64_t)(c0 + i) * a.ldo + r0 + x] = tile[x][i];
}

// The exponent that brings a largest magnitude `mx` into [2^14, 2^15); 0
// where it is zero or not finite.
__device__ __forceinline__ int plane_exp(float mx) {
    if (!(mx > 0.f) || !isfinite(mx)) return 0;
    return 14 - ilogbf(mx);
}
__device__ __forceinline__ void split_put(u16 *hi, u16 *lo, int64_t at, float v, int e) {
    const float s = ldexpf(v, e);
    const u16 h = half_down(s);
    hi[at] = h;
    // the rest of a value that is not finite would be NaN; the sum has it already
    lo[at] = isfinite(s) ? half_down(s - half_up(h)) : (u16)0;
}

__global__ __launch_bounds__(256) void split_kernel(const SplitArgs a) {
    __shared__ float mx[4];
    const int r = blockIdx.x;
    const float *in = a.in + (int64_t)(a.perm ? a.perm[r] : r) * a.ldi;
    float m = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += 256) {
        const float v = fabsf(in[c]);
        m = v > m || v != v ? v : m;
    }
    for (int o = 32; o; o >>= 1) {
        const float v = __shfl_xor(m, o);
        m = v > m || v != v ? v : m;
    }
    if ((threadIdx.x & 63) == 0) mx[threadIdx.x >> 6] = m;
    __syncthreads();
    for (int i = 0; i < 4; ++i) m = mx[i] > m || mx[i] != mx[i] ? mx[i] : m;
    const int e = plane_exp(m);
    if (threadIdx.x == 0) a.e[r] = e;
    for (int64_t c = threadIdx.x; c < a.ldo; c += 256)
        split_put(a.hi, a.lo, (int64_t)r * a.ldo + c, c < a.cols ? in[c] : 0.f, e);
}

__global__ __launch_bounds__(256) void zero_u32_kernel(unsigned *p, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i] = 0;
}
// Largest magnitudes of the columns: magnitudes order as their bits do, and
// the maximum does not depend on the order of the atomics.
__global__ __launch_bounds__(256) void colmax_kernel(const SplitArgs a) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    const int r0 = (int)((int64_t)a.rows * blockIdx.y / gridDim.y), r1 = (int)((int64_t)a.rows * (blockIdx.y + 1) / gridDim.y);
    unsigned m = 0;
    for (int r = r0; r < r1; ++r) m = max(m, __float_as_uint(a.in[(int64_t)r * a.ldi + c]) & 0x7fffffffu);
    atomicMax(a.colmax + c, m);
}
__global__ __launch_bounds__(256) void split_t_kernel(const SplitArgs a) {
    __shared__ float tile[64][65];
    const int r0 = blockIdx.x * 64, c0 = blockIdx.y * 64, x = threadIdx.x & 63, y = threadIdx.x >> 6;
    for (int i = y; i < 64; i += 4)
        tile[i][x] = r0 + i < a.rows && c0 + x < a.cols ? a.in[(int64_t)(r0 + i) * a.ldi + c0 + x] : 0.f;
    __syncthreads();
    for (int i = y; i < 64; i += 4) {
        if (c0 + i >= a.cols) break;
        const int e = plane_exp(__uint_as_float(a.colmax[c0 + i]));
        if (r0 + x < a.ldo) split_put(a.hi, a.lo, (int64_t)(c0 + i) * a.ldo + r0 + x, tile[x][i], e);
        if (blockIdx.x == 0 && x == 0) a.e[c0 + i] = e;
    }
}

template <typename A>
hipError_t launch(const void *fn, dim3 grid, int block, const A &a, hipStream_t s) {
    void *p[] = {const_cast<A *>(&a)};
    return hipLaunchKernel(fn, grid, dim3((unsigned)block), p, 0, s);
}
unsigned blocks(int64_t n, int64_t most) { return (unsigned)(n < most ? (n > 0 ? n : 1) : most); }
bool tables(const BatchTables &b) {
    return b.perm && b.run_start && b.run_id && b.run_rank && b.run_scale && b.first_run && b.items && b.chunks &&
           b.chunk_first && b.run_of && b.rows > 0 && b.runs >= 0 && b.adapters > 0 && b.rank > 0;
}

}  // namespace

hipError_t launch_shrink(const ShrinkArgs &a, hipStream_t s) {
    if (!tables(a.b) || !a.x || !a.a || a.K <= 0 || a.rp % 32 || a.rp < a.b.rank || a.b.n_items <= 0 || !(a.t || a.planes))
        return hipErrorInvalidValue;
    const dim3 grid((unsigned)a.b.n_items, (unsigned)(a.rp / 16));
    return a.f32 ? launch(reinterpret_cast<const void *>(&shrink_kernel<true>), grid, 512, a, s)
                 : launch(reinterpret_cast<const void *>(&shrink_kernel<false>), grid, 512, a, s);
}

hipError_t launch_pack_rank(const PackRankArgs &a, hipStream_t s) {
    if (!tables(a.b) || !a.in || !a.out || a.C <= 0 || a.R != a.b.rank || a.rp < a.R || a.b.runs <= 0 || a.b.runs > 65535 ||
        (a.by_rank && a.ldc < a.C))
        return hipErrorInvalidValue;
    const int64_t n = a.by_rank ? (int64_t)a.rp * a.ldc : (int64_t)a.C * a.rp;
    return launch(reinterpret_cast<const void *>(&pack_rank_kernel), dim3(blocks((n + 255) / 256, 1024), (unsigned)a.b.runs),
                  256, a, s);
}

hipError_t launch_outer(const OuterArgs &a, hipStream_t s) {
    if (!tables(a.b) || !a.p || !a.q || !a.out || a.C <= 0 || a.rp % 16 || a.rp < a.b.rank || a.b.n_chunks > 65535 ||
        a.b.adapters > 65535 || (a.b.n_chunks > 0 && !a.part))
        return hipErrorInvalidValue;
    if (a.b.n_chunks > 0) {
        const dim3 grid((unsigned)((a.C + 63) / 64), (unsigned)(a.rp / 16), (unsigned)a.b.n_chunks);
        const hipError_t e = a.f32 ? launch(reinterpret_cast<const void *>(&outer_kernel<true>), grid, 256, a, s)
                                   : launch(reinterpret_cast<const void *>(&outer_kernel<false>), grid, 256, a, s);
        if (e != hipSuccess) return e;
    }
    const int64_t n = (int64_t)a.b.rank * a.C;
    return launch(reinterpret_cast<const void *>(&outer_sum_kernel),
                  dim3(blocks((n + 255) / 256, 4096), (unsigned)a.b.adapters), 256, a, s);
}

hipError_t launch_colsum(const ColsumArgs &a, hipStream_t s) {
    if (!a.in || !a.out || !a.part || a.rows <= 0 || a.cols <= 0 || a.parts < 1 || a.parts > 65535) return hipErrorInvalidValue;
    const unsigned bx = (unsigned)((a.cols + 255) / 256);
    const hipError_t e = launch(reinterpret_cast<const void *>(&colsum_kernel), dim3(bx, (unsigned)a.parts), 256, a, s);
    if (e != hipSuccess) return e;
    return launch(reinterpret_cast<const void *>(&colsum_sum_kernel), dim3(bx), 256, a, s);
}

hipError_t launch_pad(const PadArgs &a, hipStream_t s) {
    if (!a.in || !a.out || a.rows <= 0 || a.cols <= 0 || a.ldo < (a.transposed ? a.rows : a.cols)) return hipErrorInvalidValue;
    if (!a.transposed)
        return launch(a.f32 ? reinterpret_cast<const void *>(&pad_kernel<uint32_t>) : reinterpret_cast<const void *>(&pad_kernel<u16>),
                      dim3(blocks(((int64_t)a.rows * a.ldo + 255) / 256, 8192)), 256, a, s);
    const int64_t by = (a.cols + 63) / 64;
    if (by > 65535 || a.f32) return hipErrorInvalidValue;
    return launch(reinterpret_cast<const void *>(&pad_t_kernel), dim3((unsigned)((a.ldo + 63) / 64), (unsigned)by), 256, a, s);
}

hipError_t launch_split(const SplitArgs &a, hipStream_t s) {
    if (!a.in || !a.hi || !a.lo || !a.e || a.rows <= 0 || a.cols <= 0 || a.ldo < (a.transposed ? a.rows : a.cols))
        return hipErrorInvalidValue;
    if (!a.transposed) return launch(reinterpret_cast<const void *>(&split_kernel), dim3((unsigned)a.rows), 256, a, s);
    const int64_t by = (a.cols + 63) / 64;
    if (!a.colmax || a.perm || by > 65535) return hipErrorInvalidValue;
    unsigned *cm = a.colmax;
    int n = a.cols;
    void *p[] = {&cm, &n};
    const unsigned bx = (unsigned)((a.cols + 255) / 256);
    hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(&zero_u32_kernel), dim3(bx), dim3(256), p, 0, s);
    if (e != hipSuccess) return e;
    e = launch(reinterpret_cast<const void *>(&colmax_kernel), dim3(bx, blocks((a.rows + 63) / 64, 256)), 256, a, s);
    if (e != hipSuccess) return e;
    return launch(reinterpret_cast<const void *>(&split_t_kernel), dim3((unsigned)((a.ldo + 63) / 64), (unsigned)by), 256, a, s);
}

}  // namespace gemel

// The thin products of low-rank adapters: x A^T and dy B per row, and the
// adapters' own gradients, sums over rows.
#include <hip/hip_runtime.h>

#include "op_args.h"
#include "op_moves.h"

namespace gemel {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf_up(u16 h) { return __uint_as_float((uint32_t)h << 16); }
__device__ __forceinline__ u16 bf_down(float f) { return __builtin_bit_cast(u16, (__bf16)f); }

// 16 bytes of a row from element k on; elements at k_end and beyond are zeros.
template <bool F32>
__device__ __forceinline__ uint4 chunk(const void *base, int64_t row, int k, int k_end) {
    constexpr int Q = F32 ? 4 : 8;
    if (k + Q <= k_end) return get_16b((const char *)base + (row + k) * (F32 ? 4 : 2));
    union {
        uint4 v;
        u16 h[8];
        uint32_t w[4];
    } r;
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        if constexpr (F32)
            r.w[i] = k + i < k_end ? ((const uint32_t *)base)[row + k + i] : 0u;
        else
            r.h[i] = k + i < k_end ? ((const u16 *)base)[row + k + i] : (u16)0;
    }
    return r.v;
}

// Two thin products by value; which one is read with a uniform index from
// the argument block itself (indexing the parameter would copy it).
template <typename A>
struct Two {
    A a[2];
};
template <typename A>
__device__ __forceinline__ const A &arg_of(int i) {
    return ((const Two<A> *)__builtin_amdgcn_kernarg_segment_ptr())->a[i];
}

// What becomes of a sum t (scaled) of position p and rank index q. An adapter
// whose other half is not finite (bad) spoils its own rows, here, as that
// half's copy holds zeros in those places.
__device__ __forceinline__ void put_thin(const ShrinkArgs &a, int64_t p, int q, float t, int bad) {
    if (a.t) a.t[p * a.rp + q] = t;
    if (a.planes) {
        // bf16 pair: t to 16 bits, so that its product with B is as exact as
        // the main product's sums
        const u16 h = bad ? (u16)0x7fc0 : bf_down(t);
        a.planes[p * 2 * a.rp + q] = h;
        a.planes[p * 2 * a.rp + a.rp + q] = bf_down(t - bf_up(h));
    }
}

// t[p][r] = scale * sum_k x[row p][k] a[r][k] for up to 32 positions of one
// run and RB blocks of 16 rank indices. 8 waves share the depth (or a slice of
// it), chunk by chunk, and add their sums in LDS in wave order. Reading x
// bounds it, once each wave has four chunks of every operand in flight: 16384
// bf16 rows of 4096 42 us (134 MB, 3.2 TB/s), 13784 float32 rows of 2526 41
// us (139 MB, 3.4 TB/s). Sums are float32; float32 operands go through the
// float32 MFMA unrounded.
template <bool F32, int RB>
__global__ __launch_bounds__(512) void shrink_kernel(const Two<ShrinkArgs> args) {
    const int first = arg_of<ShrinkArgs>(0).slices, second = (int)blockIdx.z >= first;
    const ShrinkArgs &a = arg_of<ShrinkArgs>(second);
    const int slice = (int)blockIdx.z - (second ? first : 0);
    __shared__ f32x4 part[8][2 * RB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), g = lane >> 4, l16 = lane & 15;
    const int *it = a.b.items + 3 * blockIdx.x;
    const int u = it[0], p0 = it[1], n = it[2];
    const int rank = a.b.run_rank[u], r0 = blockIdx.y * 16 * RB;
    constexpr int Q = F32 ? 4 : 8;   // elements of a lane's chunk
    int64_t xrow[2], arow[RB];
    bool used[RB];
#pragma unroll
    for (int i = 0; i < 2; ++i) xrow[i] = (int64_t)a.b.perm[p0 + min(16 * i + l16, n - 1)] * a.ldx;
#pragma unroll
    for (int j = 0; j < RB; ++j) {
        const int r = r0 + 16 * j + l16;
        used[j] = r < rank;
        arow[j] = ((int64_t)(a.by_run ? u : a.b.run_id[u]) * (a.by_run ? a.rp : a.b.rank) + (used[j] ? r : 0)) * a.lda;
    }
    f32x4 acc[2][RB];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < RB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto add = [&](const uint4 (&xv)[2], const uint4 (&av)[RB]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                if constexpr (F32) {
                    const f32x4 x = __builtin_bit_cast(f32x4, xv[i]), w = __builtin_bit_cast(f32x4, av[j]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x[e], acc[i][j], 0, 0, 0);
                } else {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, av[j]),
                                                                        __builtin_bit_cast(bf16x8, xv[i]), acc[i][j], 0, 0, 0);
                }
            }
    };
    if (r0 < rank) {
        int k = slice * a.per + wave * 4 * Q;   // (the wave's; its lane groups take Q each)
        const int end = min(a.K, (slice + 1) * a.per);
        // whole chunks, four rounds of them in flight: no branch may stand
        // between the loads
        const char *const xb = (const char *)a.x, *const ab = (const char *)a.a;
        constexpr int E = F32 ? 4 : 2, ROUNDS = 4;
        for (; k + (ROUNDS - 1) * 32 * Q + 4 * Q <= end; k += ROUNDS * 32 * Q) {
            uint4 xv[ROUNDS][2], av[ROUNDS][RB];
#pragma unroll
            for (int q = 0; q < ROUNDS; ++q) {
                const int kk = k + q * 32 * Q + g * Q;
#pragma unroll
                for (int i = 0; i < 2; ++i) xv[q][i] = get_16b(xb + (xrow[i] + kk) * E);
#pragma unroll
                for (int j = 0; j < RB; ++j) av[q][j] = get_16b(ab + (arow[j] + kk) * E);
            }
#pragma unroll
            for (int q = 0; q < ROUNDS; ++q) {
#pragma unroll
                for (int j = 0; j < RB; ++j) av[q][j] = used[j] ? av[q][j] : uint4{};
                add(xv[q], av[q]);
            }
        }
        for (; k < end; k += 32 * Q) {
            uint4 xv[2], av[RB];
#pragma unroll
            for (int i = 0; i < 2; ++i) xv[i] = chunk<F32>(a.x, xrow[i], k + g * Q, end);
#pragma unroll
            for (int j = 0; j < RB; ++j) av[j] = chunk<F32>(a.a, arow[j], k + g * Q, used[j] ? end : 0);
            add(xv, av);
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < RB; ++j) part[wave][i * RB + j][lane] = acc[i][j];
    int bad = 0;
    if (a.flags) {
        for (int i = threadIdx.x; i < a.n_flags; i += 512) bad |= a.flags[(int64_t)u * a.n_flags + i];
        bad = __syncthreads_or(bad);
        if (a.slices > 1 && threadIdx.x == 0) a.bad[u] = bad;
    } else {
        __syncthreads();
    }
    if (wave >= 2 * RB) return;
    f32x4 sum = part[0][wave][lane];
    for (int w = 1; w < 8; ++w) sum += part[w][wave][lane];
    const int i = wave / RB, j = wave - i * RB;
    if (16 * i + l16 >= n) return;
    const float scale = a.b.run_scale[u];
    const int64_t p = p0 + 16 * i + l16;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int q = r0 + 16 * j + 4 * g + e;
        if (a.slices > 1)
            a.part[((int64_t)slice * a.b.rows + p) * a.rp + q] = sum[e];
        else
            put_thin(a, p, q, q < rank ? sum[e] * scale : 0.f, bad);
    }
}

// The slices' sums, added in order.
__global__ __launch_bounds__(256) void shrink_sum_kernel(const Two<ShrinkArgs> args) {
    const ShrinkArgs &a = arg_of<ShrinkArgs>(blockIdx.y);
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)a.b.rows * a.rp;
    const int p = (int)(i / a.rp), q = (int)(i - (int64_t)p * a.rp);
    if (a.slices < 2 || i >= n) return;
    const int u = a.b.run_at[p];
    if (u < 0) return;
    float t = 0.f;
#pragma unroll 8
    for (int k = 0; k < a.slices; ++k) t += a.part[k * n + i];
    put_thin(a, p, q, q < a.b.run_rank[u] ? t * a.b.run_scale[u] : 0.f, a.flags ? a.bad[u] : 0);
}

// out[r][c] = sum over a chunk's positions of p(pos, r) q[row][c] for 32 r
// and 4 * CT columns, 32 positions at a time. The matrix cores want 8
// positions of a column (or of an r) in a lane, so both operands are turned
// on the way out of LDS. A float32 p beside bf16 q is multiplied as three
// bf16 pieces, which hold all of its bits; float32 q goes to the float32
// MFMA. The next 32 positions are in registers while the present ones are
// multiplied; reading q (or writing out) bounds it: both adapter gradients of
// 8192 bf16 rows of 4096 57 us (134 MB, 2.4 TB/s), dW and dx of 14 float32
// rows, 20244 -> 956, 60 us (155 MB, 2.6 TB/s).
template <bool F32, bool P32>
__device__ __forceinline__ void outer(const OuterArgs &a, int block, unsigned char *qs, float *ps) {
    constexpr int RB = 2, E = F32 ? 4 : 2, CT = F32 ? 32 : 64, COLS = 4 * CT, FC = CT / 16, PIECES = P32 ? 3 : 1;
    constexpr int PITCH = COLS * E + 16, PP = RB * 16 + 1;   // bytes; floats
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, l16 = lane & 15;
    const int across = (a.C + COLS - 1) / COLS, down = (a.R + 31) / 32;
    const int bx = block % across, by = block / across % down, bz = block / (across * down);
    const int c0 = bx * COLS, r0 = by * 32;
    int p0 = bz * a.per, n = min(a.per, a.positions - p0);
    if (a.chunks) {
        const int ch = bz / a.sub, piece = bz - ch * a.sub;
        const int all = a.chunks[3 * ch + 2], each = ((all + a.sub - 1) / a.sub + 31) / 32 * 32;
        p0 = a.chunks[3 * ch + 1] + piece * each;
        n = min(each, all - piece * each);
    }
    constexpr int Q = 16 / E, LR = COLS / Q, NQ = 32 * LR / 256, NP = 32 * RB * 16 / 256;
    uint4 q[NQ];
    float p[NP];
    // items of p along whichever of its indices is contiguous
    const bool along = a.sr == 1;
    auto p_row = [&](int i) __attribute__((always_inline)) { return along ? (i * 256 + tid) / 32 : (i * 256 + tid) % 32; };
    auto p_col = [&](int i) __attribute__((always_inline)) { return along ? (i * 256 + tid) % 32 : (i * 256 + tid) / 32; };
    const bool whole = c0 + COLS <= a.C;
    auto load = [&](int s) __attribute__((always_inline)) {
        if (whole && s + 32 <= n) {
            // (no branch between the loads)
            int64_t at[NQ];
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                const int pos = p0 + s + (i * 256 + tid) / LR;
                at[i] = (int64_t)(a.perm ? a.perm[pos] : pos) * a.ldq + c0 + (tid % LR) * Q;
            }
#pragma unroll
            for (int i = 0; i < NQ; ++i) q[i] = get_16b((const char *)a.q + at[i] * E);
        } else {
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                const int row = (i * 256 + tid) / LR, c = c0 + (tid % LR) * Q;
                const bool in = s + row < n;
                const int pos = p0 + s + row;
                q[i] = chunk<F32>(a.q, in ? (int64_t)(a.perm ? a.perm[pos] : pos) * a.ldq : 0, c, in ? a.C : 0);
            }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int row = p_row(i), r = r0 + p_col(i);
            p[i] = 0.f;
            if (s + row < n && r < a.R) {
                const int64_t at = (int64_t)(p0 + s + row) * a.sp + r * a.sr;
                p[i] = P32 ? ((const float *)a.p)[at] : bf_up(((const u16 *)a.p)[at]);
            }
        }
    };
    f32x4 acc[RB][FC];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    load(0);
    for (int s = 0; s < n; s += 32) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NQ; ++i) *(uint4 *)(qs + ((i * 256 + tid) / LR) * PITCH + (tid % LR) * 16) = q[i];
#pragma unroll
        for (int i = 0; i < NP; ++i) ps[p_row(i) * PP + p_col(i)] = p[i];
        __syncthreads();
        if (s + 32 < n) load(s + 32);
        if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float x[RB], y[FC];
#pragma unroll
                for (int i = 0; i < RB; ++i) x[i] = ps[(4 * e + g) * PP + i * 16 + l16];
#pragma unroll
                for (int j = 0; j < FC; ++j) y[j] = *(const float *)(qs + (4 * e + g) * PITCH + (wave * CT + j * 16 + l16) * 4);
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int j = 0; j < FC; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[j], acc[i][j], 0, 0, 0);
            }
        } else {
            bf16x8 x[RB][PIECES];
#pragma unroll
            for (int i = 0; i < RB; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float v = ps[(8 * g + e) * PP + i * 16 + l16];
#pragma unroll
                    for (int w = 0; w < PIECES; ++w) {
                        x[i][w][e] = (__bf16)v;
                        v -= (float)x[i][w][e];
                    }
                }
#pragma unroll
            for (int j = 0; j < FC; ++j) {
                bf16x8 y;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    y[e] = *(const __bf16 *)(qs + (8 * g + e) * PITCH + (wave * CT + j * 16 + l16) * 2);
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int w = PIECES - 1; w >= 0; --w)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i][w], y, acc[i][j], 0, 0, 0);
            }
        }
    }
    float *out = a.out + bz * a.chunk;
#pragma unroll
    for (int j = 0; j < FC; ++j) {
        const int c = c0 + wave * CT + j * 16 + l16;
        if (c >= a.C) continue;
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = r0 + i * 16 + 4 * g + e;
                if (r < a.R) out[r * a.ld + c] = acc[i][j][e];
            }
    }
}

// Several such products in one launch.
template <bool F32>
__global__ __launch_bounds__(256) void outer_kernel(const Outers args) {
    __shared__ __attribute__((aligned(16))) unsigned char qs[32 * (512 + 16)];
    __shared__ float ps[32 * 33];
    const Outers &all = *(const Outers *)__builtin_amdgcn_kernarg_segment_ptr();
    int i = 0;
    while (i + 1 < all.n && (int)blockIdx.x >= all.first[i + 1]) ++i;
    const OuterArgs &a = all.a[i];
    const int block = (int)blockIdx.x - all.first[i];
    if (F32 || a.p_f32)
        outer<F32, true>(a, block, qs, ps);
    else
        outer<F32, F32>(a, block, qs, ps);
}

template <typename A>
hipError_t launch(const void *fn, dim3 grid, int block, const A *a, int n, hipStream_t s) {
    Two<A> t{{a[0], a[n - 1]}};
    void *p[] = {&t};
    return hipLaunchKernel(fn, grid, dim3((unsigned)block), p, 0, s);
}

}  // namespace

hipError_t launch_shrink(const ShrinkArgs *a, int n, hipStream_t s) {
    if (!shrink_valid(a, n)) return hipErrorInvalidValue;
    const int slices = a[0].slices + (n > 1 ? a[1].slices : 0);
    const dim3 grid((unsigned)a[0].b.n_items, (unsigned)(a[0].rp / 32), (unsigned)slices);
    const void *fn = a[0].f32 ? reinterpret_cast<const void *>(&shrink_kernel<true, 2>)
                              : reinterpret_cast<const void *>(&shrink_kernel<false, 2>);
    const hipError_t e = launch(fn, grid, 512, a, n, s);
    if (e != hipSuccess || slices == n) return e;
    const dim3 all((unsigned)(((int64_t)a[0].b.rows * a[0].rp + 255) / 256), (unsigned)n);
    return launch(reinterpret_cast<const void *>(&shrink_sum_kernel), all, 256, a, n, s);
}

hipError_t launch_outer(const Outers &o, hipStream_t s) {
    if (o.n == 0) return hipSuccess;
    void *p[] = {const_cast<Outers *>(&o)};
    return hipLaunchKernel(o.a[0].q_f32 ? reinterpret_cast<const void *>(&outer_kernel<true>)
                                        : reinterpret_cast<const void *>(&outer_kernel<false>),
                           dim3((unsigned)o.blocks), dim3(256), p, 0, s);
}

}  // namespace gemel

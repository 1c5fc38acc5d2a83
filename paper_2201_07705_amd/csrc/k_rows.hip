// Adapted projections of few rows (up to 64): every request its own adapter,
// one row each, is the usual load of a server.
//
// Reading the weights is what bounds them, and after that the launches. Two
// launches do the work. The first holds workgroups of two kinds that do not
// wait for each other: 64 outputs by a slice of the depth (the weights, by
// direct global-to-LDS loads four steps ahead, on the matrix cores), and the
// thin products x A^T of 16 rows of one adapter by a slice of the depth. The
// second adds the slices in order, multiplies the thin sums with the rows of
// B that each output needs, and adds the bias. All sums are float32; float32
// operands stay float32.
//
// 4096 -> 4096, every row its own adapter of rank 16, bf16: one row 11 us, 64
// rows 16 us (3.4 TB/s of weights and adapters), of which two launches are 9;
// as tiles of 64 rows, copies and thin products in launches of their own 28
// and 97 us.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "op_args.h"
#include "op_moves.h"

namespace gemel {

namespace {

typedef __attribute__((address_space(3))) unsigned char lds_u8;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf_up(u16 h) { return __uint_as_float((uint32_t)h << 16); }
__device__ __forceinline__ u16 bf_down(float f) { return __builtin_bit_cast(u16, (__bf16)f); }

template <int N>
__device__ __forceinline__ void wait_vm() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}
// The loads of a step have landed in every wave, and every wave has its last
// fragments in registers: the buffer they came from may be refilled. (Their
// products do not touch memory, so only the wait keeps the reads before the
// barrier.)
template <int N>
__device__ __forceinline__ void turn() {
    __builtin_amdgcn_s_waitcnt(0xF | (0x3 << 14) | (0x7 << 4));   // LDS reads
    wait_vm<N>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// The matrix-core product of two 16-byte chunks a lane holds: 8 bf16 (32
// depths over the 4 lane groups) or 4 float32 (16 depths; element e of every
// chunk is one product of 4 depths, in an order that both operands share).
template <bool F32>
__device__ __forceinline__ f32x4 mul(const uint4 &a, const uint4 &b, f32x4 c) {
    if constexpr (F32) {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
        return c;
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                       0);
    }
}

// Bytes [at, at + 16) of a row of `end` bytes; what lies beyond is zero.
template <bool F32>
__device__ __forceinline__ uint4 chunk(const char *row, int at, int end) {
    if (at + 16 <= end) return get_16b(row + at);
    union {
        uint4 v;
        u16 h[8];
        uint32_t w[4];
    } r;
    if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = at + 4 * i < end ? *(const uint32_t *)(row + at + 4 * i) : 0u;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.h[i] = at + 2 * i < end ? *(const u16 *)(row + at + 2 * i) : (u16)0;
    }
    return r.v;
}

constexpr int ROW = ROWS_STEP;   // bytes of a row in a step
constexpr int RING = 4;

// Thin sums of item blockIdx / (rank blocks * slices): 4 waves share the slice.
template <bool F32>
__device__ __forceinline__ void thin(const RowsArgs &a, int block, f32x4 *part) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, l16 = lane & 15;
    const int slice = block % a.thin_slices, rest = block / a.thin_slices;
    const int rb = rest % a.rank_blocks, item = rest / a.rank_blocks;
    const int *it = a.b.items + 3 * item;
    const int u = it[0], p0 = it[1], n = it[2], rank = a.b.run_rank[u];
    const int elem = F32 ? 4 : 2, end = a.k_bank * elem;
    const char *x = (const char *)a.x + (int64_t)a.b.perm[p0 + min(l16, n - 1)] * a.ldx * elem;
    const int r = rb * 16 + l16;
    const bool used = r < rank;
    const char *w = (const char *)a.a + ((int64_t)a.b.run_id[u] * a.b.rank + (used ? r : 0)) * a.k_bank * elem;
    const int k0 = slice * a.thin_bytes, k1 = min(end, k0 + a.thin_bytes);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (rb * 16 < rank) {
        int k = k0 + wave * 64;   // (the wave's; its lane groups take 16 bytes each)
        // whole chunks, eight of each operand in flight: no branch may stand
        // between the loads
        for (; k + 7 * 256 + 64 <= k1; k += 8 * 256) {
            uint4 xv[8], wv[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                xv[q] = get_16b(x + k + q * 256 + g * 16);
                wv[q] = get_16b(w + k + q * 256 + g * 16);
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) acc = mul<F32>(used ? wv[q] : uint4{}, xv[q], acc);
        }
        for (; k < k1; k += 256) {
            const uint4 xv = chunk<F32>(x, k + g * 16, k1);
            const uint4 wv = chunk<F32>(w, k + g * 16, used ? k1 : 0);
            acc = mul<F32>(wv, xv, acc);
        }
    }
    part[wave * 64 + lane] = acc;
    __syncthreads();
    if (wave) return;
    for (int i = 1; i < 4; ++i) acc += part[i * 64 + lane];
    if (l16 < n)
        *(f32x4 *)(a.t + ((int64_t)slice * a.b.rows + p0 + l16) * a.rank_blocks * 16 + rb * 16 + 4 * g) =
            acc * a.b.run_scale[u];
}

// MB blocks of 16 rows.
template <bool F32, int MB>
__global__ __launch_bounds__(256) void rows_kernel(const RowsArgs a) {
    constexpr int STAGE = (64 + 16 * MB) * ROW, LOADS = 2 + (MB + 1) / 2;
    __shared__ __attribute__((aligned(1024))) unsigned char r0[STAGE + (MB & 1) * 16 * ROW], r1[STAGE + (MB & 1) * 16 * ROW],
        r2[STAGE + (MB & 1) * 16 * ROW], r3[STAGE + (MB & 1) * 16 * ROW];
    if ((int)blockIdx.x < a.thin_blocks) {
        thin<F32>(a, blockIdx.x, (f32x4 *)r0);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, l16 = lane & 15;
    const int block = blockIdx.x - a.thin_blocks, tiles = (a.N + 63) / 64;
    const int slice = block / tiles, n0 = (block - slice * tiles) * 64;
    const int elem = F32 ? 4 : 2;
    const int s0 = slice * a.steps, s1 = min(a.all_steps, s0 + a.steps);
    // load i of a thread fills slot i * 256 + tid of a buffer: row slot / 8
    // (64 weight rows, then the inputs; rows beyond the last repeat it),
    // whose position slot % 8 holds chunk (slot % 8) ^ (row / 2 % 8)
    const char *src[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int row = (i * 256 + tid) >> 3, ch = ((tid & 7) ^ ((row >> 1) & 7)) * 16;
        const int m = min(max(row - 64, 0), a.b.rows - 1);
        src[i] = i < 2 ? (const char *)a.w + (int64_t)min(n0 + row, a.N - 1) * a.ldw * elem + ch
                       : (const char *)a.x + (int64_t)m * a.ldx * elem + ch;
    }
    const int end = a.K * elem;
    int at = s0;
    auto issue = [&](unsigned char *buf) __attribute__((always_inline)) {
        // past the last step its chunks again, so that every step waits alike
        const int k = min(at, s1 - 1) * ROW;
        ++at;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int row = (i * 256 + tid) >> 3, ch = ((tid & 7) ^ ((row >> 1) & 7)) * 16;
            __builtin_amdgcn_global_load_lds(k + ch < end ? (const void *)(src[i] + k) : (const void *)a.zero,
                                             (lds_u8 *)(buf + (i * 4 + wave) * 1024), 16, 0, 0);
        }
    };
    f32x4 acc[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    unsigned char *const ring[RING] = {r0, r1, r2, r3};
#pragma unroll
    for (int i = 0; i < RING - 1; ++i) issue(ring[i]);
    const int sw = (l16 >> 1) & 7;
    auto step = [&](const unsigned char *cur, unsigned char *next) __attribute__((always_inline)) {
        turn<(RING - 2) * LOADS>();
        issue(next);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = ((h * 4 + g) ^ sw) * 16;
            const uint4 wv = *(const uint4 *)(cur + (wave * 16 + l16) * ROW + c);
#pragma unroll
            for (int i = 0; i < MB; ++i) acc[i] = mul<F32>(wv, *(const uint4 *)(cur + (64 + i * 16 + l16) * ROW + c), acc[i]);
        }
    };
    // the slices are whole rings of steps (the last may run past its end,
    // whose weights are then not multiplied)
    int s = s0;
    for (; s + RING <= s1; s += RING) {
        step(r0, r3);
        step(r1, r0);
        step(r2, r1);
        step(r3, r2);
    }
    if (s < s1) step(r0, r3);
    if (s + 1 < s1) step(r1, r0);
    if (s + 2 < s1) step(r2, r1);
    wait_vm<0>();
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int m = i * 16 + l16, n = n0 + wave * 16 + g * 4;
        if (m < a.b.rows && n < a.ldp) *(f32x4 *)(a.partial + ((int64_t)slice * a.b.rows + m) * a.ldp + n) = acc[i];
    }
}

// One row and 512 columns per workgroup. A chain of dependent loads is all
// that a short launch takes, so what a row needs of the tables lies together,
// and the slices are requested before it arrives.
template <bool F32>
__global__ __launch_bounds__(128) void rows_sum_kernel(const RowsArgs a) {
    __shared__ float ts[256];
    const int row = blockIdx.y, tid = threadIdx.x;
    const int4 info = a.b.row_info[row];   // position, run or -1, adapter, rank
    const int n = (blockIdx.x * 128 + tid) * 4;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (n < a.N) {
        const float *part = a.partial + (int64_t)row * a.ldp + n;
#pragma unroll 8
        for (int k = 0; k < a.slices; ++k) v += *(const f32x4 *)(part + (int64_t)k * a.b.rows * a.ldp);
    }
    const int u = info.y, rank = u < 0 ? 0 : info.w;
    for (int r = tid; r < rank; r += 128) {
        const float *t = a.t + (int64_t)info.x * a.rank_blocks * 16 + r;
        float x = 0.f;
#pragma unroll 4
        for (int k = 0; k < a.thin_slices; ++k) x += t[(int64_t)k * a.b.rows * a.rank_blocks * 16];
        ts[r] = x;
    }
    __syncthreads();
    if (n >= a.N) return;
    if (u >= 0) {
        const int R = a.b.rank, elem = F32 ? 4 : 2;
        const char *b = (const char *)a.bank_b + ((int64_t)info.z * a.N + n) * R * elem;
        const int left = min(4, a.N - n);
        constexpr int Q = F32 ? 4 : 8;
        const bool whole = left == 4 && rank % Q == 0;
#pragma unroll 2
        for (int r = 0; r < rank; r += Q) {
            uint4 q[4];
            if (whole) {
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = get_16b(b + ((int64_t)i * R + r) * elem);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    q[i] = i < left ? chunk<F32>(b + (int64_t)i * R * elem, r * elem, rank * elem) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < Q; ++j) {
                const float t = r + j < rank ? ts[r + j] : 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t w = (&q[i].x)[F32 ? j : j / 2];
                    v[i] += t * (F32 ? __uint_as_float(w) : bf_up((u16)(j % 2 ? w >> 16 : w & 0xffff)));
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (a.bias && n + i < a.N) v[i] += a.bias[n + i];
    const int64_t at = (int64_t)row * a.ldy + n;
    if constexpr (F32) {
        float *y = (float *)a.y + at;
        if (n + 3 < a.N) {
            put_f32x4(y, v);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i < a.N) y[i] = v[i];
        }
    } else {
        u16 *y = (u16 *)a.y + at;
        if (n + 3 < a.N) {
            put_u16x4(y, make_ushort4(bf_down(v[0]), bf_down(v[1]), bf_down(v[2]), bf_down(v[3])));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i < a.N) y[i] = bf_down(v[i]);
        }
    }
}

template <bool F32>
hipError_t go(const RowsArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)(a.thin_blocks + (a.N + 63) / 64 * a.slices));
    void *p[] = {const_cast<RowsArgs *>(&a)};
    const void *fn = nullptr;
    switch ((a.b.rows + 15) / 16) {
        case 1: fn = reinterpret_cast<const void *>(&rows_kernel<F32, 1>); break;
        case 2: fn = reinterpret_cast<const void *>(&rows_kernel<F32, 2>); break;
        case 3: fn = reinterpret_cast<const void *>(&rows_kernel<F32, 3>); break;
        case 4: fn = reinterpret_cast<const void *>(&rows_kernel<F32, 4>); break;
        default: return hipErrorInvalidValue;
    }
    const hipError_t e = hipLaunchKernel(fn, grid, dim3(256), p, 0, s);
    if (e != hipSuccess) return e;
    return hipLaunchKernel(reinterpret_cast<const void *>(&rows_sum_kernel<F32>),
                           dim3((unsigned)((a.N + 511) / 512), (unsigned)a.b.rows), dim3(128), p, 0, s);
}

}  // namespace

hipError_t launch_rows(const RowsArgs &a, hipStream_t s) {
    if (!rows_valid(a)) return hipErrorInvalidValue;
    return a.f32 ? go<true>(a, s) : go<false>(a, s);
}

}  // namespace gemel

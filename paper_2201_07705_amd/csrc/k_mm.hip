// Products of 16-bit matrices with float32 sums: C[m][n] = sum over k of
// A[m][k] * B[n][k], both operands rows of contiguous elements.
#include <hip/hip_runtime.h>

#include <climits>
#include <type_traits>

#include "op_args.h"
#include "op_moves.h"

namespace gemel {

namespace {

typedef __attribute__((address_space(3))) unsigned char lds_u8;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int BK = MM_BK;

template <int N>
__device__ __forceinline__ void wait_vm() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

__device__ __forceinline__ void wait_lgkm0() { __builtin_amdgcn_s_waitcnt(0xF | (0x3 << 14) | (0x7 << 4)); }

__device__ __forceinline__ u16 to_bf16(float f) { return __builtin_bit_cast(u16, (__bf16)f); }
__device__ __forceinline__ float half_up(u16 h) { return (float)__builtin_bit_cast(_Float16, h); }
__device__ __forceinline__ u16 to_half(float f) { return __builtin_bit_cast(u16, (_Float16)f); }

__device__ __forceinline__ f32x4 half_up4(ushort4 h) {
    return f32x4{half_up(h.x), half_up(h.y), half_up(h.z), half_up(h.w)};
}
__device__ __forceinline__ f32x4 rest4(f32x4 v) {
    return f32x4{v[0] - half_up(to_half(v[0])), v[1] - half_up(to_half(v[1])), v[2] - half_up(to_half(v[2])),
                 v[3] - half_up(to_half(v[3]))};
}

// Where an epilogue works: the first element of the tile, and whether the
// whole tile lies inside the result: then addresses are a uniform base and a
// 32-bit offset, and nothing is clamped or masked.
struct Tile {
    int z, m0, n0;
    bool inside;
};
// The byte offset of element (m, n) of the tile in a matrix of `bytes` each.
__device__ __forceinline__ uint32_t offset_of(int m, int n, int64_t ld, int bytes) {
    return ((uint32_t)m * (uint32_t)ld + (uint32_t)n) * (uint32_t)bytes;
}
template <typename P>
__device__ __forceinline__ P *at_tile(P *p, const Tile &t, int64_t z, int64_t ld) {
    return p + (int64_t)t.z * z + (int64_t)t.m0 * ld + t.n0;
}
template <typename V>
__device__ __forceinline__ V load_at(const void *base, uint32_t off) {
    return *(const V *)((const char *)base + off);
}
template <typename V>
__device__ __forceinline__ void store_at(void *base, uint32_t off, V v) {
    *(V *)((char *)base + off) = v;
}
// The same of planes (tiles begin at multiples of 32).
__device__ __forceinline__ uint32_t offset_of(int m, int n, const Planes &p) {
    return offset_of(m, p.pair ? pair_at(n) : n, p.ld, 2);
}
__device__ __forceinline__ u16 *at_tile(u16 *plane, const Tile &t, const Planes &p) {
    return plane + (int64_t)t.z * p.z + (int64_t)t.m0 * p.ld + ((int64_t)t.n0 << p.pair);
}
__device__ __forceinline__ int width(const Planes &p) { return (int)(p.ld >> p.pair); }
// Elements (m, n .. n + 3) of the tile of a matrix in planes; rows are padded
// to 64, so 4 elements stay in a row, and rows beyond the last one read it.
__device__ __forceinline__ void at4(const Planes &p, const Tile &t, int m, int n, int rows, f32x4 &hi, f32x4 &lo) {
    lo = f32x4{0.f, 0.f, 0.f, 0.f};
    if (t.inside) {
        const uint32_t off = offset_of(m, n, p);
        hi = half_up4(load_at<ushort4>(at_tile(p.hi, t, p), off));
        if (p.lo) lo = half_up4(load_at<ushort4>(at_tile(p.lo, t, p), off));
    } else {
        const int c = min(t.n0 + n, width(p) - 4);
        const int64_t at = (int64_t)t.z * p.z + (int64_t)min(t.m0 + m, rows - 1) * p.ld + (p.pair ? pair_at(c) : c);
        hi = half_up4(*(const ushort4 *)(p.hi + at));
        if (p.lo) lo = half_up4(*(const ushort4 *)(p.lo + at));
    }
}

// Values of a matrix kept as float16 planes, as pairs: the nearest half, and
// above it the rest of the value in a second half (22 bits together).
__device__ __forceinline__ uint4 pairs(f32x4 v) {
    uint4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u16 h = to_half(v[i]);
        (&r.x)[i] = h | (uint32_t)to_half(v[i] - half_up(h)) << 16;
    }
    return r;
}
__device__ __forceinline__ void put_pairs(u16 *hi, u16 *lo, uint32_t off, uint4 v) {
    store_at(hi, off, make_uint2(__builtin_amdgcn_perm(v.y, v.x, 0x05040100), __builtin_amdgcn_perm(v.w, v.z, 0x05040100)));
    if (lo)
        store_at(lo, off, make_uint2(__builtin_amdgcn_perm(v.y, v.x, 0x07060302), __builtin_amdgcn_perm(v.w, v.z, 0x07060302)));
}

// One operand's loads of a step: 16 bytes at base + off[i] into the wave's
// slots. A buffer resource keeps the base in scalar registers; every
// offset is in bounds, so its own check is not used.
template <int LOADS, int NW>
__device__ __forceinline__ void fetch(const u16 *base, const uint32_t (&off)[LOADS], unsigned char *stage, int wave) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<u16 *>(base), 0, -1, 0x00020000);
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_u8 *)(stage + (i * NW + wave) * 1024), 16, (int)off[i], 0, 0, 0);
}

// The kernel's argument block where the hardware keeps it.
__device__ __forceinline__ const MmArgs *late_args(const MmArgs &) {
    auto *p = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return (const MmArgs *)p;
}

// Brings the argument block into the scalar cache with the first loads of the
// kernel: its later part would otherwise be fetched, from host memory, only
// when the epilogue asks for it.
__device__ __forceinline__ void touch_args() {
    typedef const __attribute__((address_space(4))) int *args_t;
    const args_t p = (args_t)__builtin_amdgcn_kernarg_segment_ptr();
    int x = 0;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(MmArgs) / 4); i += 16) x |= p[i];
    asm volatile("" ::"s"(x));
}

// Tile of a workgroup: consecutive tiles on one XCD, and among them groups
// of 8 tile rows, whose operand rows then stay in its L2. Symmetric results:
// only tiles on and above the diagonal exist, row i of them paired with row
// last - i, so that each pair has as many.
template <int T>
__device__ __forceinline__ void mm_place(const MmArgs &a, int &tm, int &tn) {
    // (32: the reduction's, which covers the planes' padding to 64)
    const int tiles_m = T < 64 ? (a.M + 63) / 64 * (64 / T) : (a.M + T - 1) / T;
    const int tiles_n = T < 64 ? (a.N + 63) / 64 * (64 / T) : (a.N + T - 1) / T;
    const int G = gridDim.x;
    const int t = (G & 7) == 0 ? (int)(blockIdx.x & 7) * (G >> 3) + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
    if (a.sym) {
        const int pair = t / (tiles_n + 1), c = t - pair * (tiles_n + 1), first = tiles_n - pair;
        tm = c < first ? pair : tiles_n - 1 - pair;
        tn = tm + (c < first ? c : c - first);
        return;
    }
    const int group = t / (8 * tiles_n), first = group * 8, rows = min(8, tiles_m - first);
    const int in = t - group * 8 * tiles_n;
    tn = in / rows;
    tm = first + in - tn * rows;
}

// What the epilogue of elements (m, n .. n + 3) of the tile reads, gathered
// before any of a group's results are stored.
struct Near {
    f32x4 hi, lo;   // a matrix in planes (MIX: lo is the second matrix)
    f32x4 w;        // a diagonal, the weights, or the bias
    float d;        // POLY: the diagonal at m
    int row;        // ROWS, SCALED: output row
    int e, u;       // SCALED: its exponent, and its run or -1
    int eb[4];      // SCALED: exponents of the columns
};
template <int EPI>
__device__ __forceinline__ Near gather(const MmArgs &a, const Tile &t, int m, int n) {
    const MmOut &o = a.o;
    Near r;
    if constexpr (EPI == EPI_ROWS || EPI == EPI_SCALED) {
        const int mc = min(t.m0 + m, a.M - 1);
        r.row = o.perm ? o.perm[mc] : mc;
        r.w = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (EPI == EPI_SCALED) {
            r.e = o.ea[mc];
            r.u = a.runs > 0 ? o.run_at[mc] : -1;
            if (t.inside) {
                const uint4 x = get_16b(o.eb + t.n0 + n);
#pragma unroll
                for (int i = 0; i < 4; ++i) r.eb[i] = (int)(&x.x)[i];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) r.eb[i] = o.eb[min(t.n0 + n + i, a.N - 1)];
            }
        }
        if (o.bias && t.inside) {
            r.w = get_f32x4<f32x4>(o.bias + t.n0 + n);
        } else if (o.bias) {
#pragma unroll
            for (int i = 0; i < 4; ++i) r.w[i] = o.bias[min(t.n0 + n + i, a.N - 1)];
        }
    } else if constexpr (EPI == EPI_POLY) {
        at4(o.s, t, m, n, a.M, r.hi, r.lo);
        if (o.sdiag) {
            const float *d = o.sdiag + t.z * o.diag_z;
            r.w = *(const f32x4 *)(d + min(t.n0 + n, (int)o.diag_z - 4));
            r.d = d[min(t.m0 + m, a.M - 1)];
        }
    } else if constexpr (EPI == EPI_MIX) {
        f32x4 lo;
        at4(o.s2, t, m, n, a.M, r.lo, lo);
        r.lo += lo;
        at4(o.s, t, m, n, a.M, r.hi, lo);
        r.hi += lo;
    } else if constexpr (EPI != EPI_GRAM) {
        at4(o.s, t, m, n, a.M, r.hi, r.lo);
        if constexpr (EPI == EPI_STEP) {
            if (t.inside) {
                r.w = load_at<f32x4_any>(at_tile((const float *)o.out, t, o.z, o.ld), offset_of(m, n, o.ld, 4));
            } else {
                const float *w = (const float *)o.out + (int64_t)t.z * o.z + (int64_t)min(t.m0 + m, a.M - 1) * o.ld;
#pragma unroll
                for (int i = 0; i < 4; ++i) r.w[i] = w[min(t.n0 + n + i, a.N - 1)];
            }
        } else if (o.mdiag) {
            const float *d = o.mdiag + t.z * o.diag_z;
            if (o.diag_rows) {
                const float x = d[min(t.m0 + m, a.M - 1)];
                r.w = f32x4{x, x, x, x};
            } else {
                r.w = *(const f32x4 *)(d + min(t.n0 + n, (int)o.diag_z - 4));
            }
        }
    }
    return r;
}

// SCALED: the low-rank part of G pieces (m, n .. n + 3), added to what
// finish adds. No branch stands between the loads: rows without a run read
// the first one's and drop it.
template <int G>
__device__ __forceinline__ void low_rank(const MmArgs &a, const Tile &t, const int (&m)[G], const int (&n)[G], Near (&near)[G]) {
    const MmOut &o = a.o;
    if (a.runs <= 0) return;
    f32x4 sum[G];
#pragma unroll
    for (int g = 0; g < G; ++g) sum[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int r = 0; r < o.rank; r += 4) {   // (zeros from a run's rank on)
        f32x4 x[G], b[G][4];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            x[g] = *(const f32x4 *)(o.t + (int64_t)min(t.m0 + m[g], a.M - 1) * o.rp + r);
            const float *bx = o.bx + ((int64_t)max(near[g].u, 0) * o.rp + r) * o.ldbx + min((int64_t)t.n0 + n[g], o.ldbx - 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) b[g][i] = *(const f32x4 *)(bx + i * o.ldbx);
        }
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[g] += x[g][i] * b[g][i];
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const f32x4 w = near[g].w + sum[g];
#pragma unroll
        for (int i = 0; i < 4; ++i) near[g].w[i] = near[g].u < 0 ? near[g].w[i] : w[i];
    }
}

// The epilogue of elements (m, n .. n + 3) of the tile. M and N are the
// product's; planes are written up to their padded row lengths, with zeros
// beyond M and N, because later products read them in steps of 64. Returns
// the plane pairs.
template <int EPI>
__device__ __forceinline__ uint4 finish(const MmArgs &a, const Tile &t, int m, int n, f32x4 v, const Near &in) {
    const MmOut &o = a.o;
    const int left = a.N - t.n0 - n;                   // elements of the row from n on
    const bool there = t.inside || (t.m0 + m < a.M && left > 0);
    // cs X + cv v in X's plane units (a X + M X, v being the product of the
    // planes). Where M is a single plane, what its diagonal (most of M once X
    // is nearly orthogonal) and X have lost to rounding is put back.
    if constexpr (EPI == EPI_NEXT || EPI == EPI_ORTH || EPI == EPI_STEP) {
        v = o.cs * (in.hi + in.lo) + o.cv * v;
        if constexpr (EPI != EPI_STEP)
            if (o.mdiag) v += 0x1p-14f * (rest4(in.w) * in.hi + in.w * in.lo);
    }
    if constexpr (EPI == EPI_ROWS || EPI == EPI_SCALED) {
        if (!there) return uint4{};
        const int64_t at = (int64_t)in.row * o.ld + t.n0 + n;
        if constexpr (EPI == EPI_SCALED) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = ldexpf(v[i], -(in.e + in.eb[i]));
        }
        v += in.w;
        if (o.out_f32) {
            float *p = (float *)o.out + at;
            if (left > 3) {
                put_f32x4(p, v);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < left) p[i] = v[i];
            }
        } else {
            u16 *p = (u16 *)o.out + at;
            if (left > 3) {
                put_u16x4(p, make_ushort4(to_bf16(v[0]), to_bf16(v[1]), to_bf16(v[2]), to_bf16(v[3])));
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < left) p[i] = to_bf16(v[i]);
            }
        }
        return uint4{};
    } else if constexpr (EPI == EPI_ORTH || EPI == EPI_STEP) {
        if (!there) return uint4{};
        f32x4 x = o.lambda[t.z * ORTH_LAMBDAS] * 0x1p-13f * v;
        if constexpr (EPI == EPI_STEP) x = (1.f - o.decay) * in.w - o.rate * x;
        const bool wide = EPI == EPI_STEP || o.out_f32;
        u16 *const h = EPI == EPI_STEP ? o.copy : wide ? nullptr : (u16 *)o.out;
        if (left > 3) {
            if (wide) store_at(at_tile((float *)o.out, t, o.z, o.ld), offset_of(m, n, o.ld, 4), (f32x4_any)x);
            if (h)
                store_at(at_tile(h, t, o.z, o.ld), offset_of(m, n, o.ld, 2),
                         u16x4_any{to_bf16(x[0]), to_bf16(x[1]), to_bf16(x[2]), to_bf16(x[3])});
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= left) continue;
                if (wide) store_at(at_tile((float *)o.out, t, o.z, o.ld), offset_of(m, n + i, o.ld, 4), x[i]);
                if (h) store_at(at_tile(h, t, o.z, o.ld), offset_of(m, n + i, o.ld, 2), to_bf16(x[i]));
            }
        }
        return uint4{};
    } else {
        const Planes &p = o.p;
        f32x4 x;
        if constexpr (EPI == EPI_GRAM) {
            x = v * 0x1p-15f;
        } else if constexpr (EPI == EPI_POLY) {
            const float l = o.lambda[t.z * ORTH_LAMBDAS], l2 = l * l;
            f32x4 s = in.hi;
            if (o.sdiag) {
                // S is its plane but for the diagonal
                v += (in.d - half_up(to_half(in.d)) + rest4(in.w)) * s;
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = t.m0 + m == t.n0 + n + i ? in.d : s[i];
            } else {
                s += in.lo;
            }
            x = 0x1p14f * (float)COEF_B * 0x1p-11f * l2 * s + 0x1p14f * (float)COEF_C * 0x1p-22f * l2 * l2 * v;
        } else if constexpr (EPI == EPI_MIX) {
            x = o.cs * in.hi + o.cs2 * in.lo + o.cv * v;
            if (o.lambdas) {
                const float *l = o.lambda + t.z * ORTH_LAMBDAS, f = l[0] / l[o.lambdas];
                x *= f * f;
            }
        } else {
            const float *l = o.lambda + t.z * ORTH_LAMBDAS;
            x = l[0] / l[o.lambdas] * v;
        }
        if (!t.inside)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = t.m0 + m < a.M && i < left ? x[i] : 0.f;
        if constexpr (EPI == EPI_GRAM || EPI == EPI_POLY) {
            float *const d = EPI == EPI_GRAM ? o.sdiag : o.mdiag;
            const int i = t.m0 + m - t.n0 - n;
            if (d && i >= 0 && i < 4 && t.m0 + m < a.M) d[t.z * o.diag_z + t.m0 + m] = i == 0 ? x[0] : i == 1 ? x[1] : i == 2 ? x[2] : x[3];
        }
        const uint4 q = pairs(x);
        if (t.inside || (t.m0 + m < a.M && t.n0 + n < width(p)))
            put_pairs(at_tile(p.hi, t, p), p.lo ? at_tile(p.lo, t, p) : nullptr, offset_of(m, n, p), q);
        return q;
    }
}

// One T x T output tile per workgroup: 8 waves of 128 x 64 (T = 256) or 32 x
// 64 (T = 128, two workgroups on a compute unit), or 4 of 32 x 32 (T = 64).
// A step of depth 64 is fetched by direct global-to-LDS loads into one of
// STAGES buffers (separate arrays, so that the compiler sees which buffer a
// load in flight writes), a buffer being asked for again as soon as its last
// fragments are in registers. Slot p of a buffer holds row p / 8, 16-byte
// chunk (p % 8) ^ (row / 2 % 8): the fragment reads of 16 rows then fall on
// distinct banks. A step is PHASES pieces, each reading the next one's
// fragments, so that the matrix cores wait for LDS only across the one
// barrier of a step, and there the fragments read before it cover the others.
// Large tiles have no registers for more than a quarter step (256) or half a
// step (128) in hand; small ones take a whole one and four buffers, which is
// what latency wants.
//
// Pairs: 32 columns of hi and of lo are a step, so that its three products
// take four tiles through LDS where three plain steps of the same depth would
// take six (2048 x 1000 of 1024 pairs 27.6 -> 22.4 us).
//
// What bounds it: the matrix cores at T = 256 and 128 (25088 x 4096 of 4096
// pairs, with the update of X in both layouts: 2128 and 2113 us, 1195
// TFLOP/s of float16 products), the CU's 64 bytes a cycle from the L2 at T =
// 64 (2746 us). Below 512 tiles of 64 what a compute unit does alone counts:
// 2048 x 1000 of 1024 pairs 22.4 us at T = 64, 33.2 at 128, 95.5 at 256.
template <int T>
constexpr int mm_threads() { return mm_threads_of(T); }

template <int T, int STAGES, int PHASES, bool F16, bool PAIR, int EPI>
__global__ __launch_bounds__((mm_threads<T>()), T == 256 ? 1 : T == 128 ? 4 : 2) void mm_kernel(const MmArgs a) {
    constexpr int NT = mm_threads<T>(), NW = NT / 64, WN = T == 256 ? 4 : 2;
    constexpr int TM = T * WN / NW, TN = T / WN, FM = TM / 16, FN = TN / 16;
    constexpr int LOADS = T * 8 / NT, ROW = BK * 2;
    __shared__ __attribute__((aligned(1024))) unsigned char st0[2 * T * ROW], st1[2 * T * ROW],
        st2[STAGES > 2 ? 2 * T * ROW : 16], st3[STAGES > 3 ? 2 * T * ROW : 16];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave - wm * WN, g = lane >> 4, l16 = lane & 15;
    touch_args();
    int tm, tn;
    mm_place<T>(a, tm, tn);
    const int split = blockIdx.y, z = blockIdx.z;
    const int m0 = tm * T, n0 = tn * T;
    const int nk = (a.K + BK - 1) / BK;
    const int s0 = split * a.steps, mains = min(nk - s0, a.steps);
    // extension steps: the runs that overlap the tile's rows, in the last split
    int u = 0, ek = 0, exts = 0;
    if (EPI == EPI_ROWS && a.ext && split == a.splits - 1) {
        u = a.first_run[m0 >> 6];
        int e = u;
        while (e < a.runs && a.run_start[e] < min(m0 + T, a.M)) ++e;
        exts = (e - u) * (a.ext / BK);
    }
    const int total = mains + exts;

    // load i of a thread fills slot i * NT + tid; byte offsets from the
    // tile's first row (or, with a row table, from the matrix)
    uint32_t oa[LOADS], ob[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int row = (i * NT + tid) >> 3, ch = ((tid & 7) ^ ((row >> 1) & 7)) * 8;
        const int m = min(m0 + row, a.M - 1), n = min(n0 + row, a.N - 1);
        oa[i] = (uint32_t)((a.perm ? a.perm[m] : m - m0) * (uint32_t)a.lda + ch) * 2u;
        ob[i] = (uint32_t)((n - n0) * (uint32_t)a.ldb + ch) * 2u;
    }
    const int64_t za = (int64_t)z * a.za + (a.perm ? 0 : (int64_t)m0 * a.lda), zb = (int64_t)z * a.zb + (int64_t)n0 * a.ldb;
    // the next step's operands
    int iss = 0;
    const u16 *pa = a.a + za + s0 * BK, *pb = a.b + zb + s0 * BK;
    // Requests the next step; past the last one, the last one again (into a
    // buffer whose reads are over), so that every step waits alike.
    auto issue = [&](unsigned char *stage) __attribute__((always_inline)) {
        const bool ext = EPI == EPI_ROWS && exts > 0 && iss >= mains;
        const int kk = (s0 + min(iss, mains - 1)) * BK;
        if (EPI == EPI_ROWS && (ext || kk + BK > a.K)) {
            // rows of other runs, and chunks beyond a depth that is no
            // multiple of 64, are zeros
            const u16 *qa = pa, *qb = pb;
            int lo = 0, hi = INT_MAX;
            if (ext) {
                qa = a.t + (int64_t)m0 * a.ext + ek;
                qb = a.bx + ((int64_t)u * a.N + n0) * a.ext + ek;
                lo = a.run_start[u];
                hi = a.run_start[u + 1];
            }
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int row = (i * NT + tid) >> 3, ch = ((tid & 7) ^ ((row >> 1) & 7)) * 8;
                const bool in = ext ? m0 + row >= lo && m0 + row < hi : kk + ch < a.K;
                const uint32_t xa = ext ? (uint32_t)(row * a.ext + ch) * 2u : oa[i];
                const uint32_t xb = ext ? (uint32_t)((min(n0 + row, a.N - 1) - n0) * a.ext + ch) * 2u : ob[i];
                __builtin_amdgcn_global_load_lds(in ? (const void *)((const char *)qa + xa) : (const void *)a.zero,
                                                 (lds_u8 *)(stage + (i * NW + wave) * 1024), 16, 0, 0);
                __builtin_amdgcn_global_load_lds(ext || in ? (const void *)((const char *)qb + xb) : (const void *)a.zero,
                                                 (lds_u8 *)(stage + T * ROW + (i * NW + wave) * 1024), 16, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (ext && iss + 1 < total) {
                ek += BK;
                if (ek >= a.ext) {
                    ek = 0;
                    ++u;
                }
            }
        } else {
            fetch<LOADS, NW>(pa, oa, stage, wave);
            fetch<LOADS, NW>(pb, ob, stage + T * ROW, wave);
        }
        iss = min(iss + 1, total);
        if (iss < mains) {
            pa += BK;
            pb += BK;
        }
    };
    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    using H8 = std::conditional_t<F16, f16x8, bf16x8>;
    // fragments: of a quarter (depth half, row half), a half or a whole step,
    // and the next one's
    constexpr int NA = PHASES == 4 ? FM / 2 : PHASES == 2 ? FM : 2 * FM, NB = PHASES == 1 ? 2 * FN : FN;
    H8 fa0[NA], fa1[NA], fb0[NB], fb1[NB];
    // rows 16 apart share their swizzle: one address per depth half
    const int ra = (wm * TM + l16) * ROW, rb = T * ROW + (wn * TN + l16) * ROW;
    const int h0 = (g ^ ((l16 >> 1) & 7)) * 16, h1 = ((4 + g) ^ ((l16 >> 1) & 7)) * 16;
    auto read_a = [&](H8(&f)[NA], const unsigned char *s, int h, int row) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NA; ++i)
            f[i] = *(const H8 *)(s + ra + (PHASES == 1 && i >= FM ? h1 : h) + (row + i % FM) * 16 * ROW);
    };
    auto read_b = [&](H8(&f)[NB], const unsigned char *s, int h) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NB; ++j) f[j] = *(const H8 *)(s + rb + (PHASES == 1 && j >= FN ? h1 : h) + j % FN * 16 * ROW);
    };
    auto mul = [&](H8(&f)[NA], H8(&b)[NB], int row) __attribute__((always_inline)) {
        // a whole step: both halves of the depth, or hi lo, lo hi and hi hi
        constexpr int PRODUCTS = PHASES > 1 ? 1 : PAIR ? 3 : 2, ROWS = PHASES > 1 ? NA : FM;
#pragma unroll
        for (int q = 0; q < PRODUCTS; ++q) {
            const int ha = PAIR ? q == 1 : q, hb = PAIR ? PHASES == 1 && q == 0 : q;
#pragma unroll
            for (int i = 0; i < ROWS; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    f32x4 &c = acc[row + i][j];
                    const H8 &x = f[ha * FM + i], &y = b[hb * FN + j];
                    if constexpr (F16)
                        c = __builtin_amdgcn_mfma_f32_16x16x32_f16(y, x, c, 0, 0, 0);
                    else
                        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, x, c, 0, 0, 0);
                }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // the loads of the step after `cur`'s have landed in every wave, and
    // every wave has read the last of `cur`
    auto turn = [&]() __attribute__((always_inline)) {
        wait_lgkm0();
        wait_vm<(STAGES - 2) * 2 * LOADS>();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    // one step; set: which fragments hold the whole step (PHASES == 1), or
    // b's hi (pairs)
    auto paired = [&](unsigned char *cur, unsigned char *next, H8(&bh)[NB], H8(&bl)[NB]) __attribute__((always_inline)) {
        if constexpr (PHASES == 4) {
            read_a(fa1, cur, h1, 0);
            read_b(bl, cur, h1);
            mul(fa0, bh, 0);
            mul(fa0, bl, 0);
            read_a(fa0, cur, h0, NA);
            mul(fa1, bh, 0);
            read_a(fa1, cur, h1, NA);
            mul(fa0, bh, NA);
            mul(fa0, bl, NA);
            turn();
            issue(cur);
            read_a(fa0, next, h0, 0);
            read_b(bl, next, h0);
            mul(fa1, bh, NA);
        } else {
            read_a(fa1, cur, h1, 0);
            read_b(bl, cur, h1);
            mul(fa0, bh, 0);
            mul(fa0, bl, 0);
            turn();
            issue(cur);
            read_a(fa0, next, h0, 0);
            read_b(bl, next, h0);
            mul(fa1, bh, 0);
        }
    };
    auto step = [&](unsigned char *cur, unsigned char *next, int set) __attribute__((always_inline)) {
        if constexpr (PAIR && PHASES > 1) {
            if (set)
                paired(cur, next, fb1, fb0);
            else
                paired(cur, next, fb0, fb1);
        } else if constexpr (PHASES == 4) {
            read_a(fa1, cur, h0, NA);
            mul(fa0, fb0, 0);
            read_a(fa0, cur, h1, 0);
            read_b(fb1, cur, h1);
            mul(fa1, fb0, NA);
            read_a(fa1, cur, h1, NA);
            mul(fa0, fb1, 0);
            turn();
            issue(cur);
            read_a(fa0, next, h0, 0);
            read_b(fb0, next, h0);
            mul(fa1, fb1, NA);
        } else if constexpr (PHASES == 2) {
            read_a(fa1, cur, h1, 0);
            read_b(fb1, cur, h1);
            mul(fa0, fb0, 0);
            turn();
            issue(cur);
            read_a(fa0, next, h0, 0);
            read_b(fb0, next, h0);
            mul(fa1, fb1, 0);
        } else {
            turn();
            issue(cur);
            if (set) {
                read_a(fa0, next, h0, 0);
                read_b(fb0, next, h0);
                mul(fa1, fb1, 0);
            } else {
                read_a(fa1, next, h0, 0);
                read_b(fb1, next, h0);
                mul(fa0, fb0, 0);
            }
        }
    };
    static_assert(STAGES % 2 == 0, "a turn of the ring is a turn of the fragments");
    unsigned char *const ring[4] = {st0, st1, st2, st3};
#pragma unroll
    for (int i = 0; i < STAGES; ++i) issue(ring[i]);
    wait_vm<(STAGES - 1) * 2 * LOADS>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read_a(fa0, st0, h0, 0);
    read_b(fb0, st0, h0);
    // no way out of the loop but its end: with one the compiler spills the sums
    int left = total;
    for (; left >= STAGES; left -= STAGES) {
#pragma unroll
        for (int i = 0; i < STAGES; ++i) step(ring[i], ring[(i + 1) % STAGES], i & 1);
    }
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (left > i) step(ring[i], ring[i + 1], i & 1);
    wait_vm<0>();
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    // the argument block is read again from here on: its epilogue part would
    // otherwise sit in scalar registers through the loop
    const MmArgs &e = *late_args(a);
    // Each wave's sums pass through its own part of LDS, 64 rows at a time,
    // so that one rolled loop finishes whole rows of contiguous columns (and
    // another, for transposed outputs, whole columns). 16-byte chunk c of row
    // m sits at chunk c ^ swz(m): writes in the MFMA's layout, reads of rows
    // and reads of columns all spread over the banks.
    constexpr int RP = TM < 64 ? TM : 64, C = TN / 4, SZ = RP * TN * 4;
    static_assert(NW * SZ <= 4 * T * ROW && 2 * T * ROW % SZ == 0, "staging");
    unsigned char *const mine = wave * SZ < 2 * T * ROW ? st0 + wave * SZ : st1 + (wave * SZ - 2 * T * ROW);
    auto swz = [](int m) __attribute__((always_inline)) { return ((m & 3) * 4 + (m >> 2)) & (C - 1); };
#pragma unroll
    for (int pass = 0; pass < TM / RP; ++pass) {
        const int mb = m0 + wm * TM + pass * RP, nb = n0 + wn * TN;
        if (pass) wait_lgkm0();
#pragma unroll
        for (int i = 0; i < RP / 16; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int m = i * 16 + l16;
                *(f32x4 *)(mine + m * TN * 4 + ((j * 4 + g) ^ swz(m)) * 16) = acc[pass * (RP / 16) + i][j];
            }
        wait_lgkm0();
        asm volatile("" ::: "memory");
        const bool turned = (EPI == EPI_NEXT || ((EPI == EPI_GRAM || EPI == EPI_POLY || EPI == EPI_MIX) && e.sym && tn > tm)) &&
                            e.splits == 1;
        const Tile tile{z, mb, nb, mb + RP <= e.M && nb + TN <= e.N};
        constexpr int ITEMS = RP * C / 64, GROUP = T == 256 ? (EPI == EPI_ROWS ? 1 : 2) : T == 128 && EPI == EPI_SCALED ? 2 : 4;   // (registers)
        static_assert(ITEMS % GROUP == 0, "whole groups");
#pragma unroll 1
        for (int i0 = 0; i0 < ITEMS; i0 += GROUP) {
            f32x4 v[GROUP];
            Near near[GROUP];
#pragma unroll
            for (int i = 0; i < GROUP; ++i) {
                const int it = (i0 + i) * 64 + lane, m = it / C, c = it & (C - 1);
                v[i] = *(const f32x4 *)(mine + m * TN * 4 + (c ^ swz(m)) * 16);
                if (e.splits == 1) near[i] = gather<EPI>(e, tile, m, c * 4);
            }
            if constexpr (EPI == EPI_SCALED)
                if (e.splits == 1) {
                    int ms[GROUP], ns[GROUP];
#pragma unroll
                    for (int i = 0; i < GROUP; ++i) {
                        ms[i] = ((i0 + i) * 64 + lane) / C;
                        ns[i] = (lane & (C - 1)) * 4;
                    }
                    low_rank<GROUP>(e, tile, ms, ns, near);
                }
#pragma unroll
            for (int i = 0; i < GROUP; ++i) {
                const int it = (i0 + i) * 64 + lane, m = it / C, c = it & (C - 1);
                if (e.splits > 1) {
                    if (mb + m < e.M && nb + c * 4 < e.N)
                        store_at(e.partial + (((int64_t)split * e.batch + z) * e.M + mb) * e.ldp + nb,
                                 offset_of(m, c * 4, e.ldp, 4), v[i]);
                } else {
                    const uint4 q = finish<EPI>(e, tile, m, c * 4, v[i], near[i]);
                    if (turned) *(uint4 *)(mine + m * TN * 4 + (c ^ swz(m)) * 16) = q;
                }
            }
        }
        if (!turned) continue;
        wait_lgkm0();
        asm volatile("" ::: "memory");
        const Planes &q = EPI == EPI_NEXT ? e.o.q : e.o.p;
        const Tile flip{z, nb, mb, tile.inside};
        u16 *const hi = at_tile(q.hi, flip, q), *const lo = q.lo ? at_tile(q.lo, flip, q) : nullptr;
#pragma unroll 1
        for (int i = 0; i < TN * RP / 256; ++i) {
            const int it = i * 64 + lane;
            const int n = it / (RP / 4), m = (it % (RP / 4)) * 4;
            uint4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                (&v.x)[k] = *(const uint32_t *)(mine + (m + k) * TN * 4 + ((n >> 2) ^ swz(m + k)) * 16 + (n & 3) * 4);
            if (tile.inside || (nb + n < e.N && mb + m < width(q))) put_pairs(hi, lo, offset_of(n, m, q), v);
        }
    }
}

// Sums the splits of each element in order and applies the epilogue, one
// 32 x 32 tile per workgroup (4 elements to a thread: what takes time is the
// latency of a few loads); transposed planes go through LDS.
template <int EPI>
__global__ __launch_bounds__(256) void mm_reduce_kernel(const MmArgs a) {
    constexpr bool PLANES = EPI == EPI_GRAM || EPI == EPI_POLY || EPI == EPI_NEXT || EPI == EPI_MIX;
    __shared__ uint32_t turn[PLANES ? 32 : 1][33];
    int tm, tn;
    mm_place<32>(a, tm, tn);
    const int z = blockIdx.z, m0 = tm * 32, n0 = tn * 32;
    const Tile tile{z, m0, n0, m0 + 32 <= a.M && n0 + 32 <= a.N};
    const bool turned = EPI == EPI_NEXT || (PLANES && a.sym && tn > tm);
    const int m = threadIdx.x >> 3, n = (threadIdx.x & 7) * 4;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    Near near[1] = {gather<EPI>(a, tile, m, n)};
    if constexpr (EPI == EPI_SCALED) {
        const int ms[1] = {m}, ns[1] = {n};
        low_rank<1>(a, tile, ms, ns, near);
    }
    if (m0 + m < a.M && n0 + n < a.N) {
        const float *p = a.partial + ((int64_t)z * a.M + m0 + m) * a.ldp + n0 + n;
        const int64_t step = (int64_t)a.batch * a.M * a.ldp;
        int s = 0;
        for (; s + 4 <= a.splits; s += 4) {
            f32x4 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = *(const f32x4 *)(p + (s + i) * step);
#pragma unroll
            for (int i = 0; i < 4; ++i) v += x[i];
        }
        for (; s < a.splits; ++s) v += *(const f32x4 *)(p + s * step);
    }
    const uint4 q = finish<EPI>(a, tile, m, n, v, near[0]);
    if constexpr (PLANES) {
        if (!turned) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) turn[m][n + e] = (&q.x)[e];
        __syncthreads();
        const Planes &t = EPI == EPI_NEXT ? a.o.q : a.o.p;
        const Tile flip{z, n0, m0, tile.inside};
        u16 *const hi = at_tile(t.hi, flip, t), *const lo = t.lo ? at_tile(t.lo, flip, t) : nullptr;
        // (thread: row m of the transpose, 4 of its columns from n on)
        const uint4 x = make_uint4(turn[n][m], turn[n + 1][m], turn[n + 2][m], turn[n + 3][m]);
        if (n0 + m < a.N && m0 + n < width(t)) put_pairs(hi, lo, offset_of(m, n, t), x);
    }
}

template <int T, int STAGES, int PHASES, bool F16, bool PAIR, int EPI>
hipError_t go(const MmArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)mm_tiles(a, T), (unsigned)a.splits, (unsigned)a.batch);
    void *p[] = {const_cast<MmArgs *>(&a)};
    hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(&mm_kernel<T, STAGES, PHASES, F16, PAIR, EPI>), grid,
                                   dim3(mm_threads<T>()), p, 0, s);
    if (e != hipSuccess || a.splits == 1) return e;
    return hipLaunchKernel(reinterpret_cast<const void *>(&mm_reduce_kernel<EPI>),
                           dim3((unsigned)mm_tiles(a, 32), 1, (unsigned)a.batch), dim3(256), p, 0, s);
}

template <int EPI, bool F16, bool PAIR>
hipError_t pick(const MmArgs &a, hipStream_t s) {
    return a.tile == 256   ? go<256, 2, 4, F16, PAIR, EPI>(a, s)
           : a.tile == 128 ? go<128, 2, 2, F16, PAIR, EPI>(a, s)
                           : go<64, 4, 1, F16, PAIR, EPI>(a, s);
}
// (float16) either layout, or pairs only
template <int EPI>
hipError_t any(const MmArgs &a, hipStream_t s) {
    return a.pair ? pick<EPI, true, true>(a, s) : pick<EPI, true, false>(a, s);
}
template <int EPI>
hipError_t pairs_only(const MmArgs &a, hipStream_t s) {
    return a.pair ? pick<EPI, true, true>(a, s) : hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_mm(const MmArgs &a, hipStream_t s) {
    if (!mm_valid(a)) return hipErrorInvalidValue;
    switch (a.epi) {
        case EPI_ROWS: return a.pair ? hipErrorInvalidValue : pick<EPI_ROWS, false, false>(a, s);
        case EPI_SCALED: return pairs_only<EPI_SCALED>(a, s);
        case EPI_GRAM: return any<EPI_GRAM>(a, s);
        case EPI_POLY: return any<EPI_POLY>(a, s);
        case EPI_NEXT: return any<EPI_NEXT>(a, s);
        case EPI_ORTH: return any<EPI_ORTH>(a, s);
        case EPI_STEP: return pairs_only<EPI_STEP>(a, s);
        case EPI_MIX: return pairs_only<EPI_MIX>(a, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace gemel

// Products of two matrices in 4-bit floating point, on the matrix cores that
// take blocks and their scales as they are: y[m][n] = sum over k of x[m][k] *
// w[n][k] + bias[n].
#include <hip/hip_runtime.h>

#include <type_traits>

#include "mx_args.h"
#include "mx_device.h"

namespace gemel {

namespace {

typedef __attribute__((address_space(3))) unsigned char lds_u8;
typedef mx_f32x4 f32x4;

constexpr int ROW = MX_GROUP / 8;   // bytes of a row in a step (128 columns)
constexpr int STAGES = 4;           // a turn of the buffers is a group of scales

template <int N>
__device__ __forceinline__ void wait_vm() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}
__device__ __forceinline__ void wait_lgkm0() { __builtin_amdgcn_s_waitcnt(0xF | (0x3 << 14) | (0x7 << 4)); }

template <int LOADS, int NW>
__device__ __forceinline__ void fetch(const uint8_t *base, const uint32_t (&off)[LOADS], unsigned char *stage, int wave) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(base), 0, -1, 0x00020000);
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_u8 *)(stage + (i * NW + wave) * 1024), 16, (int)off[i], 0, 0, 0);
}

// One T x T tile per workgroup: 8 waves of 128 x 64 (T = 256) or 32 x 64 (T =
// 128), or 4 of 32 x 32 (T = 64). A step is 128 columns, 64 bytes of each row,
// fetched by direct global-to-LDS loads into one of four buffers, three steps
// ahead: a buffer is asked for again as soon as every wave has its last
// fragments in registers. Slot p of a buffer holds row p / 4, 16-byte chunk
// (p % 4) ^ (row / 2 % 4), so that the fragment reads of 16 rows fall on
// distinct banks. The scales of four steps are one word of a lane, fetched
// with the first of them.
//
// 16384 rows 4096 -> 4096 158 us (3480 TFLOP/s), 8192^3 270 to 281 (4000).
// What bounds it is not one unit: the matrix cores are busy 42% of all cycles,
// LDS 27%, at a clock that falls to 2.0 GHz; with one workgroup, two waves to
// a SIMD, they wait for each other. Trials without the fetches take 135 us,
// without the stores of the results 153, without the barriers 157. Two stages of 256 columns instead of
// four of 128, or fragments read before instead of among the products, took
// the same.
template <int T>
__global__ __launch_bounds__((mx_threads_of(T)), T == 256 ? 1 : T == 128 ? 4 : 2) void mx_mm_kernel(const MxMm a) {
    constexpr int NT = mx_threads_of(T), NW = NT / 64, WN = T == 256 ? 4 : 2;
    constexpr int TM = T * WN / NW, TN = T / WN, FM = TM / 16, FN = TN / 16;
    constexpr int LOADS = T * 4 / NT, STAGE = 2 * T * ROW;
    constexpr bool HALVES = T == 256;   // (no registers for all fragments of two steps)
    __shared__ __attribute__((aligned(1024))) unsigned char st0[STAGE], st1[STAGE], st2[STAGE], st3[STAGE], sc[2 * T * 16];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave - wm * WN, g = lane >> 4, l16 = lane & 15;
    const int M = a.x.rows, N = a.w.rows;
    // consecutive tiles on one XCD, and among them groups of 8 tile rows
    int tm, tn;
    {
        const int tiles_m = (M + T - 1) / T, tiles_n = (N + T - 1) / T, G = gridDim.x;
        const int t = (G & 7) == 0 ? (int)(blockIdx.x & 7) * (G >> 3) + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
        const int group = t / (8 * tiles_n), first = group * 8, rows = min(8, tiles_m - first);
        const int in = t - group * 8 * tiles_n;
        tn = in / rows;
        tm = first + in - tn * rows;
    }
    const int m0 = tm * T, n0 = tn * T;
    const int64_t pitch = mx_pitch(a.w.cols);
    const int s0 = (int)blockIdx.y * a.per * 4, total = min((int)(pitch / ROW) - s0, a.per * STAGES);

    uint32_t oa[LOADS], ob[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int row = (i * NT + tid) >> 2, ch = ((tid & 3) ^ ((row >> 1) & 3)) * 16;
        oa[i] = (uint32_t)(min(m0 + row, M - 1) - m0) * (uint32_t)pitch + ch;
        ob[i] = (uint32_t)(min(n0 + row, N - 1) - n0) * (uint32_t)pitch + ch;
    }
    const uint8_t *pa = a.x.codes + m0 * pitch + s0 * ROW, *pb = a.w.codes + n0 * pitch + s0 * ROW;
    // scales: 64 rows to a wave, of x for the first half of the waves that are
    // needed and of w for the rest (waves beyond repeat what others load)
    constexpr int PARTS = T / 64;
    const int part = wave % (2 * PARTS), of_w = part >= PARTS, local = (part - of_w * PARTS) * 64 + lane;
    const int srows = of_w ? N : M;
    const uint8_t *ps = (of_w ? a.w.scales : a.x.scales) + (int64_t)(s0 >> 2) * srows * 16;
    const uint32_t os = (uint32_t)min((of_w ? n0 : m0) + local, srows - 1) * 16u;
    unsigned char *const sslot = sc + of_w * T * 16 + (part - of_w * PARTS) * 1024;
    int iss = 0;
    // Requests the next step, the P-th of its four; past the last one, the last
    // one again (into a buffer whose reads are over), so that every step waits
    // alike.
    auto issue = [&](auto which, unsigned char *stage) __attribute__((always_inline)) {
        constexpr int P = decltype(which)::value;
        fetch<LOADS, NW>(pa, oa, stage, wave);
        fetch<LOADS, NW>(pb, ob, stage + T * ROW, wave);
        if constexpr (P == 0) {
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(ps), 0, -1, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_u8 *)sslot, 16, (int)os, 0, 0, 0);
        }
        if (++iss < total) {
            pa += ROW;
            pb += ROW;
            if (P == 3) ps += (int64_t)srows * 16;
        }
    };
    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr int NA = HALVES ? FM / 2 : FM;
    i32x4 fa0[NA], fa1[NA], fb0[FN], fb1[FN];
    int sa[FM], sb[FN];
    const int h = (g ^ ((l16 >> 1) & 3)) * 16;
    const int ra = (wm * TM + l16) * ROW + h, rb = T * ROW + (wn * TN + l16) * ROW + h;
    auto read_a = [&](i32x4(&f)[NA], const unsigned char *s, int row) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NA; ++i) f[i] = *(const i32x4 *)(s + ra + (row + i) * 16 * ROW);
    };
    auto read_b = [&](i32x4(&f)[FN], const unsigned char *s) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < FN; ++j) f[j] = *(const i32x4 *)(s + rb + j * 16 * ROW);
    };
    // (reads are issued before the products that they are to pass behind)
    auto behind = [&]() __attribute__((always_inline)) { __builtin_amdgcn_sched_barrier(0); };
    auto read_s = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[i] = *(const int *)(sc + (wm * TM + i * 16 + l16) * 16 + g * 4);
#pragma unroll
        for (int j = 0; j < FN; ++j) sb[j] = *(const int *)(sc + T * 16 + (wn * TN + j * 16 + l16) * 16 + g * 4);
    };
    auto mul = [&](auto which, i32x4(&f)[NA], i32x4(&b)[FN], int row) __attribute__((always_inline)) {
        constexpr int P = decltype(which)::value;
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[row + i][j] = mx_mul<P>(b[j], f[i], acc[row + i][j], sb[j], sa[row + i]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // the loads of the step after `cur`'s, the P-th, have landed in every wave,
    // and every wave has read the last of `cur`; two more steps are on their
    // way, one of which may bring scales
    auto turn = [&](auto which) __attribute__((always_inline)) {
        constexpr int P = decltype(which)::value;
        wait_lgkm0();
        wait_vm<2 * 2 * LOADS + (P == 1 || P == 2)>();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    auto step = [&](auto which, unsigned char *cur, unsigned char *next) __attribute__((always_inline)) {
        constexpr int P = decltype(which)::value;
        i32x4(&b)[FN] = P & 1 ? fb1 : fb0, (&b_next)[FN] = P & 1 ? fb0 : fb1;
        if constexpr (HALVES) {
            read_a(fa1, cur, NA);
            behind();
            mul(which, fa0, b, 0);
            turn(which);
            read_a(fa0, next, 0);
            read_b(b_next, next);
            issue(which, cur);
            behind();
            mul(which, fa1, b, NA);
        } else {
            i32x4(&f)[NA] = P & 1 ? fa1 : fa0, (&f_next)[NA] = P & 1 ? fa0 : fa1;
            turn(which);
            read_a(f_next, next, 0);
            read_b(b_next, next);
            issue(which, cur);
            behind();
            mul(which, f, b, 0);
        }
        if constexpr (P == 3) read_s();
    };
    constexpr std::integral_constant<int, 0> P0;
    constexpr std::integral_constant<int, 1> P1;
    constexpr std::integral_constant<int, 2> P2;
    constexpr std::integral_constant<int, 3> P3;
    issue(P0, st0);
    issue(P1, st1);
    issue(P2, st2);
    issue(P3, st3);
    wait_vm<3 * 2 * LOADS>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read_a(fa0, st0, 0);
    read_b(fb0, st0);
    read_s();
    // (rows of codes are whole groups of four steps)
    for (int left = total; left > 0; left -= STAGES) {
        step(P0, st0, st1);
        step(P1, st1, st2);
        step(P2, st2, st3);
        step(P3, st3, st0);
    }
    wait_vm<0>();
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    // Each wave's sums pass through its own part of LDS, 64 rows at a time, so
    // that whole rows of contiguous columns are written. 16-byte chunk c of row
    // m sits at chunk c ^ swz(m).
    constexpr int RP = TM < 64 ? TM : 64, C = TN / 4, SZ = RP * TN * 4;
    static_assert(NW * SZ <= 4 * STAGE && STAGE % SZ == 0, "staging");
    const int buffer = wave * SZ / STAGE;
    unsigned char *const mine = (buffer == 0 ? st0 : buffer == 1 ? st1 : buffer == 2 ? st2 : st3) + wave * SZ % STAGE;
    auto swz = [](int m) __attribute__((always_inline)) { return ((m & 3) * 4 + (m >> 2)) & (C - 1); };
    const int nb = n0 + wn * TN, n = nb + (lane & (C - 1)) * 4;
    const f32x4 bias = mx_bias(a.splits == 1 && n < N ? a.bias : nullptr, n, N);
#pragma unroll
    for (int pass = 0; pass < TM / RP; ++pass) {
        const int mb = m0 + wm * TM + pass * RP;
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
#pragma unroll 4
        for (int it = lane; it < RP * C; it += 64) {
            const int m = it / C, c = it & (C - 1);
            const f32x4 v = *(const f32x4 *)(mine + m * TN * 4 + (c ^ swz(m)) * 16);
            if (mb + m >= M || n >= N) continue;
            if (a.splits > 1)
                *(f32x4 *)(a.part + ((int64_t)blockIdx.y * M + mb + m) * a.ldp + n) = v;
            else
                mx_put(a.y, a.ldy, a.f32, mb + m, n, N, v + bias);
        }
        asm volatile("" ::: "memory");
    }
}

template <int T>
hipError_t go(const MxMm &a, hipStream_t s) {
    void *p[] = {const_cast<MxMm *>(&a)};
    return hipLaunchKernel(reinterpret_cast<const void *>(&mx_mm_kernel<T>),
                           dim3((unsigned)mx_mm_tiles(a), (unsigned)a.splits), dim3(mx_threads_of(T)), p, 0, s);
}

}  // namespace

hipError_t launch_mx_mm(const MxMm &a, hipStream_t s) {
    if (!mx_mm_valid(a)) return hipErrorInvalidValue;
    hipError_t e = a.tile == 256 ? go<256>(a, s) : a.tile == 128 ? go<128>(a, s) : go<64>(a, s);
    if (e != hipSuccess || a.splits == 1) return e;
    return launch_mx_sum(MxSum{a.part, a.ldp, a.splits, a.x.rows, a.w.rows, a.bias, a.y, a.ldy, a.f32}, s);
}

}  // namespace gemel

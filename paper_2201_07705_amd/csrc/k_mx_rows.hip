// Products of rows that are not quantised (bf16, or float32 as three bf16
// planes whose sum they are: every product is then exact and sums are
// float32) with 4-bit weights, and of few quantised rows.
//
// Reading the weights bounds them: a lane loads the 32 codes of one block of
// a weight row in one piece, and its registers are operands of the matrix
// cores as soon as the hardware has made bf16 of them (8 codes are 4
// conversions). The depth's order within 128 columns is the codes': lane
// group g holds the block g, and the rows are read to match. One row 4096 ->
// 4096 4.8 us (1.9 TB/s of weights, two round trips to memory), 25088 -> 4096
// 16 (3.5 TB/s).
#include <hip/hip_runtime.h>

#include "mx_args.h"
#include "mx_device.h"

namespace gemel {

namespace {

typedef mx_f32x4 f32x4;
enum { ACT_BF16, ACT_PLANES, ACT_MX };

// Up to 16 rows: 16 outputs to a workgroup, whose waves take turns at the
// groups of 512 columns. One launch: what counts is latency.
template <int ACT>
__global__ __launch_bounds__(1024) void mx_few_kernel(const MxRows a) {
    __shared__ f32x4 sums[16][64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int N = a.w.rows, K = a.w.cols, groups = (K + MX_GROUP - 1) / MX_GROUP, n0 = blockIdx.x * 16;
    const int64_t pitch = mx_pitch(K);
    const int n = min(n0 + l16, N - 1), m = min(l16, a.M - 1);
    const uint8_t *codes = a.w.codes + n * pitch + g * 16, *scales = a.w.scales + n * 16ll + g * 4;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int kg = wave; kg < groups; kg += a.waves) {
        uint4 w[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) w[s] = *(const uint4 *)(codes + kg * 256ll + s * 64);
        const uint32_t sw = *(const uint32_t *)(scales + (int64_t)kg * N * 16);
        if constexpr (ACT == ACT_MX) {
            uint4 x[4];
            const uint8_t *xc = a.q.codes + m * pitch + kg * 256ll + g * 16;
#pragma unroll
            for (int s = 0; s < 4; ++s) x[s] = *(const uint4 *)(xc + s * 64);
            const uint32_t sx = *(const uint32_t *)(a.q.scales + ((int64_t)kg * a.M + m) * 16 + g * 4);
            acc = mx_mul<0>(__builtin_bit_cast(i32x4, w[0]), __builtin_bit_cast(i32x4, x[0]), acc, (int)sw, (int)sx);
            acc = mx_mul<1>(__builtin_bit_cast(i32x4, w[1]), __builtin_bit_cast(i32x4, x[1]), acc, (int)sw, (int)sx);
            acc = mx_mul<2>(__builtin_bit_cast(i32x4, w[2]), __builtin_bit_cast(i32x4, x[2]), acc, (int)sw, (int)sx);
            acc = mx_mul<3>(__builtin_bit_cast(i32x4, w[3]), __builtin_bit_cast(i32x4, x[3]), acc, (int)sw, (int)sx);
        } else {
            constexpr int P = ACT == ACT_PLANES ? 3 : 1;
            const int c0 = kg * MX_GROUP + g * 32;
            const u16 *row = a.x + m * a.ldx;
            auto mul = [&](int s, int i, const uint4 &x) __attribute__((always_inline)) {
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mx_bf16((&w[s].x)[i], mx_scale(sw >> s * 8 & 255)),
                                                              __builtin_bit_cast(mx_bf16x8, x), acc, 0, 0, 0);
            };
            if ((kg + 1) * MX_GROUP <= K) {
                // (what fits the registers of 16 waves is in flight at once)
                constexpr int AT_ONCE = P == 1 ? 16 : 8;
#pragma unroll
                for (int i0 = 0; i0 < 16; i0 += AT_ONCE) {
                    uint4 x[P][AT_ONCE];
#pragma unroll
                    for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
                        for (int p = 0; p < P; ++p)
                            x[p][i] = get_16b(row + p * a.plane + c0 + ((i0 + i) >> 2) * 128 + ((i0 + i) & 3) * 8);
#pragma unroll
                    for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
                        for (int p = 0; p < P; ++p) mul((i0 + i) >> 2, (i0 + i) & 3, x[p][i]);
                }
            } else {
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    if (kg * MX_GROUP + s * 128 >= K) break;
#pragma unroll 1
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int i = 0; i < 4; ++i) mul(s, i, mx_chunk(row + p * a.plane, c0 + s * 128 + i * 8, K));
                }
            }
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
    for (int i = 1; i < a.waves; ++i) acc += sums[i][lane];
    if (l16 < a.M && n0 + 4 * g < N)
        mx_put(a.y, a.ldy, a.f32, l16, n0 + 4 * g, N, acc + mx_bias(a.bias, n0 + 4 * g, N));
}

// 16 MB rows and 128 NB outputs to a workgroup of 8 waves, 16 NB outputs to a
// wave, over a slice of the depth. Steps of 128 columns of the rows pass
// through two buffers of LDS (16-byte chunk c of row r at chunk c ^ r % 16:
// the fragment reads of 16 rows fall on distinct banks); rows and codes are
// loaded one or two steps ahead. A fragment of the rows serves NB products:
// with NB = 2 LDS is as busy as the matrix cores (1024 float32 rows 25088 ->
// 4096 in 510 us; NB = 4 469, 1350 TFLOP/s of bf16 products).
template <int P, int MB, int NB>
__global__ __launch_bounds__(512, 2) void mx_rows_kernel(const MxRows a) {
    constexpr int ROWS = 16 * MB, CHUNKS = P * ROWS * 16, LOADS = mx_piece_loads(P * ROWS);
    constexpr int AHEAD = P == 3 && NB == 4 ? 1 : 2;   // steps (registers)
    __shared__ uint4 st[2][CHUNKS];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int N = a.w.rows, K = a.w.cols, n0 = blockIdx.x * 128 * NB + wave * 16 * NB, m0 = blockIdx.z * ROWS;
    const int64_t pitch = mx_pitch(K);
    const int step0 = (int)blockIdx.y * a.per, steps = min((K + 127) / 128 - step0, a.per);
    uint32_t codes[NB], scales[NB];   // (from the wave's first output: up to 63 rows of 2^19 bytes)
    const uint8_t *const code0 = a.w.codes + (int64_t)min(n0, N - 1) * pitch, *const scale0 = a.w.scales + (int64_t)min(n0, N - 1) * 16;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int n = min(n0 + j * 16 + l16, N - 1) - min(n0, N - 1);
        codes[j] = (uint32_t)n * (uint32_t)pitch + g * 16;
        scales[j] = n * 16 + g * 4;
    }
    struct Ahead {
        uint4 x[LOADS], w[NB];
        uint32_t s[NB];
    } ahead[AHEAD];
    // (where the thread's pieces begin in their rows; no branch stands between
    // the loads of a whole step)
    const u16 *pieces[LOADS];
    const int col = mx_piece_col(tid);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int row = mx_piece_row(i, tid, P * ROWS), p = row / ROWS, r = row % ROWS;
        pieces[i] = a.x + p * a.plane + (int64_t)min(m0 + r, a.M - 1) * a.ldx + col;
    }
    auto load = [&](Ahead &q, int step) __attribute__((always_inline)) {
        if ((step + 1) * 128 <= K) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) q.x[i] = get_16b(pieces[i] + step * 128);
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) q.x[i] = mx_chunk(pieces[i] - col, step * 128 + col, K);
        }
        const uint8_t *const wc = code0 + step * 64ll, *const ws = scale0 + (int64_t)(step >> 2) * N * 16;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            q.w[j] = *(const uint4 *)(wc + codes[j]);
            q.s[j] = *(const uint32_t *)(ws + scales[j]);
        }
    };
    f32x4 acc[NB][MB];
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int b = 0; b < MB; ++b) acc[j][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto turn = [&](Ahead &q, uint4 *buf, int k) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int id = i * 512 + tid, r = id / 16;
            if (CHUNKS % 512 == 0 || id < CHUNKS) buf[r * 16 + ((id & 15) ^ (r & 15))] = q.x[i];
        }
        uint4 w[NB];
        float scale[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            w[j] = q.w[j];
            scale[j] = mx_scale(q.s[j] >> ((step0 + k) & 3) * 8 & 255);
        }
        __syncthreads();
        if (k + AHEAD < steps) load(q, step0 + k + AHEAD);
        // Fragments of the rows, the one of piece i, plane p, block b being the
        // (i P + p) MB + b-th: read AHEAD_READS before they are used, so that the
        // matrix cores do not wait for LDS (1024 rows 25088 -> 4096 bf16 209 us,
        // read where they are used 237; float32 469 and 498; 3 and 6 ahead
        // instead of 2 and 4 within 1.5%, with 4 to 8 registers more).
        constexpr int READS = 4 * P * MB, AHEAD_READS = NB == 4 ? 2 : 4, RING = AHEAD_READS + 1;
        mx_bf16x8 v[RING], f[NB];
        auto read = [&](int t) __attribute__((always_inline)) {
            const int i = t / (P * MB), row = t % (P * MB) * 16 + l16;
            v[t % RING] = __builtin_bit_cast(mx_bf16x8, buf[row * 16 + ((4 * g + i) ^ l16)]);
        };
#pragma unroll
        for (int t = 0; t < AHEAD_READS; ++t) read(t);
#pragma unroll
        for (int t = 0; t < READS; ++t) {
            if (t + AHEAD_READS < READS) read(t + AHEAD_READS);
            __builtin_amdgcn_sched_barrier(0);
            if (t % (P * MB) == 0)
#pragma unroll
                for (int j = 0; j < NB; ++j) f[j] = mx_bf16((&w[j].x)[t / (P * MB)], scale[j]);
            const int b = t % MB;
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[j][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[j], v[t % RING], acc[j][b], 0, 0, 0);
        }
    };
    load(ahead[0], step0);
    if (AHEAD > 1 && steps > 1) load(ahead[AHEAD - 1], step0 + 1);
    for (int k = 0; k < steps; k += 2) {
        turn(ahead[0], st[0], k);
        if (k + 1 < steps) turn(ahead[AHEAD - 1], st[1], k + 1);
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int n = n0 + j * 16 + 4 * g;
        if (n >= N) continue;
        const f32x4 bias = mx_bias(a.slices == 1 ? a.bias : nullptr, n, N);
#pragma unroll
        for (int b = 0; b < MB; ++b) {
            const int m = m0 + b * 16 + l16;
            if (m >= a.M) continue;
            if (a.slices > 1)
                *(f32x4 *)(a.part + ((int64_t)blockIdx.y * a.M + m) * a.ldp + n) = acc[j][b];
            else
                mx_put(a.y, a.ldy, a.f32, m, n, N, acc[j][b] + bias);
        }
    }
}

template <typename K>
hipError_t go(K kernel, const MxRows &a, dim3 grid, int threads, hipStream_t s) {
    void *p[] = {const_cast<MxRows *>(&a)};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3((unsigned)threads), p, 0, s);
}
template <int P, int NB>
hipError_t many(const MxRows &a, hipStream_t s) {
    const int mb = mx_row_blocks(a.M);
    const dim3 grid((unsigned)((a.w.rows + 128 * NB - 1) / (128 * NB)), (unsigned)a.slices, (unsigned)((a.M + mb * 16 - 1) / (mb * 16)));
    return mb == 2 ? go(&mx_rows_kernel<P, 2, NB>, a, grid, 512, s) : mb == 3 ? go(&mx_rows_kernel<P, 3, NB>, a, grid, 512, s)
                                                                              : go(&mx_rows_kernel<P, 4, NB>, a, grid, 512, s);
}

}  // namespace

hipError_t launch_mx_rows(const MxRows &a, hipStream_t s) {
    if (!mx_rows_valid(a)) return hipErrorInvalidValue;
    if (a.M <= MX_FEW) {
        const dim3 grid((unsigned)((a.w.rows + 15) / 16));
        return a.q.codes      ? go(&mx_few_kernel<ACT_MX>, a, grid, a.waves * 64, s)
               : a.planes > 1 ? go(&mx_few_kernel<ACT_PLANES>, a, grid, a.waves * 64, s)
                              : go(&mx_few_kernel<ACT_BF16>, a, grid, a.waves * 64, s);
    }
    hipError_t e = a.planes > 1 ? (a.wide ? many<3, 4>(a, s) : many<3, 2>(a, s)) : (a.wide ? many<1, 4>(a, s) : many<1, 2>(a, s));
    if (e != hipSuccess || a.slices == 1) return e;
    return launch_mx_sum(MxSum{a.part, a.ldp, a.slices, a.M, a.w.rows, a.bias, a.y, a.ldy, a.f32}, s);
}

}  // namespace gemel

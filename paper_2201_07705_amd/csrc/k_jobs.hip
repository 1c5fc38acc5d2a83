// Layouts and sums around the products of the operators: small pieces of
// work, several of which share a launch (alone each would cost the launch
// more than its work).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "op_args.h"
#include "op_moves.h"

namespace gemel {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf_up(u16 h) { return __uint_as_float((uint32_t)h << 16); }
__device__ __forceinline__ u16 bf_down(float f) { return __builtin_bit_cast(u16, (__bf16)f); }
__device__ __forceinline__ u16 half_down(float f) { return __builtin_bit_cast(u16, (_Float16)f); }
__device__ __forceinline__ float half_up(u16 h) { return (float)__builtin_bit_cast(_Float16, h); }

// The exponent that brings a largest magnitude, given as bits, into
// [2^14, 2^15); 0 where it is zero or not finite.
__device__ __forceinline__ int plane_exp(unsigned bits) {
    const float mx = __uint_as_float(bits);
    if (bits == 0u || bits >= 0x7f800000u) return 0;
    return 14 - ilogbf(mx);
}
// 4 values from column c (a multiple of 4) of a row of pairs on
__device__ __forceinline__ void split_put(u16 *row, int c, f32x4 v, int e) {
    u16 h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float s = ldexpf(v[i], e);
        h[i] = half_down(s);
        // the rest of a value that is not finite would be NaN; the sum has it already
        l[i] = isfinite(s) ? half_down(s - half_up(h[i])) : (u16)0;
    }
    row += pair_at(c);
    *(ushort4 *)row = make_ushort4(h[0], h[1], h[2], h[3]);
    *(ushort4 *)(row + PAIR_RUN) = make_ushort4(l[0], l[1], l[2], l[3]);
}
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// 4 consecutive float32 (`left` of them there; others zero)
__device__ __forceinline__ f32x4 load4(const float *p, int left) {
    if (left >= 4) return get_f32x4<f32x4>(p);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) v[i] = p[i];
    return v;
}

// the same of bf16
__device__ __forceinline__ f32x4 up4(const u16 *p, int left) {
    if (left >= 4) {
        const ushort4 h = get_u16x4(p);
        return f32x4{bf_up(h.x), bf_up(h.y), bf_up(h.z), bf_up(h.w)};
    }
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) v[i] = bf_up(p[i]);
    return v;
}

constexpr int CHUNK_COLS = 64;     // columns of a block of JOB_CHUNKS

// 16 bytes at a time; output rows are whole chunks of that
template <typename E>
__device__ __forceinline__ void pad(const Job &j, int block) {
    constexpr int Q = 16 / sizeof(E);
    const int across = (int)(j.ldo / Q);   // chunks of a row
    const int64_t first = (int64_t)block * PAD_ITEMS;
    const int row = (int)(first / across), at = (int)(first - (int64_t)row * across) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < PAD_ITEMS / 256; ++i) {
        const int down = (at + i * 256) / across, r = row + down, c = (at + i * 256 - down * across) * Q;
        if (r >= j.rows) continue;
        const E *in = (const E *)j.in + (int64_t)(j.perm ? j.perm[r] : r) * j.ldi + c;
        union {
            uint4 v;
            E e[Q];
        } x;
        if (c + Q <= j.cols) {
            x.v = get_16b(in);
        } else {
#pragma unroll
            for (int k = 0; k < Q; ++k) x.e[k] = c + k < j.cols ? in[k] : (E)0;
        }
        *(uint4 *)((E *)j.out + (int64_t)r * j.ldo + c) = x.v;
    }
}

// f(column, 4 values) over a row's columns up to `end` (zeros from the last
// on), from c on in steps; four loads in flight, no branch between them
template <typename F>
__device__ __forceinline__ void along(const float *in, int cols, int end, int c, int step, F &&f) {
    for (; c + 3 * step + 4 <= cols; c += 4 * step) {
        f32x4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = get_f32x4<f32x4>(in + c + k * step);
#pragma unroll
        for (int k = 0; k < 4; ++k) f(c + k * step, v[k]);
    }
    for (; c < end; c += step) f(c, load4(in + c, cols - c));
}

// A workgroup per row (137 rows of 23605: 47 -> 12 us against a wave each), or
// a wave for rows of up to SPLIT_WIDE.
__device__ __forceinline__ void split(const Job &j, int block, unsigned char *lds) {
    const bool wide = j.cols > SPLIT_WIDE;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = wide ? block : block * 4 + wave;
    if (r >= j.rows) return;
    const float *in = (const float *)j.in + (int64_t)(j.perm ? j.perm[r] : r) * j.ldi;
    const int first = (wide ? (int)threadIdx.x : lane) * 4, step = wide ? 1024 : 256;
    unsigned m = 0;
    along(in, j.cols, j.cols, first, step, [&](int, f32x4 v) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) m = max(m, magnitude(v[i]));
    });
    for (int o = 32; o; o >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, o));
    if (wide) {
        unsigned *const part = (unsigned *)lds;
        if (lane == 0) part[wave] = m;
        __syncthreads();
        m = max(max(part[0], part[1]), max(part[2], part[3]));
    }
    const int e = plane_exp(m);
    if (first == 0) j.e[r] = e;
    u16 *out = (u16 *)j.out + r * j.ldo;
    along(in, j.cols, (int)(j.ldo / 2), first, step,
          [&](int c, f32x4 v) __attribute__((always_inline)) { split_put(out, c, v, e); });
}

// 64 x 64 tiles through LDS, which holds the tile transposed. E: u16 (copied)
// or float (split).
template <typename E>
__device__ __forceinline__ void turn(const Job &j, int block, unsigned char *lds) {
    constexpr bool F = sizeof(E) == 4;
    constexpr int Q = 16 / sizeof(E), PITCH = F ? 65 : 66;
    E *const tile = (E *)lds;                             // [column][row]
    float *const part = (float *)(lds + 64 * PITCH * sizeof(E) + 8);   // [4][64]
    const int tid = threadIdx.x, across = (j.cols + 63) / 64;
    const int r0 = block / across * 64, c0 = block % across * 64;
    union Chunk {
        uint4 v;
        E e[Q];
    };
    constexpr int N = 64 * 64 / Q / 256;   // chunks of a thread
    Chunk x[N];
    const bool whole = r0 + 64 <= j.rows && c0 + 64 <= j.cols;
    if (whole) {
        // (no branch between the loads)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int k = i * 256 + tid;
            x[i].v = get_16b((const E *)j.in + (int64_t)(r0 + k / (64 / Q)) * j.ldi + c0 + k % (64 / Q) * Q);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = (i * 256 + tid) / (64 / Q), c = (i * 256 + tid) % (64 / Q) * Q;
            const E *in = (const E *)j.in + (int64_t)(r0 + r) * j.ldi + c0 + c;
#pragma unroll
            for (int k = 0; k < Q; ++k) x[i].e[k] = r0 + r < j.rows && c0 + c + k < j.cols ? in[k] : (E)0;
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int r = (i * 256 + tid) / (64 / Q), c = (i * 256 + tid) % (64 / Q) * Q;
#pragma unroll
        for (int k = 0; k < Q; ++k) tile[(c + k) * PITCH + r] = x[i].e[k];
    }
    int *const es = (int *)(part + 256);
    if (F && tid < 64 && c0 + tid < j.cols) {
        unsigned m = 0;
        for (int p = 0; p < j.parts; ++p) m = max(m, j.max[(int64_t)p * j.cols + c0 + tid]);
        es[tid] = plane_exp(m);
        if (r0 == 0) j.e[c0 + tid] = es[tid];
    }
    __syncthreads();
    for (int i = tid; i < 64 * 16; i += 256) {
        const int c = i >> 4, r = (i & 15) * 4;
        if (c0 + c >= j.cols || r0 + r >= (F ? j.ldo / 2 : j.ldo)) continue;
        const E *t = tile + c * PITCH + r;
        u16 *const out = (u16 *)j.out + (int64_t)(c0 + c) * j.ldo;
        if constexpr (F)
            split_put(out, r0 + r, f32x4{t[0], t[1], t[2], t[3]}, es[c]);
        else
            *(ushort4 *)(out + r0 + r) = make_ushort4(t[0], t[1], t[2], t[3]);
    }
    if (j.sum) {
        const int c = tid & 63, q = tid >> 6;
        float v = 0.f;
        for (int r = q * 16; r < q * 16 + 16; ++r) v += F ? (float)tile[c * PITCH + r] : bf_up((u16)tile[c * PITCH + r]);
        part[q * 64 + c] = v;
        __syncthreads();
        if (q == 0 && c0 + c < j.cols)
            j.sum[(int64_t)(block / across) * j.cols + c0 + c] = part[c] + part[64 + c] + part[128 + c] + part[192 + c];
    }
}

// [parts][cols] of column maxima (float32) or sums: 64 columns per block, 16
// threads across, 16 groups of rows.
template <bool MAX>
__device__ __forceinline__ void columns(const Job &j, int block, unsigned char *lds) {
    f32x4 *const part = (f32x4 *)lds;   // [16][16]
    const int across = (j.cols + 63) / 64, p = block / across, c = block % across * 64 + (threadIdx.x & 15) * 4;
    const int g = threadIdx.x >> 4, left = j.cols - c;
    const int r0 = (int)((int64_t)j.rows * p / j.parts), r1 = (int)((int64_t)j.rows * (p + 1) / j.parts);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](f32x4 x) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = MAX ? __uint_as_float(max(__float_as_uint(v[i]), magnitude(x[i]))) : v[i] + x[i];
    };
    const int in = left >= 4 ? 4 : left;
    int r = r0 + g;
    // (eight loads in flight, no branch between them)
    if (in == 4 && j.f32) {
        for (; r + 112 < r1; r += 128) {
            f32x4 x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = get_f32x4<f32x4>((const float *)j.in + (r + 16 * k) * j.ldi + c);
#pragma unroll
            for (int k = 0; k < 8; ++k) add(x[k]);
        }
    } else if (in == 4) {
        for (; r + 112 < r1; r += 128) {
            ushort4 x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = get_u16x4((const u16 *)j.in + (r + 16 * k) * j.ldi + c);
#pragma unroll
            for (int k = 0; k < 8; ++k) add(f32x4{bf_up(x[k].x), bf_up(x[k].y), bf_up(x[k].z), bf_up(x[k].w)});
        }
    }
    for (; r < r1 && in > 0; r += 16)
        add(j.f32 ? load4((const float *)j.in + r * j.ldi + c, in) : up4((const u16 *)j.in + r * j.ldi + c, in));
    part[g * 16 + (threadIdx.x & 15)] = v;
    __syncthreads();
    if (g) return;
    for (int k = 1; k < 16; ++k) {
        const f32x4 x = part[k * 16 + threadIdx.x];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = MAX ? __uint_as_float(max(__float_as_uint(v[i]), __float_as_uint(x[i]))) : v[i] + x[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) {
            if (MAX)
                j.max[(int64_t)p * j.cols + c + i] = __float_as_uint(v[i]);
            else
                j.sum[(int64_t)p * j.cols + c + i] = v[i];
        }
}

// 64 columns per block, 4 groups of parts
__device__ __forceinline__ void coladd(const Job &j, int block, unsigned char *lds) {
    float *const part = (float *)lds;
    const int c = block * 64 + (threadIdx.x & 63), g = threadIdx.x >> 6;
    float v = 0.f;
    if (c < j.cols) {
#pragma unroll 8
        for (int p = g; p < j.parts; p += 4) v += j.sum[(int64_t)p * j.cols + c];
    }
    part[threadIdx.x] = v;
    __syncthreads();
    if (g == 0 && c < j.cols)
        ((float *)j.out)[c] = part[threadIdx.x] + part[64 + threadIdx.x] + part[128 + threadIdx.x] + part[192 + threadIdx.x];
}

// 64 columns of a run per block, 32 rank indices at a time through LDS: both
// the input and the output are moved along their own rows, whichever index
// these have (40 adapters of 59 x 8385 to columns: 344 -> 40 us against
// stores of single elements)
__device__ __forceinline__ void pack(const Job &j, int block, unsigned char *lds) {
    uint32_t *const tile = (uint32_t *)lds;   // [32][65]
    const int width = j.by_rank ? (int)j.ldo : j.cols, across = (width + 63) / 64, u = block / across, c0 = block % across * 64;
    const int rank = j.run_rank[u], tid = threadIdx.x;
    // (a half of an adapter has at most 2^28 elements: 32-bit offsets)
    const char *const in = (const char *)j.in + (int64_t)j.run_id[u] * j.cols * j.R * (j.f32 ? 4 : 2);
    int bad = 0;
    for (int r0 = 0; r0 < j.rp; r0 += 32) {
        // (clamped, so that no branch stands between the loads)
        uint32_t x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = k * 256 + tid;
            const int r = min(r0 + (j.in_rc ? i >> 6 : i & 31), rank - 1), c = min(c0 + (j.in_rc ? i & 63 : i >> 5), j.cols - 1);
            const uint32_t at = j.in_rc ? (uint32_t)r * j.cols + c : (uint32_t)c * j.R + r;
            x[k] = j.f32 ? *(const uint32_t *)(in + at * 4u) : *(const u16 *)(in + at * 2u);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = k * 256 + tid, r = j.in_rc ? i >> 6 : i & 31, c = j.in_rc ? i & 63 : i >> 5;
            const bool there = r0 + r < rank && c0 + c < j.cols;
            const bool spoilt = there && !j.by_rank && (x[k] & 0x7f80u) == 0x7f80u;
            bad |= spoilt;
            tile[r * 65 + c] = there && !spoilt ? x[k] : 0u;
        }
        __syncthreads();
        if (j.by_rank) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int r = (k * 256 + tid) >> 6, c = tid & 63;
                if (c0 + c >= width) continue;
                const int64_t to = ((int64_t)u * j.rp + r0 + r) * j.ldo + c0 + c;
                if (j.f32)
                    ((uint32_t *)j.out)[to] = tile[r * 65 + c];
                else
                    ((u16 *)j.out)[to] = (u16)tile[r * 65 + c];
            }
        } else if (c0 + (tid >> 2) < j.cols) {
            const int c = tid >> 2, r = (tid & 3) * 8;
            uint4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k) (&v.x)[k] = tile[(r + 2 * k) * 65 + c] | tile[(r + 2 * k + 1) * 65 + c] << 16;
            u16 *out = (u16 *)j.out + ((int64_t)u * j.cols + c0 + c) * 2 * j.rp + r0 + r;
            *(uint4 *)out = v;
            *(uint4 *)(out + j.rp) = v;
        }
        __syncthreads();
    }
    if (j.by_rank) return;
    bad = __syncthreads_or(bad);
    if (tid == 0) j.flags[block] = bad;
}

// 64 columns of an adapter per block, 32 rank indices at a time
__device__ __forceinline__ void chunks(const Job &j, int block, unsigned char *lds) {
    float *const tile = (float *)lds;   // [32][65]
    const int across = (j.cols + CHUNK_COLS - 1) / CHUNK_COLS, ad = block / across, c0 = block % across * CHUNK_COLS;
    const int u = j.run_of[ad], rank = u < 0 ? 0 : j.run_rank[u];
    const int k0 = u < 0 ? 0 : j.chunk_first[u] * j.sub, k1 = u < 0 ? 0 : j.chunk_first[u + 1] * j.sub;
    float *out = (float *)j.out + (int64_t)ad * j.R * j.cols;
    const int tid = threadIdx.x, c = c0 + (tid & 63), cc = min(c, j.cols - 1);
    for (int r0 = 0; r0 < j.R; r0 += 32) {
        // thread: rank indices r0 + tid / 64 + 4 q; all Q sums of a piece are
        // asked for together
        float v[8] = {};
        auto add = [&](auto q_) __attribute__((always_inline)) {
            constexpr int Q = decltype(q_)::value;
            const float *p = j.sum + ((int64_t)k0 * j.rp + r0 + (tid >> 6)) * j.cols + cc;
#pragma unroll 4
            for (int k = k0; k < k1; ++k, p += (int64_t)j.rp * j.cols) {
#pragma unroll
                for (int q = 0; q < Q; ++q) v[q] += p[(int64_t)(4 * q) * j.cols];
            }
        };
        const int left = rank - r0;
        if (left > 16)
            add(std::integral_constant<int, 8>{});
        else if (left > 4)
            add(std::integral_constant<int, 4>{});
        else if (left > 0)
            add(std::integral_constant<int, 1>{});
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int i = (tid >> 6) + 4 * q, r = r0 + i;
            const float x = r < rank && c < j.cols ? v[q] : 0.f;
            if (j.turned)
                tile[i * 65 + (tid & 63)] = x;
            else if (r < j.R && c < j.cols)
                out[(int64_t)r * j.cols + c] = x;
        }
        if (!j.turned) continue;
        __syncthreads();
        for (int i = threadIdx.x; i < 64 * 32; i += 256) {
            const int c = i >> 5, r = i & 31;
            if (c0 + c < j.cols && r0 + r < j.R) out[(int64_t)(c0 + c) * j.R + r0 + r] = tile[r * 65 + c];
        }
        __syncthreads();
    }
}

// 1024 columns of a row per block
__device__ __forceinline__ void rows(const Job &j, int block, unsigned char *lds) {
    float *const ts = (float *)lds;   // [256]
    const int across = (j.cols + 1023) / 1024, row = block / across, c = (block % across * 256 + threadIdx.x) * 4;
    const int4 info = j.row_info[row];   // position, run or -1, adapter, rank
    const int rank = j.t && info.y >= 0 ? info.w : 0, left = j.cols - c;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (left > 0) {
#pragma unroll 8
        for (int p = 0; p < j.parts; ++p) v += *(const f32x4 *)(j.sum + ((int64_t)p * j.rows + row) * j.ldi + c);
    }
    if ((int)threadIdx.x < rank) ts[threadIdx.x] = j.t[(int64_t)info.x * j.rp + threadIdx.x];
    __syncthreads();
    if (left <= 0) return;
#pragma unroll 4
    for (int r = 0; r < rank; ++r) {
        const int64_t at = ((int64_t)info.z * j.R + r) * j.cols + c;
        v += ts[r] * (j.f32 ? load4((const float *)j.in + at, left) : up4((const u16 *)j.in + at, left));
    }
    const int64_t to = row * j.ldo + c;
    if (left >= 4) {
        if (j.f32)
            put_f32x4((float *)j.out + to, v);
        else
            put_u16x4((u16 *)j.out + to, make_ushort4(bf_down(v[0]), bf_down(v[1]), bf_down(v[2]), bf_down(v[3])));
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= left) continue;
        if (j.f32)
            ((float *)j.out)[to + i] = v[i];
        else
            ((u16 *)j.out)[to + i] = bf_down(v[i]);
    }
}

__global__ __launch_bounds__(256) void jobs_kernel(const Jobs args) {
    __shared__ __attribute__((aligned(16))) unsigned char lds[64 * 65 * 4 + 16 + 1024 + 256];
    // (a uniform index into the argument block where it lies)
    const Jobs &all = *(const Jobs *)__builtin_amdgcn_kernarg_segment_ptr();
    int i = 0;
    while (i + 1 < all.n && (int)blockIdx.x >= all.first[i + 1]) ++i;
    const Job &j = all.job[i];
    const int block = (int)blockIdx.x - all.first[i];
    switch (j.kind) {
        case JOB_PAD:
            if (j.f32)
                pad<uint32_t>(j, block);
            else
                pad<u16>(j, block);
            break;
        case JOB_SPLIT: split(j, block, lds); break;
        case JOB_TURN:
            if (j.f32)
                turn<float>(j, block, lds);
            else
                turn<u16>(j, block, lds);
            break;
        case JOB_COLMAX: columns<true>(j, block, lds); break;
        case JOB_COLSUM: columns<false>(j, block, lds); break;
        case JOB_COLADD: coladd(j, block, lds); break;
        case JOB_PACK: pack(j, block, lds); break;
        case JOB_CHUNKS: chunks(j, block, lds); break;
        case JOB_ROWS: rows(j, block, lds); break;
    }
}

}  // namespace

hipError_t launch_jobs(const Jobs &j, hipStream_t s) {
    if (j.n == 0) return hipSuccess;
    void *p[] = {const_cast<Jobs *>(&j)};
    return hipLaunchKernel(reinterpret_cast<const void *>(&jobs_kernel), dim3((unsigned)j.blocks), dim3(256), p, 0, s);
}

}  // namespace gemel

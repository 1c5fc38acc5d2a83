// The parts of an orthogonalised matrix update around its large products: the
// momentum, the norm of the update, and the scaled update as float16 planes
// in both layouts; and, for matrices with an axis of up to 64, all of it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "op_args.h"
#include "op_moves.h"

namespace gemel {

namespace {

typedef double f64x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf_up(u16 h) { return __uint_as_float((uint32_t)h << 16); }
__device__ __forceinline__ u16 half_down(float f) { return __builtin_bit_cast(u16, (_Float16)f); }
__device__ __forceinline__ float half_up(u16 h) { return (float)__builtin_bit_cast(_Float16, h); }

// The update's value at element i of the batch, once momentum is current.
__device__ __forceinline__ float update_at(const OrthArgs &a, int64_t i) {
    const float g = a.f32 ? ((const float *)a.g)[i] : bf_up(((const u16 *)a.g)[i]);
    if (!a.step) return g;
    return a.nesterov ? g + a.beta * a.m[i] : a.m[i];
}

// Sum over a workgroup of 256, the same order every time; valid in thread 0.
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double part[4];
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return part[0] + part[1] + part[2] + part[3];
}

// 4 consecutive elements of the update from element `at` on; those from
// `left` on are zeros. With a step, momentum is brought up to date first
// (FIRST) and read back later.
template <bool FIRST>
__device__ __forceinline__ f32x4 update4(const OrthArgs &a, int64_t at, int left) {
    f32x4 u = {0.f, 0.f, 0.f, 0.f};
    if (left >= 4) {
        f32x4 g;
        if (a.f32) {
            g = get_f32x4<f32x4>((const float *)a.g + at);
        } else {
            const ushort4 h = get_u16x4((const u16 *)a.g + at);
            g = f32x4{bf_up(h.x), bf_up(h.y), bf_up(h.z), bf_up(h.w)};
        }
        if (!a.step) return g;
        f32x4 m = get_f32x4<f32x4>(a.m + at);
        if (FIRST) {
            m = a.beta * m + g;
            put_f32x4(a.m + at, m);
        }
        return a.nesterov ? g + a.beta * m : m;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= left) continue;
        if (FIRST && a.step) a.m[at + i] = a.beta * a.m[at + i] + ((const float *)a.g)[at + i];
        u[i] = update_at(a, at + i);
    }
    return u;
}

// Momentum and squared sums, 4 elements at a time; reading and writing bounds
// it (4096 x 25088 with momentum 207 us, 1.23 GB, 6 TB/s).
__global__ __launch_bounds__(256) void norm_kernel(const OrthArgs a) {
    const int64_t size = (int64_t)a.rows * a.cols, base = blockIdx.y * size;
    double s = 0.;
#pragma unroll 4
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < size; i += (int64_t)a.parts * 1024) {
        const f32x4 u = update4<true>(a, base + i, (int)min((int64_t)4, size - i));
#pragma unroll
        for (int e = 0; e < 4; ++e) s += (double)u[e] * u[e];
    }
    s = block_sum(s);
    if (threadIdx.x == 0) a.sums[(int64_t)blockIdx.y * a.parts + blockIdx.x] = s;
}

// 64 x 64 tiles, in pairs 4096 x 25088 373 us (1.64 GB, 4.4 TB/s): reads and
// writes bound it. A power of two brings the norm into [0.5, 1), so that bf16
// values stay exact. What is left of the division by norm + 1e-7 is lambda[0],
// in (1, 2] unless the norm is small beside 1e-7: the planes hold X_k /
// lambda[k]. Where lambda[k] < 1/4 the polynomial is nearly its linear term,
// and a factor of 4 goes from the planes to lambda[k + 1], which keeps the
// planes below 1.21 / (1/4).
__global__ __launch_bounds__(256) void seed_kernel(const OrthArgs a) {
    __shared__ float tile[64][65];
    __shared__ int es;
    const int z = blockIdx.z;
    double s = 0.;
    for (int i = threadIdx.x; i < a.parts; i += 256) s += a.sums[(int64_t)z * a.parts + i];
    s = block_sum(s);
    if (threadIdx.x == 0) {
        const double norm = sqrt(s);
        const int e = norm > 0. && isfinite(norm) ? -1 - ilogb(norm) : 0;
        es = e;
        if (blockIdx.x == 0 && blockIdx.y == 0) {
            float l = norm > 0. || norm != norm ? (float)(1. / ldexp(norm + 1e-7, e)) : 1.f;
            for (int k = 0; k <= a.steps; ++k) {
                a.lambda[z * ORTH_LAMBDAS + k] = l;
                if (l < 0.25f) l *= 4.f;
            }
        }
    }
    __syncthreads();
    const int e = es + 13;
    const int c0 = blockIdx.x * 64, r0 = blockIdx.y * 64, x = (threadIdx.x & 15) * 4, y = threadIdx.x >> 4;
    const bool wide = a.rows <= a.cols;
    const Planes &p = wide ? a.x : a.xt, &q = wide ? a.xt : a.x;   // as the input lies, and transposed
    const int64_t base = (int64_t)z * a.rows * a.cols;
    auto put4 = [](const Planes &p, int64_t row, int n, f32x4 v) __attribute__((always_inline)) {
        const int64_t at = row + (p.pair ? pair_at(n) : n);
        const ushort4 h = make_ushort4(half_down(v[0]), half_down(v[1]), half_down(v[2]), half_down(v[3]));
        *(ushort4 *)(p.hi + at) = h;
        if (p.lo)
            *(ushort4 *)(p.lo + at) = make_ushort4(half_down(v[0] - half_up(h.x)), half_down(v[1] - half_up(h.y)),
                                                   half_down(v[2] - half_up(h.z)), half_down(v[3] - half_up(h.w)));
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + y + 16 * i, c = c0 + x;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if (r < a.rows && c < a.cols) v = update4<false>(a, base + (int64_t)r * a.cols + c, min(4, a.cols - c));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = ldexpf(v[k], e);
            tile[y + 16 * i][x + k] = v[k];
        }
        if (r < a.rows && c < p.ld >> p.pair) put4(p, z * p.z + r * p.ld, c, v);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = c0 + y + 16 * i, r = r0 + x;
        const f32x4 v = {tile[x][y + 16 * i], tile[x + 1][y + 16 * i], tile[x + 2][y + 16 * i], tile[x + 3][y + 16 * i]};
        if (c < a.cols && r < q.ld >> q.pair) put4(q, z * q.z + c * q.ld, r, v);
    }
}

// ---- thin matrices: n = min(rows, cols) <= 64 ----
//
// The iterates X_k = P_{k-1}(S_{k-1}) ... X_0 of a wide matrix share their
// row space, and their Gram matrices follow from the first: S_{k+1} = P S_k P
// with P = a I + b S_k + c S_k^2. So X is read twice: once for S_0 = X X^T,
// once for the result (product of all P) X. Small singular values grow up to
// 485 times on the way, and with them what rounding leaves in S_0: with
// float32 sums 1e-7 of S_0 became up to 3e-3 of the result, so S_0 and the
// polynomials are float64 (the f64 matrix cores are idle otherwise, and the
// work is n^2 m + 19 n^3). Three launches: 48 matrices of 16 x 4096 27 us, 1
// of 64 x 4096 74, 48 of 64 x 4096 191; as planes 324, 121 and 379 us. Wider
// ones than 64 would not have their polynomials in one workgroup's LDS.

// Partial Gram matrices. A workgroup takes stretches of 64 positions of the
// long axis through LDS ([n][64] floats, rows 68 apart), its
// 4 waves 16 positions each, and adds the waves' sums at the end. Only tiles
// on and above the diagonal are computed.
template <int NB, bool WIDE>
__global__ __launch_bounds__(256) void thin_gram_kernel(const OrthArgs a) {
    constexpr int NP = 16 * NB, TILES = NB * (NB + 1) / 2;
    __shared__ float us[NP][68];
    __shared__ double sum[16][17];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, l16 = lane & 15;
    const int z = blockIdx.y, n = WIDE ? a.rows : a.cols, m = WIDE ? a.cols : a.rows;
    const int64_t base = (int64_t)z * a.rows * a.cols;
    f64x4 acc[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) acc[t] = f64x4{0., 0., 0., 0.};
    for (int64_t k0 = (int64_t)blockIdx.x * 64; k0 < m; k0 += (int64_t)a.parts * 64) {
        __syncthreads();
        if (WIDE) {
            for (int i = tid; i < NP * 16; i += 256) {
                const int r = i >> 4, c = (i & 15) * 4;
                const f32x4 v = r < n ? update4<true>(a, base + (int64_t)r * a.cols + k0 + c, (int)min((int64_t)4, m - k0 - c))
                                      : f32x4{0.f, 0.f, 0.f, 0.f};
                *(f32x4 *)&us[r][c] = v;
            }
        } else {
            for (int i = tid; i < 64 * NP / 4; i += 256) {
                const int k = i / (NP / 4), c = (i % (NP / 4)) * 4;
                const f32x4 v = k0 + k < m ? update4<true>(a, base + (k0 + k) * a.cols + c, min(4, n - c))
                                           : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 4; ++e) us[c + e][k] = v[e];
            }
        }
        __syncthreads();
        f32x4 f[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) f[b] = *(const f32x4 *)&us[b * 16 + l16][wave * 16 + g * 4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            int t = 0;
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = i; j < NB; ++j, ++t)
                    acc[t] = __builtin_amdgcn_mfma_f64_16x16x4f64((double)f[i][e], (double)f[j][e], acc[t], 0, 0, 0);
        }
    }
    double *out = a.gram + ((int64_t)z * a.parts + blockIdx.x) * NP * NP;
    int t = 0;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = i; j < NB; ++j, ++t) {
            for (int w = 0; w < 4; ++w) {
                __syncthreads();
                if (wave == w)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        double *s = &sum[4 * e + g][l16];
                        *s = w ? *s + acc[t][e] : acc[t][e];
                    }
            }
            __syncthreads();
            const int r = tid >> 4, c = tid & 15;
            out[(i * 16 + r) * NP + j * 16 + c] = sum[r][c];
        }
}

// One workgroup per matrix: the products of symmetric polynomials of one
// matrix commute and are symmetric, so tiles on and above the diagonal
// suffice, and rows serve for columns. A wave for each of these tiles: what
// takes time is the chain of some 20 products, and before it the latency of
// reading the partial Gram matrices, which groups of 256 threads share.
template <int NB>
constexpr int poly_threads() { return NB < 3 ? 256 : NB == 3 ? 512 : 1024; }
template <int NB>
__global__ __launch_bounds__(poly_threads<NB>()) void thin_poly_kernel(const OrthArgs a) {
    constexpr int NP = 16 * NB, TILES = NB * (NB + 1) / 2, LD = NP + 2, NT = poly_threads<NB>(), GROUPS = NT / 256;
    static_assert(GROUPS <= 4 && TILES * 256 <= NP * LD || GROUPS == 1, "a buffer for each group's sums");
    __shared__ double buf[4][NP * LD];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, l16 = lane & 15;
    const int z = blockIdx.x;
    const double *part = a.gram + (int64_t)z * a.parts * NP * NP;
    double *s = buf[0], *p = buf[1], *q = buf[2], *t = buf[3];
    const int group = tid >> 8, in = tid & 255;
    // f(tile, element of S) over a thread's elements
    auto elements = [&](auto &&f) __attribute__((always_inline)) {
        int b = 0;
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = i; j < NB; ++j, ++b) f(b, i * 16 + (in >> 4), j * 16 + (in & 15));
    };
    double v[TILES];
    elements([&](int b, int r, int c) __attribute__((always_inline)) {
        v[b] = 0.;
#pragma unroll 8
        for (int k = group; k < a.parts; k += GROUPS) v[b] += part[(int64_t)k * NP * NP + r * NP + c];
        if (group) buf[group][b * 256 + in] = v[b];
    });
    __syncthreads();
    if (group == 0)
        elements([&](int b, int r, int c) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 1; k < GROUPS; ++k) v[b] += buf[k][b * 256 + in];
            s[r * LD + c] = v[b];
            if (r / 16 < c / 16) s[c * LD + r] = v[b];
        });
    __syncthreads();
    double trace = 0.;
    for (int i = 0; i < NP; ++i) trace += s[i * LD + i];
    __syncthreads();
    const double norm = sqrt(trace), inv = 1. / (norm + 1e-7);
    for (int i = tid; i < NP * LD; i += NT) s[i] = s[i] * inv * inv;
    __syncthreads();
    // out(r, c, sum over k of x[r][k] y[c][k]) for both (r, c) and (c, r)
    auto product = [&](const double *x, const double *y, auto &&out) __attribute__((always_inline)) {
        for (int b = wave; b < TILES; b += NT / 64) {
            int i = 0, j = b;
            while (j >= NB - i) {
                j -= NB - i;
                ++i;
            }
            j += i;
            f64x4 v = {0., 0., 0., 0.};
#pragma unroll
            for (int k = 0; k < NP; k += 4)
                v = __builtin_amdgcn_mfma_f64_16x16x4f64(x[(i * 16 + l16) * LD + k + g], y[(j * 16 + l16) * LD + k + g], v, 0,
                                                         0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = i * 16 + 4 * e + g, c = j * 16 + l16;
                out(r, c, v[e]);
                if (i != j) out(c, r, v[e]);
            }
        }
        __syncthreads();
    };
    for (int k = 0; k < a.steps; ++k) {
        double *const first = k ? p : q;   // the first polynomial is the product so far
        product(s, s, [&](int r, int c, double v) __attribute__((always_inline)) {
            first[r * LD + c] = (r == c ? COEF_A : 0.) + COEF_B * s[r * LD + c] + COEF_C * v;
        });
        if (k) {
            product(p, q, [&](int r, int c, double v) __attribute__((always_inline)) { t[r * LD + c] = v; });
            double *const old = q;
            q = t;
            t = old;
        }
        if (k + 1 < a.steps) {
            product(first, s, [&](int r, int c, double v) __attribute__((always_inline)) { t[r * LD + c] = v; });
            product(t, first, [&](int r, int c, double v) __attribute__((always_inline)) { s[r * LD + c] = v; });
        }
    }
    const int e = norm > 0. && isfinite(norm) ? -1 - ilogb(norm) : 0;
    const double scale = ldexp(inv, -e);
    for (int i = tid; i < NP * NP; i += NT) a.q[(int64_t)z * NP * NP + i] = (float)(q[i / NP * LD + i % NP] * scale);
    if (tid == 0) a.e[z] = e;
}

__device__ __forceinline__ u16 bf_down(float f) { return __builtin_bit_cast(u16, (__bf16)f); }

// out = q (2^e u) for 64 positions of the long axis per workgroup, float32
// products on the float32 matrix cores; bound by the reads of the update and
// the weights and the writes.
template <int NB, bool WIDE>
__global__ __launch_bounds__(256) void thin_apply_kernel(const OrthArgs a) {
    constexpr int NP = 16 * NB;
    __shared__ float us[NP][68], os[NP][68];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, l16 = lane & 15;
    const int z = blockIdx.y, n = WIDE ? a.rows : a.cols, m = WIDE ? a.cols : a.rows;
    const int64_t base = (int64_t)z * a.rows * a.cols, k0 = (int64_t)blockIdx.x * 64;
    const int ex = a.e[z];
    const float *q = a.q + (int64_t)z * NP * NP;
    auto place = [&](int i, int &r, int &c, int64_t &at, int &left) __attribute__((always_inline)) {
        // item i: 4 consecutive elements of a row as it lies in memory
        r = WIDE ? i >> 4 : i / (NP / 4);
        c = (WIDE ? i & 15 : i % (NP / 4)) * 4;
        left = WIDE ? (r < n ? (int)min((int64_t)4, m - k0 - c) : 0) : (k0 + r < m ? min(4, n - c) : 0);
        at = WIDE ? base + (int64_t)r * a.cols + k0 + c : base + (k0 + r) * a.cols + c;
    };
    for (int i = tid; i < NP * 16; i += 256) {
        int r, c, left;
        int64_t at;
        place(i, r, c, at, left);
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if (left > 0) v = update4<false>(a, at, left);
#pragma unroll
        for (int e = 0; e < 4; ++e) (WIDE ? us[r][c + e] : us[c + e][r]) = ldexpf(v[e], ex);
    }
    __syncthreads();
    // wave w: positions 16 w .. 16 w + 15, all n rows
    f32x4 acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = 0; k < NP; k += 4) {
        const float uv = us[k + g][wave * 16 + l16];
#pragma unroll
        for (int b = 0; b < NB; ++b)
            acc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(q[(b * 16 + l16) * NP + k + g], uv, acc[b], 0, 0, 0);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) os[b * 16 + 4 * g + e][wave * 16 + l16] = acc[b][e];
    __syncthreads();
    for (int i = tid; i < NP * 16; i += 256) {
        int r, c, left;
        int64_t at;
        place(i, r, c, at, left);
        if (left <= 0) continue;
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = WIDE ? os[r][c + e] : os[c + e][r];
        float *const f = a.step || a.f32 ? (float *)a.out + at : nullptr;
        u16 *const h = a.step ? (a.copy ? a.copy + at : nullptr) : a.f32 ? nullptr : (u16 *)a.out + at;
        if (left >= 4) {
            if (a.step) v = (1.f - a.decay) * get_f32x4<f32x4>(f) - a.rate * v;
            if (f) put_f32x4(f, v);
            if (h) put_u16x4(h, make_ushort4(bf_down(v[0]), bf_down(v[1]), bf_down(v[2]), bf_down(v[3])));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (e >= left) continue;
                if (a.step) v[e] = (1.f - a.decay) * f[e] - a.rate * v[e];
                if (f) f[e] = v[e];
                if (h) h[e] = bf_down(v[e]);
            }
        }
    }
}

hipError_t launch(const void *fn, dim3 grid, const OrthArgs &a, hipStream_t s, int threads = 256) {
    void *p[] = {const_cast<OrthArgs *>(&a)};
    return hipLaunchKernel(fn, grid, dim3((unsigned)threads), p, 0, s);
}
// f of the number of 16-row blocks, and whether the short axis is the rows
template <typename F>
hipError_t thin(const OrthArgs &a, F &&f) {
    const bool wide = a.rows <= a.cols;
    switch ((std::min(a.rows, a.cols) + 15) / 16) {
        case 1: return f(std::integral_constant<int, 1>{}, wide);
        case 2: return f(std::integral_constant<int, 2>{}, wide);
        case 3: return f(std::integral_constant<int, 3>{}, wide);
        case 4: return f(std::integral_constant<int, 4>{}, wide);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_norm(const OrthArgs &a, hipStream_t s) {
    if (!orth_valid(a, false)) return hipErrorInvalidValue;
    return launch(reinterpret_cast<const void *>(&norm_kernel), dim3((unsigned)a.parts, (unsigned)a.count), a, s);
}

hipError_t launch_seed(const OrthArgs &a, hipStream_t s) {
    if (!orth_valid(a, false)) return hipErrorInvalidValue;
    return launch(reinterpret_cast<const void *>(&seed_kernel),
                  dim3((unsigned)((a.cols + 63) / 64), (unsigned)((a.rows + 63) / 64), (unsigned)a.count), a, s);
}

hipError_t launch_thin_gram(const OrthArgs &a, hipStream_t s) {
    if (!orth_valid(a, true)) return hipErrorInvalidValue;
    return thin(a, [&](auto nb, bool wide) {
        constexpr int NB = decltype(nb)::value;
        return launch(wide ? reinterpret_cast<const void *>(&thin_gram_kernel<NB, true>)
                           : reinterpret_cast<const void *>(&thin_gram_kernel<NB, false>),
                      dim3((unsigned)a.parts, (unsigned)a.count), a, s);
    });
}

hipError_t launch_thin_poly(const OrthArgs &a, hipStream_t s) {
    if (!orth_valid(a, true)) return hipErrorInvalidValue;
    return thin(a, [&](auto nb, bool) {
        constexpr int NB = decltype(nb)::value;
        return launch(reinterpret_cast<const void *>(&thin_poly_kernel<NB>), dim3((unsigned)a.count), a, s,
                      poly_threads<NB>());
    });
}

hipError_t launch_thin_apply(const OrthArgs &a, hipStream_t s) {
    if (!orth_valid(a, true)) return hipErrorInvalidValue;
    return thin(a, [&](auto nb, bool wide) {
        constexpr int NB = decltype(nb)::value;
        return launch(wide ? reinterpret_cast<const void *>(&thin_apply_kernel<NB, true>)
                           : reinterpret_cast<const void *>(&thin_apply_kernel<NB, false>),
                      dim3((unsigned)((std::max(a.rows, a.cols) + 63) / 64), (unsigned)a.count), a, s);
    });
}

}  // namespace gemel

// Answers off rows of logits: log probability and rank of a label, entropy,
// the best classes; and the loss of a student against a teacher's best logits
// with its gradient.
//
// With c = log2(e) / T and t_i = (z_i - m) c, m the row's largest logit, every
// result follows from S = sum 2^t_i and A = sum 2^t_i t_i:
//   log sum = m / T + ln 2 log2 S,  log p_i = (z_i - m) / T - ln 2 log2 S,
//   entropy = ln 2 (log2 S - A / S).
//
// A row is held in registers by a team of waves, each lane pieces of 16 bytes
// of it, so that it is read once; rows that no team can hold are cut into
// chunks whose sums and best classes a second launch joins.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "answer_args.h"
#include "op_moves.h"

namespace gemel {

namespace {

typedef unsigned short u16;
typedef unsigned long long u64;
constexpr float LN2 = 0.693147180559945309417f;

__device__ __forceinline__ float infinity() { return __builtin_inff(); }
__device__ __forceinline__ float quiet() { return __builtin_nanf(""); }

// a, b, c: the largest; of a NaN and a number the number (fmaxf would first
// bring every operand into canonical form)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Reductions over a wave: rows of 16 lanes, then between them; every lane
// gets the result.
template <int CTRL, typename T>
__device__ __forceinline__ T moved(T none, T v) {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CTRL, 0xf,
                                                             0xf, false));
}
template <typename T, typename F>
__device__ __forceinline__ T wave_reduce(T v, T none, F f) {
    v = f(v, moved<0x111>(none, v));   // row_shr 1, 2, 4, 8
    v = f(v, moved<0x112>(none, v));
    v = f(v, moved<0x114>(none, v));
    v = f(v, moved<0x118>(none, v));
    v = f(v, moved<0x142>(none, v));   // row_bcast 15, 31
    v = f(v, moved<0x143>(none, v));
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float wave_max(float v) {
    return wave_reduce(v, -infinity(), [](float a, float b) { return max3(a, b, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
    return wave_reduce(v, 0.f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ int wave_sum(int v) {
    return wave_reduce(v, 0, [](int a, int b) { return a + b; });
}
__device__ __forceinline__ int wave_min(int v) {
    return wave_reduce(v, 0x7fffffff, [](int a, int b) { return min(a, b); });
}

// What a team of W waves shares is written before and read after this.
template <int W>
__device__ __forceinline__ void team_sync() {
    if constexpr (W == 1) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    } else {
        __syncthreads();
    }
}

// Classes [lo, hi) of a row in the registers of T threads: piece v of a lane begins
// at class at(v). A piece that would pass the end is moved back to end there,
// and what the piece before it holds already is -inf in it. The last L pieces
// stay in LDS between their uses.
template <bool F32, int T, int V, int L = 0>
struct Held {
    static constexpr int VEC = F32 ? 4 : 8, SIZE = F32 ? 4 : 2;
    uint4 raw[V];
    int lo, hi, tid;
    uint4 (*parked)[T];

    __device__ __forceinline__ int first(int v) const { return lo + (v * T + tid) * VEC; }
    __device__ __forceinline__ int at(int v) const { return hi - lo < VEC ? first(v) : min(first(v), hi - VEC); }
    __device__ __forceinline__ float get(int v, int j) const {
        if constexpr (F32)
            return __uint_as_float((&raw[v].x)[j]);
        else
            return __uint_as_float(j & 1 ? (&raw[v].x)[j / 2] & 0xffff0000u : (&raw[v].x)[j / 2] << 16);
    }
    // The first n elements of piece v become -inf.
    __device__ __forceinline__ void mask(int v, int n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t &x = (&raw[v].x)[i];
            if constexpr (F32)
                x = n > i ? 0xff800000u : x;
            else
                x = n > 2 * i + 1 ? 0xff80ff80u : n > 2 * i ? (x & 0xffff0000u) | 0xff80u : x;
        }
    }
    // Before piece v is used: what was made of it earlier is made again, and
    // nothing is made of it ahead (the compiler would keep every bf16 unpacked,
    // or every exponential, in several times the registers). The sums or stores
    // of the piece before are done first.
    __device__ __forceinline__ void again(int v) {
        if constexpr (L > 0)
            if (v >= V - L) raw[v] = parked[v - (V - L)][tid];
        asm volatile("" : "+v"(raw[v].x), "+v"(raw[v].y), "+v"(raw[v].z), "+v"(raw[v].w)::"memory");
    }
    __device__ __forceinline__ void park(int v) {
        if constexpr (L > 0)
            if (v >= V - L) parked[v - (V - L)][tid] = raw[v];
    }
    __device__ __forceinline__ void again(int v, float &s, float &a) {
        if constexpr (L > 0)
            if (v >= V - L) raw[v] = parked[v - (V - L)][tid];
        asm volatile("" : "+v"(raw[v].x), "+v"(raw[v].y), "+v"(raw[v].z), "+v"(raw[v].w), "+v"(s), "+v"(a));
    }
    __device__ __forceinline__ void load(const char *row, int lo_, int hi_, int tid_) {
        lo = lo_;
        hi = hi_;
        tid = tid_;
        if (hi - lo < VEC) {   // fewer classes than a piece
#pragma unroll
            for (int v = 0; v < V; ++v) mask(v, VEC);
            if (tid == 0)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    if (lo + j >= hi) continue;
                    if constexpr (F32)
                        (&raw[0].x)[j] = *(const uint32_t *)(row + (lo + j) * 4);
                    else
                        (&raw[0].x)[j / 2] = ((&raw[0].x)[j / 2] & (j & 1 ? 0xffffu : 0xffff0000u)) |
                                             (uint32_t) * (const u16 *)(row + (lo + j) * 2) << (j & 1) * 16;
                }
            return;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) raw[v] = get_16b(row + (uint32_t)at(v) * SIZE);
        const int next = T < 64 ? T : (tid & ~63) + 64;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (lo + (v * T + next) * VEC > hi) mask(v, first(v) - at(v));
    }
};

__device__ __forceinline__ float logit(const Logits &l, const char *row, int i) {
    return l.f32 ? *(const float *)(row + (int64_t)i * 4) : __uint_as_float((uint32_t) * (const u16 *)(row + (int64_t)i * 2) << 16);
}

// Sums of two parts of a row together.
__device__ __forceinline__ Part joined(const Part &x, const Part &y, float c) {
    Part p;
    p.before = x.before + y.before;
    // (NaN sums are not empty)
    if (x.s == 0.f) return Part{y.m, y.s, y.a, p.before};
    if (y.s == 0.f) return Part{x.m, x.s, x.a, p.before};
    p.m = max3(x.m, y.m, y.m);
    const float dx = (x.m - p.m) * c, dy = (y.m - p.m) * c;
    const float fx = __builtin_amdgcn_exp2f(dx), fy = __builtin_amdgcn_exp2f(dy);
    p.s = x.s * fx + y.s * fy;
    // (what is 2^-127 of the other leaves nothing, however far it is away)
    p.a = (fx > 0.f ? (x.a + dx * x.s) * fx : 0.f) + (fy > 0.f ? (y.a + dy * y.s) * fy : 0.f);
    return p;
}

// Largest elements of a lane's groups: pieces, or parts of the only one or two.
template <bool F32, int V>
struct Groups {
    static constexpr int SUB = V == 1 ? (F32 ? 2 : 4) : V == 2 ? 2 : 1, N = V * SUB, SIZE = (F32 ? 4 : 8) / SUB;
    float most[N];
};

// Sums of the elements that a wave holds (a: only with A).
//
// Where m c is of ordinary size t = z c - r, r being m c rounded, is one
// operation instead of two; its sums are then those for m but for a factor of
// 2^d, d = m c - r. (Elements that are far apart would lose bits there.)
template <bool A, bool F32, int T, int V, int L>
__device__ __forceinline__ Part wave_part(Held<F32, T, V, L> &h, float c, Groups<F32, V> &most) {
    constexpr int VEC = Held<F32, T, V>::VEC;
    using G = Groups<F32, V>;
    static_assert(!L || G::SUB == 1, "parked pieces are groups");
    float m = -infinity();
#pragma unroll
    for (int g = 0; g < G::N; ++g) {
        float &x = most.most[g];
        x = -infinity();
#pragma unroll
        for (int j = 0; j < G::SIZE; j += 2) {
            const int v = g / G::SUB, k = g % G::SUB * G::SIZE + j;
            x = max3(x, h.get(v, k), h.get(v, k + 1));
        }
        m = max3(m, x, x);
        h.park(g);
    }
    m = wave_max(m);
    const float ref = m == -infinity() ? 0.f : m, r = ref * c;
    float s = 0.f, a = 0.f;
    auto sums = [&](auto one) __attribute__((always_inline)) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            h.again(v, s, a);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float t = decltype(one)::value ? __builtin_fmaf(h.get(v, j), c, -r) : (h.get(v, j) - ref) * c;
                const float e = __builtin_amdgcn_exp2f(t);
                s += e;
                // (0 times -inf, a masked class's, has to be nothing)
                if constexpr (A) a = __builtin_fmaf(e, fmaxf(t, -1e30f), a);
            }
        }
    };
    if (fabsf(r) < 0x1p16f) {
        sums(std::true_type{});
        const float d = __builtin_fmaf(ref, c, -r), f = __builtin_amdgcn_exp2f(-d);
        a = (a - d * s) * f;
        s *= f;
    } else {
        sums(std::false_type{});
    }
    return Part{m, wave_sum(s), A ? wave_sum(a) : 0.f, 0};
}

// The team's sums from those of its waves, in every lane.
template <int W>
__device__ __forceinline__ Part team_part(Part p, Part *shared, int wave, float c) {
    if constexpr (W == 1) return p;
    if ((threadIdx.x & 63) == 0) shared[wave] = p;
    __syncthreads();
    Part sum = shared[0];
#pragma unroll
    for (int w = 1; w < W; ++w) sum = joined(sum, shared[w], c);
    return sum;
}

// A row's sums from those of its chunks, one to a lane, in every lane.
__device__ __forceinline__ Part chunks_part(const Part *part, int chunks, float c) {
    const int lane = threadIdx.x & 63;
    Part p = part[min(lane, chunks - 1)];
    const bool there = lane < chunks;
    // (NaN sums stay, whatever their reference is; an empty chunk adds nothing)
    const float m = wave_max(there ? p.m : -infinity()), d = p.s == 0.f ? 0.f : (p.m - m) * c, f = __builtin_amdgcn_exp2f(d);
    Part q;
    q.m = m;
    q.s = wave_sum(there ? p.s * f : 0.f);
    q.a = wave_sum(there && f > 0.f ? (p.a + d * p.s) * f : 0.f);
    q.before = wave_sum(there ? p.before : 0);
    return q;
}

// Half the distance of a and b: that of finite ones is finite.
__device__ __forceinline__ float half_of(float a, float b) { return 0.5f * a - 0.5f * b; }

// Loss of a row, which is 2 T times the sum of these over its entries: the
// share q of an entry times half of T (log q - log p), with half the
// distances of the teacher's value and of the logit from their row's largest,
// and half of T (ln mass - ln S). (Divided by T instead, distances would
// overflow in losses that do not.)
__device__ __forceinline__ float loss_part(float share, float half_v, float half_z, float half_sums) {
    return share > 0.f ? share * (half_v - half_z - half_sums) : 0.f;
}

struct Results {
    bool lost;      // some logit is NaN or +inf
    float log2_s;
};
__device__ __forceinline__ Results results(const Part &p) { return {!(p.s < infinity()), log2f(p.s)}; }
__device__ __forceinline__ float log_prob(const Part &p, const Results &q, float z, float inv_t) {
    if (q.lost) return quiet();
    return z == -infinity() || p.s == 0.f ? -infinity() : half_of(z, p.m) * (2.f * inv_t) - LN2 * q.log2_s;
}
// One row's outputs but for the list.
__device__ __forceinline__ void put_row(const ScoreArgs &a, int row, const Part &p, int label, float z_label) {
    const Results q = results(p);
    if (a.entropy) {
        const float h = LN2 * (q.log2_s - p.a / p.s);
        a.entropy[row] = q.lost ? quiet() : p.s == 0.f || h < 0.f ? 0.f : h;
    }
    if (a.log_sum) a.log_sum[row] = q.lost ? quiet() : p.s == 0.f ? -infinity() : p.m * a.l.inv_t + LN2 * q.log2_s;
    const bool in = label >= 0 && label < a.l.classes;
    if (a.log_prob) a.log_prob[row] = label == -1 ? 0.f : in ? log_prob(p, q, z_label, a.l.inv_t) : quiet();
    if (a.rank) a.rank[row] = in && !q.lost ? p.before : -1;
}
__device__ __forceinline__ void put_top(const ScoreArgs &a, int row, int i, const Part &p, const Results &q, float z, int index) {
    const int64_t at = (int64_t)row * a.top + i;
    if (a.top_index) a.top_index[at] = q.lost ? -1 : index;
    if (a.top_log_prob) a.top_log_prob[at] = q.lost ? quiet() : index < 0 ? -infinity() : log_prob(p, q, z, a.l.inv_t);
}

struct Best {
    float z;
    int i;
};
// A value and its class as one number: larger for what comes first.
__device__ __forceinline__ u64 key_of(float z, int index) {
    const uint32_t u = __float_as_uint(z + 0.f);   // (-0 is 0)
    const uint32_t k = u & 0x80000000u ? ~u : u | 0x80000000u;
    return index < 0 ? 0 : (u64)k << 32 | (uint32_t)~index;
}
__device__ __forceinline__ Best of_key(u64 key) {
    const uint32_t k = (uint32_t)(key >> 32);
    return key ? Best{__uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k), (int)~(uint32_t)key} : Best{-infinity(), -1};
}

// Order of floats as whole numbers.
__device__ __forceinline__ uint32_t ordered(float z) {
    const uint32_t u = __float_as_uint(z);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// The least value (in the order of `ordered`) that is known to be reached by
// `top` of N values in each lane, and few more: between lo, which enough
// reach, and hi, by halves.
template <int N>
__device__ __forceinline__ uint32_t reached(const uint32_t (&k)[N], uint32_t lo, uint32_t hi, int top) {
    while (hi - lo > 1) {
        const uint32_t t = lo + (hi - lo) / 2;
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k[i] >= t));
        if (n >= top)
            lo = t;
        else
            hi = t;
        if (n >= top && n <= top + top / 4) break;
    }
    return lo;
}
// Values that at least `top` and `part` of the wave's elements reach, and few
// more: ones that as many of its lanes' groups reach with their largest
// (-inf where there are not as many).
template <int N>
__device__ __forceinline__ void wave_reach(const float (&most)[N], float m, int top, int part, float &all, float &some) {
    uint32_t k[N], least = 0xffffffffu;
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        k[i] = ordered(most[i]);
        const bool there = most[i] > -infinity();
        least = min(least, there ? k[i] : 0xffffffffu);
        n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(there));
    }
    least = __builtin_bit_cast(uint32_t, wave_min(__builtin_bit_cast(int, least ^ 0x80000000u))) ^ 0x80000000u;
    all = some = -infinity();
    if (n < part) return;
    const uint32_t hi = ordered(m) + 1;
    uint32_t lo = least;
    if (n >= top) {
        lo = reached(k, lo, hi, top);
        all = from_ordered(lo);
    }
    some = part < top ? from_ordered(reached(k, lo, hi, part)) : all;
}

// Entries of a wave's list of candidates for the best classes.
constexpr int CANDIDATES = 256;

// The best classes of a row (or chunk) are found among the elements that
// reach the largest of the waves' values of wave_reach: each counts the ones
// before it. Where ties leave more candidates than there is room for, the
// best class behind the last one is searched `top` times.
//
// What bounds it: about 600 vector instructions for the 2048 elements of a
// wave (one exponential each) beside reading them, 866 with the 20 best, 1296
// with 64; short rows, those that a row needs once. 2048 rows of 100003 bf16
// with their 20 best: searched one after the other 1480 us, as candidates 278,
// in chunks of 4 waves instead of 8 with twice the elements 147 (the sums alone
// 95, reading 80); 16384 rows of 1001 with 5: 34 and 18 us.
template <bool F32, int W, int V>
__global__ __launch_bounds__((W == 1 ? 256 : W * 64), V < 8 ? 8 : 4) void score_kernel(const ScoreArgs a) {
    constexpr int VEC = F32 ? 4 : 8, TEAMS = answer_teams(W);
    __shared__ Part parts[W];
    __shared__ Best best[W];
    __shared__ u64 list[TEAMS * W][CANDIDATES];
    __shared__ float reaches[W], part_reaches[W];
    __shared__ int counts[W];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int team = W == 1 ? wave : 0, w = W == 1 ? 0 : wave, tid = W == 1 ? lane : (int)threadIdx.x;
    const int row = (int)blockIdx.x * TEAMS + team, chunk = blockIdx.y;
    if (row >= a.l.rows) return;   // (a wave of its own: no barrier waits for it)
    const int64_t unit = (int64_t)row * a.l.chunks + chunk;
    const char *z = (const char *)a.l.z + (int64_t)row * a.l.ld * (F32 ? 4 : 2);
    const int lo = chunk * a.l.chunk, hi = min(a.l.classes, lo + a.l.chunk);
    const int label = a.labels ? a.labels[row] : -1;
    const bool in = label >= 0 && label < a.l.classes;
    Held<F32, W * 64, V> h;
    h.load(z, lo, hi, tid);
    const float z_label = in ? logit(a.l, z, label) : 0.f;
    // the classes before the label in its piece, one for each lane
    const int piece = in ? label - (label - lo) % VEC : 0;
    const bool here = a.rank && in && w == 0 && label >= lo && label < hi;
    const float near = here && piece + lane < label ? logit(a.l, z, piece + lane) : quiet();
    Groups<F32, V> most;
    Part p = wave_part<true>(h, a.l.c, most);
    if (a.rank && in) {
        int n = 0;
        if (z_label > -infinity()) {
            // in pieces before the label's equal ones count too: what is above
            // the next smaller float
            const uint32_t u = __float_as_uint(z_label);
            const float below = __uint_as_float(z_label == 0.f ? 0x80000001u : u & 0x80000000u ? u + 1 : u - 1);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float t = h.first(v) + VEC <= label ? below : z_label;
                h.again(v);
#pragma unroll
                for (int j = 0; j < VEC; ++j) n += h.get(v, j) > t;
            }
            p.before = wave_sum(n) + __builtin_popcountll(__builtin_amdgcn_ballot_w64(near == z_label));
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int b = h.at(v), f = h.first(v);
                h.again(v);
#pragma unroll
                for (int j = 0; j < VEC; ++j) n += h.get(v, j) > -infinity() || (b + j < min(label, hi) && b + j >= f);
            }
            p.before = wave_sum(n);
        }
    }
    // what every wave's share of the best classes reaches is reached by `top`
    // of the team's elements, and so is what `top` of a single wave's reach
    float reach = 0.f, part_reach = 0.f;
    if (a.top) {
        const int part = (a.top + W - 1) / W;
        using G = Groups<F32, V>;
        if (a.top <= 24 && hi - lo >= 4 * VEC * a.top) {   // (fine groups where lanes are few)
            float x[1] = {most.most[0]};
#pragma unroll
            for (int i = 1; i < G::N; ++i) x[0] = max3(x[0], most.most[i], most.most[i]);
            wave_reach(x, p.m, a.top, part, reach, part_reach);
        } else {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = i < G::N ? most.most[i] : -infinity();
#pragma unroll
            for (int i = 4; i < G::N; ++i) x[i % 4] = max3(x[i % 4], most.most[i], most.most[i]);
            wave_reach(x, p.m, a.top, part, reach, part_reach);
        }
    }
    if constexpr (W > 1)
        if (lane == 0) {
            reaches[w] = reach;
            part_reaches[w] = part_reach;
        }
    p = team_part<W>(p, parts, w, a.l.c);   // (a barrier)
    const Results q = results(p);
    if (tid == 0) {
        if (a.l.chunks > 1)
            a.part[unit] = p;
        else
            put_row(a, row, p, label, z_label);
    }
    if (!a.top) return;
    auto put = [&](int i, const Best &b) __attribute__((always_inline)) {
        if (a.l.chunks > 1) {
            a.list_value[unit * a.top + i] = b.z;
            a.list_index[unit * a.top + i] = b.i;
        } else {
            put_top(a, row, i, p, q, b.z, b.i);
        }
    };
    if constexpr (W > 1) {
        part_reach = part_reaches[0];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            reach = max3(reach, reaches[i], reaches[i]);
            part_reach = fminf(part_reach, part_reaches[i]);
        }
        reach = max3(reach, part_reach, part_reach);
    }
    reach = max3(reach, -3.402823466e38f, -3.402823466e38f);   // (classes not offered are no candidates)
    u64 *const mine = list[team * W + w];
    int n = 0;
    if (!q.lost) {   // (chunks: another one may be; the join sees to that)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            using G = Groups<F32, V>;
            float m = most.most[v * G::SUB];
#pragma unroll
            for (int i = 1; i < G::SUB; ++i) m = max3(m, most.most[v * G::SUB + i], most.most[v * G::SUB + i]);
            if (!__builtin_amdgcn_ballot_w64(m >= reach)) continue;
            const int at = h.at(v);
            h.again(v);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float x = h.get(v, j);
                const u64 who = __builtin_amdgcn_ballot_w64(x >= reach);
                if (who) {
                    const int place = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
                    if (x >= reach && place < CANDIDATES) mine[place] = key_of(x, at + j);
                    n += __builtin_popcountll(who);
                }
            }
        }
    }
    if constexpr (W > 1)
        if (lane == 0) counts[w] = n;
    team_sync<W>();
    int total = n, largest = n;
    if constexpr (W > 1) {
        total = largest = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            total += counts[i];
            largest = max(largest, counts[i]);
        }
    }
    if (largest <= CANDIDATES) {
        for (int i = tid; i < total; i += W * 64) {
            int at = i, which = 0;
            if constexpr (W > 1)
#pragma unroll
                for (int l = 0; l + 1 < W; ++l)
                    if (which == l && at >= counts[l]) {
                        at -= counts[l];
                        ++which;
                    }
            const u64 key = list[team * W + which][at];
            int before = 0;
            for (int l = 0; l < W; ++l) {
                const u64 *const other = list[team * W + l];
                const int m = W == 1 ? n : counts[l];
#pragma unroll 4
                for (int k = 0; k < m; ++k) before += other[k] > key;
            }
            if (before < a.top) put(before, of_key(key));
        }
        for (int i = total + tid; i < a.top; i += W * 64) put(i, Best{-infinity(), -1});
        return;
    }
    Best last{infinity(), -1};
    for (int k = 0; k < a.top; ++k) {
        Best b{-infinity(), -1};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = h.at(v);
            h.again(v);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float x = h.get(v, j);
                if (x > b.z && (x < last.z || (x == last.z && at + j > last.i))) b = Best{x, at + j};
            }
        }
        const float top = wave_max(b.z);
        b.i = wave_min(b.z == top && b.i >= 0 ? b.i : 0x7fffffff);
        b.z = top;
        if constexpr (W > 1) {
            __syncthreads();
            if (lane == 0) best[w] = b;
            __syncthreads();
            b = best[0];
#pragma unroll
            for (int i = 1; i < W; ++i) {
                const Best o = best[i];
                if (o.z > b.z || (o.z == b.z && o.i < b.i)) b = o;
            }
        }
        last = b;
        if (tid == 0) put(k, b);
    }
}

// One row for each workgroup: the sums of its chunks, and the best of their
// lists.
constexpr int KEPT = 512;
template <int N>   // entries of the lists
__global__ __launch_bounds__(256) void score_join_kernel(const ScoreArgs a) {
    __shared__ u64 keys[N], kept[KEPT];
    __shared__ int left;
    const int row = blockIdx.x, tid = threadIdx.x, chunks = a.l.chunks, n = chunks * a.top;
    const int64_t at = (int64_t)row * chunks;
    const Part p = chunks_part(a.part + at, chunks, a.l.c);
    const Results q = results(p);
    if (tid == 0) {
        const int label = a.labels ? a.labels[row] : -1;
        const char *z = (const char *)a.l.z + (int64_t)row * a.l.ld * (a.l.f32 ? 4 : 2);
        put_row(a, row, p, label, label >= 0 && label < a.l.classes ? logit(a.l, z, label) : 0.f);
    }
    if (tid == 0) left = 0;
    for (int i = tid; i < n; i += 256) keys[i] = key_of(a.list_value[at * a.top + i], a.list_index[at * a.top + i]);
    __syncthreads();
    // what the last entry of any list reaches is a bound on the row's last, and
    // so is what every list's share of the best reaches: few are left, and each
    // counts the ones before it (many only where few lists hold all of the best)
    u64 least = 1, shares = ~0ull;
    const int part = (a.top + chunks - 1) / chunks;
    for (int l = 0; l < chunks && a.top; ++l) {
        const u64 last = keys[l * a.top + a.top - 1], share = keys[l * a.top + part - 1];
        least = last > least ? last : least;
        shares = share < shares ? share : shares;
    }
    least = shares > least ? shares : least;
    for (int i = tid; i < n; i += 256) {
        const u64 key = keys[i];
        if (key < least) continue;
        const int at = atomicAdd(&left, 1);
        if (at < KEPT) kept[at] = key;
    }
    __syncthreads();
    const int total = left;
    auto place = [&](u64 key, int before) __attribute__((always_inline)) {
        if (before >= a.top) return;
        const Best b = of_key(key);
        put_top(a, row, before, p, q, b.z, b.i);
    };
    if (total <= KEPT) {
        for (int i = tid; i < total; i += 256) {
            const u64 key = kept[i];
            int before = 0;
#pragma unroll 4
            for (int k = 0; k < total; ++k) before += kept[k] > key;
            place(key, before);
        }
    } else {
        for (int i = tid; i < n; i += 256) {
            const u64 key = keys[i];
            if (key < least) continue;
            int before = 0;
            for (int l = 0; l < chunks && before < a.top; ++l) {
                int x = 0, y = a.top;   // entries of the (sorted) list that come before
                while (x < y) {
                    const int m = (x + y) >> 1;
                    if (keys[l * a.top + m] > key)
                        x = m + 1;
                    else
                        y = m;
                }
                before += x;
            }
            place(key, before);
        }
    }
    // places that no class takes
    if (tid < a.top && tid >= total) put_top(a, row, tid, p, q, -infinity(), -1);
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    return (uint32_t)__builtin_bit_cast(u16, (__bf16)a) | (uint32_t)__builtin_bit_cast(u16, (__bf16)b) << 16;
}

// q = softmax of the teacher's entries v / T, p that of all of the student's
// logits z / T: loss = T^2 sum q (log q - log p), and with respect to z
//   dz = dloss T (p - q),
// entries of one class added up. Every wave of a team keeps entry i in lane
// i. What bounds it: reading and writing, which overlap only between the
// workgroups of a compute unit: 4096 rows of 65537 bf16 take 302 us where one
// fits (all pieces in registers), 245 where two do (4 of 9 pieces in LDS);
// a copy of as many bytes 201. What a lane writes for a class with an entry it overwrites itself, so
// that the order of the two stores is that of the program.
template <bool F32, int W, int V, int L = 0>
__global__ __launch_bounds__((W == 1 ? 256 : W * 64), 8) void distill_kernel(const DistillArgs a) {
    constexpr int VEC = F32 ? 4 : 8, TEAMS = answer_teams(W), SIZE = F32 ? 4 : 2;
    __shared__ Part parts[W];
    __shared__ uint4 parked[L ? L : 1][L ? W * 64 : 1];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int team = W == 1 ? wave : 0, w = W == 1 ? 0 : wave, tid = W == 1 ? lane : (int)threadIdx.x;
    const int row = (int)blockIdx.x * TEAMS + team, chunk = blockIdx.y;
    if (row >= a.l.rows) return;
    const char *z = (const char *)a.l.z + (int64_t)row * a.l.ld * SIZE;
    const int lo = chunk * a.l.chunk, hi = min(a.l.classes, lo + a.l.chunk);
    int index = -1;
    float value = 0.f;
    if (lane < a.k) {
        index = a.index[(int64_t)row * a.k + lane];
        value = a.value[(int64_t)row * a.k + lane];
    }
    const float weight = a.dloss ? a.dloss[row] : 1.f;
    Held<F32, W * 64, V, L> h;
    if constexpr (L > 0) h.parked = parked;
    h.load(z, lo, hi, tid);
    const bool bad = __builtin_amdgcn_ballot_w64(index < -1 || index >= a.l.classes) != 0;
    if (index >= a.l.classes) index = -1;
    const bool entry = index >= 0;
    const float z_entry = entry ? logit(a.l, z, index) : 0.f;
    // the teacher's side, like the student's the distance from the largest
    // value first, then scaled (finite values do not overflow); a value that is
    // NaN or +inf makes the mass NaN
    const float v = entry ? value : -infinity();
    const float v_most = wave_max(v), far = (v - (v_most == -infinity() ? 0.f : v_most)) * a.l.inv_t;
    const bool some = bad || __builtin_amdgcn_ballot_w64(!(v == -infinity())) != 0;
    const float e = entry ? expf(far) : 0.f;
    float mass = wave_sum(e);
    if (bad) mass = quiet();
    const float share = e / mass;
    Part p;
    Groups<F32, V> most;
    if (a.l.chunks > 1) {
        p = chunks_part(a.part + (int64_t)row * a.parts, a.parts, a.l.c);
    } else {
        p = team_part<W>(wave_part<false>(h, a.l.c, most), parts, w, a.l.c);
    }
    const bool lost = !(p.s < infinity()) || p.s == 0.f || mass != mass;
    const float t_entry = (z_entry - p.m) * a.l.c;
    if (a.loss && w == 0 && chunk == 0) {
        const float half_sums = 0.5f * a.t * (logf(mass) - LN2 * log2f(p.s));
        const float sum = wave_sum(loss_part(share, half_of(v, v_most), half_of(z_entry, p.m), half_sums));
        if (lane == 0) a.loss[row] = !some ? 0.f : lost ? quiet() : 2.f * a.t * sum;
    }
    if (!a.dz) return;
    char *const d = (char *)a.dz + (int64_t)row * a.ldd * SIZE;
    auto put = [](char *d, int i, float g) __attribute__((always_inline)) {
        if constexpr (F32)
            *(float *)(d + (uint32_t)i * 4) = g;
        else
            *(u16 *)(d + (uint32_t)i * 2) = __builtin_bit_cast(u16, (__bf16)g);
    };
    // (a row without entries gives nothing, whatever it holds)
    const float coef = !some ? 0.f : lost ? quiet() : weight * a.t, by = coef / p.s;
    auto gradient = [&](float x) __attribute__((always_inline)) {
        return some ? by * __builtin_amdgcn_exp2f((x - p.m) * a.l.c) : 0.f;
    };
#pragma unroll
    for (int v = 0; v < V; ++v) {
        h.again(v);
        uint4 x;
        if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) (&x.x)[j] = __float_as_uint(gradient(h.get(v, j)));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) (&x.x)[j] = pack2(gradient(h.get(v, 2 * j)), gradient(h.get(v, 2 * j + 1)));
        }
        const int f = h.first(v);
        if (f + VEC <= hi) *(u32x4_any *)(d + (uint32_t)f * SIZE) = __builtin_bit_cast(u32x4_any, x);
    }
    __builtin_amdgcn_sched_barrier(0);
    // the last classes, where they do not fill a piece
    const int tail = lo + (hi - lo) / VEC * VEC;
    if (tid == (hi - lo) / VEC % (W * 64))
#pragma unroll 1
        for (int i = tail; i < hi; ++i) put(d, i, gradient(logit(a.l, z, i)));
    if (!some) return;
    // this wave's classes with an entry
    const int piece = entry ? (index - lo) / VEC % (W * 64) : -1;
    u64 mine = __builtin_amdgcn_ballot_w64(entry && index >= lo && index < hi && piece >> 6 == w);
    while (mine) {
        const int i = __builtin_ctzll(mine);
        mine &= mine - 1;
        const int cls = __builtin_amdgcn_readlane(index, i), owner = __builtin_amdgcn_readlane(piece, i) & 63;
        const float q = wave_sum(index == cls ? share : 0.f);
        const float t = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(t_entry), i));
        const float g = by * __builtin_amdgcn_exp2f(t) - coef * q;
        if (lane == owner) put(d, cls, g);
    }
}

// ---- rows of few classes: 16 lanes to a row, 4 rows to a wave ----
//
// A wave to a row leaves most lanes idle and repeats what is done once for
// each row: 97344 rows of 80 float32 classes, loss and gradient of 10 entries,
// 60 us against 17 (reading and writing take 14).

// Reductions over 16 lanes, by rotation: every lane gets the same bits.
template <typename T, typename F>
__device__ __forceinline__ T row_reduce(T v, F f) {
    v = f(v, moved<0x128>(v, v));   // row_ror 8, 4, 2, 1
    v = f(v, moved<0x124>(v, v));
    v = f(v, moved<0x122>(v, v));
    return f(v, moved<0x121>(v, v));
}
__device__ __forceinline__ float row_max(float v) {
    return row_reduce(v, [](float a, float b) { return max3(a, b, b); });
}
__device__ __forceinline__ float row_sum(float v) {
    return row_reduce(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ int row_sum(int v) {
    return row_reduce(v, [](int a, int b) { return a + b; });
}
__device__ __forceinline__ int row_min(int v) {
    return row_reduce(v, [](int a, int b) { return min(a, b); });
}

// Sums of a row that 16 lanes hold.
template <bool A, bool F32, int V>
__device__ __forceinline__ Part row_part(const Held<F32, 16, V> &h, float c) {
    constexpr int VEC = Held<F32, 16, V>::VEC;
    float m = -infinity(), s = 0.f, a = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < VEC; j += 2) m = max3(m, h.get(v, j), h.get(v, j + 1));
    m = row_max(m);
    const float ref = m == -infinity() ? 0.f : m;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float t = (h.get(v, j) - ref) * c;
            const float e = __builtin_amdgcn_exp2f(t);
            s += e;
            if constexpr (A) a = __builtin_fmaf(e, fmaxf(t, -1e30f), a);
        }
    return Part{m, row_sum(s), A ? row_sum(a) : 0.f, 0};
}

template <bool F32, int V>
__global__ __launch_bounds__(256) void score_small_kernel(const ScoreArgs a) {
    constexpr int VEC = F32 ? 4 : 8;
    const int lane = threadIdx.x & 15, at_row = blockIdx.x * 16 + (threadIdx.x >> 4), row = min(at_row, a.l.rows - 1);
    const bool there = at_row < a.l.rows;
    const char *z = (const char *)a.l.z + (int64_t)row * a.l.ld * (F32 ? 4 : 2);
    const int label = a.labels ? a.labels[row] : -1;
    const bool in = label >= 0 && label < a.l.classes;
    Held<F32, 16, V> h;
    h.load(z, 0, a.l.classes, lane);
    const float z_label = in ? logit(a.l, z, label) : 0.f;
    Part p = row_part<true>(h, a.l.c);
    float x[V * VEC];
    int n = 0;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int i = h.at(v) + j;
            x[v * VEC + j] = h.get(v, j);
            if (i < h.first(v) || i >= a.l.classes) continue;
            n += x[v * VEC + j] > z_label || (x[v * VEC + j] == z_label && i < label);
        }
    p.before = row_sum(n);
    const Results q = results(p);
    if (lane == 0 && there) put_row(a, row, p, label, z_label);
    for (int k = 0; k < a.top; ++k) {
        Best b{-infinity(), 0x7fffffff};
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (x[v * VEC + j] > b.z) b = Best{x[v * VEC + j], h.at(v) + j};
        const float top = row_max(b.z);
        b.i = row_min(b.z == top ? b.i : 0x7fffffff);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (h.at(v) + j == b.i) x[v * VEC + j] = -infinity();
        if (lane == 0 && there) put_top(a, row, k, p, q, top, top == -infinity() ? -1 : b.i);
    }
}

// E entries to a lane.
template <bool F32, int V, int E>
__global__ __launch_bounds__(256) void distill_small_kernel(const DistillArgs a) {
    constexpr int VEC = F32 ? 4 : 8, SIZE = F32 ? 4 : 2;
    const int lane = threadIdx.x & 15, at_row = blockIdx.x * 16 + (threadIdx.x >> 4), row = min(at_row, a.l.rows - 1);
    const bool there = at_row < a.l.rows;
    const char *z = (const char *)a.l.z + (int64_t)row * a.l.ld * SIZE;
    int index[E];
    float v[E], z_entry[E], share[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const bool here = i * 16 + lane < a.k;
        const int64_t at = (int64_t)row * a.k + (here ? i * 16 + lane : 0);
        index[i] = here ? a.index[at] : -1;
        v[i] = a.value[at];
    }
    const float weight = a.dloss ? a.dloss[row] : 1.f;
    Held<F32, 16, V> h;
    h.load(z, 0, a.l.classes, lane);
    int wrong = 0, some = 0;
    float v_most = -infinity();
#pragma unroll
    for (int i = 0; i < E; ++i) {
        wrong |= index[i] < -1 || index[i] >= a.l.classes;
        if (index[i] >= a.l.classes || index[i] < 0) index[i] = -1;
        z_entry[i] = index[i] >= 0 ? logit(a.l, z, index[i]) : 0.f;
        if (index[i] < 0) v[i] = -infinity();
        some |= !(v[i] == -infinity());
        v_most = max3(v_most, v[i], v[i]);
    }
    wrong = row_sum(wrong);
    some = row_sum(some | wrong);
    v_most = row_max(v_most);
    float mass = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        // (the distance first, then scaled: finite values do not overflow)
        const float far = (v[i] - (v_most == -infinity() ? 0.f : v_most)) * a.l.inv_t;
        share[i] = index[i] >= 0 ? expf(far) : 0.f;
        mass += share[i];
    }
    mass = wrong ? quiet() : row_sum(mass);
#pragma unroll
    for (int i = 0; i < E; ++i) share[i] /= mass;
    const Part p = row_part<false>(h, a.l.c);
    const bool lost = !(p.s < infinity()) || p.s == 0.f || mass != mass;
    if (a.loss) {
        const float half_sums = 0.5f * a.t * (logf(mass) - LN2 * log2f(p.s));
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) sum += loss_part(share[i], half_of(v[i], v_most), half_of(z_entry[i], p.m), half_sums);
        sum = row_sum(sum);
        if (lane == 0 && there) a.loss[row] = !some ? 0.f : lost ? quiet() : 2.f * a.t * sum;
    }
    if (!a.dz || !there) return;
    char *const d = (char *)a.dz + (int64_t)row * a.ldd * SIZE;
    const float coef = !some ? 0.f : lost ? quiet() : weight * a.t, by = coef / p.s;
    auto gradient = [&](float x) __attribute__((always_inline)) {
        return some ? by * __builtin_amdgcn_exp2f((x - p.m) * a.l.c) : 0.f;
    };
    auto put = [&](int i, float g) __attribute__((always_inline)) {
        if constexpr (F32)
            *(float *)(d + (uint32_t)i * 4) = g;
        else
            *(u16 *)(d + (uint32_t)i * 2) = __builtin_bit_cast(u16, (__bf16)g);
    };
#pragma unroll
    for (int k = 0; k < V; ++k) {
        uint4 x;
        if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) (&x.x)[j] = __float_as_uint(gradient(h.get(k, j)));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) (&x.x)[j] = pack2(gradient(h.get(k, 2 * j)), gradient(h.get(k, 2 * j + 1)));
        }
        const int f = h.first(k);
        if (f + VEC <= a.l.classes) *(u32x4_any *)(d + (uint32_t)f * SIZE) = __builtin_bit_cast(u32x4_any, x);
    }
    const int tail = a.l.classes / VEC * VEC + lane;
    if (tail < a.l.classes) put(tail, gradient(logit(a.l, z, tail)));
    if (!some) return;
    // classes with an entry are written again, by the entry's lane, after the
    // stores of the whole row (the wave's own, which stay in order); entries of
    // one class write the same
    float q[E];
#pragma unroll
    for (int i = 0; i < E; ++i) q[i] = 0.f;
    auto add = [&](auto which, int i) __attribute__((always_inline)) {
        constexpr int J = decltype(which)::value;   // (row_newbcast J)
        const int cls = moved<0x150 + J>(0, index[i]);
        const float s = moved<0x150 + J>(0.f, share[i]);
#pragma unroll
        for (int k = 0; k < E; ++k) q[k] += index[k] == cls ? s : 0.f;
    };
#pragma unroll
    for (int i = 0; i < E; ++i) {
        if (i * 16 >= a.k) break;
#define ENTRY(J) \
    if (i * 16 + J < a.k) add(std::integral_constant<int, J>{}, i)
        ENTRY(0); ENTRY(1); ENTRY(2); ENTRY(3); ENTRY(4); ENTRY(5); ENTRY(6); ENTRY(7);
        ENTRY(8); ENTRY(9); ENTRY(10); ENTRY(11); ENTRY(12); ENTRY(13); ENTRY(14); ENTRY(15);
#undef ENTRY
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (index[i] >= 0) put(index[i], by * __builtin_amdgcn_exp2f((z_entry[i] - p.m) * a.l.c) - coef * q[i]);
}

template <typename A, typename K>
hipError_t go(K kernel, const A &a, hipStream_t s) {
    void *p[] = {const_cast<A *>(&a)};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)answer_groups(a.l), (unsigned)a.l.chunks),
                           dim3((unsigned)answer_threads(a.l.waves)), p, 0, s);
}

template <bool F32, int V>
hipError_t distill_small(const DistillArgs &a, hipStream_t s) {
    return a.k <= 16 ? go(&distill_small_kernel<F32, V, 1>, a, s) : go(&distill_small_kernel<F32, V, 4>, a, s);
}

template <bool F32>
hipError_t score_form(const ScoreArgs &a, hipStream_t s) {
    switch (a.l.waves * 100 + a.l.vecs) {
        case 1: return go(&score_small_kernel<F32, 1>, a, s);
        case 2: return go(&score_small_kernel<F32, 2>, a, s);
        case 101: return go(&score_kernel<F32, 1, 1>, a, s);
        case 102: return go(&score_kernel<F32, 1, 2>, a, s);
        case 104: return go(&score_kernel<F32, 1, 4>, a, s);
        case 402: return go(&score_kernel<F32, 4, 2>, a, s);
        case 404: return go(&score_kernel<F32, 4, 4>, a, s);
        case 804: return go(&score_kernel<F32, 8, 4>, a, s);
        case 808: return go(&score_kernel<F32, 8, 8>, a, s);
    }
    return hipErrorInvalidValue;
}
template <bool F32>
hipError_t distill_form(const DistillArgs &a, hipStream_t s) {
    switch (a.l.waves * 100 + a.l.vecs) {
        case 1: return distill_small<F32, 1>(a, s);
        case 2: return distill_small<F32, 2>(a, s);
        case 101: return go(&distill_kernel<F32, 1, 1>, a, s);
        case 102: return go(&distill_kernel<F32, 1, 2>, a, s);
        case 104: return go(&distill_kernel<F32, 1, 4>, a, s);
        case 402: return go(&distill_kernel<F32, 4, 2>, a, s);
        case 404: return go(&distill_kernel<F32, 4, 4>, a, s);
        case 804: return go(&distill_kernel<F32, 8, 4>, a, s);
        case 1604: return go(&distill_kernel<F32, 16, 4>, a, s);
        case 1609: return go(&distill_kernel<F32, 16, 9, 4>, a, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_score(const ScoreArgs &a, hipStream_t s) {
    if (!score_valid(a)) return hipErrorInvalidValue;
    return a.l.f32 ? score_form<true>(a, s) : score_form<false>(a, s);
}

hipError_t launch_score_join(const ScoreArgs &a, hipStream_t s) {
    if (!score_valid(a) || a.l.chunks < 2 || a.l.rows * 256ll > 0xffffffffll) return hipErrorInvalidValue;
    void *p[] = {const_cast<ScoreArgs *>(&a)};
    const void *kernel = a.l.chunks * a.top <= 1024 ? reinterpret_cast<const void *>(&score_join_kernel<1024>)
                                                    : reinterpret_cast<const void *>(&score_join_kernel<ANSWER_MAX_CHUNKS * TOP_MAX>);
    return hipLaunchKernel(kernel, dim3((unsigned)a.l.rows), dim3(256), p, 0, s);
}

hipError_t launch_distill(const DistillArgs &a, hipStream_t s) {
    if (!distill_valid(a)) return hipErrorInvalidValue;
    return a.l.f32 ? distill_form<true>(a, s) : distill_form<false>(a, s);
}

}  // namespace gemel

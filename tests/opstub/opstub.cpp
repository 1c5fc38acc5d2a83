// CPU stand-in for the kernels of the operators that serve and retrain merged
// layers. Compiled with their host code (operators.cpp, op_plan.cpp), the
// stand-in runtime of ../hoststub and AddressSanitizer: device memory is host
// memory, request tables hold their real values, and every launch checks that
// each range its kernel would read or write is one that may be accessed.
// (Pieces of a workspace have poisoned gaps between them in such a build.)
#include <sanitizer/asan_interface.h>

#include <algorithm>
#include <cstdio>
#include <string>

#include "hip/hip_runtime.h"
#include "op_args.h"

using namespace gemel;

namespace {
long violations = 0, launches = 0;
std::string last;
const char *kernel = "";

void wrong(const char *what, const void *p, long long bytes) {
    char buf[256];
    std::snprintf(buf, sizeof buf, "%s: %s [%p, +%lld)", kernel, what, p, bytes);
    if (violations++ < 5) std::fprintf(stderr, "opstub violation: %s\n", buf);
    last = buf;
}
void touch(const char *what, const void *p, int64_t bytes) {
    if (bytes <= 0) return;
    if (!p || __asan_region_is_poisoned(const_cast<void *>(p), (size_t)bytes)) wrong(what, p, bytes);
}
// rows of `cols` elements, `ld` apart, in the order of `perm` (or as they lie)
void touch_rows(const char *what, const void *p, int64_t rows, int64_t cols, int64_t ld, int elem, const int *perm = nullptr) {
    if (perm) touch("row table", perm, rows * 4);
    for (int64_t r = 0; r < rows; ++r)
        touch(what, (const char *)p + (perm ? perm[r] : r) * ld * elem, cols * elem);
}
void touch_planes(const char *what, const Planes &p, int64_t rows, int batch) {
    for (int z = 0; z < batch; ++z) {
        touch(what, p.hi + z * p.z, rows * p.ld * 2);
        if (p.lo && !p.pair) touch(what, p.lo + z * p.z, rows * p.ld * 2);
    }
}
hipError_t begin(const char *name, bool valid) {
    kernel = name;
    if (!valid) return hipErrorInvalidValue;
    ++launches;
    return hipSuccess;
}
#define BEGIN(name, valid) \
    if (begin(name, valid) != hipSuccess) return hipErrorInvalidValue

void touch_tables(const BatchTables &b) {
    touch("perm", b.perm, b.rows * 4ll);
    touch("run_start", b.run_start, (b.runs + 1) * 4ll);
    touch("run_id", b.run_id, b.runs * 4ll);
    touch("run_rank", b.run_rank, b.runs * 4ll);
    touch("run_scale", b.run_scale, b.runs * 4ll);
    touch("items", b.items, b.n_items * 12ll);
    touch("run_at", b.run_at, b.rows * 4ll);
}
}  // namespace

#undef hipDeviceSynchronize
#undef hipHostFree
static long device_waits = 0;
static hipError_t event_answer = hipSuccess;

extern "C" {
hipError_t hipEventQuery(hipEvent_t) { return event_answer; }
hipError_t opstub_device_synchronize() {
    ++device_waits;
    return hipDeviceSynchronize();
}
// (which waits for the device too)
hipError_t opstub_host_free(void *p) {
    ++device_waits;
    return hipHostFree(p);
}
long opstub_device_waits() { return device_waits; }
// What every event answers from now on (0: passed, 600: not yet).
void opstub_events_answer(int e) { event_answer = (hipError_t)e; }
long opstub_violations() { return violations; }
long opstub_launches() { return launches; }
const char *opstub_last() { return last.c_str(); }
}

namespace gemel {

hipError_t launch_mm(const MmArgs &a, hipStream_t) {
    BEGIN("launch_mm", mm_valid(a));
    const MmOut &o = a.o;
    const int64_t M = a.M, N = a.N;
    touch("zero", a.zero, 16);
    for (int z = 0; z < a.batch; ++z) {
        touch_rows("a", a.a + z * a.za, M, a.K, a.lda, 2, a.perm);
        touch_rows("b", a.b + z * a.zb, N, a.K, a.ldb, 2);
    }
    if (a.perm)
        for (int64_t m = 0; m < M; ++m)
            if (a.perm[m] < 0 || a.perm[m] >= a.perm_rows) wrong("perm value", a.perm + m, a.perm[m]);
    if (a.ext) {
        touch("t", a.t, M * a.ext * 2);
        touch("bx", a.bx, a.runs * N * a.ext * 2);
        touch("run_start", a.run_start, (a.runs + 1) * 4ll);
        touch("first_run", a.first_run, ((M + 63) / 64 + 1) * 4);
    }
    if (a.splits > 1) touch("partial", a.partial, (int64_t)a.splits * a.batch * M * a.ldp * 4);
    if (a.epi == EPI_ROWS || a.epi == EPI_SCALED) {
        touch_rows("out", o.out, M, N, o.ld, a.epi == EPI_SCALED || o.out_f32 ? 4 : 2, o.perm);
        if (o.bias) touch("bias", o.bias, N * 4);
        if (a.epi == EPI_ROWS) return hipSuccess;
        touch("ea", o.ea, M * 4);
        touch("eb", o.eb, N * 4);
        if (a.runs > 0) {
            touch("run_at", o.run_at, M * 4);
            touch("thin sums", o.t, M * o.rp * 4);
            touch("bx", o.bx, (int64_t)a.runs * o.rp * o.ldbx * 4);
        }
        return hipSuccess;
    }
    if (o.sdiag) touch("sdiag", o.sdiag, a.batch * o.diag_z * 4);
    if (o.mdiag) touch("mdiag", o.mdiag, a.batch * o.diag_z * 4);
    if (a.epi != EPI_GRAM) {
        touch("lambda", o.lambda, ((a.batch - 1) * ORTH_LAMBDAS + 1 + o.lambdas) * 4ll);
        touch_planes("s", o.s, M, a.batch);
    }
    if (a.epi == EPI_MIX) touch_planes("s2", o.s2, M, a.batch);
    if (a.epi == EPI_ORTH || a.epi == EPI_STEP) {
        for (int z = 0; z < a.batch; ++z) {
            const int e = a.epi == EPI_STEP || o.out_f32 ? 4 : 2;
            touch_rows("out", (char *)o.out + z * o.z * e, M, N, o.ld, e);
            if (o.copy) touch_rows("copy", o.copy + z * o.z, M, N, o.ld, 2);
        }
        return hipSuccess;
    }
    touch_planes("p", o.p, M, a.batch);
    if (o.p.ld < N * (1 + o.p.pair)) wrong("p is narrow", o.p.hi, o.p.ld);
    if (a.epi == EPI_NEXT) {
        touch_planes("q", o.q, N, a.batch);
        if (o.q.ld < M * (1 + o.q.pair)) wrong("q is narrow", o.q.hi, o.q.ld);
    }
    return hipSuccess;
}

hipError_t launch_rows(const RowsArgs &a, hipStream_t) {
    BEGIN("launch_rows", rows_valid(a));
    const int e = a.f32 ? 4 : 2, rows = a.b.rows;
    touch("zero", a.zero, 16);
    touch_rows("x", a.x, rows, a.K, a.ldx, e);
    touch_rows("w", a.w, a.N, a.K, a.ldw, e);
    touch("partial", a.partial, (int64_t)a.slices * rows * a.ldp * 4);
    touch("row_info", a.b.row_info, rows * 16ll);
    if (a.bias) touch("bias", a.bias, a.N * 4ll);
    touch_rows("y", a.y, rows, a.N, a.ldy, e);
    if (!a.thin_blocks) return hipSuccess;
    touch_tables(a.b);
    touch("t", a.t, (int64_t)a.thin_slices * rows * a.rank_blocks * 64);
    for (int i = 0; i < a.b.n_items; ++i) {
        const int *it = a.b.items + 3 * i, u = it[0];
        if (it[2] < 1 || it[2] > 16 || it[1] < 0 || it[1] + it[2] > rows) wrong("item", it, it[2]);
        const int64_t id = a.b.run_id[u], rank = a.b.run_rank[u];
        touch("a", (const char *)a.a + id * a.b.rank * a.k_bank * e, rank * a.k_bank * e);
        touch("b", (const char *)a.bank_b + id * a.N * a.b.rank * e, (int64_t)a.N * a.b.rank * e);
    }
    return hipSuccess;
}

hipError_t launch_shrink(const ShrinkArgs *all, int n, hipStream_t) {
    BEGIN("launch_shrink", shrink_valid(all, n));
    for (int k = 0; k < n; ++k) {
        const ShrinkArgs &a = all[k];
        const BatchTables &b = a.b;
        const int e = a.f32 ? 4 : 2;
        touch_tables(b);
        for (int i = 0; i < b.n_items; ++i) {
            const int *it = b.items + 3 * i, u = it[0];
            if (it[2] < 1 || it[2] > 32 || it[1] < 0 || it[1] + it[2] > b.rows) wrong("item", it, it[2]);
            touch_rows("x", a.x, it[2], a.K, a.ldx, e, b.perm + it[1]);
            touch_rows("a", (const char *)a.a + (a.by_run ? (int64_t)u * a.rp : (int64_t)b.run_id[u] * b.rank) * a.lda * e,
                       b.run_rank[u], a.K, a.lda, e);
        }
        if (a.slices > 1) touch("part", a.part, (int64_t)a.slices * b.rows * a.rp * 4);
        if (a.flags) touch("flags", a.flags, (int64_t)b.runs * a.n_flags * 4);
        if (a.flags && a.slices > 1) touch("bad", a.bad, b.runs * 4ll);
        if (a.t) touch("t", a.t, (int64_t)b.rows * a.rp * 4);
        if (a.planes) touch("planes", a.planes, (int64_t)b.rows * a.rp * 4);
    }
    return hipSuccess;
}

hipError_t launch_outer(const Outers &o, hipStream_t) {
    if (o.n == 0) return hipSuccess;
    BEGIN("launch_outer", true);
    for (int k = 0; k < o.n; ++k) {
        const OuterArgs &a = o.a[k];
        const int pe = a.p_f32 ? 4 : 2, qe = a.q_f32 ? 4 : 2;
        for (int bz = 0; bz < a.n_chunks; ++bz) {
            int p0 = bz * a.per, n = std::min(a.per, a.positions - p0);
            if (a.chunks) {
                const int ch = bz / a.sub, piece = bz - ch * a.sub;
                touch("chunks", a.chunks + 3 * ch, 12);
                const int whole = a.chunks[3 * ch + 2], each = ((whole + a.sub - 1) / a.sub + 31) / 32 * 32;
                p0 = a.chunks[3 * ch + 1] + piece * each;
                n = std::min(each, whole - piece * each);
            }
            touch_rows("out", a.out + bz * a.chunk, a.R, a.C, a.ld, 4);
            if (n <= 0) continue;
            if (a.sr == 1)
                touch_rows("p", (const char *)a.p + p0 * a.sp * pe, n, a.R, a.sp, pe);
            else
                touch_rows("p", (const char *)a.p + p0 * (int64_t)pe, a.R, n, a.sr, pe);
            if (a.perm)
                touch_rows("q", a.q, n, a.C, a.ldq, qe, a.perm + p0);
            else
                touch_rows("q", (const char *)a.q + p0 * a.ldq * qe, n, a.C, a.ldq, qe);
        }
    }
    return hipSuccess;
}

hipError_t launch_jobs(const Jobs &all, hipStream_t) {
    if (all.n == 0) return hipSuccess;
    BEGIN("launch_jobs", true);
    for (int k = 0; k < all.n; ++k) {
        const Job &j = all.job[k];
        const int e = j.f32 ? 4 : 2;
        const int64_t rows = j.rows, cols = j.cols;
        static const char *const names[] = {"pad", "split", "turn", "colmax", "colsum", "coladd", "pack", "chunks", "rows"};
        kernel = names[j.kind];
        switch (j.kind) {
            case JOB_PAD:
            case JOB_SPLIT:
                touch_rows("in", j.in, rows, cols, j.ldi, e, j.perm);
                touch("out", j.out, rows * j.ldo * (j.kind == JOB_SPLIT ? 2 : e));
                if (j.kind == JOB_SPLIT) touch("e", j.e, rows * 4);
                break;
            case JOB_TURN:
                touch_rows("in", j.in, rows, cols, j.ldi, e);
                touch("out", j.out, cols * j.ldo * 2);
                if (j.f32) touch("e", j.e, cols * 4);
                if (j.f32) touch("max", j.max, j.parts * cols * 4);
                if (j.sum) touch("sum", j.sum, (rows + 63) / 64 * cols * 4);
                break;
            case JOB_COLMAX:
            case JOB_COLSUM:
                touch_rows("in", j.in, rows, cols, j.ldi, e);
                touch("result", j.kind == JOB_COLMAX ? (void *)j.max : j.sum, j.parts * cols * 4);
                break;
            case JOB_COLADD:
                touch("sum", j.sum, j.parts * cols * 4);
                touch("out", j.out, cols * 4);
                break;
            case JOB_PACK:
                touch("run_id", j.run_id, j.n * 4ll);
                touch("run_rank", j.run_rank, j.n * 4ll);
                for (int u = 0; u < j.n; ++u) touch("in", (const char *)j.in + j.run_id[u] * cols * j.R * e, cols * j.R * e);
                touch("out", j.out, j.by_rank ? j.n * j.rp * j.ldo * e : j.n * cols * 2 * j.rp * 2);
                if (!j.by_rank) touch("flags", j.flags, j.n * ((cols + 63) / 64) * 4);
                break;
            case JOB_CHUNKS:
                touch("run_of", j.run_of, j.n * 4ll);
                touch("out", j.out, j.n * j.R * cols * 4);
                for (int ad = 0; ad < j.n; ++ad) {
                    const int u = j.run_of[ad];
                    if (u < 0) continue;
                    touch("chunk_first", j.chunk_first + u, 8);
                    const int64_t k0 = (int64_t)j.chunk_first[u] * j.sub, k1 = (int64_t)j.chunk_first[u + 1] * j.sub;
                    touch("sum", j.sum + k0 * j.rp * cols, (k1 - k0) * j.rp * cols * 4);
                }
                break;
            case JOB_ROWS:
                touch("row_info", j.row_info, rows * 16);
                touch("sum", j.sum, j.parts * rows * j.ldi * 4);
                touch_rows("out", j.out, rows, cols, j.ldo, e);
                for (int64_t r = 0; j.t && r < rows; ++r) {
                    const int4 i = j.row_info[r];
                    if (i.y < 0) continue;
                    touch("t", j.t + (int64_t)i.x * j.rp, i.w * 4ll);
                    touch("in", (const char *)j.in + (int64_t)i.z * j.R * cols * e, i.w * cols * e);
                }
                break;
            default: wrong("kind", &j, j.kind);
        }
    }
    return hipSuccess;
}

static void touch_update(const OrthArgs &a) {
    const int64_t size = (int64_t)a.count * a.rows * a.cols;
    touch("g", a.g, size * (a.f32 ? 4 : 2));
    if (a.step) touch("m", a.m, size * 4);
}
hipError_t launch_norm(const OrthArgs &a, hipStream_t) {
    BEGIN("launch_norm", orth_valid(a, false));
    touch_update(a);
    touch("sums", a.sums, (int64_t)a.count * a.parts * 8);
    return hipSuccess;
}
hipError_t launch_seed(const OrthArgs &a, hipStream_t) {
    BEGIN("launch_seed", orth_valid(a, false));
    const int64_t n = std::min(a.rows, a.cols), m = std::max(a.rows, a.cols);
    touch_update(a);
    touch("sums", a.sums, (int64_t)a.count * a.parts * 8);
    touch("lambda", a.lambda, a.count * ORTH_LAMBDAS * 4ll);
    touch_planes("x", a.x, n, a.count);
    touch_planes("xt", a.xt, m, a.count);
    return hipSuccess;
}
hipError_t launch_thin_gram(const OrthArgs &a, hipStream_t) {
    BEGIN("launch_thin_gram", orth_valid(a, true));
    const int64_t np = op_round_up(std::min(a.rows, a.cols), 16);
    touch_update(a);
    touch("gram", a.gram, a.count * a.parts * np * np * 8);
    return hipSuccess;
}
hipError_t launch_thin_poly(const OrthArgs &a, hipStream_t) {
    BEGIN("launch_thin_poly", orth_valid(a, true));
    const int64_t np = op_round_up(std::min(a.rows, a.cols), 16);
    touch("gram", a.gram, a.count * a.parts * np * np * 8);
    touch("q", a.q, a.count * np * np * 4);
    touch("e", a.e, a.count * 4ll);
    return hipSuccess;
}
hipError_t launch_thin_apply(const OrthArgs &a, hipStream_t) {
    BEGIN("launch_thin_apply", orth_valid(a, true));
    const int64_t size = (int64_t)a.count * a.rows * a.cols;
    touch_update(a);
    touch("out", a.out, size * (a.step || a.f32 ? 4 : 2));
    if (a.copy) touch("copy", a.copy, size * 2);
    return hipSuccess;
}

}  // namespace gemel

extern "C" {
// The grid (threads across) that a product of this shape would be launched
// with, and 0 where its plan does not fit one.
long long opstub_product_threads(int m, int n, int k, int batch, int pair, int sym) {
    MmArgs a{};
    a.M = m;
    a.N = n;
    a.K = k;
    a.batch = batch;
    a.pair = pair;
    a.sym = sym;
    mm_plan(a);
    return mm_fits(a) ? mm_tiles(a, a.tile) * mm_threads_of(a.tile) : 0;
}
}

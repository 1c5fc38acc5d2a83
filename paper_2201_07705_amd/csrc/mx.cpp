// The operators of matrices in microscaled 4-bit floating point: argument
// checks, workspaces, and the order of their kernels.
#include <climits>

#include "mx_args.h"
#include "op_call.h"

using namespace gemel;
using namespace gemel::op;

namespace {

constexpr int64_t MAX_ROWS = 1 << 22;
constexpr int64_t PIECE = 1ll << 27;   // values of float32 rows whose planes (6 bytes each) a pass holds, about
constexpr int64_t COPIES = 1ll << 30;  // values of copied bf16 rows that a pass holds

gemel_status check_mx(gemel_ctx *ctx, const char *what, const gemel_mx *q, Mx *out) {
    if (!q) return fail(ctx, GEMEL_EINVAL, std::string(what) + " is null");
    if (q->rows < 0 || q->rows > MAX_ROWS || q->cols < 1 || q->cols > MX_MAX_COLS)
        return fail(ctx, GEMEL_EINVAL, std::string(what) + " must have 0.." + std::to_string(MAX_ROWS) + " rows of 1.." +
                                           std::to_string(MX_MAX_COLS) + " columns");
    *out = Mx{(uint8_t *)q->codes, (uint8_t *)q->scales, q->rows, q->cols};
    if (q->rows == 0) return GEMEL_OK;
    if (!q->codes || !q->scales) return fail(ctx, GEMEL_EINVAL, std::string(what) + ": codes or scales are null");
    if ((uintptr_t)q->codes % 16 || (uintptr_t)q->scales % 16)
        return fail(ctx, GEMEL_EINVAL, std::string(what) + ": codes and scales must be aligned to 16 bytes");
    return GEMEL_OK;
}
Range codes_of(const Mx &q, bool out) { return range("codes", q.codes, q.rows * mx_pitch(q.cols), out); }
Range scales_of(const Mx &q, bool out) { return range("scales", q.scales, q.rows * mx_groups(q.cols) * 16, out); }

gemel_status check_type(gemel_ctx *ctx, int32_t dtype) {
    return dtype == GEMEL_F32 || dtype == GEMEL_BF16 ? GEMEL_OK : fail(ctx, GEMEL_EINVAL, "unknown type of values");
}

// y of rows that are not quantised.
struct Wide {
    const void *x;
    int64_t ldx;
    int M;
    Mx w;
    const float *bias;
    char *y;
    int64_t ldy;
    bool f32;
};

// float32 rows, and bf16 ones where that is expected to take less time: the
// weights are expanded in registers (float32, planes below each other through
// the bf16 product instead: 1024 rows 25088 -> 4096 469 us and 685, 16384 rows
// 8.2 and 8.9 ms, 4096 -> 4096 1.25 and 1.7). Planes of float32 rows are made
// for a piece of the rows at a time, which bounds the workspace.
gemel_status in_registers(Call &c, const Wide &p) {
    gemel_ctx *ctx = c.ctx;
    const int64_t ld = op_round_up(p.w.cols, 8);
    const int each = p.f32 ? (int)std::min<int64_t>(p.M, std::max<int64_t>(1024, std::min(MX_MOST, PIECE / ld / 64 * 64))) : p.M;
    auto plan = [&](int rows) {
        MxRows a{};
        a.w = p.w;
        a.planes = p.f32 ? 3 : 1;
        a.M = rows;
        mx_rows_plan(a);
        return a;
    };
    const MxRows whole = plan(each), last = p.M % each ? plan(p.M % each) : whole;
    auto partial = [](const MxRows &a) { return a.slices > 1 ? (int64_t)a.slices * a.M * a.ldp : 0; };
    const size_t o_x = c.lay.take(p.f32 ? 3 * each * ld : 0, 2), o_part = c.lay.take(std::max(partial(whole), partial(last)), 4);
    if (c.lay.bytes)
        if (gemel_status s = workspace(c)) return s;
    for (int r = 0; r < p.M; r += each) {
        MxRows a = p.M - r < each ? last : whole;
        a.x = (const u16 *)p.x;
        a.ldx = p.ldx;
        if (p.f32) {
            const MxPlanes split{(const float *)p.x + r * p.ldx, p.ldx, c.at<u16>(o_x), ld, a.M, p.w.cols};
            OPCHK(launch_mx_planes(split, c.stream), "planes");
            a.x = split.out;
            a.ldx = ld;
            a.plane = a.M * ld;
        }
        a.bias = p.bias;
        a.y = p.y + (int64_t)r * p.ldy * (p.f32 ? 4 : 2);
        a.ldy = p.ldy;
        a.f32 = p.f32;
        a.part = c.at<float>(o_part);
        OPCHK(launch_mx_rows(a, c.stream), "product");
    }
    return GEMEL_OK;
}

// Rows that the bf16 product reads where they are (without a row table it
// takes any number of them).
bool in_place(const Wide &p) {
    return (uintptr_t)p.x % 16 == 0 && p.ldx % 8 == 0 && p.w.cols % 8 == 0 && p.ldx <= MM_MAX_LD;
}

// bf16 rows otherwise: the weights are expanded to bf16 once and go through
// the bf16 product, which needs a copy of rows that are not aligned, of as many
// at a time as bound the workspace. Which of
// the two is taken: up to MX_ROWS rows never this one, slower at each of 10
// shapes of 256 to 1024 rows; beyond, the one of the smaller estimate, both a
// fit to these shapes of up to 16384 rows: what is taken is 1.5% from the
// faster one in the mean, 26% at worst. 25088 -> 4096: 1024 rows 209 us in
// registers, expanded once 248, 2048 rows 393 and 398, 4096 rows 781 and 689;
// 1000 -> 1000 4096 rows 16.3 and 25.6; 21990 -> 856 (copied) 3451 rows 183
// and 321.
gemel_status expanded(Call &c, const Wide &p, MmArgs m) {
    gemel_ctx *ctx = c.ctx;
    const int64_t Kp = m.K;
    const bool copy = !in_place(p);
    const int each = copy ? (int)std::min<int64_t>(p.M, std::max<int64_t>(1024, COPIES / Kp / 256 * 256)) : p.M;
    if (!mm_fits(m)) return fail(ctx, GEMEL_EINVAL, "the product is too large");
    m.M = each;   // (tiles and splits stay those of all rows)
    const size_t o_w = c.lay.take(p.w.rows * Kp, 2), o_x = c.lay.take(copy ? each * Kp : 0, 2), o_part = c.lay.take(partial_floats(m), 4);
    if (gemel_status s = workspace(c)) return s;
    MxCast cast{};
    cast.q = p.w;
    cast.out = c.at<u16>(o_w);
    cast.ld = Kp;
    cast.out_cols = (int)Kp;
    OPCHK(launch_mx_values(cast, c.stream), "weights");
    m.b = (const u16 *)cast.out;
    m.ldb = Kp;
    m.zero = (const u16 *)c.st->zero;
    m.partial = c.at<float>(o_part);
    m.o.ld = p.ldy;
    m.o.bias = p.bias;
    for (int r = 0; r < p.M; r += each) {
        m.M = std::min(each, p.M - r);
        m.a = (const u16 *)p.x + r * p.ldx;
        m.lda = p.ldx;
        if (copy) {
            Jobs jobs;
            Job j{};
            j.kind = JOB_PAD;
            j.in = m.a;
            j.ldi = p.ldx;
            j.rows = m.M;
            j.cols = p.w.cols;
            j.out = c.at<u16>(o_x);
            j.ldo = Kp;
            if (!add_job(jobs, j)) return fail(ctx, GEMEL_EINVAL, "x is too large");
            OPCHK(launch_jobs(jobs, c.stream), "copies");
            m.a = c.at<u16>(o_x);
            m.lda = Kp;
        }
        m.o.out = (u16 *)p.y + r * p.ldy;
        OPCHK(launch_mm(m, c.stream), "product");
    }
    return GEMEL_OK;
}

gemel_status wide_product(Call &c, const Wide &p) {
    if (p.f32 || p.M <= MX_ROWS) return in_registers(c, p);
    MmArgs m{};
    m.M = p.M;
    m.N = p.w.rows;
    m.K = (int)op_round_up(p.w.cols, 8);
    m.batch = 1;
    m.epi = EPI_ROWS;
    const double bytes = 2.0 * p.M * p.w.cols;   // of the rows; microseconds
    double once = 7 + std::max(0.8 * mm_plan(m), bytes / 2.3e6) + 2.5 * p.w.rows * p.w.cols / 2.4e6;
    if (!in_place(p)) once += 5.4 + 2 * bytes / 2.3e6;
    MxRows a{};
    a.w = p.w;
    a.planes = 1;
    a.M = p.M;
    return p.M <= MX_MOST && (!mm_fits(m) || mx_rows_plan(a) <= once) ? in_registers(c, p) : expanded(c, p, m);
}

gemel_status both_quantized(Call &c, const Mx &x, const Mx &w, const float *bias, void *y, int64_t ldy, bool f32) {
    gemel_ctx *ctx = c.ctx;
    if (x.rows <= MX_FEW) {
        MxRows a{};
        a.w = w;
        a.q = x;
        a.planes = 1;
        a.M = x.rows;
        mx_rows_plan(a);
        a.bias = bias;
        a.y = y;
        a.ldy = ldy;
        a.f32 = f32;
        OPCHK(launch_mx_rows(a, c.stream), "product");
        return GEMEL_OK;
    }
    MxMm a{};
    a.x = x;
    a.w = w;
    mx_mm_plan(a);
    if (a.splits > 1) {
        const size_t o_part = c.lay.take((int64_t)a.splits * x.rows * a.ldp, 4);
        if (gemel_status s = workspace(c)) return s;
        a.part = c.at<float>(o_part);
    }
    a.bias = bias;
    a.y = y;
    a.ldy = ldy;
    a.f32 = f32;
    OPCHK(launch_mx_mm(a, c.stream), "product");
    return GEMEL_OK;
}

}  // namespace

extern "C" {

gemel_status gemel_mx_quantize(gemel_ctx *ctx, const void *x, int64_t x_stride, int32_t dtype, const gemel_mx *out,
                               void *hip_stream) {
    if (!ctx) return GEMEL_EINVAL;
    return guarded(ctx, [&]() -> gemel_status {
        MxCast a{};
        if (gemel_status s = check_type(ctx, dtype)) return s;
        if (gemel_status s = check_mx(ctx, "out", out, &a.q)) return s;
        if (a.q.rows == 0) return GEMEL_OK;
        const int64_t e = dtype == GEMEL_F32 ? 4 : 2;
        if (gemel_status s = check_rows(ctx, "x", x, x_stride, a.q.cols, e)) return s;
        if (gemel_status s = apart(ctx, {codes_of(a.q, true), scales_of(a.q, true),
                                         range("x", x, a.q.rows, a.q.cols, x_stride, e, false)}))
            return s;
        DeviceScope scope(ctx->device);
        State *st;
        if (gemel_status s = ready(ctx, (hipStream_t)hip_stream, &st)) return s;
        a.x = x;
        a.ld = x_stride;
        a.f32 = dtype == GEMEL_F32;
        OPCHK(launch_mx_quantize(a, (hipStream_t)hip_stream), "quantisation");
        return GEMEL_OK;
    });
}

gemel_status gemel_mx_dequantize(gemel_ctx *ctx, const gemel_mx *q, void *out, int64_t out_stride, int32_t dtype,
                                 void *hip_stream) {
    if (!ctx) return GEMEL_EINVAL;
    return guarded(ctx, [&]() -> gemel_status {
        MxCast a{};
        if (gemel_status s = check_type(ctx, dtype)) return s;
        if (gemel_status s = check_mx(ctx, "q", q, &a.q)) return s;
        if (a.q.rows == 0) return GEMEL_OK;
        const int64_t e = dtype == GEMEL_F32 ? 4 : 2;
        if (gemel_status s = check_rows(ctx, "out", out, out_stride, a.q.cols, e)) return s;
        if (gemel_status s = apart(ctx, {range("out", out, a.q.rows, a.q.cols, out_stride, e, true), codes_of(a.q, false),
                                         scales_of(a.q, false)}))
            return s;
        DeviceScope scope(ctx->device);
        State *st;
        if (gemel_status s = ready(ctx, (hipStream_t)hip_stream, &st)) return s;
        a.out = out;
        a.ld = out_stride;
        a.f32 = dtype == GEMEL_F32;
        a.out_cols = a.q.cols;
        OPCHK(launch_mx_values(a, (hipStream_t)hip_stream), "values");
        return GEMEL_OK;
    });
}

gemel_status gemel_mx_product(gemel_ctx *ctx, int32_t rows, const void *x, int64_t x_stride, const gemel_mx *xq,
                              const gemel_mx *weight, const float *bias, void *y, int64_t y_stride, void *hip_stream) {
    if (!ctx) return GEMEL_EINVAL;
    return guarded(ctx, [&]() -> gemel_status {
        Mx q{}, w{};
        if (gemel_status s = check_mx(ctx, "weight", weight, &w)) return s;
        if (w.rows < 1) return fail(ctx, GEMEL_EINVAL, "weight has no rows");
        if ((x != nullptr) == (xq != nullptr) && rows != 0) return fail(ctx, GEMEL_EINVAL, "either x or xq must be given");
        if (rows < 0 || rows > MAX_ROWS) return fail(ctx, GEMEL_EINVAL, "rows must be in 0.." + std::to_string(MAX_ROWS));
        if (xq) {
            if (gemel_status s = check_mx(ctx, "xq", xq, &q)) return s;
            if (q.rows != rows || q.cols != w.cols)
                return fail(ctx, GEMEL_EINVAL, "xq must have `rows` rows of as many columns as weight");
        }
        if (rows == 0) return GEMEL_OK;
        const bool f32 = ctx->dtype == GEMEL_F32;
        const int64_t e = f32 ? 4 : 2;
        if (x)
            if (gemel_status s = check_rows(ctx, "x", x, x_stride, w.cols, e)) return s;
        if (gemel_status s = check_rows(ctx, "y", y, y_stride, w.rows, e)) return s;
        if (gemel_status s = check_aligned(ctx, "bias", bias, 4)) return s;
        if (gemel_status s = apart(ctx, {range("y", y, rows, w.rows, y_stride, e, true),
                                         range("x", x, rows, w.cols, x_stride, e, false), codes_of(q, false), scales_of(q, false),
                                         codes_of(w, false), scales_of(w, false), range("bias", bias, w.rows * 4ll, false)}))
            return s;
        DeviceScope scope(ctx->device);
        State *st;
        if (gemel_status s = ready(ctx, (hipStream_t)hip_stream, &st)) return s;
        Call c{ctx, st, (hipStream_t)hip_stream, nullptr, {}, nullptr};
        if (xq) return both_quantized(c, q, w, bias, y, y_stride, f32);
        const Wide p{x, x_stride, rows, w, bias, (char *)y, y_stride, f32};
        return wide_product(c, p);
    });
}

}  // extern "C"

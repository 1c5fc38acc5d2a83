// The operators that read answers off logits and distil them: argument checks,
// and the order of their kernels.
#include <cmath>

#include "answer_args.h"
#include "op_call.h"

using namespace gemel;
using namespace gemel::op;

namespace {

constexpr int64_t MAX_ROWS = 1 << 22, MAX_CLASSES = 1 << 20;
constexpr float MIN_T = 1e-6f, MAX_T = 1e6f;

// Logits [rows][classes]; *out is what the kernels are told of them.
gemel_status check_logits(gemel_ctx *ctx, int32_t rows, int32_t classes, const void *z, int64_t stride, int32_t dtype, float t,
                          Logits *out) {
    if (rows < 0 || rows > MAX_ROWS) return fail(ctx, GEMEL_EINVAL, "rows must be in 0.." + std::to_string(MAX_ROWS));
    if (classes < 1 || classes > MAX_CLASSES)
        return fail(ctx, GEMEL_EINVAL, "classes must be in 1.." + std::to_string(MAX_CLASSES));
    if (dtype != GEMEL_F32 && dtype != GEMEL_BF16) return fail(ctx, GEMEL_EINVAL, "unknown type of logits");
    if (!(t >= MIN_T && t <= MAX_T)) return fail(ctx, GEMEL_EINVAL, "temperature must be in 1e-6..1e6");
    if (rows == 0) return GEMEL_OK;
    if (gemel_status s = check_rows(ctx, "logits", z, stride, classes, dtype == GEMEL_F32 ? 4 : 2)) return s;
    *out = Logits{};
    out->z = z;
    out->ld = stride;
    out->f32 = dtype == GEMEL_F32;
    out->rows = rows;
    out->classes = classes;
    out->inv_t = 1.f / t;
    out->c = (float)(1.4426950408889634 / t);
    return GEMEL_OK;
}
Range logit_range(const Logits &l) { return range("logits", l.z, l.rows, l.classes, l.ld, l.f32 ? 4 : 2, false); }

gemel_status check_entries(gemel_ctx *ctx, int32_t rows, int32_t k, const int32_t *index, const float *value, const float *dloss) {
    if (k < 1 || k > TOP_MAX) return fail(ctx, GEMEL_EINVAL, "entries must be in 1.." + std::to_string(TOP_MAX));
    if (rows == 0) return GEMEL_OK;
    if (!index) return fail(ctx, GEMEL_EINVAL, "indices is null");
    if (!value) return fail(ctx, GEMEL_EINVAL, "values is null");
    if (gemel_status s = check_aligned(ctx, "indices", index, 4)) return s;
    if (gemel_status s = check_aligned(ctx, "values", value, 4)) return s;
    return check_aligned(ctx, "dloss", dloss, 4);
}

gemel_status log_probs(gemel_ctx *ctx, const Logits &l, const int32_t *labels, int top, const gemel_answers &o, hipStream_t stream) {
    ScoreArgs a{};
    a.l = l;
    a.labels = labels;
    a.top = o.top_indices || o.top_log_probs ? top : 0;
    a.log_prob = o.log_prob;
    a.rank = o.rank;
    a.entropy = o.entropy;
    a.log_sum = o.log_sum;
    a.top_index = o.top_indices;
    a.top_log_prob = o.top_log_probs;
    score_plan(a.l, a.top);
    DeviceScope scope(ctx->device);
    State *st;
    if (gemel_status s = ready(ctx, stream, &st)) return s;
    if (a.l.chunks == 1) {
        OPCHK(launch_score(a, stream), "log probabilities");
        return GEMEL_OK;
    }
    Call c{ctx, st, stream, nullptr, {}, nullptr};
    const int64_t units = (int64_t)l.rows * a.l.chunks;
    const size_t o_part = c.lay.take(units, sizeof(Part)), o_value = c.lay.take(units * a.top, 4),
                 o_index = c.lay.take(units * a.top, 4);
    if (gemel_status s = workspace(c)) return s;
    a.part = c.at<Part>(o_part);
    a.list_value = c.at<float>(o_value);
    a.list_index = c.at<int>(o_index);
    OPCHK(launch_score(a, stream), "log probabilities");
    OPCHK(launch_score_join(a, stream), "log probabilities of wide rows");
    return GEMEL_OK;
}

// (dz and loss may be null)
gemel_status distill(gemel_ctx *ctx, DistillArgs a, hipStream_t stream) {
    distill_plan(a.l);
    DeviceScope scope(ctx->device);
    State *st;
    if (gemel_status s = ready(ctx, stream, &st)) return s;
    if (a.l.chunks > 1) {
        Call c{ctx, st, stream, nullptr, {}, nullptr};
        ScoreArgs sums{};
        sums.l = a.l;
        score_plan(sums.l, 0);
        a.parts = sums.l.chunks;
        const size_t o_part = c.lay.take((int64_t)a.l.rows * a.parts, sizeof(Part));
        if (gemel_status s = workspace(c)) return s;
        a.part = sums.part = c.at<Part>(o_part);
        OPCHK(launch_score(sums, stream), "sums of wide rows");
    }
    OPCHK(launch_distill(a, stream), "distillation");
    return GEMEL_OK;
}

}  // namespace

extern "C" {

gemel_status gemel_log_probs(gemel_ctx *ctx, int32_t rows, int32_t classes, const void *logits, int64_t logits_stride,
                             int32_t dtype, const int32_t *labels, int32_t top, float temperature, const gemel_answers *out,
                             void *hip_stream) {
    if (!ctx) return GEMEL_EINVAL;
    return guarded(ctx, [&]() -> gemel_status {
        Logits l;
        if (gemel_status s = check_logits(ctx, rows, classes, logits, logits_stride, dtype, temperature, &l)) return s;
        if (top < 0 || top > TOP_MAX) return fail(ctx, GEMEL_EINVAL, "top must be in 0.." + std::to_string(TOP_MAX));
        if (!out) return fail(ctx, GEMEL_EINVAL, "out is null");
        if (rows == 0) return GEMEL_OK;
        const gemel_answers &o = *out;
        if ((o.log_prob || o.rank) && !labels) return fail(ctx, GEMEL_EINVAL, "labels is null");
        if (!o.log_prob && !o.rank && !o.entropy && !o.log_sum && (!top || (!o.top_indices && !o.top_log_probs)))
            return fail(ctx, GEMEL_EINVAL, "no output is asked for");
        const int64_t n = (int64_t)rows * 4;
        const std::vector<Range> all = {range("log_prob", o.log_prob, n, true), range("rank", o.rank, n, true),
                                        range("entropy", o.entropy, n, true), range("log_sum", o.log_sum, n, true),
                                        range("top_indices", top ? o.top_indices : nullptr, n * top, true),
                                        range("top_log_probs", top ? o.top_log_probs : nullptr, n * top, true),
                                        range("labels", labels, n, false), logit_range(l)};
        for (size_t i = 0; i + 1 < all.size(); ++i)
            if (gemel_status s = check_aligned(ctx, all[i].what, (const void *)all[i].lo, 4)) return s;
        if (gemel_status s = apart(ctx, all)) return s;
        return log_probs(ctx, l, labels, top, o, (hipStream_t)hip_stream);
    });
}

gemel_status gemel_distill(gemel_ctx *ctx, int32_t rows, int32_t classes, const void *logits, int64_t logits_stride, int32_t dtype,
                           const int32_t *indices, const float *values, int32_t entries, float temperature, float *loss,
                           void *hip_stream) {
    if (!ctx) return GEMEL_EINVAL;
    return guarded(ctx, [&]() -> gemel_status {
        DistillArgs a{};
        if (gemel_status s = check_logits(ctx, rows, classes, logits, logits_stride, dtype, temperature, &a.l)) return s;
        if (gemel_status s = check_entries(ctx, rows, entries, indices, values, nullptr)) return s;
        if (rows == 0) return GEMEL_OK;
        if (!loss) return fail(ctx, GEMEL_EINVAL, "loss is null");
        if (gemel_status s = check_aligned(ctx, "loss", loss, 4)) return s;
        const int64_t n = (int64_t)rows * 4;
        if (gemel_status s = apart(ctx, {range("loss", loss, n, true), range("indices", indices, n * entries, false),
                                         range("values", values, n * entries, false), logit_range(a.l)}))
            return s;
        a.index = indices;
        a.value = values;
        a.k = entries;
        a.t = temperature;
        a.loss = loss;
        return distill(ctx, a, (hipStream_t)hip_stream);
    });
}

gemel_status gemel_distill_backward(gemel_ctx *ctx, int32_t rows, int32_t classes, const float *dloss, const void *logits,
                                    int64_t logits_stride, int32_t dtype, const int32_t *indices, const float *values,
                                    int32_t entries, float temperature, void *dlogits, int64_t dlogits_stride, float *loss,
                                    void *hip_stream) {
    if (!ctx) return GEMEL_EINVAL;
    return guarded(ctx, [&]() -> gemel_status {
        DistillArgs a{};
        if (gemel_status s = check_logits(ctx, rows, classes, logits, logits_stride, dtype, temperature, &a.l)) return s;
        if (gemel_status s = check_entries(ctx, rows, entries, indices, values, dloss)) return s;
        if (rows == 0) return GEMEL_OK;
        const int64_t e = a.l.f32 ? 4 : 2, n = (int64_t)rows * 4;
        if (gemel_status s = check_rows(ctx, "dlogits", dlogits, dlogits_stride, classes, e)) return s;
        if (gemel_status s = check_aligned(ctx, "loss", loss, 4)) return s;
        if (gemel_status s = apart(ctx, {range("dlogits", dlogits, rows, classes, dlogits_stride, e, true),
                                         range("loss", loss, n, true), range("dloss", dloss, n, false),
                                         range("indices", indices, n * entries, false),
                                         range("values", values, n * entries, false), logit_range(a.l)}))
            return s;
        a.index = indices;
        a.value = values;
        a.k = entries;
        a.t = temperature;
        a.dloss = dloss;
        a.loss = loss;
        a.dz = dlogits;
        a.ldd = dlogits_stride;
        return distill(ctx, a, (hipStream_t)hip_stream);
    });
}

}  // extern "C"

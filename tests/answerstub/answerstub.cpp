// CPU stand-in for the kernels of answers, distillation and 4-bit matrices,
// beside that of ../opstub: every launch checks that its operands and results
// are, as wholes, ranges that may be accessed. The addresses that threads form
// inside of them are the kernels' own; they are enumerated for the rows of x of
// mx_rows_kernel alone (touch_pieces here, and pieces.cpp).
#include <sanitizer/asan_interface.h>

#include <cstdio>
#include <string>

#include "hip/hip_runtime.h"
#include "answer_args.h"
#include "mx_args.h"

using namespace gemel;

namespace {
long violations = 0, launches = 0;
std::string last, names;
const char *kernel = "";

void touch(const char *what, const void *p, int64_t bytes) {
    if (bytes <= 0) return;
    if (p && !__asan_region_is_poisoned(const_cast<void *>(p), (size_t)bytes)) return;
    char buf[256];
    std::snprintf(buf, sizeof buf, "%s: %s [%p, +%lld)", kernel, what, p, (long long)bytes);
    if (violations++ < 5) std::fprintf(stderr, "answerstub violation: %s\n", buf);
    last = buf;
}
void touch_rows(const char *what, const void *p, int64_t rows, int64_t cols, int64_t ld, int elem) {
    for (int64_t r = 0; r < rows; ++r) touch(what, (const char *)p + r * ld * elem, cols * elem);
}
void touch_mx(const char *what, const Mx &q) {
    touch(what, q.codes, q.rows * mx_pitch(q.cols));
    touch(what, q.scales, q.rows * mx_groups(q.cols) * 16);
}
bool begin(const char *name, bool valid) {
    kernel = name;
    if (valid) ++launches;
    if (valid) names += std::string(names.empty() ? "" : " ") + name;
    return valid;
}
#define BEGIN(name, valid) \
    if (!begin(name, valid)) return hipErrorInvalidValue
}  // namespace

extern "C" {
long answerstub_violations() { return violations; }
long answerstub_launches() { return launches; }
const char *answerstub_last() { return last.c_str(); }
const char *answerstub_names() {
    static std::string out;
    out = names;
    names.clear();
    return out.c_str();
}
}

namespace gemel {

static void touch_logits(const Logits &l) { touch_rows("logits", l.z, l.rows, l.classes, l.ld, l.f32 ? 4 : 2); }

static void touch_answers(const ScoreArgs &a) {
    const int64_t rows = a.l.rows;
    if (a.labels) touch("labels", a.labels, rows * 4);
    if (a.log_prob) touch("log_prob", a.log_prob, rows * 4);
    if (a.rank) touch("rank", a.rank, rows * 4);
    if (a.entropy) touch("entropy", a.entropy, rows * 4);
    if (a.log_sum) touch("log_sum", a.log_sum, rows * 4);
    if (a.top_index) touch("top_index", a.top_index, rows * a.top * 4);
    if (a.top_log_prob) touch("top_log_prob", a.top_log_prob, rows * a.top * 4);
}
static void touch_chunks(const ScoreArgs &a) {
    const int64_t units = (int64_t)a.l.rows * a.l.chunks;
    touch("part", a.part, units * sizeof(Part));
    touch("list_value", a.list_value, units * a.top * 4);
    touch("list_index", a.list_index, units * a.top * 4);
}
hipError_t launch_score(const ScoreArgs &a, hipStream_t) {
    BEGIN("score", score_valid(a));
    touch_logits(a.l);
    if (a.l.chunks > 1)
        touch_chunks(a);
    else
        touch_answers(a);
    return hipSuccess;
}
hipError_t launch_score_join(const ScoreArgs &a, hipStream_t) {
    BEGIN("join", score_valid(a) && a.l.chunks > 1);
    touch_chunks(a);
    touch_answers(a);
    return hipSuccess;
}
hipError_t launch_distill(const DistillArgs &a, hipStream_t) {
    BEGIN("distill", distill_valid(a));
    touch_logits(a.l);
    touch("index", a.index, (int64_t)a.l.rows * a.k * 4);
    touch("value", a.value, (int64_t)a.l.rows * a.k * 4);
    if (a.dloss) touch("dloss", a.dloss, a.l.rows * 4ll);
    if (a.loss) touch("loss", a.loss, a.l.rows * 4ll);
    if (a.dz) touch_rows("dz", a.dz, a.l.rows, a.l.classes, a.ldd, a.l.f32 ? 4 : 2);
    if (a.l.chunks > 1) touch("part", a.part, (int64_t)a.l.rows * a.parts * sizeof(Part));
    return hipSuccess;
}

hipError_t launch_mx_quantize(const MxCast &a, hipStream_t) {
    BEGIN("quantize", mx_cast_valid(a, false));
    touch_rows("x", a.x, a.q.rows, a.q.cols, a.ld, a.f32 ? 4 : 2);
    touch_mx("q", a.q);
    return hipSuccess;
}
hipError_t launch_mx_values(const MxCast &a, hipStream_t) {
    BEGIN("values", mx_cast_valid(a, true));
    touch_rows("out", a.out, a.q.rows, a.out_cols, a.ld, a.f32 ? 4 : 2);
    touch_mx("q", a.q);
    return hipSuccess;
}
hipError_t launch_mx_planes(const MxPlanes &a, hipStream_t) {
    BEGIN("planes", mx_planes_valid(a));
    touch_rows("x", a.x, a.rows, a.cols, a.ldx, 4);
    touch("planes", a.out, 3 * a.rows * a.ld * 2);
    return hipSuccess;
}
hipError_t launch_mx_sum(const MxSum &a, hipStream_t) {
    BEGIN("sum", mx_sum_valid(a));
    touch("part", a.part, a.parts * a.rows * a.ldp * 4);
    if (a.bias) touch("bias", a.bias, a.cols * 4ll);
    touch_rows("y", a.y, a.rows, a.cols, a.ldy, a.f32 ? 4 : 2);
    return hipSuccess;
}
// What the threads of mx_rows_kernel read of x: the pieces of a whole step and
// of the last one, with the kernel's own map (the whole steps between them
// end before the columns do).
static void touch_pieces(const MxRows &a) {
    const int rows = 16 * mx_row_blocks(a.M), all = a.planes * rows, last = (a.w.cols - 1) / 128;
    for (int m0 = 0; m0 < a.M; m0 += rows)
        for (int i = 0; i < mx_piece_loads(all); ++i)
            for (int t = 0; t < MX_PIECE_THREADS; ++t) {
                const int row = mx_piece_row(i, t, all), m = m0 + row % rows < a.M ? m0 + row % rows : a.M - 1;
                const u16 *p = a.x + row / rows * a.plane + m * a.ldx;
                for (int step : {0, last}) {
                    const int c = step * 128 + mx_piece_col(t);
                    touch("a piece of x", p + c, mx_piece_cols(c, a.w.cols) * 2);
                }
            }
}
hipError_t launch_mx_rows(const MxRows &a, hipStream_t) {
    BEGIN(a.M <= MX_FEW ? "few" : "rows", mx_rows_valid(a));
    touch_mx("w", a.w);
    if (a.M > MX_FEW) touch_pieces(a);
    if (a.q.codes)
        touch_mx("q", a.q);
    else
        for (int p = 0; p < a.planes; ++p) touch_rows("x", a.x + p * a.plane, a.M, a.w.cols, a.ldx, 2);
    if (a.bias) touch("bias", a.bias, a.w.rows * 4ll);
    if (a.slices > 1) touch("part", a.part, (int64_t)a.slices * a.M * a.ldp * 4);
    touch_rows("y", a.y, a.M, a.w.rows, a.ldy, a.f32 ? 4 : 2);
    return hipSuccess;
}
hipError_t launch_mx_mm(const MxMm &a, hipStream_t) {
    BEGIN("mm", mx_mm_valid(a));
    touch_mx("x", a.x);
    touch_mx("w", a.w);
    if (a.bias) touch("bias", a.bias, a.w.rows * 4ll);
    if (a.splits > 1) touch("part", a.part, (int64_t)a.splits * a.x.rows * a.ldp * 4);
    touch_rows("y", a.y, a.x.rows, a.w.rows, a.ldy, a.f32 ? 4 : 2);
    return hipSuccess;
}

}  // namespace gemel

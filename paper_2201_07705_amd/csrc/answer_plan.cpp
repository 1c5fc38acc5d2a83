// Launch shapes and checks of the kernels that read answers off logits. Plain
// host code, which CPU builds share.
#include <algorithm>

#include "answer_args.h"
#include "op_args.h"

namespace gemel {

const AnswerForm answer_forms[ANSWER_FORMS] = {
    {0, 1}, {0, 2}, {1, 1}, {1, 2}, {1, 4}, {4, 2}, {4, 4}, {8, 4}, {8, 8}, {16, 4}, {16, 9}};

namespace {
void cut(Logits &l, const AnswerForm &f) {
    l.waves = f.waves;
    l.vecs = f.vecs;
    l.chunk = answer_lanes(f.waves) * f.vecs * answer_vec(l.f32);
    l.chunks = (l.classes + l.chunk - 1) / l.chunk;
}
bool form_of(const Logits &l) {
    for (const AnswerForm &f : answer_forms)
        if (l.waves == f.waves && l.vecs == f.vecs) return true;
    return false;
}
}  // namespace

int64_t answer_groups(const Logits &l) {
    const int teams = answer_teams(l.waves);
    return ((int64_t)l.rows + teams - 1) / teams;
}

static bool threads_fit(const Logits &l) { return answer_groups(l) * answer_threads(l.waves) <= MAX_THREADS; }

// The smallest form that holds a row (16 lanes search each of the best
// classes in turn: only a few; 65536 rows of 80 classes, 16 lanes against a
// wave: 5 best 17 and 48 us, 20 best 46 and 92, 64 best in a wave 74); wide
// rows in chunks of 4 waves of 4 pieces (2048 rows of 100003 bf16, 20 best:
// 147 us; of 2 pieces 205, of 4 and 8 pieces in 8 waves 200 and 218), larger
// ones only where there would be more than 64.
void score_plan(Logits &l, int top) {
    for (int i = top <= 32 ? 0 : 2; i < 9; ++i) {
        cut(l, answer_forms[i]);
        if (l.chunks <= (i < 6 ? 1 : ANSWER_MAX_CHUNKS)) return;
    }
}
// The smallest form that holds a row; rows beyond the largest in chunks of
// its own after a pass for their sums (2048 rows of 100003 bf16 287 us, of
// which the sums take 95; held in one workgroup's registers, 16 waves of 16
// pieces spill). So are 2^22 rows that would take 16 waves each, more threads
// than a launch has.
void distill_plan(Logits &l) {
    for (int i : {0, 1, 2, 3, 4, 5, 6, 7, 9, 10}) {
        cut(l, answer_forms[i]);
        if (l.chunks == 1 && threads_fit(l)) return;
    }
    cut(l, answer_forms[6]);
}

static bool logits_valid(const Logits &l) {
    return l.z && l.rows > 0 && l.classes > 0 && l.ld >= l.classes && form_of(l) && l.chunk > 0 &&
           l.chunk <= answer_lanes(l.waves) * l.vecs * answer_vec(l.f32) && l.chunks >= 1 && l.chunks <= 65535 &&
           (int64_t)l.chunk * l.chunks >= l.classes && (int64_t)l.chunk * (l.chunks - 1) < l.classes && l.c > 0 && l.inv_t > 0 &&
           (uintptr_t)l.z % (l.f32 ? 4 : 2) == 0 && threads_fit(l);
}

bool score_valid(const ScoreArgs &a) {
    if (!logits_valid(a.l) || a.top < 0 || a.top > TOP_MAX || a.l.waves > 8 || a.l.chunks > ANSWER_MAX_CHUNKS)
        return false;
    if (a.l.chunks > 1 && (!a.part || (a.top && (!a.list_value || !a.list_index)))) return false;
    return (a.log_prob || a.rank) ? a.labels != nullptr : true;
}

bool distill_valid(const DistillArgs &a) {
    return logits_valid(a.l) && a.k >= 1 && a.k <= TOP_MAX && a.index && a.value && (a.loss || a.dz) && a.t > 0 &&
           (!a.dz || (a.ldd >= a.l.classes && (uintptr_t)a.dz % (a.l.f32 ? 4 : 2) == 0)) &&
           (a.l.chunks == 1 || (a.part && a.parts >= 1 && a.parts <= ANSWER_MAX_CHUNKS));
}

}  // namespace gemel

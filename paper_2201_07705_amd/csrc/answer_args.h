// Argument blocks and launchers of the operators that read answers off logits
// and distil them. Each launcher checks on the host (answer_plan.cpp) that its
// block matches what the kernel and grid assume and returns
// hipErrorInvalidValue instead of launching otherwise.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gemel {

constexpr int TOP_MAX = 64;              // entries of a row: one for each lane of a wave
constexpr int ANSWER_MAX_CHUNKS = 64;    // parts of a row: one for each lane of a wave

// Rows of logits, and how they are cut: a team of `waves` waves (0: of 16
// lanes) holds `vecs` pieces of 16 bytes in each lane, `chunk` classes of a
// row at most.
struct Logits {
    const void *z;
    int64_t ld;
    int f32, rows, classes;
    float inv_t, c;      // 1 / temperature, and log2(e) of that
    int waves, vecs;     // a form of answer_forms
    int chunk, chunks;   // classes of a team, and teams of a row
};
// A chunk's largest logit m, and its sums of 2^t and 2^t t, t = (z - m) c; no
// class is offered where s is 0.
struct Part {
    float m, s, a;
    int before;          // classes of the chunk that come before the label
};

struct ScoreArgs {
    Logits l;
    const int *labels;   // [rows] or null
    int top;
    // outputs, each may be null
    float *log_prob;
    int *rank;
    float *entropy, *log_sum;
    int *top_index;      // [rows][top]
    float *top_log_prob;
    // chunks > 1: [rows][chunks], and the best `top` of each
    Part *part;
    float *list_value;
    int *list_index;
};

struct DistillArgs {
    Logits l;
    const int *index;    // [rows][k] classes, -1: no entry
    const float *value;  // [rows][k]
    int k;
    float t;             // temperature
    const float *dloss;  // [rows] or null (1)
    float *loss;         // [rows] or null
    void *dz;            // or null
    int64_t ldd;
    const Part *part;    // chunks > 1: [rows][parts] sums of the row's parts
    int parts;
};

struct AnswerForm {
    int waves, vecs;
};
constexpr int ANSWER_FORMS = 11;
extern const AnswerForm answer_forms[ANSWER_FORMS];
constexpr int answer_vec(int f32) { return f32 ? 4 : 8; }   // classes of a piece
// Rows that a workgroup holds at once
constexpr int answer_teams(int waves) { return waves == 0 ? 16 : waves == 1 ? 4 : 1; }
constexpr int answer_lanes(int waves) { return waves == 0 ? 16 : waves * 64; }   // of a team
constexpr int answer_threads(int waves) { return answer_teams(waves) * answer_lanes(waves); }

void score_plan(Logits &l, int top);
void distill_plan(Logits &l);
bool score_valid(const ScoreArgs &a);
bool distill_valid(const DistillArgs &a);
int64_t answer_groups(const Logits &l);   // workgroups, for each chunk

hipError_t launch_score(const ScoreArgs &a, hipStream_t s);
// chunks > 1: joins what launch_score has left for each chunk
hipError_t launch_score_join(const ScoreArgs &a, hipStream_t s);
hipError_t launch_distill(const DistillArgs &a, hipStream_t s);

}  // namespace gemel

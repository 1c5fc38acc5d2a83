// Argument blocks and launchers of the operators that serve and retrain
// merged layers: adapted projections, their gradients, and orthogonalised
// matrix updates. Each launcher checks on the host (op_plan.cpp) that its
// block matches what the kernel and grid assume and returns
// hipErrorInvalidValue instead of launching otherwise.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gemel {

typedef unsigned short u16;

// Threads of a grid along one axis (the runtime's limit).
constexpr int64_t MAX_THREADS = 0xffffffffll;

constexpr int64_t op_round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// What a product does with its sums v (float32) of element (m, n).
enum MmEpi {
    EPI_ROWS = 0,   // out[perm[m]][n] = v + bias[n], in the context's type
    EPI_SCALED = 1, // out[perm[m]][n] = v * 2^-(ea[m] + eb[n]) + low-rank part + bias[n], float32
    EPI_GRAM = 2,   // S = v * 2^-26, stored * 2^11 as planes, with its mirror image
    EPI_POLY = 3,   // M = b l^2 S + c l^4 v 2^-22, stored * 2^14 as planes, with its mirror image
    EPI_NEXT = 4,   // X = f (cs X + cv v), in plane units (2^13), in both layouts
    EPI_ORTH = 5,   // out[m][n] = l 2^-13 (cs X + cv v), in the context's type
    EPI_STEP = 6,   // w = (1 - decay) w - rate * l 2^-13 (cs X + cv v), and its copy
    EPI_MIX = 7     // f (cs S + cs2 S2 + cv v), in plane units, with its mirror image
};

// 16-bit planes of a matrix: hi, and lo (the rest; null = not kept). Rows of
// ld elements, z elements between the matrices of a batch. Separate arrays,
// or (pair) one whose rows alternate 32 elements of hi with the same 32 of
// lo, which is then hi + 32: what a product of pairs reads together lies
// together.
struct Planes {
    u16 *hi, *lo;
    int64_t ld, z;
    int pair;
};
constexpr int PAIR_RUN = 32;
// Where element n of a row is in an array of pairs (4 elements from a
// multiple of 4 on are consecutive in either layout).
__host__ __device__ constexpr int pair_at(int n) { return 2 * n - (n & (PAIR_RUN - 1)); }

struct MmOut {
    void *out;            // ROWS, SCALED, ORTH, STEP (w)
    int64_t ld, z;
    int out_f32;          // ROWS, ORTH: float32 instead of bf16
    const float *bias;    // [N] or null
    const int *perm;      // output row of product row m, or null
    const int *ea, *eb;   // SCALED
    // SCALED: low-rank part, sum over r < rank of t[m][r] * bx[run][r][n]
    // where the row has a run (run_at[m] >= 0); rank a multiple of 4, rows of
    // bx ldbx apart, a multiple of 4
    const float *t, *bx;
    const int *run_at;
    int rp, rank;
    int64_t ldbx;
    Planes p, q;          // GRAM, POLY, MIX: p; NEXT: p = [m][n], q = [n][m]
    Planes s, s2;         // POLY, MIX: S; NEXT, ORTH, STEP: X as the product's rows lie
    float cs, cs2, cv;
    int lambdas;          // f = lambda[0] / lambda[lambdas], MIX: squared (0: 1)
    // diagonals of S and M, kept unrounded where these are single planes
    // ([batch][diag_z]): GRAM and POLY write theirs, POLY reads S's, NEXT,
    // ORTH and STEP read M's, by output row or column
    float *sdiag, *mdiag;
    int64_t diag_z;
    int diag_rows;
    const float *lambda;  // l of each matrix, ORTH_LAMBDAS apart
    u16 *copy;            // STEP: bf16 copy of w or null
    float rate, decay;    // STEP
};

// C[m][n] = sum over k of a[row m][k] * b[n][k]. Operands are rows of
// contiguous 16-bit elements (bf16 for EPI_ROWS, else float16); 16-byte
// aligned, ld a multiple of 8; where K is not a multiple of 64 chunks of 8
// beyond K are read as zeros (K a multiple of 8). pair: rows of pairs, K
// counting both planes; the products hi hi, hi lo and lo hi are summed.
struct MmArgs {
    const u16 *a, *b;
    int64_t lda, ldb, za, zb;
    int pair, M, N, K, batch;
    int epi;
    int sym;              // only tiles on and above the diagonal
    int tile;             // 64, 128 or 256 (mm_plan)
    int splits, steps;    // depth splits, and steps of 64 in each
    float *partial;       // [splits][batch][M][ldp] with splits > 1
    int64_t ldp;
    const u16 *zero;      // 16 zero bytes or more
    const int *perm;      // row of a behind product row m, or null
    int64_t perm_rows;    // rows that it points into
    // low-rank extension of the depth (bf16): t [M][ext] rows against
    // bx [run][N][ext], where the row's run is the one holding m
    const u16 *t, *bx;
    int ext, runs;        // ext a multiple of 64, 0 = none
    const int *run_start; // [runs + 1]; rows before run_start[0] have none
    const int *first_run; // [ceil(M / 64) + 1] first run ending after row 64 i
    MmOut o;
};
// Longest rows: a tile's byte offsets fit 32 bits (and with a row table the
// whole matrix's: perm_rows * lda up to 2^30 elements).
constexpr int64_t MM_MAX_LD = 1 << 22;
constexpr int MM_BK = 64;   // depth of a step: a 128-byte line of each row
double mm_plan(MmArgs &a);   // tile, splits, steps, ldp of a shape; the microseconds expected
int64_t mm_tiles(const MmArgs &a, int T);   // T x T tiles of a result (32: the sum of splits)
constexpr int mm_threads_of(int tile) { return tile == 64 ? 256 : 512; }
bool mm_fits(const MmArgs &a);    // the sizes of a planned product, before it has operands
bool mm_valid(const MmArgs &a);
hipError_t launch_mm(const MmArgs &a, hipStream_t s);

constexpr int ROWS_MAX = 64;   // rows that launch_rows takes

// Requests grouped by adapter, as tables in device memory.
struct BatchTables {
    const int *perm;       // [rows] row behind position p
    const int *run_start;  // [runs + 1] positions
    const int *run_id;     // [runs] adapter
    const int *run_rank;   // [runs]
    const float *run_scale;// [runs]
    const int *first_run;  // [ceil(rows / 64) + 1]
    const int *items;      // [n_items][3]: run, first position, positions (<= 16, or 32 with more than ROWS_MAX rows)
    const int *chunks;     // [n_chunks][3]: run, first position, positions
    const int *chunk_first;// [runs + 1] chunks of a run
    const int *run_of;     // [adapters] run or -1
    const int *run_at;     // [rows] run of position p or -1
    const int4 *row_info;  // [rows], batches of up to ROWS_MAX rows: position, run or -1, adapter, rank
    int rows, runs, adapters, rank, n_items, n_chunks, per_chunk;   // per_chunk: most positions of a chunk
};

// y of up to ROWS_MAX rows. x and w in place: 16-byte aligned rows, K a
// multiple of 8 (bf16) or 4 (f32).
struct RowsArgs {
    const void *x, *w, *a, *bank_b;
    const float *bias;
    void *y;
    int64_t ldx, ldw, ldy;
    int f32, K, N;
    int k_bank;            // row length of a (K of x and w may be padded)
    const void *zero;      // 16 zero bytes or more
    // rows_plan: slices of the depth in steps of 128 bytes, and of the thin
    // products in bytes
    int all_steps, steps, slices, rank_blocks, thin_bytes, thin_slices, thin_blocks;
    int64_t ldp;
    float *partial;        // [slices][rows][ldp]
    float *t;              // [thin_slices][rows][rank_blocks * 16]
    BatchTables b;
};
constexpr int ROWS_STEP = 128;   // bytes of a row in a step
void rows_plan(RowsArgs &a);
bool rows_valid(const RowsArgs &a);
hipError_t launch_rows(const RowsArgs &a, hipStream_t s);

// t[p][r] = scale * sum over k of x[perm[p]][k] * a[run][r][k]
struct ShrinkArgs {
    const void *x;
    const void *a;         // rows of K (by_run: packed, [runs][rp][lda]; else [adapters][rank][K])
    int64_t ldx, lda;
    int by_run, f32, K, rp;
    int slices, per;       // shrink_plan: the depth in slices of `per`
    float *part;           // [slices][rows][rp] with slices > 1
    // null, or JOB_PACK's flags of the other half ([runs][n_flags]): planes of
    // a run with any set are NaN; bad: [runs], with slices > 1
    const int *flags;
    int n_flags;
    int *bad;
    u16 *planes;           // [rows][2 rp] hi | lo, or null
    float *t;              // [rows][rp]
    BatchTables b;
};
void shrink_plan(ShrinkArgs &a, int n);   // slices, per; n products go in one launch
bool shrink_valid(const ShrinkArgs *a, int n);
// One or two thin products (of one batch) in a launch (two, where the depth is cut).
hipError_t launch_shrink(const ShrinkArgs *a, int n, hipStream_t s);

// out[chunk][r][c] = sum over the chunk's positions of p(pos, r) * q[perm[pos]][c],
// p(pos, r) = p[pos * sp + r * sr], r < R, c < C.
struct OuterArgs {
    const void *p;
    const void *q;
    int64_t sp, sr, ldq;
    int p_f32, q_f32;      // types (a float32 q goes with a float32 p)
    int R, C;
    const int *perm;       // or null
    float *out;
    int64_t ld, chunk;     // distance of rows, and of chunks
    // [n_chunks / sub][3]: .., first position, positions, each of them in
    // `sub` pieces of which the last ones may be empty; null: `per` positions
    // in each
    const int *chunks;
    int n_chunks, sub, positions, per;
};
constexpr int MAX_OUTER = 4;
struct Outers {
    int n = 0, blocks = 0;
    int first[MAX_OUTER + 1] = {};
    OuterArgs a[MAX_OUTER];
};
bool add_outer(Outers &o, const OuterArgs &a);   // false: not valid
hipError_t launch_outer(const Outers &o, hipStream_t s);

// Small pieces of work around the products, several in one launch. Blocks of
// one job do not depend on those of another.
enum JobKind {
    // out[r][c], c < ldo: rows (perm[r]) of `in` copied, zeros from cols on;
    // ldo whole 16-byte chunks
    JOB_PAD,
    // float32 rows (perm[r]) as float16 pairs of in * 2^e, one exponent per
    // row (its largest value lands in [2^14, 2^15)): out, e. ldo counts both
    // planes, a multiple of 128
    JOB_SPLIT,
    // out[c][r], r < ldo: the transpose, zeros from rows on; float32 as
    // pairs (ldo as for SPLIT) with one exponent per output row, from the maxima of
    // JOB_COLMAX. sum: NULL, or [ceil(rows / 64)][cols] sums of 64 rows
    JOB_TURN,
    JOB_COLMAX,            // max [parts][cols]: largest magnitudes (as bits)
    JOB_COLSUM,            // sum [parts][cols]
    JOB_COLADD,            // out[c] = sum over parts of sum[part][c]
    // adapter halves per run, in [adapters][C][R] (or in_rc [R][C]):
    // out[run][C][2 rp] with each row's ranks twice (bf16), or by_rank:
    // out[run][rp][ldo]. Rank indices from the run's rank on are zeros, and
    // so are columns beyond C. Not by_rank, values that are not finite become
    // zeros too, and flags [runs][ceil(C / 64)] say where there were any: in
    // the product rows of other runs meet them as factors of zero
    JOB_PACK,
    // out[adapter] = sum over its chunks' pieces of part [piece][rp][C], as [R][C] or
    // (turned) [C][R]; zeros for adapters without rows, and from an
    // adapter's rank on
    JOB_CHUNKS,
    // up to ROWS_MAX rows: out[r][c], rows ldo apart, = sum over parts of
    // sum [part][rows][ldi] + sum over rank of t[position][rank] *
    // in[adapter][rank][c], in the type f32 says
    JOB_ROWS
};
struct Job {
    int kind, blocks, f32, rows, cols, parts;
    const void *in;
    void *out;
    int *e;
    unsigned *max;
    float *sum;
    int64_t ldi, ldo;
    const int *perm;
    int in_rc, by_rank, turned, R, rp, n;   // PACK: n runs, CHUNKS: n adapters; columns in cols
    int sub;               // CHUNKS: pieces of a chunk
    int *flags;            // PACK, not by_rank
    const int *run_id, *run_rank, *run_of, *chunk_first;
    const int4 *row_info;
    const float *t;
};
constexpr int PAD_ITEMS = 1024;    // 16-byte chunks of a block of JOB_PAD
constexpr int SPLIT_WIDE = 1024;   // longest row that JOB_SPLIT gives to a wave
constexpr int MAX_JOBS = 6;
struct Jobs {
    int n = 0, blocks = 0;
    int first[MAX_JOBS + 1] = {};
    Job job[MAX_JOBS];
};
bool add_job(Jobs &j, const Job &job);   // sets its blocks; false: not valid
hipError_t launch_jobs(const Jobs &j, hipStream_t s);

// ---- orthogonalised updates ----
constexpr double COEF_A = 3.4445, COEF_B = -4.7750, COEF_C = 2.0315;
constexpr int ORTH_MAX_STEPS = 16, ORTH_LAMBDAS = ORTH_MAX_STEPS + 1;
constexpr int THIN_MAX = 64;

// One batch of `count` row-major [rows][cols] matrices.
struct OrthArgs {
    const void *g;         // update, or the gradient of a step
    float *m;              // step: momentum (null otherwise)
    int f32;               // type of g and of `out`
    int step, nesterov;
    float beta;
    int rows, cols, count, steps;
    int parts;             // partial sums per matrix
    // planes of X_k / lambda[k], X_k the k-th iterate
    double *sums;          // [count][parts] squared sums
    float *lambda;         // [count][ORTH_LAMBDAS]
    Planes x;              // [n][ld >= m]: the wide orientation
    Planes xt;             // [m][ld >= n]
    // thin matrices: n = min(rows, cols) <= THIN_MAX
    double *gram;          // [count][parts][np * np], np = n rounded up to 16
    float *q;              // [count][np * np]: out = q * (2^e u)
    int *e;                // [count]
    void *out;             // result, or the weights of a step
    u16 *copy;
    float rate, decay;
};
bool orth_valid(const OrthArgs &a, bool thin);
hipError_t launch_norm(const OrthArgs &a, hipStream_t s);   // momentum and squared sums
hipError_t launch_seed(const OrthArgs &a, hipStream_t s);   // planes of the scaled update, lambda
hipError_t launch_thin_gram(const OrthArgs &a, hipStream_t s);   // momentum and partial Gram matrices
hipError_t launch_thin_poly(const OrthArgs &a, hipStream_t s);   // q, e
hipError_t launch_thin_apply(const OrthArgs &a, hipStream_t s);  // out

}  // namespace gemel

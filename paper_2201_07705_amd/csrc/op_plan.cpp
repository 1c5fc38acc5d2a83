// Launch shapes and checks of the operators' kernels: tiles, depth splits and
// slices from the sizes, and whether an argument block is one that its kernel
// and grid can take. Plain host code, which CPU builds share.
#include <algorithm>

#include "op_args.h"

namespace gemel {

int64_t mm_tiles(const MmArgs &a, int T) {
    const int64_t tm = T < 64 ? (a.M + 63) / 64 * (64 / T) : (a.M + T - 1) / T;
    const int64_t tn = T < 64 ? (a.N + 63) / 64 * (64 / T) : (a.N + T - 1) / T;
    return a.sym ? tm * (tm + 1) / 2 : tm * tn;
}

// Tile and depth splits, by the estimated time of the launch: the turns that
// the compute units take, each a step's time for every step and a fixed part
// for the pipeline's start and the epilogue; and, where the depth is split,
// writing and reading the partial sums and the second launch. The times are
// a fit to 23 shapes from 128 x 128 x 8192 to 25088 x 4096 x 4096 at every
// tile and up to 32 splits, within 9% of the measured ones; for each of these
// shapes the tile and split chosen is the fastest one measured. What splits
// are for: a symmetric 512 x 512 result of depth 4608 takes 16.3 us whole and
// 10.2 in 4 splits, one of 4096 x 4096 and 25088 pairs 1322 and 1089 us in 7
// (its 136 tiles of 256 leave half of the 256 compute units idle); 2048 x
// 1000 of 1024 pairs is fastest whole (22.4 us).
double mm_plan(MmArgs &a) {
    struct Form {
        int tile, slots;                        // workgroups that run at once
        double alone, full, fixed, fixed_part;  // microseconds; with partial sums out
    };
    static const Form single[] = {
        {256, 256, 1.40, 1.40, 30.0, 6.5}, {128, 512, 0.48, 0.87, 12.3, 3.4}, {64, 512, 0.12, 0.36, 6.7, 2.5}};
    static const Form pair[] = {
        {256, 256, 2.05, 2.05, 50.0, 7.0}, {128, 512, 0.56, 1.20, 12.5, 3.6}, {64, 512, 0.16, 0.44, 6.3, 2.0}};
    const Form *const forms = a.pair ? pair : single;
    const int steps = (a.K + MM_BK - 1) / MM_BK;
    double best = 1e30;
    for (int i = 0; i < 3; ++i) {   // (the 256 form first: there is always one)
        const Form &f = forms[i];
        if (f.tile < 256 && mm_tiles(a, f.tile) * mm_threads_of(f.tile) > MAX_THREADS) continue;
        const int64_t tiles = mm_tiles(a, f.tile) * a.batch;
        for (int want = 1; want <= 32 && want <= std::max(1, steps / 4); ++want) {
            const int per = (steps + want - 1) / want, splits = (steps + per - 1) / per;
            if (splits != want) continue;
            const int64_t groups = tiles * splits, whole = groups / f.slots, rest = groups % f.slots;
            const double fixed = splits > 1 ? f.fixed_part : f.fixed;
            double us = (double)whole * (per * f.full + fixed);
            if (rest) us += per * (rest > 256 ? f.full : f.alone) + fixed;
            const double bytes = (double)splits * a.batch * a.M * op_round_up(a.N, 4) * (a.sym ? 2 : 4);
            if (splits > 1) us += 4.8 + 0.13 * splits + 2 * bytes / 5.5e6;
            if (splits > 1 && bytes > 1e9) continue;
            if (us < best) {
                best = us;
                a.tile = f.tile;
                a.steps = per;
                a.splits = splits;
            }
        }
    }
    a.ldp = op_round_up(a.N, 4);
    return best;
}

bool mm_fits(const MmArgs &a) {
    return a.M > 0 && a.N > 0 && a.K > 0 && a.K <= MM_MAX_LD && a.batch > 0 && a.batch <= 65535 &&
           mm_tiles(a, a.tile) * mm_threads_of(a.tile) <= MAX_THREADS &&
           (a.splits <= 1 || mm_tiles(a, 32) * 256 <= MAX_THREADS);
}

bool mm_valid(const MmArgs &a) {
    const int nk = (a.K + MM_BK - 1) / MM_BK;
    if (a.K % 8 || a.lda % 8 || a.ldb % 8 || a.lda > MM_MAX_LD || a.ldb > MM_MAX_LD ||
        (a.perm && a.perm_rows * a.lda > (1ll << 30)) || (a.tile != 64 && a.tile != 128 && a.tile != 256) || a.za % 8 ||
        a.zb % 8 || a.lda < a.K || a.ldb < a.K || !a.zero || a.splits < 1 || a.steps < 1 ||
        a.ext % MM_BK || (int64_t)a.splits * a.steps < nk || (int64_t)(a.splits - 1) * a.steps >= nk)
        return false;
    if (!a.a || !a.b || (uintptr_t)a.a % 16 || (uintptr_t)a.b % 16) return false;
    if (a.splits > 1 && (!a.partial || a.ldp % 4 || a.ldp < a.N)) return false;
    if (a.ext && (!a.t || !a.bx || a.runs < 1 || !a.run_start || !a.first_run || a.batch != 1))
        return false;
    if (a.sym && a.M != a.N) return false;
    if (a.epi == EPI_SCALED && (!a.o.ea || !a.o.eb ||
                                (a.runs > 0 && (!a.o.t || !a.o.bx || !a.o.run_at || a.o.rank % 4 || a.o.rank > a.o.rp ||
                                                a.o.ldbx % 4 || a.o.ldbx < a.N))))
        return false;
    if (a.epi != EPI_ROWS && (a.K % MM_BK || a.ext)) return false;
    return mm_fits(a);
}

// Slices of the depth: as many workgroups as run at once (three on a compute
// unit with up to 32 rows, else two), and at least four steps in each; thin
// products 2 KB of each row in a slice, which may take half of those places,
// of float32 a third. 64 rows of 64 adapters, 4096 -> 4096: float32 93 us
// where they may take all (one slice is left), 50 for half, 44 for a third;
// bf16 15.6 for half (4 slices), 17.8 for a third (5).
void rows_plan(RowsArgs &a) {
    const int elem = a.f32 ? 4 : 2;
    a.all_steps = (int)(((int64_t)a.K * elem + ROWS_STEP - 1) / ROWS_STEP);
    a.rank_blocks = (a.b.rank + 15) / 16;
    a.thin_bytes = 2048;
    a.thin_slices = (int)(((int64_t)a.K * elem + a.thin_bytes - 1) / a.thin_bytes);
    a.thin_blocks = a.b.runs ? a.b.n_items * a.rank_blocks * a.thin_slices : 0;
    const int tiles = (a.N + 63) / 64, slots = a.b.rows <= 32 ? 768 : 512;
    const int want = std::max(1, std::min({(slots - std::min(a.thin_blocks, slots / (a.f32 ? 3 : 2))) / tiles, (a.all_steps + 3) / 4, 64}));
    a.steps = (a.all_steps + want - 1) / want;
    a.slices = (a.all_steps + a.steps - 1) / a.steps;
    a.ldp = op_round_up(a.N, 4);
}

bool rows_valid(const RowsArgs &a) {
    const int q = a.f32 ? 4 : 8;
    return !(!a.x || !a.w || !a.y || !a.partial || !a.zero || a.b.rows < 1 || a.b.rows > ROWS_MAX || a.N < 1 || a.K < 1 ||
             a.slices < 1 || a.steps < 1 || (int64_t)(a.slices - 1) * a.steps >= a.all_steps ||
             (int64_t)a.slices * a.steps < a.all_steps || (uintptr_t)a.x % 16 || (uintptr_t)a.w % 16 || a.ldx % q || a.ldw % q ||
             a.K % q || a.ldx < a.K || a.ldw < a.K || a.k_bank > a.K || a.k_bank < 1 || a.ldp < a.N || a.ldp % 4 ||
             (int64_t)a.K * (a.f32 ? 4 : 2) > (1 << 30) ||
             (a.thin_blocks && (!a.a || !a.bank_b || !a.t || a.b.rank > 256)));
}

namespace {
bool tables(const BatchTables &b) {
    return b.perm && b.run_start && b.run_id && b.run_rank && b.run_scale && b.first_run && b.items && b.chunks &&
           b.chunk_first && b.run_of && b.run_at && b.rows > 0 && b.runs > 0 && b.adapters > 0 && b.rank > 0;
}
}  // namespace

// A workgroup takes 2 us for every 512 (float32) or 1024 columns, and adding
// slices a launch of 5 us: the depth is cut where few workgroups would have
// more than 8 us of it, into as many as the card holds at once.
void shrink_plan(ShrinkArgs &a, int n) {
    const int turn = a.f32 ? 512 : 1024, turns = (a.K + turn - 1) / turn;
    const int64_t groups = (int64_t)a.b.n_items * (a.rp / 32) * n;
    a.slices = 1;
    a.per = a.K;
    if (turns <= 4 || groups > 256) return;
    const int want = (int)std::min<int64_t>(turns, 512 / std::max<int64_t>(1, groups));
    a.per = (turns + want - 1) / want * turn;
    a.slices = (a.K + a.per - 1) / a.per;
}

bool shrink_valid(const ShrinkArgs *a, int n) {
    if (n < 1 || n > 2) return false;
    for (int i = 0; i < n; ++i)
        if (!tables(a[i].b) || !a[i].x || !a[i].a || a[i].K <= 0 || a[i].rp % 32 || a[i].rp < a[i].b.rank ||
            a[i].b.n_items <= 0 || !(a[i].t || a[i].planes) || a[i].rp != a[0].rp || a[i].f32 != a[0].f32 ||
            a[i].b.items != a[0].b.items || a[i].slices < 1 || a[i].per < 1 || (int64_t)a[i].slices * a[i].per < a[i].K ||
            (int64_t)(a[i].slices - 1) * a[i].per >= a[i].K || (a[i].slices > 1 && !a[i].part) ||
            (a[i].flags && (a[i].n_flags < 1 || (a[i].slices > 1 && !a[i].bad))))
            return false;
    return true;
}

bool add_outer(Outers &o, const OuterArgs &a) {
    if (o.n >= MAX_OUTER || !a.p || !a.q || !a.out || a.R < 1 || a.C < 1 || a.n_chunks < 1 || (a.sp != 1 && a.sr != 1) ||
        a.ld < a.C || (a.q_f32 && !a.p_f32) || (o.n && a.q_f32 != o.a[0].q_f32) ||
        (a.chunks && (a.sub < 1 || a.n_chunks % a.sub)) ||
        (!a.chunks && (a.per < 1 || a.positions < 1 || (int64_t)a.n_chunks * a.per < a.positions ||
                       (int64_t)(a.n_chunks - 1) * a.per >= a.positions)))
        return false;
    const int cols = a.q_f32 ? 128 : 256;
    const int64_t blocks = (int64_t)((a.C + cols - 1) / cols) * ((a.R + 31) / 32) * a.n_chunks;
    if ((blocks + o.blocks) * 256 > MAX_THREADS) return false;
    o.a[o.n] = a;
    o.first[o.n] = o.blocks;
    o.blocks += (int)blocks;
    o.first[++o.n] = o.blocks;
    return true;
}

bool add_job(Jobs &all, const Job &in) {
    if (all.n >= MAX_JOBS) return false;
    Job &j = all.job[all.n];
    j = in;
    const int64_t across = ((int64_t)j.cols + 63) / 64;
    int64_t blocks = 0;
    bool ok = j.cols > 0;
    switch (j.kind) {
        case JOB_PAD:
            ok = ok && j.in && j.out && j.rows > 0 && j.ldo >= j.cols && j.ldo % (j.f32 ? 4 : 8) == 0;
            blocks = ((int64_t)j.rows * (j.ldo / (j.f32 ? 4 : 8)) + PAD_ITEMS - 1) / PAD_ITEMS;
            break;
        case JOB_SPLIT:
            ok = ok && j.in && j.out && j.e && j.rows > 0 && j.ldo / 2 >= j.cols && j.ldo % (4 * PAIR_RUN) == 0;
            blocks = j.cols > SPLIT_WIDE ? j.rows : ((int64_t)j.rows + 3) / 4;
            break;
        case JOB_TURN:
            ok = ok && j.in && j.out && j.rows > 0 && j.ldo / (j.f32 ? 2 : 1) >= j.rows && j.ldo % (j.f32 ? 4 * PAIR_RUN : 4) == 0 &&
                 (!j.f32 || (j.e && j.max && j.parts > 0));
            blocks = across * ((j.ldo / (j.f32 ? 2 : 1) + 63) / 64);
            ok = ok && (!j.sum || blocks == across * ((j.rows + 63) / 64));
            break;
        case JOB_COLMAX:
            ok = ok && j.in && j.max && j.rows > 0 && j.parts > 0 && j.f32;
            blocks = across * j.parts;
            break;
        case JOB_COLSUM:
            ok = ok && j.in && j.sum && j.rows > 0 && j.parts > 0;
            blocks = across * j.parts;
            break;
        case JOB_COLADD:
            ok = ok && j.sum && j.out && j.parts > 0;
            blocks = across;
            break;
        case JOB_PACK:
            ok = ok && j.in && j.out && j.run_id && j.run_rank && j.R > 0 && j.rp >= j.R && j.rp % 32 == 0 && j.n > 0 &&
                 (j.by_rank ? j.ldo >= j.cols : !j.f32 && j.flags);
            blocks = (j.by_rank ? (j.ldo + 63) / 64 : across) * j.n;
            break;
        case JOB_CHUNKS:
            ok = ok && j.sum && j.sub > 0 && j.out && j.run_of && j.run_rank && j.chunk_first && j.R > 0 && j.rp >= j.R && j.n > 0;
            blocks = across * j.n;
            break;
        case JOB_ROWS:
            ok = ok && j.sum && j.out && j.row_info && j.rows > 0 && j.rows <= ROWS_MAX && j.parts > 0 && j.ldi >= j.cols &&
                 j.ldi % 4 == 0 && j.ldo >= j.cols && (!j.t || (j.in && j.R > 0 && j.R <= 256 && j.rp >= j.R));
            blocks = (((int64_t)j.cols + 1023) / 1024) * j.rows;
            break;
        default: ok = false;
    }
    if (!ok || blocks < 1 || (blocks + all.blocks) * 256 > MAX_THREADS) return false;
    j.blocks = (int)blocks;
    all.first[all.n] = all.blocks;
    all.blocks += j.blocks;
    all.first[++all.n] = all.blocks;
    return true;
}

bool orth_valid(const OrthArgs &a, bool thin) {
    if (!a.g || a.rows <= 0 || a.cols <= 0 || a.count <= 0 || a.count > 65535 || a.parts <= 0 || a.steps < 1 ||
        a.steps > ORTH_MAX_STEPS || (a.step && (!a.m || !a.f32)))
        return false;
    if (thin) return std::min(a.rows, a.cols) <= THIN_MAX && a.gram && a.q && a.e && a.out;
    return a.sums && a.lambda && a.x.hi && a.xt.hi && (a.rows + 63) / 64 <= 65535;
}

}  // namespace gemel

// Launch shapes and checks of the kernels of 4-bit matrices. Plain host code,
// which CPU builds share.
#include <algorithm>

#include "mx_args.h"
#include "op_args.h"

namespace gemel {

namespace {
bool mx_there(const Mx &q) {
    return q.codes && q.scales && q.rows > 0 && q.cols > 0 && q.cols <= MX_MAX_COLS && (uintptr_t)q.codes % 16 == 0 &&
           (uintptr_t)q.scales % 16 == 0;
}
}  // namespace

bool mx_cast_valid(const MxCast &a, bool values) {
    const int e = a.f32 ? 4 : 2;
    if (!mx_there(a.q)) return false;
    if (values) return a.out && (uintptr_t)a.out % e == 0 && a.out_cols >= 1 && a.out_cols <= MX_MAX_COLS && a.ld >= a.out_cols;
    return a.x && (uintptr_t)a.x % e == 0 && a.ld >= a.q.cols;
}

bool mx_planes_valid(const MxPlanes &a) {
    return a.x && a.out && a.rows > 0 && a.cols > 0 && a.ldx >= a.cols && a.ld >= a.cols && a.ld % 8 == 0 &&
           (uintptr_t)a.out % 16 == 0 && (uintptr_t)a.x % 4 == 0;
}

bool mx_sum_valid(const MxSum &a) {
    return a.part && a.parts > 0 && a.rows > 0 && a.cols > 0 && a.ldp >= a.cols && a.ldp % 4 == 0 && a.y && a.ldy >= a.cols &&
           (uintptr_t)a.part % 16 == 0;
}

// Up to MX_FEW rows: 16 outputs to a workgroup, whose waves (at most 16) have
// a group of 512 columns or more each; no slices. Beyond: slices until the
// card is full, of at least 4 steps; 512 outputs to a workgroup where that
// leaves enough of them (37 rows 4096 -> 4096, whose 32 steps fill few
// workgroups: 18.5 us with 512, 13.7 with 256; float32 25088 -> 4096 42 and
// 47). 16 rows 4096 -> 4096 7.7 us, 17 rows 11.5.
void mx_rows_plan(MxRows &a) {
    a.ldp = op_round_up(a.w.rows, 4);
    a.per = a.slices = 1;
    if (a.M <= MX_FEW) {
        a.waves = (int)std::min<int64_t>(mx_groups(a.w.cols), 16);
        return;
    }
    a.waves = 8;
    const int steps = (a.w.cols + 127) / 128, rows = 16 * mx_row_blocks(a.M);
    const int64_t down = (a.M + rows - 1) / rows;
    a.wide = (a.w.rows + 511) / 512 * down * (steps / 4) >= 256;
    const int n = a.wide ? 512 : 256;
    const int64_t tiles = (a.w.rows + n - 1) / n * down;
    const int want = (int)std::max<int64_t>(1, std::min<int64_t>(steps / 4, 256 / tiles));
    a.per = (steps + want - 1) / want;
    a.slices = (steps + a.per - 1) / a.per;
}

bool mx_rows_valid(const MxRows &a) {
    const int steps = (a.w.cols + 127) / 128;
    if (!mx_there(a.w) || a.M < 1 || !a.y || a.ldy < a.w.rows) return false;
    if (a.M <= MX_FEW) {
        if (a.waves < 1 || a.waves > 16) return false;
    } else {
        if (a.waves != 8 || a.slices < 1 || a.per < 1 || (int64_t)a.slices * a.per < steps || (int64_t)(a.slices - 1) * a.per >= steps ||
            a.slices > 65535 || a.q.codes || a.M > MX_MOST)
            return false;
        if (a.slices > 1 && (!a.part || a.ldp < a.w.rows || a.ldp % 4)) return false;
    }
    if (a.q.codes) return mx_there(a.q) && a.q.cols == a.w.cols && a.q.rows == a.M;
    return a.x && (a.planes == 1 || a.planes == 3) && a.ldx >= a.w.cols;
}

int64_t mx_mm_tiles(const MxMm &a) {
    return (int64_t)((a.x.rows + a.tile - 1) / a.tile) * ((a.w.rows + a.tile - 1) / a.tile);
}

// The largest tile that still fills the card, cut over the depth where even
// small ones do not. 4096 -> 4096: 4096 rows in tiles of 256 41 us (3360
// TFLOP/s), 2048 in tiles of 128 26 (2630).
void mx_mm_plan(MxMm &a) {
    const int groups = (int)mx_groups(a.w.cols);
    a.splits = 1;
    a.ldp = op_round_up(a.w.rows, 4);
    for (int tile : {256, 128, 64}) {
        a.tile = tile;
        if (mx_mm_tiles(a) >= 256) break;
    }
    const int64_t tiles = mx_mm_tiles(a);
    const int want = (int)std::max<int64_t>(1, std::min<int64_t>({256 / tiles, groups, 16}));
    a.per = (groups + want - 1) / want;
    a.splits = (groups + a.per - 1) / a.per;
}

bool mx_mm_valid(const MxMm &a) {
    const int groups = (int)mx_groups(a.w.cols);
    return mx_there(a.x) && mx_there(a.w) && a.x.cols == a.w.cols && (a.tile == 64 || a.tile == 128 || a.tile == 256) && a.y &&
           a.ldy >= a.w.rows && a.splits >= 1 && a.splits <= 65535 && a.per >= 1 && a.per * a.splits >= groups &&
           a.per * (a.splits - 1) < groups && (a.splits == 1 || (a.part && a.ldp >= a.w.rows && a.ldp % 4 == 0)) &&
           mx_mm_tiles(a) * mx_threads_of(a.tile) <= MAX_THREADS;
}

}  // namespace gemel

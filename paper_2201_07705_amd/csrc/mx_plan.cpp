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
// a group of 512 columns or more each; no slices (16 rows 4096 -> 4096 7.7 us,
// 17 rows 11.5). Beyond: 256 or 512 outputs to a workgroup and slices of the
// depth, by the estimated time: the turns that the 256 compute units take,
// each a step's time for every step (expanding weights, and products) and a
// fixed part, and the sums of slices. The times are a fit to 10 shapes of 20
// to 16384 rows, forms and slices, 10% off in the mean square; the form taken
// is 0.6% from the fastest one measured in the mean and 24% at worst (2048
// outputs of 512 columns). What is at stake: bf16 25088 -> 4096 37 rows 23.4
// us with 256 outputs, 27.0 with 512, 2048 rows 463 and 393; 1024 rows 4096 ->
// 4096 39.9 whole with 256, 51.3 in two slices with 512.
double mx_rows_plan(MxRows &a) {
    a.ldp = op_round_up(a.w.rows, 4);
    a.per = a.slices = 1;
    a.wide = 0;
    if (a.M <= MX_FEW) {
        a.waves = (int)std::min<int64_t>(mx_groups(a.w.cols), 16);
        return 0;
    }
    a.waves = 8;
    const int steps = (a.w.cols + 127) / 128, blocks = mx_row_blocks(a.M), down = (a.M + 16 * blocks - 1) / (16 * blocks);
    double best = 1e30;
    for (int wide = 0; wide < 2; ++wide) {
        const int n = wide ? 512 : 256, products = a.planes * blocks * (wide ? 4 : 2);
        const double step = wide ? 0.71 + 0.063 * products : 0.47 + 0.07 * products;   // microseconds
        const double fixed = a.planes == 1 ? (wide ? 12 : 5) : (wide ? 7.5 : 6.5);
        const int64_t tiles = (int64_t)((a.w.rows + n - 1) / n) * down;
        const int most = (int)std::max<int64_t>(1, std::min<int64_t>({steps / 2, 512 / tiles, 64}));
        for (int want = 1; want <= most; ++want) {
            const int per = (steps + want - 1) / want;
            if ((steps + per - 1) / per != want) continue;
            const double bytes = want > 1 ? 4.0 * want * a.M * a.ldp : 0;
            if (bytes > 1e9) break;
            double us = 2 + (double)((tiles * want + 255) / 256) * (per * step + fixed);
            if (want > 1) us += 2.5 + 0.1 * want + 2 * bytes / 6.2e6;
            if (us < best) {
                best = us;
                a.wide = wide;
                a.per = per;
                a.slices = want;
            }
        }
    }
    return best;
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

// Argument blocks and launchers of the operators of matrices in microscaled
// 4-bit floating point. Each launcher checks on the host (mx_plan.cpp) that
// its block matches what the kernel and grid assume and returns
// hipErrorInvalidValue instead of launching otherwise.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gemel {

typedef unsigned short u16;

// Rows of 4-bit codes, two to a byte, and a scale byte for each block of 32
// columns, in groups of 512 columns. Rows of codes are padded with zeros to
// whole groups (256 bytes, four steps of a product). Scales lie group by
// group, 16 bytes for each row of the matrix: byte 4 g + s belongs to the block g of the
// group's s-th 128 columns, so that a lane of a product (which holds the
// block g of every step) finds its scales of four steps in one word.
constexpr int MX_BLOCK = 32, MX_GROUP = 512;
struct Mx {
    uint8_t *codes;
    uint8_t *scales;
    int rows, cols;
};
constexpr int64_t mx_groups(int64_t cols) { return (cols + MX_GROUP - 1) / MX_GROUP; }
constexpr int64_t mx_pitch(int64_t cols) { return mx_groups(cols) * (MX_GROUP / 2); }
constexpr int64_t MX_MAX_COLS = 1 << 20;

struct MxCast {
    Mx q;
    const void *x;        // quantise: rows ld apart
    void *out;            // values: rows ld apart, columns [0, out_cols) (zeros beyond cols)
    int64_t ld;
    int f32, out_cols;
};
bool mx_cast_valid(const MxCast &a, bool values);
hipError_t launch_mx_quantize(const MxCast &a, hipStream_t s);
hipError_t launch_mx_values(const MxCast &a, hipStream_t s);

// float32 rows as three bf16 planes whose sum they are: [3][rows][ld]
struct MxPlanes {
    const float *x;
    int64_t ldx;
    u16 *out;
    int64_t ld;           // a multiple of 8, zeros from cols on
    int rows, cols;
};
bool mx_planes_valid(const MxPlanes &a);
hipError_t launch_mx_planes(const MxPlanes &a, hipStream_t s);

// y[m][n] = bias[n] + sum over parts of part[i][m][n] (rows ldp apart)
struct MxSum {
    const float *part;
    int64_t ldp;
    int parts, rows, cols;
    const float *bias;
    void *y;
    int64_t ldy;
    int f32;
};
bool mx_sum_valid(const MxSum &a);
hipError_t launch_mx_sum(const MxSum &a, hipStream_t s);

// Rows that are not quantised against 4-bit weights w: bf16 rows, or three
// planes of float32 ones. Up to MX_FEW rows the waves of a workgroup split
// the depth; beyond that they split the outputs and share the rows in LDS.
constexpr int MX_FEW = 16, MX_ROWS = 1024;   // MX_ROWS: of bf16 always, more by estimate; float32 rows always
constexpr int64_t MX_MOST = 1 << 19;         // rows of a launch
struct MxRows {
    Mx w;
    const u16 *x;
    int64_t ldx, plane;   // rows, and planes, apart
    int planes;           // 1 or 3
    Mx q;                 // instead of x: quantised rows (up to MX_FEW)
    int M;
    // mx_rows_plan: up to MX_FEW rows, waves of a workgroup; else steps of 128
    // columns in a slice, slices, and whether a workgroup takes 512 outputs
    // instead of 256
    int waves, per, slices, wide;
    const float *bias;
    void *y;
    int64_t ldy;
    int f32;              // type of y
    float *part;          // slices > 1: [slices][M][ldp]
    int64_t ldp;
};
// 16 rows each, of a workgroup: as few as hold all rows, or 4 (3 where that
// pads a tenth less)
constexpr int mx_row_blocks(int M) {
    return M <= 32 ? 2 : M <= 48 ? 3 : M <= 64 || 10 * ((M + 47) / 48 * 48) > 9 * ((M + 63) / 64 * 64) ? 4 : 3;
}
// Beyond MX_FEW rows: the rows of a workgroup (of every plane, below each
// other) pass through LDS in steps of 128 columns, in pieces of 8: load i of
// thread t of 512 brings the piece at columns mx_piece_col(t) of the step, of
// row mx_piece_row(i, t, rows). Where rows are no multiple of 32, threads that
// are left over load the last row once more.
constexpr int MX_PIECE_THREADS = 512;
constexpr int mx_piece_loads(int rows) { return (rows * 16 + MX_PIECE_THREADS - 1) / MX_PIECE_THREADS; }
constexpr int mx_piece_col(int thread) { return thread % 16 * 8; }
constexpr int mx_piece_row(int i, int thread, int rows) {
    const int row = (i * MX_PIECE_THREADS + thread) / 16;
    return row < rows ? row : rows - 1;
}
// Columns of the piece at column c that there are.
constexpr int mx_piece_cols(int c, int cols) { return c + 8 <= cols ? 8 : c < cols ? cols - c : 0; }
double mx_rows_plan(MxRows &a);   // the microseconds expected
bool mx_rows_valid(const MxRows &a);
hipError_t launch_mx_rows(const MxRows &a, hipStream_t s);

// Both sides quantised: tiles of T x T.
struct MxMm {
    Mx x, w;
    int tile, per, splits;   // mx_mm_plan: groups of 512 columns in a split
    const float *bias;
    void *y;
    int64_t ldy;
    int f32;
    float *part;             // splits > 1: [splits][x.rows][ldp]
    int64_t ldp;
};
void mx_mm_plan(MxMm &a);
bool mx_mm_valid(const MxMm &a);
constexpr int mx_threads_of(int tile) { return tile == 64 ? 256 : 512; }
int64_t mx_mm_tiles(const MxMm &a);
hipError_t launch_mx_mm(const MxMm &a, hipStream_t s);

}  // namespace gemel

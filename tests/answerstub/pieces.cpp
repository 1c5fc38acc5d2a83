// Every address that the products of more than MX_FEW rows with 4-bit weights
// form for the rows, enumerated with the kernel's own map from threads to
// pieces: prints how many reads leave their row, and how many pieces do not
// come from where their place in LDS says. argv[1] "mistaken": the address of
// a thread that is left over takes the columns of the last piece while the
// bound takes those of the thread, which has to be found out.
#include <algorithm>
#include <cstdio>
#include <cstring>

#include "mx_args.h"

using namespace gemel;

int main(int argc, char **argv) {
    const bool mistaken = argc > 1 && !std::strcmp(argv[1], "mistaken");
    long outside = 0, displaced = 0, reads = 0;
    int most = 0;   // elements beyond the end of the last row
    bool seen[5] = {};
    for (int planes : {1, 3})
        for (int M : {17, 31, 32, 33, 37, 40, 48, 49, 63, 64, 65, 96, 97, 129, 144, 145, 200, 300}) {
            const int blocks = mx_row_blocks(M), rows = 16 * blocks, all = planes * rows;
            seen[blocks] = true;
            for (int K = 1; K <= 1300; K += K < 400 ? 1 : 37)
                for (int m0 = 0; m0 < M; m0 += rows)
                    for (int i = 0; i < mx_piece_loads(all); ++i)
                        for (int t = 0; t < MX_PIECE_THREADS; ++t) {
                            const int id = i * MX_PIECE_THREADS + t, row = mx_piece_row(i, t, all), col = mx_piece_col(t);
                            if (row < 0 || row >= all) ++outside;
                            if (id < all * 16 && (row != id / 16 || col != id % 16 * 8)) ++displaced;
                            const int m = std::min(m0 + row % rows, M - 1);
                            for (int step = 0; step * 128 < K; ++step) {
                                const int at = mistaken ? std::min(id, all * 16 - 1) % 16 * 8 : col;
                                const bool whole = (step + 1) * 128 <= K;
                                const int n = whole ? 8 : mx_piece_cols(step * 128 + col, K);
                                ++reads;
                                if (n == 0 || (n > 0 && step * 128 + at + n <= K)) continue;
                                ++outside;
                                if (m == M - 1) most = std::max(most, step * 128 + at + n - K);
                            }
                        }
        }
    std::printf("%ld %ld %d %d %d\n", outside, displaced, most, reads > 0, seen[2] && seen[3] && seen[4]);
}

// The forms that rows of logits take at the limits of what the calls accept:
// prints how many of them have no launch that is valid, and how many were
// tried. Addresses are not used.
#include <cstdio>
#include <initializer_list>

#include "answer_args.h"
#include "op_args.h"

using namespace gemel;

int main() {
    void *const p = (void *)4096;
    long bad = 0, all = 0;
    for (int f32 : {0, 1})
        for (int rows : {1, 65536, (1 << 22) - 1, 1 << 22})
            for (int classes = 1; classes <= 1 << 20; classes = classes < 16 ? classes + 1 : classes * 9 / 8)
                for (int edge = -1; edge <= 1; ++edge)
                    for (int k : {1, 32, 33, 64}) {
                        Logits l{};
                        l.z = p;
                        l.f32 = f32;
                        l.rows = rows;
                        // (the plan's own edges too: powers of two, and nine of them)
                        int c = classes;
                        for (int w = 64; w <= 1 << 20; w *= 2)
                            if (c > w - w / 8 && c <= w) c = w + edge;
                        l.classes = c < 1 ? 1 : c > 1 << 20 ? 1 << 20 : c;
                        l.ld = 1 << 20;
                        l.inv_t = l.c = 1.f;
                        ScoreArgs s{};
                        s.l = l;
                        score_plan(s.l, s.top = k);
                        s.part = (Part *)p;
                        s.list_value = (float *)p;
                        s.list_index = (int *)p;
                        DistillArgs d{};
                        d.l = l;
                        distill_plan(d.l);
                        ScoreArgs sums{};
                        sums.l = d.l;
                        score_plan(sums.l, 0);
                        sums.part = (Part *)p;
                        d.index = (int *)p;
                        d.value = (float *)p;
                        d.k = k;
                        d.t = 1.f;
                        d.loss = (float *)p;
                        d.dz = p;
                        d.ldd = 1 << 20;
                        d.part = (Part *)p;
                        d.parts = sums.l.chunks;
                        const bool fine = score_valid(s) && distill_valid(d) && (d.l.chunks == 1 || score_valid(sums));
                        if (!fine && bad++ < 3) std::fprintf(stderr, "f32 %d: %d x %d, %d\n", f32, rows, l.classes, k);
                        ++all;
                    }
    std::printf("%ld %ld\n", bad, all);
}

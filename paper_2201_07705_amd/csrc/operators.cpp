// The operators that serve and retrain merged layers: argument checks,
// request tables, workspaces, and the order of their kernels.
#include <climits>
#include <cmath>

#include "op_call.h"

using namespace gemel;
using namespace gemel::op;

namespace {

constexpr int64_t MAX_ROWS = 1 << 22, MAX_DIM = 1 << 20, MAX_COUNT = 65535;
constexpr int64_t NARROW = 64;   // outputs whose dW is summed without copies of x
constexpr int MAX_RANK = 256, MAX_STEPS = ORTH_MAX_STEPS;

// Makes tables whose calls are over spare. A stream that cannot be asked (it
// was destroyed) leaves them to the next wait for the device.
void reclaim(State &st) {
    constexpr int LOOK = 8;   // unfinished ones that are asked for in a call
    int busy = 0;
    for (size_t i = 0; i < st.retired.size();) {
        Retired &r = st.retired[i];
        bool lost = false, done = true;
        r.events.reserve(r.events.size() + r.streams.size());
        st.events.reserve(st.events.size() + r.events.size() + r.streams.size() + 1);
        while (!lost && !r.streams.empty()) {
            hipEvent_t e = nullptr;
            if (st.events.empty()) {
                lost = hipEventCreateWithFlags(&e, hipEventDisableTiming) != hipSuccess;
            } else {
                e = st.events.back();
                st.events.pop_back();
            }
            if (!lost && hipEventRecord(e, r.streams.back()) != hipSuccess) {
                st.events.push_back(e);
                lost = true;
            }
            if (lost) break;
            r.events.push_back(e);
            r.streams.pop_back();
        }
        for (size_t k = 0; !lost && done && busy < LOOK && k < r.events.size(); ++k) {
            const hipError_t q = hipEventQuery(r.events[k]);
            done = q == hipSuccess;
            lost = !done && q != hipErrorNotReady;
        }
        if (lost) (void)hipGetLastError();
        if (!lost && (!done || busy >= LOOK)) {
            ++busy;
            ++i;
            continue;
        }
        (lost ? st.held : st.spare).push_back({r.dev, r.bytes});
        st.events.insert(st.events.end(), r.events.begin(), r.events.end());
        st.retired.erase(st.retired.begin() + (std::ptrdiff_t)i);
    }
}

gemel_status upload(gemel_ctx *ctx, State &st, const std::vector<int32_t> &words, Batch &b) {
    size_t want = 64 << 10;
    while (want < words.size() * 4) want *= 2;
    auto fits = [&]() {
        for (size_t i = 0; i < st.spare.size(); ++i)
            if (st.spare[i].second == want) return (int)i;
        return -1;
    };
    st.outgrown.reserve(st.outgrown.size() + 1);
    int at = fits();
    if (at < 0) {
        reclaim(st);
        at = fits();
    }
    if (at < 0 && st.held.size() >= 32) {
        OPCHK(hipDeviceSynchronize(), "hipDeviceSynchronize");
        st.spare.insert(st.spare.end(), st.held.begin(), st.held.end());
        st.held.clear();
        at = fits();
    }
    if (at >= 0) {
        b.dev = st.spare[(size_t)at].first;
        st.spare.erase(st.spare.begin() + at);
    } else {
        OPCHK(hipMalloc(&b.dev, want), "request tables");
    }
    b.bytes = want;
    hipError_t e = hipSuccess;
    if (st.pinned_bytes < want) {
        if (st.pinned) st.outgrown.push_back(st.pinned);
        st.pinned = nullptr;
        st.pinned_bytes = 0;
        e = hipHostMalloc(&st.pinned, want, hipHostMallocDefault);
        if (e == hipSuccess) st.pinned_bytes = want;
    }
    if (e == hipSuccess) {
        std::memcpy(st.pinned, words.data(), words.size() * 4);
        e = hipMemcpyAsync(b.dev, st.pinned, words.size() * 4, hipMemcpyHostToDevice, st.side);
    }
    if (e == hipSuccess) e = hipStreamSynchronize(st.side);
    if (e != hipSuccess) {
        (void)hipFree(b.dev);
        b.dev = nullptr;
        return hip_fail(ctx, e, "request tables");
    }
    return GEMEL_OK;
}

gemel_status make_batch(gemel_ctx *ctx, const int32_t *ids, const int32_t *n_rows, int n_req, int n_ad, int max_rank,
                        const int32_t *ranks, const float *scales, int32_t *out_id) {
    int64_t rows = 0;
    for (int i = 0; i < n_req; ++i) rows += n_rows[i];
    // rows by adapter: slot 0 none, slot 1 + a adapter a
    std::vector<int> start((size_t)n_ad + 2, 0);
    for (int i = 0; i < n_req; ++i) start[(size_t)(ids[i] + 1)] += n_rows[i];
    std::vector<int> at((size_t)n_ad + 1);
    int sum = 0;
    for (int s = 0; s <= n_ad; ++s) {
        at[(size_t)s] = sum;
        sum += start[(size_t)s];
    }
    std::vector<int> perm((size_t)rows);
    for (int i = 0, row = 0; i < n_req; ++i)
        for (int k = 0; k < n_rows[i]; ++k) perm[(size_t)at[(size_t)(ids[i] + 1)]++] = row++;
    std::vector<int> run_start, run_id, run_rank, run_of((size_t)n_ad, -1), items, chunks, chunk_first;
    std::vector<float> run_scale;
    // chunks of rows whose gradient sums are kept apart and then added in
    // order: about 32 over the batch, so that few adapters still fill the card
    const int per_chunk = (int)std::max<int64_t>(64, op_round_up((rows + 31) / 32, 16));
    for (int a = 0; a < n_ad; ++a) {
        const int n = start[(size_t)a + 1];
        if (!n) continue;
        const int u = (int)run_id.size(), p0 = at[(size_t)a + 1] - n;
        run_of[(size_t)a] = u;
        run_start.push_back(p0);
        run_id.push_back(a);
        run_rank.push_back(ranks ? ranks[a] : max_rank);
        run_scale.push_back(scales ? scales[a] : 1.f);
        const int per_item = rows > ROWS_MAX ? 32 : 16;
        for (int p = 0; p < n; p += per_item)
            for (int v : {u, p0 + p, std::min(per_item, n - p)}) items.push_back(v);
        chunk_first.push_back((int)chunks.size() / 3);
        for (int p = 0; p < n; p += per_chunk)
            for (int v : {u, p0 + p, std::min(per_chunk, n - p)}) chunks.push_back(v);
    }
    std::vector<int> run_at((size_t)rows, -1);
    run_start.push_back((int)rows);
    for (size_t u = 0; u < run_id.size(); ++u)
        std::fill(run_at.begin() + run_start[u], run_at.begin() + run_start[u + 1], (int)u);
    chunk_first.push_back((int)chunks.size() / 3);
    const int runs = (int)run_id.size();
    std::vector<int> first_run;
    for (int64_t p = 0, u = 0; p <= rows + 63; p += 64) {
        while (u < runs && run_start[(size_t)u + 1] <= p) ++u;
        first_run.push_back((int)u);
    }
    std::vector<int> info;
    for (int i = 0, row = 0; rows <= ROWS_MAX && i < n_req; ++i)
        for (int k = 0; k < n_rows[i]; ++k, ++row) {
            const int pos = (int)(std::find(perm.begin(), perm.end(), row) - perm.begin());
            const int u = ids[i] < 0 ? -1 : run_of[(size_t)ids[i]];
            for (int v : {pos, u, ids[i], u < 0 ? 0 : run_rank[(size_t)u]}) info.push_back(v);
        }
    std::vector<int32_t> words;
    auto add = [&](const void *p, size_t n) {
        const size_t o = words.size();
        words.resize(o + (size_t)op_round_up((int64_t)std::max<size_t>(n, 1), 4));
        if (n) std::memcpy(words.data() + o, p, n * 4);
        return o;
    };
    const size_t o_perm = add(perm.data(), perm.size()), o_start = add(run_start.data(), run_start.size()),
                 o_id = add(run_id.data(), run_id.size()), o_rank = add(run_rank.data(), run_rank.size()),
                 o_scale = add(run_scale.data(), run_scale.size()), o_first = add(first_run.data(), first_run.size()),
                 o_items = add(items.data(), items.size()), o_chunks = add(chunks.data(), chunks.size()),
                 o_cf = add(chunk_first.data(), chunk_first.size()), o_of = add(run_of.data(), run_of.size()),
                 o_info = add(info.data(), info.size()), o_at = add(run_at.data(), run_at.size());
    DeviceScope scope(ctx->device);
    State *st = nullptr;
    if (gemel_status s = ready(ctx, &st)) return s;
    auto b = std::make_unique<Batch>();
    size_t id = 0;
    while (id < st->batches.size() && st->batches[id]) ++id;
    if (id == st->batches.size()) st->batches.emplace_back();
    // (giving back allocates nothing)
    st->retired.reserve(st->retired.size() + st->batches.size());
    st->spare.reserve(st->spare.size() + st->batches.size());
    st->held.reserve(st->held.size() + st->batches.size());
    if (gemel_status s = upload(ctx, *st, words, *b)) return s;
    const int *d = (const int *)b->dev;
    BatchTables &t = b->t;
    t.perm = d + o_perm;
    t.run_start = d + o_start;
    t.run_id = d + o_id;
    t.run_rank = d + o_rank;
    t.run_scale = (const float *)(d + o_scale);
    t.first_run = d + o_first;
    t.items = d + o_items;
    t.chunks = d + o_chunks;
    t.chunk_first = d + o_cf;
    t.run_of = d + o_of;
    t.run_at = d + o_at;
    t.row_info = (const int4 *)(d + o_info);
    t.rows = (int)rows;
    t.runs = runs;
    t.adapters = n_ad;
    t.rank = max_rank;
    t.n_items = (int)items.size() / 3;
    t.n_chunks = (int)chunks.size() / 3;
    t.per_chunk = per_chunk;
    st->batches[id] = std::move(b);
    *out_id = (int32_t)id;
    return GEMEL_OK;
}

gemel_status check_projection(gemel_ctx *ctx, const gemel_projection *p, bool adapters) {
    if (!p) return fail(ctx, GEMEL_EINVAL, "proj is null");
    if (p->n_in < 1 || p->n_out < 1 || p->n_in > MAX_DIM || p->n_out > MAX_DIM)
        return fail(ctx, GEMEL_EINVAL, "n_in and n_out must be in 1.." + std::to_string(MAX_DIM));
    if (!p->weight) return fail(ctx, GEMEL_EINVAL, "weight is null");
    if (p->weight_stride < p->n_in) return fail(ctx, GEMEL_EINVAL, "weight_stride is smaller than n_in");
    if (adapters && (!p->a || !p->b)) return fail(ctx, GEMEL_EINVAL, "the batch uses adapters: a and b must be given");
    const int64_t e = ctx->dtype == GEMEL_F32 ? 4 : 2;
    if (gemel_status s = check_aligned(ctx, "a", p->a, e)) return s;
    return check_aligned(ctx, "b", p->b, e);
}
// ---- jobs around the products ----

Job job(int kind, const void *in, int64_t ldi, int rows, int cols, bool f32) {
    Job j{};
    j.kind = kind;
    j.in = in;
    j.ldi = ldi;
    j.rows = rows;
    j.cols = cols;
    j.f32 = f32;
    return j;
}

// A 16-bit copy of an operand: bf16 rows padded, float32 as pairs.
struct Copy {
    size_t o = 0, o_e = 0, o_max = 0;
    int64_t ld = 0;
    int parts = 0;
};
// `rows` rows of `cols` in the copy
Copy plan_copy(Call &c, int64_t rows, int64_t cols, bool f32, bool turned) {
    Copy p;
    p.ld = op_round_up(cols, 64) * (f32 ? 2 : 1);
    p.o = c.lay.take(rows * p.ld, 2);
    if (f32) {
        p.o_e = c.lay.take(rows, 4);
        // column maxima by stretches of the input's rows
        p.parts = (int)std::min<int64_t>(32, (cols + 63) / 64);
        if (turned) p.o_max = c.lay.take(p.parts * rows, 4);
    }
    return p;
}
// The jobs that fill it from `in` (rows ldi apart; turned: the copy is its
// transpose).
bool add_copy(Call &c, const Copy &p, const void *in, int64_t ldi, int rows, int cols, bool f32, bool turned, const int *perm,
              float *sum, Jobs &first, Jobs &second) {
    Job j = job(turned ? JOB_TURN : f32 ? JOB_SPLIT : JOB_PAD, in, ldi, turned ? cols : rows, turned ? rows : cols, f32);
    j.out = c.at<u16>(p.o);
    j.e = c.at<int>(p.o_e);
    j.max = c.at<unsigned>(p.o_max);
    j.ldo = p.ld;
    j.parts = p.parts;
    j.perm = perm;
    j.sum = sum;
    if (turned && f32) {
        Job m = j;
        m.kind = JOB_COLMAX;
        if (!add_job(first, m)) return false;
    }
    return add_job(second, j);
}

// Copies as the operands of a product.
void operands(Call &c, MmArgs &m, const Copy &a, const Copy &b) {
    m.a = c.at<u16>(a.o);
    m.b = c.at<u16>(b.o);
    m.lda = a.ld;
    m.ldb = b.ld;
    m.o.ea = c.at<int>(a.o_e);
    m.o.eb = c.at<int>(b.o_e);
    m.o.out_f32 = 1;
}

// The adapted product out[row] = in[row] * w^T + low-rank part, where `in`
// has K columns and the N rows of the other operand are at w.
struct Adapted {
    const void *in;
    int64_t ld_in;
    int K, N;
    const void *w;       // [N][K] rows ld_w apart, or (w_t) [K][N]
    int64_t ld_w;
    bool w_t;
    const void *bank;    // the adapter half with N
    int bank_rc;         // it lies [rank][N], not [N][rank]
    const float *bias;
    void *out;
    int64_t ld_out;
    u16 *planes = nullptr;   // the thin product (bf16)
    float *t = nullptr;      // (float32)
    // layout
    bool pad_in = false, pad_w = false;
    Copy c_in, c_w;
    size_t o_bank = 0, o_flags = 0;
    MmArgs mm{};
};

// Sizes; returns the floats of partial sums that the product wants.
int64_t plan_adapted(Call &c, const BatchTables &b, bool f32, Adapted &p) {
    const int rp = (int)op_round_up(b.rank, 32);
    MmArgs &m = p.mm;
    m.M = b.rows;
    m.N = p.N;
    m.batch = 1;
    m.pair = f32;
    m.epi = f32 ? EPI_SCALED : EPI_ROWS;
    p.pad_in = f32 || !in_place(p.in, b.rows, p.ld_in, p.K);
    p.pad_w = f32 || p.w_t || !in_place(p.w, p.N, p.ld_w, p.K);
    m.K = f32 ? (int)(2 * op_round_up(p.K, 64)) : p.K % 8 == 0 ? p.K : (int)op_round_up(p.K, 64);
    mm_plan(m);
    if (p.pad_in) p.c_in = plan_copy(c, b.rows, p.K, f32, false);
    if (p.pad_w) p.c_w = plan_copy(c, p.N, p.K, f32, p.w_t);
    if (b.runs) p.o_bank = c.lay.take((int64_t)b.runs * op_round_up(p.N, 4) * rp, 4);
    if (b.runs && !f32) p.o_flags = c.lay.take((int64_t)b.runs * ((p.N + 63) / 64 + 1), 4);   // flags, and one for each run
    return partial_floats(m);
}

bool add_adapted(Call &c, const BatchTables &b, bool f32, Adapted &p, Jobs &first, Jobs &second) {
    const int rp = (int)op_round_up(b.rank, 32);
    if (p.pad_in && !add_copy(c, p.c_in, p.in, p.ld_in, b.rows, p.K, f32, false, b.perm, nullptr, first, second)) return false;
    if (p.pad_w && !add_copy(c, p.c_w, p.w, p.ld_w, p.N, p.K, f32, p.w_t, nullptr, nullptr, first, second)) return false;
    if (!b.runs) return true;
    Job k = job(JOB_PACK, p.bank, 0, 0, p.N, f32);
    k.out = c.at<char>(p.o_bank);
    k.in_rc = p.bank_rc;
    k.by_rank = f32;
    k.R = b.rank;
    k.rp = rp;
    k.n = b.runs;
    k.ldo = op_round_up(p.N, 4);
    k.run_id = b.run_id;
    k.run_rank = b.run_rank;
    if (!f32) k.flags = c.at<int>(p.o_flags);
    return add_job(second, k);
}

gemel_status run_adapted(Call &c, const BatchTables &b, bool f32, Adapted &p, float *partial) {
    gemel_ctx *ctx = c.ctx;
    const int rp = (int)op_round_up(b.rank, 32);
    MmArgs &m = p.mm;
    if (f32) {
        operands(c, m, p.c_in, p.c_w);
        m.o.t = p.t;
        m.o.bx = c.at<float>(p.o_bank);
        m.o.run_at = b.run_at;
        m.o.rp = rp;
        m.o.rank = (int)op_round_up(b.rank, 4);
        m.o.ldbx = op_round_up(p.N, 4);
    } else {
        m.a = p.pad_in ? c.at<u16>(p.c_in.o) : (const u16 *)p.in;
        m.b = p.pad_w ? c.at<u16>(p.c_w.o) : (const u16 *)p.w;
        m.lda = p.pad_in ? p.c_in.ld : p.ld_in;
        m.ldb = p.pad_w ? p.c_w.ld : p.ld_w;
        m.perm = p.pad_in ? nullptr : b.perm;   // copies are in the order of positions
        m.perm_rows = b.rows;
        if (b.runs) {
            m.ext = 2 * rp;
            m.t = p.planes;
            m.bx = c.at<u16>(p.o_bank);
        }
    }
    m.runs = b.runs;
    m.run_start = b.run_start;
    m.first_run = b.first_run;
    m.zero = (const u16 *)c.st->zero;
    m.partial = partial;
    m.o.perm = b.perm;
    m.o.out = p.out;
    m.o.ld = p.ld_out;
    m.o.bias = p.bias;
    OPCHK(launch_mm(m, c.stream), "product");
    return GEMEL_OK;
}

gemel_status get_batch(gemel_ctx *ctx, int32_t id, State **st, Batch **b) {
    State *s = static_cast<State *>(ctx->operators.get());
    if (!s || id < 0 || (size_t)id >= s->batches.size() || !s->batches[(size_t)id])
        return fail(ctx, GEMEL_EINVAL, "unknown batch id " + std::to_string(id));
    *st = s;
    *b = s->batches[(size_t)id].get();
    return GEMEL_OK;
}

ShrinkArgs shrink(const BatchTables &b, bool f32, const void *x, int64_t ldx, int K, const void *a, int64_t lda, bool by_run,
                  int n) {
    ShrinkArgs s{};
    s.x = x;
    s.a = a;
    s.ldx = ldx;
    s.lda = lda;
    s.by_run = by_run;
    s.f32 = f32;
    s.K = K;
    s.rp = (int)op_round_up(b.rank, 32);
    s.b = b;
    shrink_plan(s, n);
    return s;
}

// The thin product takes over what JOB_PACK found in the other half.
void spoil(Call &c, const Adapted &p, ShrinkArgs &s) {
    s.n_flags = (p.N + 63) / 64;
    s.flags = c.at<int>(p.o_flags);
    s.bad = c.at<int>(p.o_flags) + (int64_t)s.b.runs * s.n_flags;
}

int64_t part_floats(const ShrinkArgs &s) { return s.slices > 1 ? (int64_t)s.slices * s.b.rows * s.rp : 0; }

// Few rows: k_rows.hip, on copies of the operands that it cannot read in
// place.
gemel_status adapt_rows(Call &c, const BatchTables &b, bool f32, const gemel_projection *proj, const void *x, int64_t ldx,
                        void *y, int64_t ldy) {
    gemel_ctx *ctx = c.ctx;
    const int64_t e = f32 ? 4 : 2, q = 16 / e, K = proj->n_in, N = proj->n_out, Kp = op_round_up(K, q);
    auto fits = [&](const void *p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld % q == 0 && K % q == 0; };
    const bool copy_x = !fits(x, ldx), copy_w = !fits(proj->weight, proj->weight_stride);
    RowsArgs a{};
    a.f32 = f32;
    a.K = (int)Kp;
    a.N = (int)N;
    a.b = b;
    rows_plan(a);
    const size_t o_x = c.lay.take(copy_x ? b.rows * Kp : 0, e), o_w = c.lay.take(copy_w ? N * Kp : 0, e),
                 o_p = c.lay.take((int64_t)a.slices * b.rows * a.ldp, 4),
                 o_t = c.lay.take(a.thin_blocks ? (int64_t)a.thin_slices * b.rows * a.rank_blocks * 16 : 0, 4);
    if (gemel_status s = workspace(c)) return s;
    a.x = x;
    a.ldx = ldx;
    a.w = proj->weight;
    a.ldw = proj->weight_stride;
    Jobs jobs;
    if (copy_x) {
        Job j = job(JOB_PAD, x, ldx, b.rows, (int)K, f32);
        a.x = j.out = c.at<char>(o_x);
        a.ldx = j.ldo = Kp;
        if (!add_job(jobs, j)) return fail(ctx, GEMEL_EINVAL, "x is too large");
    }
    if (copy_w) {
        Job j = job(JOB_PAD, proj->weight, proj->weight_stride, (int)N, (int)K, f32);
        a.w = j.out = c.at<char>(o_w);
        a.ldw = j.ldo = Kp;
        if (!add_job(jobs, j)) return fail(ctx, GEMEL_EINVAL, "weight is too large");
    }
    OPCHK(launch_jobs(jobs, c.stream), "copies");
    a.a = proj->a;
    a.bank_b = proj->b;
    a.bias = proj->bias;
    a.y = y;
    a.ldy = ldy;
    a.k_bank = (int)K;
    a.zero = c.st->zero;
    a.partial = c.at<float>(o_p);
    a.t = c.at<float>(o_t);
    OPCHK(launch_rows(a, c.stream), "product");
    return GEMEL_OK;
}

gemel_status adapt(gemel_ctx *ctx, int32_t id, const gemel_projection *proj, const void *x, int64_t ldx, void *y,
                   int64_t ldy, hipStream_t stream) {
    State *st;
    Batch *bt;
    if (gemel_status s = get_batch(ctx, id, &st, &bt)) return s;
    const BatchTables &b = bt->t;
    if (gemel_status s = check_projection(ctx, proj, b.runs > 0)) return s;
    if (b.rows == 0) return GEMEL_OK;
    const bool f32 = ctx->dtype == GEMEL_F32;
    const int64_t e = f32 ? 4 : 2, K = proj->n_in, N = proj->n_out, bank = (int64_t)b.adapters * b.rank;
    if (gemel_status s = check_rows(ctx, "x", x, ldx, K, e)) return s;
    if (gemel_status s = check_rows(ctx, "y", y, ldy, N, e)) return s;
    if (gemel_status s = check_rows(ctx, "weight", proj->weight, proj->weight_stride, K, e)) return s;
    if (gemel_status s = check_aligned(ctx, "bias", proj->bias, 4)) return s;
    if (gemel_status s = apart(ctx, {range("y", y, b.rows, N, ldy, e, true),
                                     range("x", x, b.rows, K, ldx, e, false),
                                     range("weight", proj->weight, N, K, proj->weight_stride, e, false),
                                     range("bias", proj->bias, N * 4, false), range("a", proj->a, bank * K * e, false),
                                     range("b", proj->b, bank * N * e, false)}))
        return s;
    DeviceScope scope(ctx->device);
    Call c{ctx, st, stream, bt, {}, nullptr};
    if (b.rows <= ROWS_MAX) return adapt_rows(c, b, f32, proj, x, ldx, y, ldy);
    const int rp = (int)op_round_up(b.rank, 32);
    Adapted p{};
    p.in = x;
    p.ld_in = ldx;
    p.K = (int)K;
    p.N = (int)N;
    p.w = proj->weight;
    p.ld_w = proj->weight_stride;
    p.w_t = false;
    p.bank = proj->b;
    p.bank_rc = 0;
    p.bias = proj->bias;
    p.out = y;
    p.ld_out = ldy;
    ShrinkArgs t = shrink(b, f32, x, ldx, (int)K, proj->a, K, false, 1);
    const size_t o_t = c.lay.take(b.runs ? (int64_t)b.rows * rp : 0, 4),
                 o_tp = c.lay.take(b.runs ? part_floats(t) : 0, 4);
    const size_t o_part = c.lay.take(plan_adapted(c, b, f32, p), 4);
    if (!mm_fits(p.mm)) return fail(ctx, GEMEL_EINVAL, "the projection is too large");
    if (gemel_status s = workspace(c)) return s;
    Jobs first, second;
    if (!add_adapted(c, b, f32, p, first, second)) return fail(ctx, GEMEL_EINVAL, "the projection is too large");
    OPCHK(launch_jobs(second, stream), "copies");
    if (b.runs) {
        (f32 ? (void *&)p.t : (void *&)p.planes) = c.at<void>(o_t);
        t.planes = p.planes;
        t.t = p.t;
        if (!f32) spoil(c, p, t);
        t.part = c.at<float>(o_tp);
        OPCHK(launch_shrink(&t, 1, stream), "thin product");
    }
    return run_adapted(c, b, f32, p, c.at<float>(o_part));
}

// Cuts a product over many positions into stretches: about three workgroups
// on each compute unit, `groups` of them for each stretch.
void stretches(OuterArgs &o, int64_t groups) {
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>({(768 + groups - 1) / groups, (o.positions + 63) / 64, 64}));
    o.per = (int)op_round_up((o.positions + want - 1) / want, 32);
    o.n_chunks = (o.positions + o.per - 1) / o.per;
}

gemel_status zero_out(Call &c, float *p, int64_t n) {
    gemel_ctx *ctx = c.ctx;
    for (int64_t at = 0; p && at < n; at += 1 << 30)
        OPCHK(launch_fill_u32((uint32_t *)p + at, (size_t)std::min<int64_t>(n - at, 1 << 30), 0, Sink{c.stream}), "fill");
    return GEMEL_OK;
}

gemel_status backward(gemel_ctx *ctx, int32_t id, const gemel_projection *proj, const void *x, int64_t ldx, const void *dy,
                      int64_t lddy, void *dx, int64_t lddx, float *dw, float *dbias, float *da, float *db,
                      hipStream_t stream) {
    State *st;
    Batch *bt;
    if (gemel_status s = get_batch(ctx, id, &st, &bt)) return s;
    const BatchTables &b = bt->t;
    if (gemel_status s = check_projection(ctx, proj, b.runs > 0 && (dx || da || db))) return s;
    const bool f32 = ctx->dtype == GEMEL_F32;
    const int64_t e = f32 ? 4 : 2, K = proj->n_in, N = proj->n_out, M = b.rows, bank = (int64_t)b.adapters * b.rank;
    if (M > 0) {
        if (gemel_status s = check_rows(ctx, "x", x, ldx, K, e)) return s;
        if (gemel_status s = check_rows(ctx, "dy", dy, lddy, N, e)) return s;
        if (dx)
            if (gemel_status s = check_rows(ctx, "dx", dx, lddx, K, e)) return s;
        if (gemel_status s = check_rows(ctx, "weight", proj->weight, proj->weight_stride, K, e)) return s;
    }
    for (const auto &g : {std::make_pair("dweight", dw), {"dbias", dbias}, {"da", da}, {"db", db}})
        if (gemel_status s = check_aligned(ctx, g.first, g.second, 4)) return s;
    if (gemel_status s = apart(ctx, {range("dx", dx, M, K, lddx, e, true), range("dweight", dw, N * K * 4, true),
                                     range("dbias", dbias, N * 4, true), range("da", da, bank * K * 4, true),
                                     range("db", db, bank * N * 4, true), range("x", x, M, K, ldx, e, false),
                                     range("dy", dy, M, N, lddy, e, false),
                                     range("weight", proj->weight, N, K, proj->weight_stride, e, false),
                                     range("a", proj->a, bank * K * e, false), range("b", proj->b, bank * N * e, false)}))
        return s;
    if (!dx && !dw && !dbias && !da && !db) return GEMEL_OK;
    DeviceScope scope(ctx->device);
    Call c{ctx, st, stream, bt, {}, nullptr};
    if (M == 0) {
        if (gemel_status s = zero_out(c, da, bank * K)) return s;
        if (gemel_status s = zero_out(c, db, bank * N)) return s;
        if (gemel_status s = zero_out(c, dw, N * K)) return s;
        return zero_out(c, dbias, N);
    }
    float *const no_da = b.runs ? nullptr : da, *const no_db = b.runs ? nullptr : db;   // zeros
    if (!b.runs) da = db = nullptr;
    const int rp = (int)op_round_up(b.rank, 32);
    const int64_t Np = op_round_up(N, 64);
    const bool need_u = b.runs && (dx || da), need_t = b.runs && db;
    // few rows: W is read as it lies for dx, and dW written as the product
    // of a few columns of dy and rows of x, without copies of either (bf16
    // 4096 -> 4096, an adapter for each row: 1 row 90 -> 79 us, 64 rows 275 ->
    // 136; float32 132 -> 80 and 252 -> 150)
    const bool few = M <= ROWS_MAX;
    // few float32 outputs: dW in stretches of rows that read x as it lies,
    // where the transposed pairs of x and the maxima for them would cost more
    // than the product (16384 x 4096, 10 outputs 298 -> 64 us, 64 303 -> 114;
    // 4096 x 512, 64 29 -> 18; at 100 outputs 512 x 4096 takes 26, not 23).
    // bf16 copies are cheap, and the tiles faster: 64 outputs 87 us, not 113.
    // More than 2^21 float32 rows go the same way, whatever the outputs: their
    // transposed pairs would be longer than a product's rows can be (256
    // columns, 128 outputs: 2^21 rows as pairs 4.5 ms, 64 more rows 1.9)
    const bool narrow = dw && !few && f32 && (N <= NARROW || 2 * op_round_up(M, 64) > MM_MAX_LD),
               tiled = dw && !few && !narrow;
    // U = scale dy B and T = scale x A^T
    ShrinkArgs thin[2];
    const int n_thin = need_u + need_t;
    if (need_u) thin[0] = shrink(b, f32, dy, lddy, (int)N, nullptr, Np, true, n_thin);
    if (need_t) thin[need_u] = shrink(b, f32, x, ldx, (int)K, proj->a, K, false, n_thin);
    size_t o_thin[2] = {};
    for (int i = 0; i < n_thin; ++i) o_thin[i] = c.lay.take(part_floats(thin[i]), 4);
    const size_t o_u = c.lay.take(need_u ? M * rp : 0, 4), o_up = c.lay.take(need_u && !f32 && !few ? M * rp : 0, 4),
                 o_t = c.lay.take(need_t ? M * rp : 0, 4), o_bt = c.lay.take(need_u ? b.runs * rp * Np : 0, e);
    int64_t part = 0;
    Adapted p{};
    OuterArgs rows_dx{};
    if (dx && few) {
        OuterArgs &o = rows_dx;
        o.p = dy;
        o.sp = 1;
        o.sr = lddy;
        o.q = proj->weight;
        o.ldq = proj->weight_stride;
        o.p_f32 = o.q_f32 = f32;
        o.R = (int)M;
        o.C = (int)K;
        o.ld = op_round_up(K, 4);
        o.chunk = M * o.ld;
        o.positions = (int)N;
        stretches(o, (K + (f32 ? 127 : 255)) / (f32 ? 128 : 256) * ((M + 31) / 32));
        part = o.n_chunks * o.chunk;
    } else if (dx) {
        p.in = dy;
        p.ld_in = lddy;
        p.K = (int)N;
        p.N = (int)K;
        p.w = proj->weight;
        p.ld_w = proj->weight_stride;
        p.w_t = true;
        p.bank = proj->a;
        p.bank_rc = 1;
        p.out = dx;
        p.ld_out = lddx;
        part = plan_adapted(c, b, f32, p);
        if (!mm_fits(p.mm)) return fail(ctx, GEMEL_EINVAL, "the projection is too large");
    }
    // dW = dy^T x, on transposed copies of both
    MmArgs w{};
    Copy c_dy, c_x;
    OuterArgs rows_dw{};
    size_t o_dw = 0;   // (beside the other sums: one launch writes them all)
    if (narrow) {
        OuterArgs &o = rows_dw;
        o.p = dy;
        o.sp = lddy;
        o.sr = 1;
        o.q = x;
        o.ldq = ldx;
        o.p_f32 = o.q_f32 = f32;
        o.R = (int)N;
        o.C = (int)K;
        o.ld = K;
        o.chunk = N * K;
        o.positions = (int)M;
        stretches(o, (K + (f32 ? 127 : 255)) / (f32 ? 128 : 256) * ((N + 31) / 32));
        if (o.n_chunks > 1) o_dw = c.lay.take(o.n_chunks * o.chunk, 4);
    }
    if (tiled) {
        w.M = (int)N;
        w.N = (int)K;
        w.K = (int)op_round_up(M, 64) * (f32 ? 2 : 1);
        w.batch = 1;
        w.pair = f32;
        w.epi = f32 ? EPI_SCALED : EPI_ROWS;
        mm_plan(w);
        if (!mm_fits(w)) return fail(ctx, GEMEL_EINVAL, "the projection is too large");
        c_dy = plan_copy(c, N, M, f32, true);
        c_x = plan_copy(c, K, M, f32, true);
        part = std::max(part, partial_floats(w));
    }
    // column sums of dy: of 64 rows each where dy is transposed anyway
    const int sums = (int)(tiled ? (M + 63) / 64 : std::min<int64_t>(128, (M + 63) / 64));
    const size_t o_sum = c.lay.take(dbias && !few ? sums * N : 0, 4);
    // pieces of the adapters' chunks: where these have few columns, enough for
    // three workgroups on each compute unit
    auto pieces = [&](int64_t C) {
        const int64_t groups = b.n_chunks * (rp / 32) * ((C + (f32 ? 127 : 255)) / (f32 ? 128 : 256));
        return (int)std::max<int64_t>(1, std::min<int64_t>(768 / std::max<int64_t>(groups, 1), b.per_chunk / 64));
    };
    const size_t o_da = c.lay.take(da ? (int64_t)b.n_chunks * pieces(K) * rp * K : 0, 4),
                 o_db = c.lay.take(db ? (int64_t)b.n_chunks * pieces(N) * rp * N : 0, 4), o_part = c.lay.take(part, 4);
    if (gemel_status s = workspace(c)) return s;

    Jobs first, second, last;
    Outers outers;
    bool ok = !dx || few || add_adapted(c, b, f32, p, first, second);
    float *const sum = dbias && !few ? c.at<float>(o_sum) : dbias;
    if (dw && few) {
        OuterArgs o{};
        o.p = dy;
        o.sp = lddy;
        o.sr = 1;
        o.q = x;
        o.ldq = ldx;
        o.p_f32 = o.q_f32 = f32;
        o.R = (int)N;
        o.C = (int)K;
        o.out = dw;
        o.ld = K;
        o.positions = o.per = (int)M;
        o.n_chunks = 1;
        ok = ok && add_outer(outers, o);
    }
    if (dx && few) {
        rows_dx.out = c.at<float>(o_part);
        ok = ok && add_outer(outers, rows_dx);
    }
    if (narrow) {
        const bool joined = rows_dw.n_chunks > 1;
        rows_dw.out = joined ? c.at<float>(o_dw) : dw;
        ok = ok && add_outer(outers, rows_dw);
        if (joined) {
            Job j = job(JOB_COLADD, nullptr, 0, 0, (int)(N * K), true);
            j.sum = rows_dw.out;
            j.parts = rows_dw.n_chunks;
            j.out = dw;
            ok = ok && add_job(last, j);
        }
    }
    if (tiled) {
        ok = ok && add_copy(c, c_dy, dy, lddy, (int)N, (int)M, f32, true, nullptr, sum, first, second);
        ok = ok && add_copy(c, c_x, x, ldx, (int)K, (int)M, f32, true, nullptr, nullptr, first, second);
    } else if (dbias) {
        Job j = job(JOB_COLSUM, dy, lddy, (int)M, (int)N, f32);
        j.sum = sum;
        j.parts = few ? 1 : sums;
        ok = ok && add_job(second, j);
    }
    if (need_u) {
        Job j = job(JOB_PACK, proj->b, 0, 0, (int)N, f32);
        j.out = c.at<char>(o_bt);
        j.by_rank = 1;
        j.R = b.rank;
        j.rp = rp;
        j.n = b.runs;
        j.ldo = Np;
        j.run_id = b.run_id;
        j.run_rank = b.run_rank;
        ok = ok && add_job(second, j);
    }
    if (dbias && !few) {
        Job j = job(JOB_COLADD, nullptr, 0, 0, (int)N, true);
        j.sum = sum;
        j.parts = sums;
        j.out = dbias;
        ok = ok && add_job(last, j);
    }
    float *const t = need_t ? c.at<float>(o_t) : nullptr, *const u = need_u ? c.at<float>(o_u) : nullptr;
    auto adapter_gradient = [&](const float *left, const void *right, int64_t ld, int64_t C, size_t o_sums, float *out, int turned) {
        OuterArgs o{};
        o.p = left;
        o.sp = rp;
        o.sr = 1;
        o.q = right;
        o.ldq = ld;
        o.p_f32 = 1;
        o.q_f32 = f32;
        o.R = rp;
        o.C = (int)C;
        o.perm = b.perm;
        o.out = c.at<float>(o_sums);
        o.ld = C;
        o.chunk = rp * C;
        o.chunks = b.chunks;
        o.sub = pieces(C);
        o.n_chunks = b.n_chunks * o.sub;
        ok = ok && add_outer(outers, o);
        Job j = job(JOB_CHUNKS, nullptr, 0, 0, (int)C, true);
        j.sum = o.out;
        j.out = out;
        j.sub = o.sub;
        j.turned = turned;
        j.R = b.rank;
        j.rp = rp;
        j.n = b.adapters;
        j.run_of = b.run_of;
        j.run_rank = b.run_rank;
        j.chunk_first = b.chunk_first;
        ok = ok && add_job(last, j);
    };
    if (da) adapter_gradient(u, x, ldx, K, o_da, da, 0);
    if (db) adapter_gradient(t, dy, lddy, N, o_db, db, 1);
    if (dx && few) {
        Job j = job(JOB_ROWS, proj->a, rows_dx.ld, (int)M, (int)K, f32);
        j.sum = rows_dx.out;
        j.parts = rows_dx.n_chunks;
        j.out = dx;
        j.ldo = lddx;
        j.row_info = b.row_info;
        j.t = u;
        j.R = b.rank;
        j.rp = rp;
        ok = ok && add_job(last, j);
    }
    if (!ok) return fail(ctx, GEMEL_EINVAL, "the projection is too large");

    if (gemel_status s = zero_out(c, no_da, bank * K)) return s;
    if (gemel_status s = zero_out(c, no_db, bank * N)) return s;
    OPCHK(launch_jobs(first, stream), "column maxima");
    OPCHK(launch_jobs(second, stream), "copies");
    for (int i = 0; i < n_thin; ++i) thin[i].part = c.at<float>(o_thin[i]);
    if (need_u) {
        p.planes = f32 || few ? nullptr : c.at<u16>(o_up);
        p.t = u;
        thin[0].a = c.at<char>(o_bt);
        thin[0].planes = dx ? p.planes : nullptr;
        if (thin[0].planes) spoil(c, p, thin[0]);
        thin[0].t = u;
    }
    if (need_t) thin[need_u].t = t;
    if (n_thin) OPCHK(launch_shrink(thin, n_thin, stream), "thin products");
    if (dx && !few)
        if (gemel_status s = run_adapted(c, b, f32, p, c.at<float>(o_part))) return s;
    if (tiled) {
        operands(c, w, c_dy, c_x);
        w.zero = (const u16 *)st->zero;
        w.partial = c.at<float>(o_part);
        w.o.out = dw;
        w.o.ld = K;
        OPCHK(launch_mm(w, stream), "product");
    }
    OPCHK(launch_outer(outers, stream), "gradients");
    OPCHK(launch_jobs(last, stream), "sums");
    return GEMEL_OK;
}

// ---- orthogonalised updates ----

// Thin matrices: their Gram matrix, its polynomials, and the result.
gemel_status orthogonal_thin(Call &c, OrthArgs o) {
    gemel_ctx *ctx = c.ctx;
    const int n = std::min(o.rows, o.cols), m = std::max(o.rows, o.cols), np = (int)op_round_up(n, 16);
    // stretches of 64 positions for each workgroup: enough workgroups for
    // two on each compute unit, few enough that one adds their sums
    o.parts = (int)std::max<int64_t>(1, std::min<int64_t>({(m + 63) / 64, 64, (1024 + o.count - 1) / o.count}));
    const size_t og = c.lay.take((int64_t)o.count * o.parts * np * np, 8), oq = c.lay.take((int64_t)o.count * np * np, 4),
                 oe = c.lay.take(o.count, 4);
    if (gemel_status s = workspace(c)) return s;
    o.gram = c.at<double>(og);
    o.q = c.at<float>(oq);
    o.e = c.at<int>(oe);
    OPCHK(launch_thin_gram(o, c.stream), "Gram matrix");
    OPCHK(launch_thin_poly(o, c.stream), "polynomials");
    OPCHK(launch_thin_apply(o, c.stream), "result");
    return GEMEL_OK;
}

// Newton-Schulz on the wide orientation X [n][m], n <= m: S = X X^T,
// M = b S + c S^2, X <- a X + M X. All operands are read along their rows,
// so X is kept in both layouts and S and M, being symmetric, in one.
//
// Where it costs less, two steps share S: with P = a I + M, S' = P S P
// follows from S alone, and X moves on by P' P = a^2 I + Mq at once. What S
// has lost to rounding then grows by one more polynomial, up to 12 times,
// which pairs can afford (2^-22 of S, spread over a whole row) and longer
// chains could not (485 times after five).
//
// bf16 updates take one float16 product of planes where float32 ones take
// three of pairs (hi hi, hi lo, lo hi). What rounding would cost them is in a X: noise of 2^-12 of
// X's large directions, spread over all small ones, would grow with these up
// to 485 times. So X keeps its rest (lo) for that term, while M, S and X in M
// X, whose rounding lands in the directions that are large already or is
// averaged over a whole row, do without, except for their diagonals: once X
// is nearly orthogonal these are most of S and M.
gemel_status orthogonal(Call &c, OrthArgs o) {
    gemel_ctx *ctx = c.ctx;
    if (std::min(o.rows, o.cols) <= THIN_MAX) return orthogonal_thin(c, o);
    const int steps = o.steps;
    const bool step = o.step;
    const int n = std::min(o.rows, o.cols), m = std::max(o.rows, o.cols);
    const int64_t np = op_round_up(n, 64), mp = op_round_up(m, 64), size = (int64_t)o.rows * o.cols;
    const bool lo = step || o.f32, wide = o.rows <= o.cols;
    const int all = o.count;
    // matrices at a time: planes of at most 4 GiB
    const int64_t each = 12 * np * mp + 20 * np * np;
    const int group = (int)std::max<int64_t>(1, std::min<int64_t>(all, (int64_t)(4ll << 30) / each));
    auto planes = [&](int64_t rows, int64_t ld, bool rest) {
        if (lo) ld *= 2;   // pairs
        Planes p{nullptr, nullptr, ld, rows * ld, lo};
        const size_t a = c.lay.take(group * rows * ld, 2), b = rest && !lo ? c.lay.take(group * rows * ld, 2) : 0;
        p.hi = (u16 *)a;
        p.lo = (u16 *)b;
        return p;
    };
    Planes x = planes(n, mp, true), t0 = planes(m, np, true), t1 = planes(m, np, true), s = planes(n, np, lo),
           p = planes(n, np, lo);
    o.parts = (int)std::min<int64_t>(1024, (size + 4095) / 4096);
    const size_t o_sums = c.lay.take((int64_t)group * o.parts, 8), o_lambda = c.lay.take(group * ORTH_LAMBDAS, 4),
                 o_sd = c.lay.take(lo ? 0 : group * np, 4), o_md = c.lay.take(lo ? 0 : group * np, 4);
    MmArgs gram{}, poly{}, next{}, last{}, mix{};
    int64_t part = 0;
    auto shape = [&](MmArgs &a, int M, int N, int64_t K, int epi, bool sym) {
        a.M = M;
        a.N = N;
        a.K = (int)K * (lo ? 2 : 1);
        a.batch = group;
        a.pair = lo;
        a.epi = epi;
        a.sym = sym;
        const double us = mm_plan(a);
        part = std::max(part, partial_floats(a));
        return us;
    };
    const int final = step ? EPI_STEP : EPI_ORTH;
    const double us_gram = shape(gram, n, n, mp, EPI_GRAM, true), us_poly = shape(poly, n, n, np, EPI_POLY, true),
                 us_next = shape(next, m, n, np, EPI_NEXT, false);
    (void)(wide ? shape(last, n, m, np, final, false) : shape(last, m, n, np, final, false));
    // two steps at once: a Gram matrix and an update of X less, three
    // products of n x n matrices more. 512 x 4608 256 -> 240 us, 2048 x 8192
    // 1706 -> 1397, 4096 x 25088 17.3 -> 12.3 ms; at a ratio of 0.93 (1000 x
    // 2048) 261 -> 274 us
    const bool paired = lo && steps > 1 && 3 * us_poly < 0.85 * (us_gram + us_next);
    Planes t{}, m0{}, q{};
    if (paired) {
        (void)shape(mix, n, n, np, EPI_MIX, true);
        t = planes(n, np, true);
        m0 = planes(n, np, true);
        q = planes(n, np, true);
    }
    const size_t o_part = c.lay.take(part, 4);
    for (const MmArgs *a : {&gram, &poly, &next, &last})
        if (!mm_fits(*a)) return fail(ctx, GEMEL_EINVAL, "the matrices are too large");
    if (gemel_status e = workspace(c)) return e;
    for (Planes *b : {&x, &t0, &t1, &s, &p, &t, &m0, &q}) {
        if (!b->ld) continue;
        b->hi = c.at<u16>((size_t)b->hi);
        b->lo = b->pair ? b->hi + PAIR_RUN : b->lo ? c.at<u16>((size_t)b->lo) : nullptr;
    }
    o.sums = c.at<double>(o_sums);
    o.lambda = c.at<float>(o_lambda);
    const int64_t ge = o.f32 ? 4 : 2;
    const char *g0 = (const char *)o.g;
    float *mom0 = o.m;
    const float A = (float)COEF_A;
    for (int at = 0; at < all; at += group) {
        const int count = std::min(group, all - at);
        o.count = count;
        o.g = g0 + at * size * ge;
        o.m = mom0 ? mom0 + at * size : nullptr;
        // a bf16 update is its own float16 plane
        o.x = x;
        o.xt = t0;
        if (!lo) o.x.lo = o.xt.lo = nullptr;
        OPCHK(launch_norm(o, c.stream), "norm");
        OPCHK(launch_seed(o, c.stream), "scaled update");
        // l * r of one batch, into a
        auto planes_of = [&](MmArgs &a, const Planes &l, const Planes &r) {
            a.a = l.hi;
            a.b = r.hi;
            a.lda = l.ld;
            a.ldb = r.ld;
            a.za = l.z;
            a.zb = r.z;
            a.batch = count;
            a.zero = (const u16 *)c.st->zero;
            a.partial = c.at<float>(o_part);
            a.o.sdiag = lo ? nullptr : c.at<float>(o_sd);
            a.o.mdiag = lo ? nullptr : c.at<float>(o_md);
            a.o.diag_z = np;
        };
        auto polynomial = [&](int k, const Planes &to) {
            planes_of(poly, s, s);
            poly.o.s = s;
            poly.o.p = to;
            poly.o.lambda = o.lambda + k;
            return launch_mm(poly, c.stream);
        };
        // to = f^2 (cs u + cs2 v + cv l r)
        auto mixed = [&](const Planes &to, const Planes &l, const Planes &r, const Planes &u, float cs, const Planes &v, float cs2,
                         float cv, int lambdas, int k) {
            planes_of(mix, l, r);
            mix.o.p = to;
            mix.o.s = u;
            mix.o.s2 = v;
            mix.o.cs = cs;
            mix.o.cs2 = cs2;
            mix.o.cv = cv;
            mix.o.lambdas = lambdas;
            mix.o.lambda = o.lambda + k;
            return launch_mm(mix, c.stream);
        };
        Planes from = o.xt, to = t1, now = o.x;
        for (int k = 0; k < steps;) {
            const int by = paired && k + 2 <= steps ? 2 : 1;
            planes_of(gram, now, now);
            gram.o.p = s;
            OPCHK(launch_mm(gram, c.stream), "product");
            const Planes *mul = &p;
            if (by == 2) {
                OPCHK(polynomial(k, m0), "product");
                OPCHK(mixed(t, m0, s, s, A, s, 0.f, 0x1p-14f, 0, k), "product");            // P S
                OPCHK(mixed(s, t, m0, t, A, t, 0.f, 0x1p-14f, 1, k), "product");            // f^2 P S P
                OPCHK(polynomial(k + 1, p), "product");
                OPCHK(mixed(q, p, m0, p, A * 0.25f, m0, A * 0.25f, 0x1p-16f, 0, k), "product");    // P' P - a^2 I, * 2^12
                mul = &q;
            } else {
                OPCHK(polynomial(k, p), "product");
            }
            const float cs = by == 2 ? A * A : A, cv = by == 2 ? 0x1p-12f : 0x1p-14f;
            if (k + by < steps) {
                planes_of(next, from, *mul);
                next.o.s = from;
                next.o.p = to;
                now = x;
                if (!lo && (!wide || k + 2 < steps)) now.lo = nullptr;   // nobody reads it
                next.o.q = now;
                next.o.lambda = o.lambda + k;
                next.o.lambdas = by;
                next.o.cs = cs;
                next.o.cv = cv;
                OPCHK(launch_mm(next, c.stream), "product");
                const Planes read = from.lo ? from : t0;
                from = to;
                to = read;
            } else {
                if (wide)
                    planes_of(last, *mul, from);
                else
                    planes_of(last, from, *mul);
                last.o.s = wide ? now : from;
                last.o.diag_rows = wide;
                last.o.ld = o.cols;
                last.o.z = size;
                last.o.out_f32 = o.f32;
                last.o.out = (char *)o.out + at * size * (step ? 4 : ge);
                last.o.copy = o.copy ? o.copy + at * size : nullptr;
                last.o.rate = o.rate;
                last.o.decay = o.decay;
                last.o.lambda = o.lambda + k;
                last.o.cs = cs;
                last.o.cv = cv;
                OPCHK(launch_mm(last, c.stream), "product");
            }
            k += by;
        }
    }
    return GEMEL_OK;
}

gemel_status check_matrices(gemel_ctx *ctx, int count, int rows, int cols, int steps) {
    if (count < 0 || count > MAX_COUNT) return fail(ctx, GEMEL_EINVAL, "count must be in 0.." + std::to_string(MAX_COUNT));
    if (rows < 1 || cols < 1 || rows > MAX_DIM || cols > MAX_DIM)
        return fail(ctx, GEMEL_EINVAL, "rows and cols must be in 1.." + std::to_string(MAX_DIM));
    if (steps < 1 || steps > MAX_STEPS) return fail(ctx, GEMEL_EINVAL, "steps must be in 1.." + std::to_string(MAX_STEPS));
    return GEMEL_OK;
}

}  // namespace

extern "C" {

gemel_status gemel_adapter_batch(gemel_ctx *ctx, const int32_t *adapter_ids, const int32_t *n_rows, int32_t n_requests,
                                 int32_t n_adapters, int32_t max_rank, const int32_t *ranks, const float *scales,
                                 int32_t *out_batch) {
    if (!ctx) return GEMEL_EINVAL;
    return guarded(ctx, [&]() -> gemel_status {
        if (!out_batch) return fail(ctx, GEMEL_EINVAL, "out_batch is null");
        if (n_requests < 0 || (n_requests > 0 && (!adapter_ids || !n_rows)))
            return fail(ctx, GEMEL_EINVAL, "bad request arrays");
        if (n_adapters < 1 || n_adapters > MAX_COUNT)
            return fail(ctx, GEMEL_EINVAL, "n_adapters must be in 1.." + std::to_string(MAX_COUNT));
        if (max_rank < 1 || max_rank > MAX_RANK)
            return fail(ctx, GEMEL_EINVAL, "max_rank must be in 1.." + std::to_string(MAX_RANK));
        int64_t rows = 0;
        for (int i = 0; i < n_requests; ++i) {
            if (adapter_ids[i] < -1 || adapter_ids[i] >= n_adapters)
                return fail(ctx, GEMEL_EINVAL, "request " + std::to_string(i) + ": unknown adapter " + std::to_string(adapter_ids[i]));
            if (n_rows[i] < 0) return fail(ctx, GEMEL_EINVAL, "request " + std::to_string(i) + ": negative row count");
            rows += n_rows[i];
        }
        if (rows > MAX_ROWS) return fail(ctx, GEMEL_EINVAL, "a batch holds at most " + std::to_string(MAX_ROWS) + " rows");
        for (int a = 0; a < n_adapters; ++a) {
            if (ranks && (ranks[a] < 1 || ranks[a] > max_rank))
                return fail(ctx, GEMEL_EINVAL, "adapter " + std::to_string(a) + ": rank must be in 1..max_rank");
            if (scales && !std::isfinite(scales[a]))
                return fail(ctx, GEMEL_EINVAL, "adapter " + std::to_string(a) + ": scale is not finite");
        }
        return make_batch(ctx, adapter_ids, n_rows, n_requests, n_adapters, max_rank, ranks, scales, out_batch);
    });
}

gemel_status gemel_adapter_batch_free(gemel_ctx *ctx, int32_t batch) {
    if (!ctx) return GEMEL_EINVAL;
    return guarded(ctx, [&]() -> gemel_status {
        State *st;
        Batch *b;
        if (gemel_status s = get_batch(ctx, batch, &st, &b)) return s;
        if (b->held)
            st->held.push_back({b->dev, b->bytes});
        else if (b->streams.empty())
            st->spare.push_back({b->dev, b->bytes});
        else
            st->retired.push_back({b->dev, b->bytes, std::move(b->streams), {}});
        st->batches[(size_t)batch].reset();
        return GEMEL_OK;
    });
}

gemel_status gemel_adapt(gemel_ctx *ctx, int32_t batch, const gemel_projection *proj, const void *x, int64_t x_stride,
                         void *y, int64_t y_stride, void *hip_stream) {
    if (!ctx) return GEMEL_EINVAL;
    return guarded(ctx, [&]() { return adapt(ctx, batch, proj, x, x_stride, y, y_stride, (hipStream_t)hip_stream); });
}

gemel_status gemel_adapt_backward(gemel_ctx *ctx, int32_t batch, const gemel_projection *proj, const void *x,
                                  int64_t x_stride, const void *dy, int64_t dy_stride, void *dx, int64_t dx_stride,
                                  float *dweight, float *dbias, float *da, float *db, void *hip_stream) {
    if (!ctx) return GEMEL_EINVAL;
    return guarded(ctx, [&]() {
        return backward(ctx, batch, proj, x, x_stride, dy, dy_stride, dx, dx_stride, dweight, dbias, da, db,
                        (hipStream_t)hip_stream);
    });
}

gemel_status gemel_orthogonalize(gemel_ctx *ctx, int32_t count, int32_t rows, int32_t cols, const void *g, void *out,
                                 int32_t steps, void *hip_stream) {
    if (!ctx) return GEMEL_EINVAL;
    return guarded(ctx, [&]() -> gemel_status {
        if (gemel_status s = check_matrices(ctx, count, rows, cols, steps)) return s;
        if (count == 0) return GEMEL_OK;
        const int64_t e = ctx->dtype == GEMEL_F32 ? 4 : 2, bytes = (int64_t)count * rows * cols * e;
        if (gemel_status s = check_rows(ctx, "g", g, cols, cols, e)) return s;
        if (gemel_status s = check_rows(ctx, "out", out, cols, cols, e)) return s;
        if (gemel_status s = apart(ctx, {range("out", out, bytes, true), range("g", g, bytes, false)})) return s;
        DeviceScope scope(ctx->device);
        State *st;
        if (gemel_status s = ready(ctx, &st)) return s;
        Call c{ctx, st, (hipStream_t)hip_stream, nullptr, {}, nullptr};
        OrthArgs o{};
        o.g = g;
        o.f32 = ctx->dtype == GEMEL_F32;
        o.rows = rows;
        o.cols = cols;
        o.count = count;
        o.steps = steps;
        o.out = out;
        return orthogonal(c, o);
    });
}

gemel_status gemel_muon_step(gemel_ctx *ctx, int32_t count, int32_t rows, int32_t cols, float *w, float *momentum,
                             const float *g, void *copy, float lr, float beta, float weight_decay, int32_t nesterov,
                             int32_t steps, void *hip_stream) {
    if (!ctx) return GEMEL_EINVAL;
    return guarded(ctx, [&]() -> gemel_status {
        if (gemel_status s = check_matrices(ctx, count, rows, cols, steps)) return s;
        if (!std::isfinite(lr) || !std::isfinite(beta) || !std::isfinite(weight_decay))
            return fail(ctx, GEMEL_EINVAL, "lr, beta and weight_decay must be finite");
        if (count == 0) return GEMEL_OK;
        const int64_t n = (int64_t)count * rows * cols;
        if (gemel_status s = check_rows(ctx, "w", w, cols, cols, 4)) return s;
        if (gemel_status s = check_rows(ctx, "momentum", momentum, cols, cols, 4)) return s;
        if (gemel_status s = check_rows(ctx, "g", g, cols, cols, 4)) return s;
        if (copy && ctx->dtype != GEMEL_BF16) return fail(ctx, GEMEL_EINVAL, "copy is for bf16 contexts: w is float32 already");
        if (copy)
            if (gemel_status s = check_rows(ctx, "copy", copy, cols, cols, 2)) return s;
        if (gemel_status s = apart(ctx, {range("w", w, n * 4, true), range("momentum", momentum, n * 4, true),
                                         range("copy", copy, n * 2, true), range("g", g, n * 4, false)}))
            return s;
        DeviceScope scope(ctx->device);
        State *st;
        if (gemel_status s = ready(ctx, &st)) return s;
        Call c{ctx, st, (hipStream_t)hip_stream, nullptr, {}, nullptr};
        OrthArgs o{};
        o.g = g;
        o.m = momentum;
        o.f32 = 1;
        o.step = 1;
        o.nesterov = nesterov != 0;
        o.beta = beta;
        o.rows = rows;
        o.cols = cols;
        o.count = count;
        o.steps = steps;
        o.out = w;
        o.copy = (u16 *)copy;
        o.rate = (float)((double)lr * std::sqrt(std::max(1., (double)rows / cols)));
        o.decay = (float)((double)lr * weight_decay);
        return orthogonal(c, o);
    });
}

}  // extern "C"

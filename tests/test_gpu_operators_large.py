"""The operators at sizes where they change how they work: long depths that
are cut and joined, tiles of every size with ragged edges, results wider than
one tile, and Newton-Schulz steps taken in pairs. Definitions and tolerances
are those of the small cases."""

import pytest

from test_gpu_operators import (check, close, ctxs, near, orthogonal, problem,  # noqa: F401
                                rand, reference, batch_of, DT)

pytestmark = pytest.mark.gpu

SHAPES = [
    # rows per request, adapters, bank, rank, n_in, n_out
    ([80], [0], 1, 20, 5003, 70),                   # thin sums in slices
    ([1, 0, 9], [1, 0, 1], 3, 4, 9001, 5501),       # the same, few rows
    ([70, 3], [0, -1], 2, 40, 70, 9000),            # only one of the two
    ([100, 30, 10], [1, 0, 1], 2, 8, 20001, 140),   # split depth
    ([19000, 33], [0, 1], 2, 8, 120, 100),          # split over the rows
    ([2000, 65, 2034], [2, -1, 0], 3, 24, 520, 4100),
    ([4200], [0], 1, 48, 4104, 136),
    ([520, 1], [0, 1], 2, 16, 1, 3000),
    ([60], [0], 1, 7, 4999, 3),
    ([3000, 71], [1, -1], 2, 8, 301, 41),           # few outputs, joined
    ([65], [0], 1, 8, 130, 64),                     # few outputs, one stretch
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_adapt_and_gradients(ctxs, dtype, case):  # noqa: F811
    n_rows, ids, bank, rank, k, n = SHAPES[case]
    check(ctxs[dtype], problem(dtype, n_rows, ids, bank, rank, k, n, 100 + case))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_some_gradients_alone(ctxs, dtype):  # noqa: F811
    """Each gradient asked for by itself, with cut depths and without."""
    ctx = ctxs[dtype]
    for rows in ([12, 4], [90, 40]):
        s = problem(dtype, rows, [1, 0], 2, 12, 5200, 2600, 7)
        b = batch_of(ctx, s)
        want = reference(s)
        for name in ("x", "weight", "bias", "a", "b"):
            got = ctx.adapt_backward(b, s["dy"], s["x"], s["w"], s["a"], s["b"],
                                     needs=(name,))
            assert set(got) == {name}
            close(name, got[name], want[name])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(2050, 6200), (6200, 2050), (1030, 1025),
                                       (700, 9000), (3001, 90)])
def test_orthogonalize(ctxs, dtype, rows, cols):  # noqa: F811
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows)
    g = rand(gen, rows, cols, dtype=DT[dtype])
    near(ctxs[dtype].orthogonalize(g), orthogonal(g),
         2.0 ** -8 if dtype == "bf16" else 2.0 ** -17)


@pytest.mark.parametrize("rows,cols", [(2050, 6201), (6201, 2050)])
def test_muon_step(ctxs, rows, cols):  # noqa: F811
    import torch
    gen = torch.Generator(device="cuda").manual_seed(cols)
    f64 = torch.float64
    w, m, g = (rand(gen, rows, cols, std=s, dtype=torch.float32)
               for s in (1.0, 1e-2, 1e-2))
    w0, m1 = w.clone(), 0.95 * m.to(f64) + g.to(f64)
    o = orthogonal(g.to(f64) + 0.95 * m1)
    rate = 0.3 * max(1.0, rows / cols) ** 0.5
    copy = torch.empty_like(w, dtype=torch.bfloat16)
    ctxs["bf16"].muon_step(w, m, g, lr=0.3, momentum=0.95, weight_decay=0.1,
                           copy=copy)
    want = (1 - 0.3 * 0.1) * w0.to(f64) - rate * o
    assert ((m.to(f64) - m1).abs() <= 2.0 ** -22 * (1.95 * m1.abs() + g.abs())).all()
    assert (w.to(f64) - want).norm() <= rate * 2.0 ** -17 * o.norm() + 2.0 ** -22 * w0.norm()
    assert torch.equal(copy, w.bfloat16())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_operands_dropped_while_another_stream_works(ctxs, dtype):  # noqa: F811
    """Operands that nobody holds after the call, and memory of the current
    stream asked for and filled at once."""
    import torch
    ctx = ctxs[dtype]
    s = problem(dtype, [300, 200], [1, 0], 2, 8, 1024, 512, 21)
    b = batch_of(ctx, s)
    want = ctx.adapt(b, s["x"], s["w"], s["a"], s["b"])
    wide = ctx.adapt_backward(b, s["dy"], s["x"], s["w"], s["a"], s["b"])
    o = ctx.orthogonalize(s["w"])
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    outs = []
    for _ in range(10):
        copies = [s[q].clone() for q in ("x", "w", "a", "b", "dy")]
        st.wait_stream(torch.cuda.current_stream())
        outs.append((ctx.adapt(b, *copies[:4], stream=st),
                     ctx.adapt_backward(b, copies[4], *copies[:4], stream=st),
                     ctx.orthogonalize(copies[1], stream=st)))
        shapes = [t.shape for t in copies]
        del copies
        for shape in shapes:
            torch.full(shape, float("nan"), dtype=DT[dtype], device="cuda")
    torch.cuda.synchronize()
    for y, grads, q in outs:
        assert torch.equal(y, want) and torch.equal(q, o)
        assert all(torch.equal(grads[name], wide[name]) for name in wide)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[5, 6, 4], [70, 80, 30], [40, 30, 7]])
@pytest.mark.parametrize("k,n", [(96, 104), (9000, 200), (200, 9000)])
def test_an_adapter_that_is_not_finite_spoils_its_own_rows(ctxs, dtype, rows, k, n):  # noqa: F811
    """Requests of a spoilt adapter, a sound one and none, in one tile."""
    import torch
    ctx = ctxs[dtype]
    s = problem(dtype, rows, [0, 1, -1], 2, 8, k, n, 31)
    want = reference(s)
    b = batch_of(ctx, s)
    own, rest = slice(0, rows[0]), slice(rows[0], None)
    for half, spoilt, at in (("b", float("nan"), (0, 3, 2)), ("b", float("inf"), (0, n - 1, 0)),
                             ("a", float("nan"), (0, 5, k - 1)), ("a", float("-inf"), (0, 7, 1))):
        t = dict(s, **{half: s[half].clone()})
        t[half][at] = spoilt
        y = ctx.adapt(b, s["x"], s["w"], t["a"], t["b"], bias=s["bias"])
        close("y", y[rest], tuple(q[rest] for q in want["y"]))
        assert not bool(torch.isfinite(y[own, at[1] if half == "b" else 0].float()).any())
        got = ctx.adapt_backward(b, s["dy"], s["x"], s["w"], t["a"], t["b"])
        close("x", got["x"][rest], tuple(q[rest] for q in want["x"]))
        assert not bool(torch.isfinite(got["x"][own, at[2] if half == "a" else 0].float()).any())
        for name in ("weight", "bias"):
            close(name, got[name], want[name])
        for name in ("a", "b"):
            close(name, got[name][1:], tuple(q[1:] for q in want[name]))


def test_a_graph_outlives_its_workspace(ctxs):  # noqa: F811
    """Replays after a larger call has grown the stream's workspace."""
    import torch
    ctx = ctxs["bf16"]
    s = problem("bf16", [90, 45], [1, 0], 2, 8, 136, 104, 41)
    big = problem("bf16", [4000], [0], 1, 8, 4096, 2048, 42)
    b, bb = batch_of(ctx, s), batch_of(ctx, big)
    want = ctx.adapt(b, s["x"], s["w"], s["a"], s["b"])
    out = torch.zeros_like(want)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        ctx.adapt(b, s["x"], s["w"], s["a"], s["b"])   # grows the workspace
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        ctx.adapt(b, s["x"], s["w"], s["a"], s["b"], out=out)
    with torch.cuda.stream(st):
        ctx.adapt_backward(bb, big["dy"], big["x"], big["w"], big["a"], big["b"])
    torch.cuda.synchronize()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)

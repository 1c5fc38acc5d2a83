"""Batches of requests made and dropped while the device works on."""

import time

import pytest

from test_gpu_operators import batch_of, close, ctxs, problem, reference  # noqa: F401

pytestmark = pytest.mark.gpu


def busy(stream, ms=400):
    """Products on `stream` for about that long, and an event behind them."""
    import torch
    a = torch.randn(4096, 4096, device="cuda").bfloat16()
    b = torch.empty_like(a)
    torch.mm(a, a, out=b)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(20):
        torch.mm(a, a, out=b)
    torch.cuda.synchronize()
    each = (time.perf_counter() - t) / 20
    with torch.cuda.stream(stream):
        for _ in range(int(ms * 1e-3 / each)):
            torch.mm(a, a, out=b)
        e = torch.cuda.Event()
        e.record()
    return e


def test_new_batches_do_not_wait_for_other_work(ctxs):  # noqa: F811
    import torch
    ctx = ctxs["bf16"]
    s = problem("bf16", [20, 30], [1, 0], 2, 8, 64, 48, 8)
    want = reference(s)["y"]
    batch_of(ctx, s).close()
    args = (s["x"], s["w"], s["a"], s["b"])
    # streams share the device's queues, in which work keeps its order: a
    # stream whose work a copy does not stand behind
    for stream in [torch.cuda.Stream() for _ in range(8)]:
        e = busy(stream)
        batch_of(ctx, s).close()
        if not e.query():
            break
        torch.cuda.synchronize()
    else:
        pytest.skip("every stream's queue is the copies' own")
    with torch.cuda.stream(stream):
        b = batch_of(ctx, s)
        outs = [ctx.adapt(b, *args, bias=s["bias"])]   # behind the busy work
        b.close()
    # many more than are kept before anything is waited for: some never used,
    # some used on the busy stream
    for i in range(200):
        b = batch_of(ctx, s)
        if i % 4 == 0:
            with torch.cuda.stream(stream):
                outs.append(ctx.adapt(b, *args, bias=s["bias"]))
        b.close()
    assert not e.query()   # all that while the work went on
    torch.cuda.synchronize()
    for y in outs:
        assert torch.equal(y, outs[0])
    close("y", outs[0], want)


def test_graphs_of_streams_of_their_own_replay_together(ctxs):  # noqa: F811
    """Each holds the workspace of the stream that it was captured on, so
    their replays on other streams need no order."""
    import torch
    ctx = ctxs["bf16"]
    work = []
    for i in range(2):
        s = problem("bf16", [700 + 50 * i, 90], [1, 0], 2, 16, 1032, 776, 60 + i)
        b, st = batch_of(ctx, s), torch.cuda.Stream()
        args = (s["x"], s["w"], s["a"], s["b"])
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            want = [ctx.adapt(b, *args), ctx.adapt_backward(b, s["dy"], *args)["weight"]]
        torch.cuda.synchronize()
        outs = [torch.zeros_like(t) for t in want]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            ctx.adapt(b, *args, out=outs[0])
            ctx.adapt_backward(b, s["dy"], *args, needs=("weight",), outputs={"weight": outs[1]})
        work.append((graph, torch.cuda.Stream(), want, outs, (s, b)))
    for _ in range(6):
        for _, _, _, outs, _ in work:
            for t in outs:
                t.zero_()
        torch.cuda.synchronize()
        for graph, on, _, _, _ in work:
            with torch.cuda.stream(on):
                graph.replay()
                graph.replay()
        torch.cuda.synchronize()
        for _, _, want, outs, _ in work:
            assert all(torch.equal(p, q) for p, q in zip(want, outs))


def test_the_current_stream_without_the_private_entry(ctxs, monkeypatch):  # noqa: F811
    import torch
    from paper_2201_07705_amd import gemel as G
    st = torch.cuda.Stream()
    for on in (torch.cuda.current_stream(), st):
        with torch.cuda.stream(on):
            assert G._current_stream(0) == on.cuda_stream
            with monkeypatch.context() as m:
                m.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
                assert G._current_stream(0) == on.cuda_stream
                ctxs["bf16"].orthogonalize(torch.ones(8, 8, device="cuda", dtype=torch.bfloat16))

"""Drive a CPU build of the operators' host code (stand-in HIP runtime,
bounds-checked launchers, AddressSanitizer) through calls of given sizes. Run
as a subprocess with libasan preloaded: argv is the library and a JSON list of
calls; prints one JSON line with each call's status, message and launches,
and the violations found."""

import ctypes
import json
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, ROOT)

from paper_2201_07705_amd import gemel as G  # noqa: E402

I32 = ctypes.c_int32


class Driver:
    def __init__(self, path):
        self.L = L = G.load(path)
        L.hipMalloc.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_size_t]
        L.hipFree.argtypes = [ctypes.c_void_p]
        L.opstub_violations.restype = L.opstub_launches.restype = ctypes.c_long
        L.hoststub_violations.restype = ctypes.c_long
        L.hoststub_set_capturing.argtypes = [ctypes.c_void_p]
        L.opstub_last.restype = ctypes.c_char_p
        L.opstub_device_waits.restype = L.hoststub_allocs.restype = ctypes.c_long
        self.ctx = {}
        for dtype, code in (("f32", G.F32), ("bf16", G.BF16)):
            h = ctypes.c_void_p()
            assert L.gemel_create(ctypes.byref(h), 0, code, 0) == G.OK
            self.ctx[dtype] = h
        self.held = []

    def memory(self, rows, cols, stride, elem, shift=0):
        """Device memory of exactly that many rows, `shift` elements into it."""
        p = ctypes.c_void_p()
        n = ((rows - 1) * stride + cols) * elem if rows > 0 else 0
        assert self.L.hipMalloc(ctypes.byref(p), max(n, 0) + shift * elem) == 0
        self.held.append(p)
        return p.value + shift * elem

    def drop(self):
        for p in self.held:
            self.L.hipFree(p)
        self.held = []

    def projection(self, c, ctx):
        e = 4 if c["dtype"] == "f32" else 2
        rows, k, n, bank, rank = sum(c["n_rows"]), c["k"], c["n"], c["bank"], c["rank"]
        pad, shift = c.get("pad", 0), c.get("shift", 0)
        L, out = self.L, I32(-1)
        ids, nr = c["ids"], c["n_rows"]
        ranks = c.get("ranks")
        st = L.gemel_adapter_batch(
            ctx, (I32 * max(len(ids), 1))(*ids), (I32 * max(len(ids), 1))(*nr),
            len(ids), bank, rank, None if ranks is None else (I32 * bank)(*ranks),
            None, ctypes.byref(out))
        if st != G.OK:
            return st
        w = self.memory(n, k, k + pad, e, shift)
        p = G.Projection(k, n, w, k + pad, self.memory(1, n, n, 4),
                         self.memory(bank * rank, k, k, e),
                         self.memory(bank * n, rank, rank, e))
        if c.get("bare"):
            p.a = p.b = None
        off = c.get("off", {})   # bytes that a pointer is moved by
        for name in off:
            if not name.startswith("d"):
                setattr(p, name, getattr(p, name) + off[name])
        x = self.memory(rows, k, k + pad, e, shift)
        if c["op"] == "adapt":
            if "beside" in c:   # y: columns of the matrix that x lies in
                y, ldy = x + c["beside"] * e, k + pad + c.get("skew", 0)
            else:
                y, ldy = self.memory(rows, n, n + pad, e, shift), n + pad
            st = L.gemel_adapt(ctx, out.value, ctypes.byref(p), x, k + pad, y, ldy, None)
        else:
            needs = c.get("needs", ["x", "weight", "bias", "a", "b"])
            shapes = {"weight": (n, k), "bias": (1, n), "a": (bank * rank, k),
                      "b": (bank * n, rank)}
            g = {name: self.memory(r, q, q, 4) + off.get("d" + name, 0) if name in needs else None
                 for name, (r, q) in shapes.items()}
            dx = self.memory(rows, k, k + pad, e, shift) if "x" in needs else None
            st = L.gemel_adapt_backward(
                ctx, out.value, ctypes.byref(p), x, k + pad,
                self.memory(rows, n, n + pad, e, shift), n + pad, dx, k + pad,
                g["weight"], g["bias"], g["a"], g["b"], None)
        message = L.gemel_last_error(ctx)
        assert L.gemel_adapter_batch_free(ctx, out.value) == G.OK
        return st, message

    def matrices(self, c, ctx):
        L = self.L
        count, rows, cols = c["count"], c["rows"], c["cols"]
        e = 4 if c["dtype"] == "f32" else 2
        total = count * rows
        if c["op"] == "orthogonalize":
            st = L.gemel_orthogonalize(ctx, count, rows, cols, self.memory(total, cols, cols, e),
                                       self.memory(total, cols, cols, e), c.get("steps", 5), None)
        else:
            w, m, g = (self.memory(total, cols, cols, 4) for _ in range(3))
            copy = self.memory(total, cols, cols, 2) if c["dtype"] == "bf16" else None
            st = L.gemel_muon_step(ctx, count, rows, cols, w, m, g, copy, .1, .9, .01, 1,
                                   c.get("steps", 5), None)
        return st, L.gemel_last_error(ctx)

    def rounds(self, c):
        """A server's rounds: each makes a batch, uses it on one of the
        streams and gives it back, while events answer c["answer"]. The waits
        for the device and the memory that only the batches took."""
        L, ctx, out = self.L, self.ctx["bf16"], I32(-1)
        streams = [None]
        for _ in range(c["streams"] - 1):
            s = ctypes.c_void_p()
            assert L.hipStreamCreateWithFlags(ctypes.byref(s), 1) == 0
            streams.append(s)
        k, n = 16, 24
        p = G.Projection(k, n, self.memory(n, k, k, 2), k, None, self.memory(8, k, k, 2), self.memory(n, 8, 8, 2))
        x, y = self.memory(4, k, k, 2), self.memory(4, n, n, 2)
        res = []
        for answer in c["answers"]:
            L.opstub_events_answer(answer)
            waits, allocs = L.opstub_device_waits(), L.hoststub_allocs()
            for i in range(c["rounds"]):
                assert L.gemel_adapter_batch(ctx, (I32 * 1)(0), (I32 * 1)(4), 1, 1, 8, None, None,
                                             ctypes.byref(out)) == G.OK
                s = streams[i % len(streams)]
                # (rounds of the first phase are not captured)
                L.hoststub_set_capturing(s if c.get("capture") and res else None)
                assert L.gemel_adapt(ctx, out.value, ctypes.byref(p), x, k, y, n, s) == G.OK
                L.hoststub_set_capturing(None)
                assert L.gemel_adapter_batch_free(ctx, out.value) == G.OK
            res.append([L.opstub_device_waits() - waits, L.hoststub_allocs() - allocs])
        L.opstub_events_answer(0)
        return res

    def growing(self, c):
        """Batches of ever more rows; the waits for the device."""
        L, ctx, out = self.L, self.ctx["f32"], I32(-1)
        waits = L.opstub_device_waits()
        for rows in c["n_rows"]:
            assert L.gemel_adapter_batch(ctx, (I32 * 1)(0), (I32 * 1)(rows), 1, 1, 8, None, None,
                                         ctypes.byref(out)) == G.OK
            assert L.gemel_adapter_batch_free(ctx, out.value) == G.OK
        return L.opstub_device_waits() - waits

    def threads(self, c):
        """Calls on hipStreamPerThread, one after the other, from threads of
        their own that stay alive: the memory that each took, and the waits
        for the device of batches that are given back."""
        import threading
        L, ctx, out = self.L, self.ctx["f32"], I32(-1)
        w, x, y = self.memory(8, 8, 8, 4), self.memory(90, 8, 8, 4), self.memory(90, 8, 8, 4)
        p = G.Projection(8, 8, w, 8, None, None, None)
        took, end, turn = [], threading.Event(), threading.Event()

        def one():
            for _ in range(2):
                assert L.gemel_adapter_batch(ctx, (I32 * 1)(-1), (I32 * 1)(90), 1, 1, 8, None, None,
                                             ctypes.byref(out)) == G.OK
                before = L.hoststub_allocs()
                assert L.gemel_adapt(ctx, out.value, ctypes.byref(p), x, 8, y, 8, 2) == G.OK
                took.append(L.hoststub_allocs() - before)
                assert L.gemel_adapter_batch_free(ctx, out.value) == G.OK
            turn.set()
            end.wait()

        alive = []
        for _ in range(c["threads"]):
            turn.clear()
            alive.append(threading.Thread(target=one))
            alive[-1].start()
            turn.wait()
        end.set()
        for t in alive:
            t.join()
        return took

    def call(self, c):
        if c["op"] == "threads":
            res = self.threads(c)
            self.drop()
            return res
        if c["op"] == "growing":
            return self.growing(c)
        if c["op"] == "rounds":
            res = self.rounds(c)
            self.drop()
            return res
        ctx = self.ctx[c["dtype"]]
        before = self.L.opstub_launches()
        st, message = (self.projection if "k" in c else self.matrices)(c, ctx)
        self.drop()
        return {"status": st, "message": (message or b"").decode() if st else "",
                "launches": self.L.opstub_launches() - before}


def main():
    d = Driver(sys.argv[1])
    calls = [d.call(c) for c in json.loads(sys.argv[2])]
    for h in d.ctx.values():
        assert d.L.gemel_destroy(h) == G.OK
    print(json.dumps({"calls": calls, "violations": d.L.opstub_violations() + d.L.hoststub_violations(),
                      "last": (d.L.opstub_last() or b"").decode()}))


if __name__ == "__main__":
    main()

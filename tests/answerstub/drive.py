"""Drive a CPU build of the host code of answers, distillation and 4-bit
matrices (stand-in HIP runtime, bounds-checked launchers, AddressSanitizer).
Run as a subprocess with libasan preloaded: argv is the library and a JSON
list of calls; prints one JSON line with each call's status, message and
kernels, and the violations found."""

import ctypes
import json
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, ROOT)

from paper_2201_07705_amd import gemel as G  # noqa: E402


class Driver:
    def __init__(self, path):
        self.L = L = G.load(path)
        L.hipMalloc.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_size_t]
        L.hipFree.argtypes = [ctypes.c_void_p]
        for name in ("answerstub_violations", "opstub_violations", "hoststub_violations", "opstub_launches"):
            getattr(L, name).restype = ctypes.c_long
        L.answerstub_names.restype = L.answerstub_last.restype = ctypes.c_char_p
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

    def matrix(self, rows, cols, change=()):
        """Codes and scales, to their last byte."""
        codes, scales = ((rows, 256 * -(-cols // 512)), (-(-cols // 512), rows * 16))
        return G.Mx(rows, cols, self.memory(*codes, codes[1], 1) + change[0] if change else self.memory(*codes, codes[1], 1),
                    self.memory(*scales, scales[1], 1) + (change[1] if change else 0))

    def capture(self):
        """A context's first call on a stream that is captured, and the same
        call before and after another one."""
        L, h, s = self.L, ctypes.c_void_p(), ctypes.c_void_p()
        L.hoststub_set_capturing.argtypes = [ctypes.c_void_p]
        assert L.gemel_create(ctypes.byref(h), 0, G.BF16, 0) == G.OK
        assert L.hipStreamCreateWithFlags(ctypes.byref(s), 1) == 0
        a = G.Answers(entropy=self.memory(4, 1, 1, 4))
        narrow, wide = self.memory(4, 100, 100, 4), self.memory(4, 9000, 9000, 4)
        res = []
        for captured, z, n in ((1, narrow, 100), (0, narrow, 100), (1, narrow, 100), (1, wide, 9000), (0, wide, 9000), (1, wide, 9000)):
            L.hoststub_set_capturing(s if captured else None)
            res.append(L.gemel_log_probs(h, 4, n, z, n, G.F32, None, 0, 1.0, a, s))
            L.hoststub_set_capturing(None)
        assert L.gemel_destroy(h) == G.OK
        return res

    def call(self, c):
        L, op = self.L, c["op"]
        if op == "capture":
            return self.capture()
        ctx = self.ctx[c.get("ctx", "bf16")]
        e = 4 if c["dtype"] == "f32" else 2
        code = G.F32 if c["dtype"] == "f32" else G.BF16
        rows, pad, shift = c["rows"], c.get("pad", 0), c.get("shift", 0)
        others = L.opstub_launches()   # (copies and bf16 products, among them)
        off = c.get("off", {})   # bytes that a pointer is moved by

        def mem(name, r, q):
            return self.memory(1, r * q, r * q, 4) + off.get(name, 0)

        if op in ("log_probs", "distill", "distill_backward"):
            k, n = c["k"], c["classes"]
            z = self.memory(rows, n, n + pad, e, shift) + off.get("logits", 0)
            if op == "log_probs":
                needs = c.get("needs", [f[0] for f in G.Answers._fields_])
                a = G.Answers(**{name: mem(name, rows, k if name.startswith("top") else 1) for name in needs})
                st = L.gemel_log_probs(ctx, rows, n, z, n + pad, code, None if c.get("bare") else mem("labels", rows, 1), k,
                                       c.get("t", 1.0), a, None)
            else:
                index, value, loss = mem("indices", rows, k), mem("values", rows, k), mem("loss", rows, 1)
                if op == "distill":
                    st = L.gemel_distill(ctx, rows, n, z, n + pad, code, index, value, k, c.get("t", 1.0), loss, None)
                else:
                    d = z + c["beside"] * e if "beside" in c else self.memory(rows, n, n + pad, e, shift)
                    st = L.gemel_distill_backward(ctx, rows, n, mem("dloss", rows, 1), z, n + pad, code, index, value, k,
                                                  c.get("t", 1.0), d, n + pad, loss if c.get("loss", 1) else None, None)
        elif op in ("quantize", "dequantize"):
            x = self.memory(rows, c["cols"], c["cols"] + pad, e, shift) + off.get("x", 0)
            q = self.matrix(rows, c["cols"], (off.get("codes", 0), off.get("scales", 0)))
            st = L.gemel_mx_quantize(ctx, x, c["cols"] + pad, code, q, None) if op == "quantize" else \
                L.gemel_mx_dequantize(ctx, q, x, c["cols"] + pad, code, None)
        else:
            k, n = c["k"], c["n"]
            w = self.matrix(n, k, (off.get("codes", 0), off.get("scales", 0)))
            x = q = None
            if c["acts"] != "mx":
                x = self.memory(rows, k, k + pad, e, shift) + off.get("x", 0)
            if c["acts"] != "float":
                q = self.matrix(rows, k + c.get("more", 0))
            y = x + c["beside"] * e if "beside" in c else self.memory(rows, n, n + pad, e, shift)
            bias = self.memory(1, n, n, 4) + off.get("bias", 0) if c.get("bias", 1) else None
            st = L.gemel_mx_product(self.ctx[c["dtype"]], rows, x, k + pad, q, w, bias, y,
                                    (k if "beside" in c else n) + pad, None)
            ctx = self.ctx[c["dtype"]]
        for p in self.held:
            L.hipFree(p)
        self.held = []
        return {"status": st, "message": (L.gemel_last_error(ctx) or b"").decode() if st else "",
                "kernels": L.answerstub_names().decode(), "others": L.opstub_launches() - others}


def main():
    d = Driver(sys.argv[1])
    calls = [d.call(c) for c in json.loads(sys.argv[2])]
    for h in d.ctx.values():
        assert d.L.gemel_destroy(h) == G.OK
    print(json.dumps({"calls": calls, "violations": d.L.answerstub_violations() + d.L.opstub_violations() +
                      d.L.hoststub_violations(), "last": (d.L.answerstub_last() or b"").decode()}))


if __name__ == "__main__":
    main()

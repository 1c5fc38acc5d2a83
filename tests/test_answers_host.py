"""The host code of answers, distillation and 4-bit matrices (checks, plans,
workspaces, argument blocks) compiled for the CPU with AddressSanitizer and
driven through calls of many shapes. Every launch checks that its operands and
results may be accessed as wholes: they are allocated to their last byte, and
the pieces of a workspace have gaps between them that may not be touched. What
a kernel's threads address within them is not looked at, but for the rows of
products with more than 16 of them. No GPU is needed."""

import json
import os
import random
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUB = os.path.join(ROOT, "tests", "answerstub")
OPS = os.path.join(ROOT, "tests", "opstub")
HOST = os.path.join(ROOT, "tests", "hoststub")
LIB = os.path.join(ROOT, "_build", "libgemel_answers.so")
CSRC = os.path.join(ROOT, "paper_2201_07705_amd", "csrc")


@pytest.fixture(scope="module")
def lib():
    os.makedirs(os.path.dirname(LIB), exist_ok=True)
    tmp = f"{LIB}.{os.getpid()}"
    flags = ["g++", "-std=c++17", "-g", "-O1", "-fsanitize=address", "-fno-omit-frame-pointer", "-fPIC", f"-I{OPS}", f"-I{HOST}",
             f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}"]
    sources = [os.path.join(OPS, "opstub.cpp"), os.path.join(STUB, "answerstub.cpp")]
    sources += [os.path.join(CSRC, name + ".cpp") for name in ("registry", "plan", "batching", "operators", "op_plan", "answers",
                                                               "answer_plan", "mx", "mx_plan")]
    objects = [f"{tmp}.{k}.o" for k in range(len(sources) + 1)]
    jobs = [flags + ["-c", src, "-o", obj] for src, obj in zip(sources, objects)]
    # (the runtime's own stand-in is compiled without what the operators' adds to it)
    jobs.append([f for f in flags if f != f"-I{OPS}"] + ["-c", os.path.join(HOST, "hoststub.cpp"), "-o", objects[-1]])
    with ThreadPoolExecutor(max_workers=8) as ex:
        list(ex.map(subprocess.check_call, jobs))
    subprocess.check_call(flags + ["-shared"] + objects + ["-o", tmp])
    for obj in objects:
        os.remove(obj)
    os.replace(tmp, LIB)
    return LIB


def drive(lib, calls):
    asan = subprocess.check_output(["gcc", "-print-file-name=libasan.so"], text=True).strip()
    env = dict(os.environ, LD_PRELOAD=asan, ASAN_OPTIONS="detect_leaks=0:allocator_may_return_null=1")
    r = subprocess.run(["python", os.path.join(STUB, "drive.py"), lib, json.dumps(calls)], capture_output=True, text=True,
                       env=env, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    return json.loads(r.stdout.strip().splitlines()[-1])


def sound(lib, calls):
    out = drive(lib, calls)
    for c, o in zip(calls, out["calls"]):
        assert o["status"] == 0 and o["kernels"], (c, o)
    assert out["violations"] == 0, out["last"]
    return [o["kernels"] for o in out["calls"]]


def _log(rng, lo, hi):
    import math
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


@pytest.mark.parametrize("seed", range(3))
def test_logits_stay_in_their_memory(lib, seed):
    rng = random.Random(seed)
    calls = []
    for _ in range(150):
        classes = _log(rng, 1, 1 << 20)
        c = {"op": rng.choice(["log_probs", "distill", "distill_backward"]), "dtype": rng.choice(["f32", "bf16"]),
             "ctx": rng.choice(["f32", "bf16"]), "rows": _log(rng, 1, max(1, min(3000, 3000000 // classes))),
             "classes": classes, "k": _log(rng, 1, 64)}
        if rng.random() < .5:
            c.update(pad=rng.randint(0, 9), shift=rng.randint(0, 3))
        if c["op"] == "log_probs" and rng.random() < .5:
            c["needs"] = rng.sample(["log_prob", "rank", "entropy", "log_sum", "top_indices", "top_log_probs"], rng.randint(1, 5))
        calls.append(c)
    sound(lib, calls)


def test_every_form_of_rows(lib):
    """The widest rows of each form and those beyond; many rows; chunks."""
    calls, kernels = [], []
    for dtype, vec in (("f32", 4), ("bf16", 8)):
        for lanes in (16, 32, 64, 128, 256, 512, 1024, 2048, 4096, 16 * 64 * 9):
            for classes in (lanes * vec, lanes * vec + 1):
                for op in ("log_probs", "distill_backward"):
                    calls.append({"op": op, "dtype": dtype, "rows": 3, "classes": classes, "k": 9})
        calls += [{"op": op, "dtype": dtype, "rows": 2, "classes": 1 << 20, "k": 64} for op in ("log_probs", "distill_backward")]
        calls.append({"op": "log_probs", "dtype": dtype, "rows": 1 << 20, "classes": 2, "k": 2})
    for c, k in zip(calls, sound(lib, calls)):
        wide = c["classes"] > ((4096 if c["dtype"] == "f32" else 8192) if c["op"] == "log_probs" else
                               9216 * (4 if c["dtype"] == "f32" else 8))
        kernels.append(k)
        assert k == {("log_probs", 0): "score", ("log_probs", 1): "score join", ("distill_backward", 0): "distill",
                     ("distill_backward", 1): "score distill"}[c["op"], wide], (c, k)


@pytest.mark.parametrize("seed", range(3))
def test_matrices_stay_in_their_memory(lib, seed):
    rng = random.Random(50 + seed)
    calls = []
    for _ in range(120):
        dtype = rng.choice(["f32", "bf16"])
        c = {"op": rng.choice(["quantize", "dequantize", "product", "product", "product"]), "dtype": dtype,
             "rows": _log(rng, 1, 2000)}
        if c["op"] == "product":
            c.update(k=_log(rng, 1, 6000), n=_log(rng, 1, 3000), acts=rng.choice(["float", "mx"]), bias=rng.randint(0, 1))
            if rng.random() < .5:
                c["k"] = 8 * ((c["k"] + 7) // 8)
        else:
            c.update(cols=_log(rng, 1, 6000), ctx=rng.choice(["f32", "bf16"]))
        if rng.random() < .4:
            c.update(pad=rng.randint(0, 9), shift=rng.randint(0, 3))
        calls.append(c)
    sound(lib, calls)


def test_every_path_of_products(lib):
    p = {"op": "product", "dtype": "bf16", "acts": "float", "k": 1000, "n": 300}
    f = dict(p, dtype="f32")
    q = dict(p, acts="mx")
    calls = [dict(p, rows=16), dict(f, rows=16), dict(q, rows=16), dict(p, rows=17), dict(f, rows=17), dict(q, rows=17),
             dict(p, rows=1024), dict(p, rows=1025), dict(p, rows=1025, k=1001), dict(f, rows=1025), dict(q, rows=5000, n=4096),
             dict(p, rows=17, k=100), dict(q, rows=17, k=100), dict(p, rows=5000, k=4096), dict(p, rows=8192, k=515, n=9000),
             dict(p, rows=3451, k=3001, n=90), dict(p, rows=257, k=300000, n=5)]
    want = ["few", "planes few", "few", "rows", "planes rows", "mm", "rows", "rows", "rows", "planes rows", "mm", "rows", "mm",
            "values", "values", "rows", "rows"]
    assert sound(lib, calls) == want


def test_float32_rows_beyond_one_piece(lib):
    """2^27 values whose planes are held bound a pass: pieces, the last one
    shorter, of few rows or the only one."""
    c = {"op": "product", "dtype": "f32", "acts": "float", "k": 200000, "n": 10, "bias": 0}
    want = {1024: "planes rows", 1025: "planes rows planes few", 2100: "planes rows planes rows planes rows"}
    assert sound(lib, [dict(c, rows=r) for r in want]) == list(want.values())


def test_many_short_float32_rows(lib):
    c = {"op": "product", "dtype": "f32", "acts": "float", "k": 3, "n": 2, "bias": 0}
    assert sound(lib, [dict(c, rows=(1 << 19) + 1), dict(c, rows=1 << 19)]) == ["planes rows planes few", "planes rows"]


def test_what_may_be_captured(lib):
    """Neither a context's first call nor one that its stream's workspace is
    too small for; nothing else needs a call before."""
    assert drive(lib, [{"op": "capture"}])["calls"] == [[-7, 0, 0, -7, 0, 0]]


def test_the_check_itself(lib):
    """Operands that begin one element before their memory are found out."""
    for c in ({"op": "log_probs", "dtype": "bf16", "rows": 5, "classes": 100, "k": 3, "off": {"logits": -2}},
              {"op": "quantize", "dtype": "f32", "rows": 5, "cols": 100, "off": {"x": -4}},
              {"op": "product", "dtype": "bf16", "acts": "mx", "rows": 5, "k": 100, "n": 9, "off": {"codes": 16}}):
        assert drive(lib, [c])["violations"] > 0, c


def test_pointers_that_are_not_aligned_are_refused(lib):
    calls, names = [], []
    for dtype, e in (("bf16", 2), ("f32", 4)):
        a = {"op": "log_probs", "dtype": dtype, "rows": 5, "classes": 100, "k": 3}
        d = dict(a, op="distill_backward")
        for name in ("log_prob", "rank", "entropy", "log_sum", "top_indices", "top_log_probs", "labels"):
            calls.append(dict(a, off={name: 2}))
            names.append(name)
        for name in ("indices", "values", "dloss", "loss"):
            calls.append(dict(d, off={name: 1}))
            names.append(name)
        calls.append(dict(a, off={"logits": 1}))
        names.append("logits")
        for name in ("codes", "scales"):
            calls += [{"op": op, "dtype": dtype, "rows": 5, "cols": 40, "off": {name: 8}} for op in ("quantize", "dequantize")]
            names += ["codes and scales"] * 2
        calls.append({"op": "quantize", "dtype": dtype, "rows": 5, "cols": 40, "off": {"x": 1}})
        names.append("x")
        calls.append({"op": "product", "dtype": dtype, "acts": "float", "rows": 5, "k": 40, "n": 9, "off": {"bias": 2}})
        names.append("bias")
    for c, name, o in zip(calls, names, drive(lib, calls)["calls"]):
        assert o["status"] == -1 and not o["kernels"] and name in o["message"] and "aligned" in o["message"], (c, o)


def test_outputs_that_overlap_are_refused(lib):
    d = {"op": "distill_backward", "dtype": "bf16", "rows": 6, "classes": 40, "k": 3}
    p = {"op": "product", "dtype": "bf16", "acts": "float", "rows": 6, "k": 24, "n": 16}
    good = [dict(d, pad=40, beside=40), dict(p, pad=16, beside=24)]
    bad = [dict(d, pad=40, beside=b) for b in (0, 39, 41)] + [dict(d, beside=0)] + [dict(p, pad=16, beside=b) for b in (0, 23)]
    out = drive(lib, good + bad)["calls"]
    for c, o in zip(good, out):
        assert o["status"] == 0, (c, o)
    for c, o in zip(bad, out[len(good):]):
        assert o["status"] == -1 and "overlaps" in o["message"] and not o["kernels"], (c, o)


def test_rows_both_ways_or_neither_are_refused(lib):
    p = {"op": "product", "dtype": "bf16", "rows": 6, "k": 24, "n": 16}
    both, more = drive(lib, [dict(p, acts="both"), dict(p, acts="mx", more=1)])["calls"]
    assert both["status"] == -1 and "either x or xq" in both["message"]
    assert more["status"] == -1 and "columns" in more["message"]

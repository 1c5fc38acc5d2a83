"""The operators' host code (request tables, workspaces, plans and argument
blocks) compiled for the CPU with AddressSanitizer and driven through calls
of many shapes. Every launch checks that each range its kernel would read or
write may be accessed: operands and results are allocated to their last
element, and the pieces of a workspace have gaps between them that may not
be touched. No GPU is needed."""

import json
import os
import random
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUB = os.path.join(ROOT, "tests", "opstub")
HOST = os.path.join(ROOT, "tests", "hoststub")
LIB = os.path.join(ROOT, "_build", "libgemel_ops.so")
CSRC = os.path.join(ROOT, "paper_2201_07705_amd", "csrc")


@pytest.fixture(scope="module")
def opslib():
    os.makedirs(os.path.dirname(LIB), exist_ok=True)
    tmp = f"{LIB}.{os.getpid()}"
    flags = ["g++", "-std=c++17", "-g", "-O1", "-fsanitize=address", "-fno-omit-frame-pointer", "-fPIC"]
    dirs = [f"-I{HOST}", f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}"]
    sources = {os.path.join(HOST, "hoststub.cpp"): [], os.path.join(STUB, "opstub.cpp"): [f"-I{STUB}"]}
    for name in ("registry", "plan", "batching", "operators", "op_plan"):
        sources[os.path.join(CSRC, name + ".cpp")] = [f"-I{STUB}"]
    objects = [f"{tmp}.{k}.o" for k in range(len(sources))]
    with ThreadPoolExecutor(max_workers=8) as ex:
        list(ex.map(subprocess.check_call, [flags + first + dirs + ["-c", src, "-o", obj]
                                            for (src, first), obj in zip(sources.items(), objects)]))
    subprocess.check_call(flags + ["-shared"] + objects + ["-o", tmp])
    for obj in objects:
        os.remove(obj)
    os.replace(tmp, LIB)
    return LIB


def drive(lib, calls):
    asan = subprocess.check_output(["gcc", "-print-file-name=libasan.so"], text=True).strip()
    env = dict(os.environ, LD_PRELOAD=asan, ASAN_OPTIONS="detect_leaks=0:allocator_may_return_null=1")
    r = subprocess.run(["python", os.path.join(STUB, "drive.py"), lib, json.dumps(calls)],
                       capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    return json.loads(r.stdout.strip().splitlines()[-1])


def sound(lib, calls):
    out = drive(lib, calls)
    assert len(out["calls"]) == len(calls)
    for c, o in zip(calls, out["calls"]):
        assert o["status"] == 0, (c, o)
    assert sum(o["launches"] for o in out["calls"]) > len(calls)
    assert out["violations"] == 0, out["last"]


def _log(rng, lo, hi):
    import math
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def projection(rng, op, rows):
    bank, rank = _log(rng, 1, 12), _log(rng, 1, 256)
    n = rng.randint(1, min(rows, 9))
    cuts = sorted(rng.randint(0, rows) for _ in range(n - 1))
    n_rows = [b - a for a, b in zip([0] + cuts, cuts + [rows])]
    c = {"op": op, "dtype": rng.choice(["bf16", "f32"]), "n_rows": n_rows,
         "ids": [rng.randint(-1, bank - 1) for _ in n_rows], "bank": bank, "rank": rank,
         "ranks": [rng.randint(1, rank) for _ in range(bank)],
         "k": _log(rng, 1, 5000), "n": _log(rng, 1, 3000)}
    if rng.random() < .5:
        c["k"], c["n"] = 8 * ((c["k"] + 7) // 8), 8 * ((c["n"] + 7) // 8)
    if rng.random() < .4:
        c.update(pad=rng.randint(1, 9), shift=rng.randint(0, 3))
    if op == "adapt_backward" and rng.random() < .4:
        c["needs"] = [q for q in ("x", "weight", "bias", "a", "b") if rng.random() < .5] or ["x"]
    return c


@pytest.mark.parametrize("seed", range(6))
def test_projections_stay_in_their_memory(opslib, seed):
    rng = random.Random(seed)
    calls = []
    for op in ("adapt", "adapt_backward"):
        for _ in range(25):
            calls.append(projection(rng, op, _log(rng, 1, 64)))
            calls.append(projection(rng, op, _log(rng, 65, 3000)))
    sound(opslib, calls)


def test_workspaces_of_small_calls_after_large_ones(opslib):
    """The same workspace, laid out anew by every call."""
    one = {"op": "adapt_backward", "dtype": "f32", "n_rows": [1200, 7], "ids": [0, 1], "bank": 2, "rank": 40,
           "k": 1030, "n": 520}
    calls = []
    for rows in ([1200, 7], [3], [70], [0], [64], [65]):
        for dtype in ("f32", "bf16"):
            for op in ("adapt", "adapt_backward"):
                calls.append(dict(one, op=op, dtype=dtype, n_rows=rows, ids=[0, 1][:len(rows)]))
                # thin products and sums in slices
                calls.append(dict(one, op=op, dtype=dtype, n_rows=rows, ids=[0, 1][:len(rows)], k=20001, n=70))
                calls.append(dict(one, op=op, dtype=dtype, n_rows=rows, ids=[0, 1][:len(rows)], k=70, n=20001))
    sound(opslib, calls)


@pytest.mark.parametrize("seed", range(3))
def test_matrices_stay_in_their_memory(opslib, seed):
    rng = random.Random(100 + seed)
    calls = []
    for op in ("orthogonalize", "muon"):
        for dtype in ("bf16", "f32"):
            for _ in range(12):
                rows, cols = _log(rng, 1, 1500), _log(rng, 1, 1500)
                calls.append({"op": op, "dtype": dtype, "count": _log(rng, 1, 6), "rows": rows, "cols": cols,
                              "steps": rng.randint(1, 8)})
            # steps in pairs, odd and even, and batches of several groups
            calls += [{"op": op, "dtype": dtype, "count": 2, "rows": 512, "cols": 4608, "steps": s} for s in (2, 4, 5)]
            calls.append({"op": op, "dtype": dtype, "count": 140, "rows": 1100, "cols": 1030, "steps": 2})
    sound(opslib, calls)


def test_the_check_itself(opslib):
    """Operands that begin one element before their memory are found out."""
    c = {"op": "adapt", "dtype": "bf16", "n_rows": [90], "ids": [0], "bank": 1, "rank": 8, "k": 64, "n": 72}
    assert drive(opslib, [dict(c, shift=-1)])["violations"] > 0


def test_long_batches_of_float32(opslib):
    """Rows beyond those that a transposed copy of pairs can hold, with few
    and many outputs, and each gradient alone."""
    rows = (1 << 21) + 1
    c = {"op": "adapt_backward", "dtype": "f32", "n_rows": [rows - 5, 5], "ids": [0, 1], "bank": 2, "rank": 2,
         "k": 4, "n": 65}
    sound(opslib, [c, dict(c, needs=["weight"]), dict(c, k=130, n=3, needs=["weight", "bias"]),
                   dict(c, dtype="bf16", needs=["weight"]), dict(c, op="adapt")])


def test_products_of_any_size_have_a_grid(opslib):
    """The largest batches with thousands of outputs, and every other shape
    that memory could hold, fit the 2^32 threads of a grid."""
    code = ("import ctypes, json, sys; L = ctypes.CDLL(sys.argv[1]); f = L.opstub_product_threads; "
            "f.restype = ctypes.c_longlong; print(json.dumps([f(*c) for c in json.loads(sys.argv[2])]))")
    shapes = [[1 << 22, 8256, 8, 1, 0, 0], [1 << 22, 16500, 4096, 1, 0, 0], [1 << 22, 33000, 64, 1, 1, 0],
              [1 << 20, 130000, 64, 1, 0, 0], [1 << 22, 1, 8, 1, 0, 0], [64, 1 << 20, 1 << 20, 1, 0, 0],
              [65, 1 << 20, 64, 1, 0, 0], [90000, 90000, 90112, 1, 0, 1], [4096, 25088, 8192, 1, 1, 0]]
    asan = subprocess.check_output(["gcc", "-print-file-name=libasan.so"], text=True).strip()
    r = subprocess.run(["python", "-c", code, opslib, json.dumps(shapes)], capture_output=True, text=True,
                       env=dict(os.environ, LD_PRELOAD=asan, ASAN_OPTIONS="detect_leaks=0"))
    threads = json.loads(r.stdout)
    assert all(0 < t < 1 << 32 for t in threads), threads


def test_batches_given_back_wait_for_nothing(opslib):
    """While the work of earlier rounds runs on, a server's new batches take
    new tables and never wait for the device; once it is over they take the
    old ones. Tables of a destroyed stream or a graph wait for the device."""
    rounds = {"op": "rounds", "rounds": 100}
    (warm, busy, free), = drive(opslib, [dict(rounds, streams=3, answers=[0, 600, 0])])["calls"]
    assert warm[0] == 0 and busy[0] == 0 and free[0] == 0
    assert 100 >= busy[1] >= 90 and free[1] == 0
    (lost,), = drive(opslib, [dict(rounds, streams=1, answers=[709])])["calls"]
    assert lost[0] == 3 and lost[1] <= 40
    (_, graph), = drive(opslib, [dict(rounds, streams=2, answers=[0, 0], rounds=130, capture=1)])["calls"]
    assert 1 <= graph[0] <= 2


def test_columns_of_one_matrix_are_apart(opslib):
    """x and y side by side in one matrix, in either order; refused where any
    byte is shared."""
    c = {"op": "adapt", "dtype": "bf16", "n_rows": [70], "ids": [0], "bank": 1, "rank": 4, "k": 24, "n": 16}
    good = [dict(c, pad=16, beside=24), dict(c, pad=40, beside=30), dict(c, pad=40, beside=48),
            dict(c, pad=40, beside=24 - 64 + 24), dict(c, pad=16, beside=-16), dict(c, n_rows=[1], beside=24)]
    bad = [dict(c, pad=16, beside=b) for b in (23, 25, 0, -1, -15, -17, 40, 63)] + [dict(c, pad=16, beside=24, skew=1)]
    out = drive(opslib, good + bad)["calls"]
    for q, o in zip(good, out):
        assert o["status"] == 0, (q, o)
    for q, o in zip(bad, out[len(good):]):
        assert o["status"] == -1 and "y overlaps x" in o["message"] and o["launches"] == 0, (q, o)


def test_pointers_that_are_not_aligned_are_refused(opslib):
    calls, names = [], []
    for dtype, e in (("bf16", 2), ("f32", 4)):
        c = {"op": "adapt_backward", "dtype": dtype, "n_rows": [70], "ids": [0], "bank": 1, "rank": 4, "k": 24, "n": 16}
        for name, size in (("bias", 4), ("a", e), ("b", e), ("dweight", 4), ("dbias", 4), ("da", 4), ("db", 4)):
            for by in range(1, size):
                if name != "bias":
                    calls.append(dict(c, off={name: by}))
                    names.append(name)
                if name in ("bias", "a", "b"):
                    calls.append(dict(c, op="adapt", off={name: by}))
                    names.append(name)
    for c, name, o in zip(calls, names, drive(opslib, calls)["calls"]):
        assert o["status"] == -1 and o["launches"] == 0 and o["message"] == f"{name} is not aligned to its type", (c, o)
    # gradients do not read the bias
    assert drive(opslib, [dict(c, off={"bias": 1})])["calls"][0]["status"] == 0


def test_the_shared_gradients_need_no_adapters(opslib):
    """dweight and dbias of a batch with adapters, without the bank; what the
    bank enters is refused without it."""
    calls = []
    for dtype in ("bf16", "f32"):
        for rows in ([40], [90, 30]):
            c = {"op": "adapt_backward", "dtype": dtype, "n_rows": rows, "ids": [0, 1][:len(rows)], "bank": 2,
                 "rank": 4, "k": 24, "n": 16, "bare": 1}
            calls += [dict(c, needs=["weight", "bias"]), dict(c, needs=["weight"]), dict(c, needs=["bias"])]
            calls += [dict(c, needs=[q]) for q in ("x", "a", "b")] + [dict(c, op="adapt")]
    out = drive(opslib, calls)
    assert out["violations"] == 0
    for q, o in zip(calls, out["calls"]):
        if q["op"] == "adapt" or set(q["needs"]) & {"x", "a", "b"}:
            assert o["status"] == -1 and o["launches"] == 0 and "a and b must be given" in o["message"], (q, o)
        else:
            assert o["status"] == 0, (q, o)


def test_larger_batches_wait_for_nothing(opslib):
    """Neither new tables nor the memory that they are staged in."""
    out = drive(opslib, [{"op": "growing", "n_rows": [1, 10000, 100, 40000, 1 << 20, 1 << 21, 5, 1 << 22]}])
    assert out["calls"] == [0] and out["violations"] == 0


def test_each_thread_has_its_own_per_thread_stream(opslib):
    """hipStreamPerThread is one handle for many streams, which do not wait
    for each other and so share no workspace."""
    out = drive(opslib, [{"op": "threads", "threads": 3}])
    assert out["calls"] == [[1, 0] * 3] and out["violations"] == 0

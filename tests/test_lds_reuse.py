"""Kernels that refill LDS by direct global-to-LDS loads.

Such a load is issued by any wave of a workgroup as soon as the barrier that
frees its buffer is behind it, so every wave's reads of that buffer must have
arrived before the wave enters the barrier: in program order their results
may be used later, and the barrier alone does not wait for them. The test
compiles such kernels and follows every path through the
resulting code: no barrier of a kernel with direct loads may be reached with
LDS reads outstanding. No GPU is needed."""

import os
import re
import subprocess

import pytest

from paper_2201_07705_amd import build as B

SOURCES = ["k_rows.hip", "k_mm.hip", "k_fc.hip", "k_stem.hip"]

READ = re.compile(r"ds_(read|load|bpermute|permute)")
DIRECT = re.compile(r"(global|buffer)_load_\w+ .*\blds\b|(global|buffer)_load_lds")


def kernels(asm):
    """Instructions of each kernel, with the labels among them."""
    out, name = {}, None
    for line in asm.splitlines():
        line = line.split(";")[0].rstrip()
        m = re.match(r"(_Z\w+):", line)
        if m:
            name = m.group(1)
            out[name] = []
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name is not None and re.match(r"\.LBB\w+:|\s+[a-z]", line):
            out[name].append(line.strip())
    return out


def outstanding_at_barriers(code):
    """Most LDS reads that any path has outstanding at each s_barrier."""
    labels = {i.rstrip(":"): k for k, i in enumerate(code) if i.startswith(".LBB")}
    most, todo, worst = {0: 0}, [0], {}
    while todo:
        k = todo.pop()
        n = most[k]
        i = code[k]
        op = i.split()[0]
        nexts = [k + 1]
        if READ.match(op):
            n += 1
        elif op == "s_waitcnt":
            m = re.search(r"lgkmcnt\((\d+)\)", i)
            if m:
                n = min(n, int(m.group(1)))
        elif op == "s_barrier":
            worst[k] = max(worst.get(k, 0), n)
        elif op == "s_endpgm":
            nexts = []
        elif op == "s_branch":
            nexts = [labels[i.split()[1]]]
        elif op.startswith("s_cbranch"):
            nexts.append(labels[i.split()[1]])
        n = min(n, 16)   # (a loop of reads without a wait)
        for q in nexts:
            if q < len(code) and most.get(q, -1) < n:
                most[q] = n
                todo.append(q)
    return worst


def assembly(src, tmp_path):
    out = str(tmp_path / "k.s")
    subprocess.check_call([B.HIPCC] + [f for f in B.FLAGS if f != "-fPIC"] +
                          ["--cuda-device-only", "-S", os.path.join(B.CSRC, src), "-o", out],
                          stderr=subprocess.DEVNULL)
    with open(out) as f:
        return f.read()


def test_the_walk_itself():
    loop = ["ds_read_b128 v[0:3], v9", "s_waitcnt lgkmcnt(0)", ".LBB0_1:", "s_barrier",
            "ds_read_b128 v[0:3], v9", "s_cbranch_scc1 .LBB0_2", "s_waitcnt vmcnt(0) lgkmcnt(0)",
            ".LBB0_2:", "s_barrier", "s_waitcnt lgkmcnt(0)", "s_cbranch_scc0 .LBB0_1", "s_endpgm"]
    assert outstanding_at_barriers(loop) == {3: 0, 8: 1}
    loop.remove("s_cbranch_scc1 .LBB0_2")
    assert outstanding_at_barriers(loop) == {3: 0, 7: 0}


@pytest.mark.parametrize("src", SOURCES)
def test_no_lds_read_is_outstanding_where_its_buffer_is_given_free(src, tmp_path):
    seen, bad = 0, {}
    for name, code in kernels(assembly(src, tmp_path)).items():
        if not any(DIRECT.match(i) for i in code):
            continue
        at = outstanding_at_barriers(code)
        seen += len(at)
        late = sorted(n for n in at.values() if n)
        if late:
            bad[name] = late
    assert seen > 0
    assert not bad, bad

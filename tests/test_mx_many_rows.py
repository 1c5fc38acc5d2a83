"""Products of many bf16 rows with 4-bit weights on the CPU (the host code of
test_answers_host.py): which rows are read where they are, which are copied,
and how many at a time. No GPU is needed."""

from test_answers_host import drive, lib  # noqa: F401


def test_rows_are_copied_only_where_they_are_not_aligned(lib):  # noqa: F811
    """An expansion of the weights, then one product; a copy before it where
    rows or their pointer are not aligned to 16 bytes, of 2^30 values at most."""
    p = {"op": "product", "dtype": "bf16", "acts": "float", "k": 512, "n": 8}
    calls = [dict(p, rows=(1 << 21) + 8), dict(p, rows=(1 << 21) + 8, shift=1), dict(p, rows=1 << 21, pad=1),
             dict(p, rows=(1 << 20) + 1, k=1016, pad=8), dict(p, rows=600000, k=8, pad=8), dict(p, rows=600000, k=8, pad=3)]
    out = drive(lib, calls)
    assert out["violations"] == 0, out["last"]
    for c, o in zip(calls, out["calls"]):
        assert o["status"] == 0 and o["kernels"] == "values", (c, o)
    assert [o["others"] for o in out["calls"]] == [1, 4, 2, 1, 1, 2]

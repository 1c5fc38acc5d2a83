"""The products of 4-bit matrices refill LDS by direct loads too: no barrier
that frees a buffer is reached with reads of it outstanding, and they keep
their sums and fragments in registers. No GPU is needed."""

from test_lds_reuse import DIRECT, assembly, kernels, outstanding_at_barriers


def test_no_lds_read_is_outstanding_where_its_buffer_is_given_free(tmp_path):
    seen = 0
    for name, code in kernels(assembly("k_mx_mm.hip", tmp_path)).items():
        assert any(DIRECT.match(i) for i in code), name
        at = outstanding_at_barriers(code)
        assert not any(at.values()), (name, at)
        seen += len(at)
        # the matrix instructions take their operands as they were read
        assert sum(i.startswith("v_mfma_scale") for i in code) >= 16, name
    assert seen > 0

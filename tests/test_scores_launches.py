"""How the gradient of scores is cut into launches (host rules, no GPU)."""
import pytest


@pytest.mark.parametrize("vocab", [1, 357, 4608, 8185, 8186, 16377, 16378, 16400, 32000, 50257, 128256, 1 << 20, 1 << 30])
def test_launches_begin_where_vectors_do(lib, vocab):
    """Rows of any pitch: with a multiple of 8 tokens a launch its first row is a multiple of 16 bytes from the first of all, in either type, and what the kernel reads and writes 16
    bytes at a time from there is aligned.  And a launch, of 256 threads for each 8192 words, has fewer than 2^32 threads."""
    each = lib.burst_lm_head_scores_bwd_plan(lib.scores_shape(1 << 25, vocab))
    assert each >= 8 and each % 8 == 0
    assert each * -(-(vocab + 7) // 8192) * 256 < 1 << 32


def test_refusals(lib):
    import ctypes as C
    raw, out = lib.raw(), (C.c_int64 * 1)()
    for bad in (lib.scores_shape(-1, 10), lib.scores_shape(1, 0), lib.scores_shape(1, 10, 0, 0.0)):
        assert raw.burst_lm_head_scores_bwd_plan(C.byref(bad), out) == lib.BURST_ERR_INVALID_ARG
    assert raw.burst_lm_head_scores_bwd_plan(C.byref(lib.scores_shape(1, 10)), None) == lib.BURST_ERR_INVALID_ARG
    assert raw.burst_lm_head_scores_bwd_plan(None, out) == lib.BURST_ERR_INVALID_ARG

"""CPU tests of the limits of rows written into a paged cache and read back (nothing is launched)."""

import pytest

from tests.test_cache_host import INT_MAX, SHAPE, _append, _cache, _read


@pytest.mark.parametrize("nseq, heads, most", [(64, 32, (1 << 20)), (1, 1 << 20, 2048), (3, 5, INT_MAX // 15 + 1)])
def test_pairs_that_a_counter_does_not_hold_are_refused(nseq, heads, most):
    assert _append(_cache(nseq=nseq, heads=heads), skipped=0xd000, max_new=most) == SHAPE


def test_rows_beyond_a_launch_are_refused():
    """(rows + 64 sequences) x heads below 2^28 is always taken; what is far beyond is not."""
    for nseq, heads, rows in ((1, 32, 1 << 24), (64, 32, 1 << 24), (4096, 8000, 4096 * 16)):
        assert _read(_cache(nseq=nseq, heads=heads), num_rows=rows, max_rows=INT_MAX) == SHAPE
    for nseq, heads, rows in ((1, 32, 1 << 26), (64, 32, 1 << 26)):
        assert _append(_cache(nseq=nseq, heads=heads), num_rows=rows, max_new=INT_MAX) == SHAPE

"""CPU tests of outputs whose rows share elements, which the calls around attention in a step refuse, and of layouts in which they do not (refused for another
reason here, a later one: nothing is launched)."""

import itertools

import numpy as np
import pytest

from tests.test_cache_host import ALIGN, INT_MAX, PARAMS, SHAPE, WORKSPACE, _cache
from tests.test_step_host import _bwd, _chunk, _fwd


def _overlap(D, dims):
    at = np.zeros(1, dtype=np.int64)
    for n, stride in dims:
        at = (at[:, None] + np.arange(n) * stride).ravel()
    return bool(np.any(np.diff(np.sort(at)) < D))


def _rope(dims, D, back):
    """The status of a call whose outputs lie so (their inputs lie apart), with frequencies that are refused after the strides are."""
    a, b = ("in", "out") if back else ("out", "in")
    kw = {"%s_stride_%s" % (a, x): s for x, (_, s) in zip("bht", dims)}
    kw.update({"%s_stride_%s" % (b, x): s for x, s in zip("bht", (1 << 30, 1 << 20, 1024))})
    kw.update(batch=dims[0][0], heads=dims[1][0], seqlen=dims[2][0], head_dim=D, rotary_dim=32, inv_freq=0x7002)
    return (_bwd if back else _fwd)(**kw)


def _rows(dims, D):
    """The same of a chunk, whose workspace is refused."""
    fmt = dict(head_dim=D, heads=dims[1][0], page_stride=64 * 128, tok_stride=128)
    return _chunk(_cache(**fmt), num_rows=dims[0][0], max_new=dims[0][0], q_stride_row=dims[0][1], q_stride_head=dims[1][1], num_splits=2, ws=None,
                  params=dict(PARAMS, num_heads=dims[1][0]))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("back", [False, True])
def test_rows_of_rotations(D, back):
    apart = [((2, 15 * D), (3, 5 * D), (5, D)), ((2, 15 * D), (3, D), (5, 3 * D)), ((2, 45 * D), (3, D), (5, 9 * D)), ((2, D), (3, 2 * D), (5, 6 * D)),
             ((1, 0), (3, D), (5, 3 * D)), ((2, 15 * D), (1, 0), (5, D)), ((2, 5 * D), (1, 8), (1, 0)), ((1, 0), (1, 0), (1, 0)),
             ((2, 3 * D), (2, 2 * D), (1, 0)), ((2, 3 * D), (1, 0), (2, 2 * D))]  # (the last two: between each other)
    for dims in apart:
        assert not _overlap(D, dims) and _rope(dims, D, back) == ALIGN, dims
    for dims in (((2, 0), (3, 5 * D), (5, D)), ((2, 15 * D), (3, 0), (5, D)), ((2, 15 * D), (3, D), (5, 0)), ((2, 15 * D), (3, D - 8), (5, 3 * D)),
                 ((2, 15 * D), (3, D), (5, D)), ((2, 15 * D), (3, D), (5, 2 * D)), ((2, 15 * D), (3, D), (5, 3 * D - 8)), ((2, 14 * D), (3, 5 * D), (5, D)),
                 ((1 << 10, 0), (3, 5 * D), (5, D)), ((2, 8), (1, 0), (1, 0)), ((2, 3 * D), (3, 2 * D), (2, 6 * D - 8))):
        assert _overlap(D, dims) and _rope(dims, D, back) == SHAPE, dims


def test_rows_of_chunks():
    for D in (64, 128):
        for dims in (((5, 3 * D), (3, D)), ((5, D), (3, 5 * D)), ((5, 3 * D + 8), (3, D)), ((5, 2 * D), (2, 3 * D)), ((1, 0), (3, D)), ((5, D), (1, 0))):
            overlap = _overlap(D, dims)
            assert _rows(dims, D) == (SHAPE if overlap else WORKSPACE), dims
        for dims in (((5, 0), (3, D)), ((5, 3 * D), (3, 0)), ((5, 2 * D), (3, D)), ((5, 3 * D - 8), (3, D)), ((5, D), (3, D)), ((5, 8), (1, 0))):
            assert _overlap(D, dims) and _rows(dims, D) == SHAPE, dims


@pytest.mark.parametrize("seed", range(4))
def test_strides_of_any_kind(seed):
    rng = np.random.default_rng(seed)
    seen = []
    for _ in range(400):
        dims = [(int(rng.integers(1, 6)), 8 * int(rng.integers(0, 90))) for _ in range(3)]
        overlap = _overlap(64, dims)
        seen.append(overlap)
        assert _rope(dims, 64, seed % 2) == (SHAPE if overlap else ALIGN), dims
        assert _rows(dims[1:], 64) == (SHAPE if _overlap(64, dims[1:]) else WORKSPACE), dims
    assert 20 < sum(seen) < 380


def test_large_sizes_and_strides():
    for order in itertools.permutations([(2, 1 << 40), (1 << 12, 1 << 20), (1 << 10, 64)]):
        assert _rope(order, 64, False) == ALIGN
    for order in itertools.permutations([(2, 1 << 31), (1 << 12, 1 << 20), (1 << 10, 64)]):
        assert _rope(order, 64, False) == SHAPE
    assert _rope([(1 << 12, 1 << 40), (3, 1 << 40), (1 << 10, 64)], 64, True) == SHAPE
    assert _rows([(INT_MAX, 0), (3, 128)], 128) == _rows([(INT_MAX, 128), (3, 128)], 128) == SHAPE


def test_inputs_may_be_broadcast():
    """Of the forward, and the gradients of results of the backward."""
    wide = dict(batch=2, heads=3, seqlen=5, inv_freq=0x7002)
    for none in ("b", "h", "t"):
        assert _fwd(**wide, **{"in_stride_" + none: 0}) == ALIGN
        assert _bwd(**wide, **{"out_stride_" + none: 0}) == ALIGN
        assert _bwd(**wide, **{"in_stride_" + none: 0}) == SHAPE and _fwd(**wide, **{"out_stride_" + none: 0}) == SHAPE

"""Infinities and NaN in values of V that a chunk's rows attend, where the maximum of a row's scores moves on the same 64 tokens."""

import numpy as np
import pytest

from paper_2407_17678_amd import synth
from tests import gpu_util as G
from tests.test_gpu_chunk import Chunk

pytestmark = pytest.mark.gpu


def _put(c, which, head, token, values, feature=slice(None)):
    """Of sequence 0, in the cache (which: 0 K, 1 V)."""
    case = c.c
    case.pools.data[which][case.table[0, head, token // c.S], token % c.S, feature] = values


def _check(c, head, spots, clean, got, far=lambda row, token: False):
    """spots: (token, feature, value) in V.  A row has, in the feature of those that it attends, their sum; where one's probability is out of reach (far) it may also be
    NaN; everything else is what it is without them, to the last bit."""
    keeps, touched = c.c.keeps(head), 0
    for i in range(c.new[0]):
        at, row = c.start[0] + i, c.cu[0] + i
        features = set()
        for f in {f for _, f, _ in spots}:
            here = [(t, x) for t, g, x in spots if g == f and t <= at and keeps(at // c.S, t // c.S)]
            if not here:
                continue
            features.add(f)
            touched += 1
            value, want = got[row, head, f], sum(x for _, x in here)
            if np.isnan(want):
                assert np.isnan(value), (i, f, value)
            elif any(far(at, t) for t, _ in here):
                assert np.isnan(value) or value == want, (i, f, value)
            else:
                assert value == want, (i, f, value)
        rest = [f for f in range(c.D) if f not in features]
        assert np.array_equal(got[row, head, rest], clean[row, head, rest]), i
    return touched


@pytest.mark.parametrize("S, before", [(16, 0), (32, 0), (64, 0), (16, 5), (32, 69), (128, 130)])
@pytest.mark.parametrize("new", [64, 70, 128, 150, 300])
@pytest.mark.parametrize("D, splits", [(64, 1), (128, 1), (64, 3)])
def test_first_tokens_that_a_row_attends(S, before, new, D, splits):
    """A window of one block: a row's first token may lie anywhere in 64 that are read together."""
    c = Chunk("bf16", D, S, [before + new], [new], 2, local=1, stride=0, seed=S)
    clean, clean_lse, _ = c.run(splits=splits)
    spots = [(t, (7 * t) % (D - 3), np.inf if t % 2 else -np.inf) for t in range(0, before + new, 9)]
    spots += [(t, D - 1, x) for t, x in ((before + 8, np.inf), (before + 43, -np.inf), (before + 45, np.inf), (before + 62, np.nan))]
    for t, f, x in spots:
        _put(c, 1, 1, t, x, f)
    got, lse, _ = c.run(splits=splits)
    assert np.array_equal(lse, clean_lse) and np.array_equal(got[:, 0], clean[:, 0])
    assert _check(c, 1, spots, clean, got) > new / 2


@pytest.mark.parametrize("new", [20, 50, 110, 150])
@pytest.mark.parametrize("S, D", [(64, 64), (128, 128), (32, 64)])
@pytest.mark.parametrize("down", [False, True])
def test_scores_that_exceed_all_before_them_by_hundreds(new, S, D, down):
    """All queries alike, one token in 64 beside whose score the others' are out of reach of 32 bits: from that token on a row is it alone."""
    length = 130 + new
    c = Chunk("bf16", D, S, [length], [new], 1, dense=1, seed=S)
    one = np.sign(np.random.default_rng(5).standard_normal(D)).astype(np.float32)
    c.q[:] = synth.round_to_bf16_bits(one)
    # a score of 100 sqrt(D) times the token's turn, 800 and more apart
    turns = list(range(40, length, 64))
    for n, t in enumerate(turns):
        keys = G.to_dev(synth.round_to_bf16_bits(one * np.float32(100 * (len(turns) - n if down else n + 1))))
        _put(c, 0, 0, t, keys)
    clean, clean_lse, _ = c.run()
    # one in each of the tokens that a row may be, one in a token just before it and one just after
    spots = [x for n, t in enumerate(turns) for x in ((t, 3 * n, np.inf), (t - 25, 3 * n + 1, -np.inf), (t + 2, 3 * n + 2, np.inf) if t + 2 < length else (t, 3 * n, np.inf))]
    for t, f, x in spots:
        _put(c, 1, 0, t, x, f)
    got, lse, _ = c.run()
    assert np.array_equal(lse, clean_lse)

    def far(at, t):
        seen = [u for u in turns if u <= at]
        return t != (seen[0] if down else seen[-1])
    assert _check(c, 0, spots, clean, got, far) > 0
    for i in range(new):  # (the oracle of such a row is one token of V)
        at = c.start[0] + i
        seen = [u for u in turns if u <= at]
        assert np.array_equal(clean[c.cu[0] + i, 0], c.c.v[0][0][seen[0] if down else seen[-1]])

"""Values of V that are not numbers, in blocks that every row of a tree keeps beside others that only one row keeps, and in drafted nodes: a node that attends
a NaN, or infinities of both signs, has NaN there, whichever wavefront or split met which."""

import numpy as np
import pytest

from oracle import s2_oracle as orc
from tests import gpu_util as G
from tests.test_gpu_tree import Case

pytestmark = pytest.mark.gpu

INF, MINUS_INF, NAN = 0x7F80, 0xFF80, 0x7FC0
S, D, FEATURE, TOKEN = 16, 64, 5, 3


def _row_values(bits):
    return float(G.bits_f64(np.array([bits], dtype=np.uint16))[0])


def _sum(values):
    """What an attended set of values gives where all probabilities are above 0: their sum, as far as it is not finite."""
    with np.errstate(invalid="ignore"):
        return float(np.sum(values)) if values else 0.0


@pytest.mark.parametrize("T", [12, 24, 40])
@pytest.mark.parametrize("splits", [1, 3])
def test_what_two_wavefronts_meet_is_one_sum(T, splits):
    """Row L // S of a chain keeps fourteen blocks, the next rows one less each at the beginning: the first block is only the first row's, the
    last ones are everybody's."""
    L = 16 * 19 + 15
    par = np.stack([np.arange(-1, T - 1, dtype=np.int32)])
    c = Case("bf16", D, S, [L], 1, par, local=14, stride=0)
    keeps, row0 = c.keeps(0), L // S
    clean = {blk: c.pools.data[1][c.table[0, 0, blk], TOKEN, FEATURE].clone() for blk in range(6, 20)}
    mine = row0 - 13

    def put(blk, bits):
        c.pools.data[1][c.table[0, 0, blk], TOKEN, FEATURE] = clean[blk] if bits is None else G.to_dev(np.array([bits], dtype=np.uint16))[0]

    for blk in (10, 13, 14, 15, 16, 17, 18, 19):
        for here, there in ((NAN, INF), (MINUS_INF, INF), (INF, INF), (MINUS_INF, MINUS_INF), (INF, NAN)):
            put(blk, here)
            put(mine, there)
            o, lse, _ = c.run(splits=splits)
            assert np.all(np.isfinite(lse))
            for i in range(T):
                row = (L + i) // S
                want = _sum([_row_values(x) for j, x in ((blk, here), (mine, there)) if keeps(row, j)])
                got = o[0, 0, i, FEATURE]
                if np.isfinite(want):
                    assert np.isfinite(got), (blk, hex(here), hex(there), i, got)
                else:
                    assert got == want or (np.isnan(got) and np.isnan(want)), (blk, hex(here), hex(there), i, got, want)
            assert np.all(np.isfinite(np.delete(o[0, 0], FEATURE, -1)))
            put(blk, None)
            put(mine, None)


@pytest.mark.parametrize("T", [12, 24, 40])
@pytest.mark.parametrize("splits", [1, 3])
def test_what_the_cache_and_a_node_hold_is_one_sum(T, splits):
    """One value in a block that all rows keep, another in the second node: the nodes below it have both, the first and its other children the first."""
    L = 16 * 19 + 2
    par = np.stack([np.arange(-1, T - 1, dtype=np.int32)])
    par[0, 4] = 0
    c = Case("bf16", D, S, [L], 1, par, local=14, stride=0)
    chains = orc.tree_chains(par[0])
    keeps = c.keeps(0)
    for blk in (10, 14, 16, 18):
        page = c.table[0, 0, blk]
        was = c.pools.data[1][page, TOKEN, FEATURE].clone()
        for here, there in ((NAN, INF), (MINUS_INF, INF), (INF, INF), (INF, NAN)):
            c.pools.data[1][page, TOKEN, FEATURE] = G.to_dev(np.array([here], dtype=np.uint16))[0]
            c.vd[0, 0, 1, FEATURE] = there
            o, _, _ = c.run(splits=splits)
            for i, chain in enumerate(chains):
                row = (L + len(chain) - 1) // S
                values = [here] * keeps(row, blk) + [there] * (1 in chain and keeps(row, (L + 1) // S))
                want, got = _sum([_row_values(x) for x in values]), o[0, 0, i, FEATURE]
                if np.isfinite(want):
                    assert np.isfinite(got)
                else:
                    assert got == want or (np.isnan(got) and np.isnan(want)), (blk, hex(here), hex(there), i, got, want)
        c.pools.data[1][page, TOKEN, FEATURE] = was

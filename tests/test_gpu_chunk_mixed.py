"""Chunks of several kinds in one launch, more sequences than a wavefront has lanes, rows that attend more units than are looked up at a time, and caches beyond 4 GB."""

import numpy as np
import pytest
import torch

from paper_2407_17678_amd import binding as B
from paper_2407_17678_amd import synth
from tests import cache_util as U
from tests import gpu_util as G
from tests.test_gpu_chunk import FORMATS, Chunk
from tests.test_gpu_tree import _ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D, S", [(128, 64), (64, 64), (128, 16), (64, 16), (128, 32), (64, 128)])
@pytest.mark.parametrize("splits", [0, 3])
def test_short_chunks_among_long_ones(fmt, D, S, splits):
    new = [150, 1, 20, 32, 33, 7, 0, 129]
    lens = [n + (37 * i) % (3 * S) for i, n in enumerate(new)]
    lens[2], lens[3] = 128 - 12 + 20, 128 + 32  # (rows on both sides of a tile's edge, and from one on)
    Chunk(fmt, D, S, lens, new, 2, local=2, stride=3, seed=splits, evict=[(2, 0, 0), (5, 1, 0)]).check(splits=splits)


@pytest.mark.parametrize("new", [[1, 0, 3, 2, 5] * 14, [1, 20, 40] * 23, [3] * 66 + [200, 0, 140], [0] * 130 + [70], [2] * 64 + [66], [66] + [2] * 63])
def test_more_sequences_than_lanes(new):
    lens = [n + (29 * i) % 90 for i, n in enumerate(new)]
    Chunk("mxfp8", 64, 32, lens, new, 1, local=2, stride=3).check()
    Chunk("bf16", 64, 64, lens, new, 2, local=1, stride=4).check(max_new=max(new) + 1000)


@pytest.mark.parametrize("S", [16, 64])
def test_values_that_are_not_numbers_in_a_short_chunk_among_long_ones(S):
    """V of an earlier block of the short chunk's sequence; K and V behind its end: only the rows that attend them are touched, of their own sequence and head."""
    c = Chunk("bf16", 64, S, [170, 4 * S + 9], [150, 9], 2, local=1, stride=3, seed=S)
    clean, clean_lse, _ = c.run()
    case, start = c.c, c.start[1]
    for h in range(2):
        for j in range(start // S):
            case.pools.data[1][case.table[1, h, j], 3, 5] = float("nan")
    o, lse, _ = c.run()
    assert np.array_equal(o[c.cu[0]:c.cu[1]], clean[c.cu[0]:c.cu[1]]) and np.array_equal(lse, clean_lse)
    touched = 0
    for h in range(2):
        for i in range(9):
            row, block = c.cu[1] + i, (start + i) // S
            bad = any(case.keeps(h)(block, j) for j in range(start // S))
            touched += bad
            assert np.isnan(o[row, h, 5]) == bad
            assert np.array_equal(np.delete(o[row, h], 5), np.delete(clean[row, h], 5))
    assert touched > 0


def _dense_chunk(fmt, D, S, blocks, T, splits, far=0, seed=0):
    """The last T tokens of a dense sequence over `blocks` blocks whose pages repeat twelve of them, against the same attention in 64 bits on the device.
    far: bytes from page to page."""
    pages, L, H = 12, blocks * S - S // 2, 2
    rng = np.random.default_rng([seed, D, S, T])
    bits = [synth.normal_bf16(rng, (pages * S, 1, D)) for _ in "kv"]
    pools = U.Pools(fmt, pages, S, D)
    if far:
        pools.data = [torch.empty(pages * far, dtype=torch.uint8, device="cuda").view(x.dtype).as_strided(x.shape, (far // x.element_size(), x.stride(1), 1))
                      for x in pools.data]
    own = pools.cache(_ints(np.arange(pages).reshape(1, 1, pages)))
    B.s2_kv_append_paged(own, G.to_dev(bits[0]), G.to_dev(bits[1]), _ints([0, pages * S]), _ints([0]), pages * S)
    k, v = (torch.from_numpy(U.held_rows(x, fmt)[2][:, 0]).cuda().view(pages, S, D) for x in bits)
    table = rng.integers(0, pages, size=(1, H, blocks)).astype(np.int32)
    cache, params, scale = pools.cache(_ints(table)), B.layout_params(H, 1, S, 1, 0, dense=1), D ** -0.5
    q = synth.normal_bf16(rng, (T, H, D))
    dq = G.to_dev(q)
    o, lse, missing = torch.empty_like(dq), torch.empty((H, T), dtype=torch.float32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.s2_attn_chunk_workspace_bytes(1, H, T, T, D, blocks * S, splits), dtype=torch.uint8, device="cuda")
    B.s2_attn_chunk_paged(params, cache, dq, _ints([0, T]), _ints([L - T]), o, lse, scale, ws, T, missing=missing, num_splits=splits)
    torch.cuda.synchronize()
    assert int(missing.item()) == 0
    later = torch.arange(L, device="cuda") > torch.arange(L - T, L, device="cuda")[:, None]
    for h in range(H):
        at = torch.from_numpy(table[0, h].astype(np.int64)).cuda()
        keys, values = (x[at].flatten(0, 1)[:L] for x in (k, v))
        s = (torch.from_numpy(G.bits_f64(q[:, h])).cuda() @ keys.T * scale).masked_fill(later, -np.inf)
        p = torch.softmax(s, -1)
        want, weight = (p @ values).cpu().numpy(), (p @ values.abs()).cpu().numpy()
        assert np.all(np.abs(G.to_f64(o)[:, h] - want) <= U.attention_bound(want, weight))
        assert np.all(np.abs(G.to_f64(lse)[h] - torch.logsumexp(s, -1).cpu().numpy()) <= U.LSE_BOUND)


# a workgroup looks up 64 units of 64 tokens at a time (16 of blocks under 64); of up to 32 rows two pairs of wavefronts take as many each
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T", [12, 24, 40, 150])
@pytest.mark.parametrize("D, S, blocks", [(64, 16, 2 * 64 + 9), (128, 32, 2 * 32 + 5), (64, 64, 2 * 64 + 3), (128, 128, 64 + 3), (128, 16, 5 * 64 + 30), (128, 64, 300)])
def test_long_rows(fmt, T, D, S, blocks):
    _dense_chunk(fmt, D, S, blocks, T, 1)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T, splits", [(5, 0), (20, 1), (50, 2), (200, 1)])
def test_pages_beyond_4_gb(fmt, T, splits):
    _dense_chunk(fmt, 128, 64, 20, T, splits, far=(1 << 29) + 4096)

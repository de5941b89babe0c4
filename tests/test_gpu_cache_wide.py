"""Attention over a paged cache where a launch has many workgroups, or a split more units than its lanes look up at a time; and tiles of rows written at their largest."""

import numpy as np
import pytest
import torch

from paper_2407_17678_amd import binding as B
from paper_2407_17678_amd import synth
from tests import cache_util as U
from tests import gpu_util as G
from tests.test_gpu_tree import Case, _ints, random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("D, S", [(128, 64), (64, 16), (128, 16), (64, 64), (128, 32), (64, 128)])
@pytest.mark.parametrize("splits", [0, 3])
def test_decode_of_more_than_256_workgroups(fmt, D, S, splits):
    """Four wavefronts to a workgroup instead of eight."""
    rng = np.random.default_rng([D, S])
    lens = list(rng.integers(1, 6 * S, size=29)) + [1, 6 * S]
    Case(fmt, D, S, [int(x) for x in lens], 9, None, evict=[(3, 1, 0), (30, 8, 5)], seed=splits).check(splits=splits)


def _same_rows_elsewhere(fmt, D, S, blocks, T, splits, seed=0):
    """A dense sequence over `blocks` blocks whose pages repeat twelve of them, against the same attention in 64 bits on the device."""
    pages, L, H = 12, blocks * S - S // 2, 2
    rng = np.random.default_rng([seed, D, S, T])
    bits = [synth.normal_bf16(rng, (pages * S, 1, D)) for _ in "kv"]
    pools = U.Pools(fmt, pages, S, D)
    own = pools.cache(_ints(np.arange(pages).reshape(1, 1, pages)))
    B.s2_kv_append_paged(own, G.to_dev(bits[0]), G.to_dev(bits[1]), _ints([0, pages * S]), _ints([0]), pages * S)
    k, v = (torch.from_numpy(U.held_rows(x, fmt)[2][:, 0]).cuda().view(pages, S, D) for x in bits)
    max_blocks = blocks + -(-max(T, 1) // S) + 1
    table = rng.integers(0, pages, size=(1, H, max_blocks)).astype(np.int32)
    cache = pools.cache(_ints(table))
    params = B.layout_params(H, 1, S, 1, 0, dense=1)
    scale, N = D ** -0.5, max(T, 1)
    q, kd, vd = (synth.normal_bf16(rng, (1, H, N, D)) for _ in range(3))
    dq, dk, dv = (G.to_dev(x) for x in (q, kd, vd))
    o, lse = torch.empty_like(dq), torch.empty((1, H, N), dtype=torch.float32, device="cuda")
    missing = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.s2_attn_tree_workspace_bytes(1, H, N, D, max_blocks * S, splits), dtype=torch.uint8, device="cuda")
    parents = random_tree(rng, N) if T else None
    if T:
        B.s2_attn_tree_paged(params, cache, dq, dk, dv, _ints(parents[None]), _ints([L]), o, lse, scale, ws, missing=missing, num_splits=splits)
    else:
        B.s2_attn_decode_paged_cache(params, cache, dq[:, :, 0], _ints([L]), o[:, :, 0], lse[..., 0], scale, ws, missing=missing, num_splits=splits)
    torch.cuda.synchronize()
    assert int(missing.item()) == 0
    f64 = lambda x: torch.from_numpy(G.bits_f64(x)).cuda()  # noqa: E731
    up = torch.eye(N, dtype=torch.float64, device="cuda")
    for i in range(N if T else 0):
        if parents[i] >= 0:
            up[i] += up[int(parents[i])]
    for h in range(H):
        at = torch.from_numpy(table[0, h].astype(np.int64)).cuda()
        keys, values = (x[at].flatten(0, 1)[:L] for x in (k, v))
        s = f64(q)[0, h] @ keys.T * scale
        if T:
            drafted = torch.where(up > 0, f64(q)[0, h] @ f64(kd)[0, h].T * scale, -np.inf)
            s, values = torch.cat([s, drafted], 1), torch.cat([values, f64(vd)[0, h]])
        p = torch.softmax(s, -1)
        want, weight = (p @ values).cpu().numpy(), (p @ values.abs()).cpu().numpy()
        assert np.all(np.abs(G.to_f64(o)[0, h] - want) <= U.attention_bound(want, weight))
        assert np.all(np.abs(G.to_f64(lse)[0, h] - torch.logsumexp(s, -1).cpu().numpy()) <= U.LSE_BOUND)


# blocks so that one split has more units than are looked up at a time: a decode step's wavefronts (8, and 4 where there are more workgroups) take 64 each (16 of
# blocks under 64), the two pairs of a tree of up to 32 nodes 64 each, the workgroup of a larger tree 64
@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("D, S, blocks", [(64, 16, 8 * 64 + 9), (128, 32, 8 * 32 + 5), (64, 64, 8 * 64 + 3), (128, 128, 8 * 32 + 3), (128, 16, 2 * 8 * 64 + 70)])
def test_long_rows_of_decode_steps(fmt, D, S, blocks):
    _same_rows_elsewhere(fmt, D, S, blocks, 0, 1)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("T", [12, 24, 40])
@pytest.mark.parametrize("D, S, blocks", [(64, 16, 2 * 64 + 9), (128, 32, 2 * 32 + 5), (64, 64, 2 * 64 + 3), (128, 128, 64 + 3), (128, 16, 5 * 64 + 30), (128, 64, 300)])
def test_long_rows_of_trees(fmt, T, D, S, blocks):
    _same_rows_elsewhere(fmt, D, S, blocks, T, 1)


@pytest.mark.parametrize("T", [0, 12, 24, 40])
@pytest.mark.parametrize("S", [16, 64])
def test_long_rows_in_splits(T, S):
    _same_rows_elsewhere("mxfp8", 64, S, 1200 if S == 16 else 700, T, 2)
    _same_rows_elsewhere("mxfp4", 64, S, 1200 if S == 16 else 700, T, 0)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("evicted", [0.0, 0.5, 0.97])
def test_prompts_of_many_tiles(fmt, D, evicted):
    """Tiles of 16 rows to a wavefront that writes: the same bytes as the rows written one sequence and 16 rows at a time, which are tiles of fewer."""
    nseq, H, S, n = 4, 32, 64, 520  # 4 x 33 tiles x 32 heads: more than 2048
    rng = np.random.default_rng([D, int(100 * evicted)])
    blocks = -(-n // S)
    table = rng.permutation(nseq * H * blocks).reshape(nseq, H, blocks)
    table[rng.random(table.shape) < evicted] = -1
    bits = [G.to_dev(synth.normal_bf16(rng, (nseq * n, H, D))) for _ in "kv"]
    pools, other = (U.Pools(fmt, nseq * H * blocks, S, D) for _ in range(2))
    skipped = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.s2_kv_append_paged(pools.cache(_ints(table)), *bits, _ints(np.arange(nseq + 1) * n), _ints([0] * nseq), n, skipped=skipped)
    for b in range(nseq):
        one = other.cache(_ints(table[b:b + 1]))
        for lo in range(0, n, 16):
            m = min(16, n - lo)
            B.s2_kv_append_paged(one, *(x[b * n + lo:b * n + lo + m] for x in bits), _ints([0, m]), _ints([lo]), m)
    torch.cuda.synchronize()
    for w in range(2):
        for a, c in zip(pools.host(w), other.host(w)):
            assert (a is None and c is None) or np.array_equal(a, c)
    rows = np.clip(n - np.arange(blocks) * S, 0, S)
    assert int(skipped.item()) == int(((table < 0) * rows).sum())
    # and one block against the oracle's search
    b, h, j = np.argwhere(table >= 0)[0]
    held, byte, _ = U.held_rows(bits[0][b * n + j * S:b * n + (j + 1) * S, h].cpu().view(torch.int16).numpy().view(np.uint16), fmt)
    got, got_byte = pools.host(0)
    assert np.array_equal(got[table[b, h, j]], held) and (byte is None or np.array_equal(got_byte[table[b, h, j]], byte))

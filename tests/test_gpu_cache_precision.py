"""Probabilities of attention over a paged cache keep 16 bits or more on their way to V: a tree's node is held to what a decode step gives."""

import numpy as np
import pytest
import torch

from paper_2407_17678_amd import binding as B
from tests import cache_util as U
from tests import gpu_util as G
from tests.test_gpu_tree import Case, random_tree

pytestmark = pytest.mark.gpu


def _bound(c, want, weight):
    """O's own rounding is half a step of bf16, 2^-8 of the value.  A score is a sum of D products that are exact in 32 bits: off by D 2^-23 of the sum of their
    magnitudes (whichever way the sum rounds), and by 2^-21 of itself and 2^-21 with the scaling, the maximum and the exponential.  It enters p_j, and the sum that
    divides.  p_j to 16 bits: 2^-16.  Sums of n values: n 2^-23.  All of them relative to weight = sum_j p_j |v_j|."""
    q, kd = np.abs(G.bits_f64(c.q)), np.abs(G.bits_f64(c.kd))
    sums, n = [], max(c.lens) + c.T
    for b in range(c.nseq):
        for h in range(c.H):
            keys = np.concatenate([np.abs(c.k[b][h]), kd[b, h] if c.tree else kd[b, h][:0]])
            sums.append((q[b, h] @ keys.T).max())
    most = max(sums) * c.scale
    eps = 2 * (c.D * 2.0 ** -23 * most + 2.0 ** -21 * (most + 1)) + 2.0 ** -16 + n * 2.0 ** -23
    assert eps < 2.0 ** -10, eps  # (a probability rounded to bf16 is off by up to 2^-8)
    return 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -7) + eps * weight


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("T", [1, 9, 24, 50])
@pytest.mark.parametrize("S, lens", [(16, [3, 6, 20, 0]), (64, [2, 9, 70, 1])])
def test_trees(fmt, T, S, lens):
    rng = np.random.default_rng([T, S])
    c = Case(fmt, 64, S, lens, 6, np.stack([random_tree(rng, T) for _ in lens]), local=3)
    o, _, _ = c.run()
    want, _, weight, _ = c.oracle()
    off = np.abs(o - want) - _bound(c, want, weight)
    assert np.all(off <= 0), (float(off.max()), int((off > 0).sum()))


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("strided", [False, True])
def test_decode_steps(fmt, strided):
    for S, lens in ((16, [3, 6, 20, 1]), (64, [2, 9, 70, 4])):
        c = Case(fmt, 64, S, lens, 6, None, local=3)
        o, _, _ = c.run(strided=strided)
        want, _, weight, _ = c.oracle()
        off = np.abs(o - want) - _bound(c, want, weight)
        assert np.all(off <= 0), (float(off.max()), int((off > 0).sum()))


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
def test_a_chain_is_as_many_decode_steps(fmt):
    """The last node of a chain of T, and a decode step over the cache that the same rows have been written into."""
    H, D, S, L = 4, 64, 16, 21
    for T in (3, 20, 40):
        par = np.arange(-1, T - 1, dtype=np.int32)[None]
        c = Case(fmt, D, S, [L], H, par, local=2, stride=3, seed=T)
        # (what the cache would hold of the nodes: in 8 and 4 bits they are other values, so the tree is asked with those)
        rows = [U.held_rows(x[0].transpose(1, 0, 2), fmt) for x in (c.kd, c.vd)]
        values = [torch.from_numpy(r[2]).to(torch.bfloat16).cuda() for r in rows]
        bits = [v.transpose(0, 1).contiguous().view(torch.int16).cpu().numpy().view(np.uint16)[None] for v in values]
        c.kd, c.vd = bits
        tree, _, _ = c.run()
        cache = c.pools.cache(torch.from_numpy(c.table).cuda())
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        B.s2_kv_append_paged(cache, G.to_dev(c.kd)[0].transpose(0, 1), G.to_dev(c.vd)[0].transpose(0, 1), ints([0, T]), ints([L]), T)
        q = G.to_dev(c.q)[:, :, T - 1].contiguous()
        o = torch.empty_like(q)
        ws = torch.empty(B.s2_attn_tree_workspace_bytes(1, H, 1, D, c.max_blocks * S), dtype=torch.uint8, device="cuda")
        B.s2_attn_decode_paged_cache(c.params, cache, q, ints([L + T]), o, None, c.scale, ws)
        torch.cuda.synchronize()
        want, _, weight, _ = c.oracle()
        off = np.abs(G.to_f64(o)[0] - tree[0, :, -1]) - 2 * _bound(c, want, weight)[0, :, -1]
        assert np.all(off <= 0), float(off.max())

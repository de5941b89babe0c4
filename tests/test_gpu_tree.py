"""Attention over a paged cache in bf16, 8 and 4 bits, a decode step or a tree of drafted tokens, against the fp64 oracle on the values the cache stands for."""

import numpy as np
import pytest
import torch

from oracle import s2_oracle as orc
from paper_2407_17678_amd import binding as B
from paper_2407_17678_amd import synth
from tests import cache_util as U
from tests import gpu_util as G

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(np.asarray(x).tolist(), dtype=torch.int32, device="cuda")


def random_tree(rng, T, used=None):
    par = np.array([rng.integers(-1, i) if i else -1 for i in range(T)], dtype=np.int32)
    par[used if used is not None else T:] = -2
    return par


class Case:
    """A cache on the device and on the host, a batch of trees (or, tree=False, one query to a sequence)."""

    def __init__(self, fmt, D, S, lens, H, parents, local=2, stride=3, window=0, dense=0, base=0, max_blocks=None, gap=0, seed=0, evict=(), mask=None,
                 spread=1.0):
        rng = np.random.default_rng([seed, D, S, H])
        self.fmt, self.D, self.S, self.H, self.lens, self.base = fmt, D, S, H, list(lens), base
        self.tree = parents is not None
        self.parents = parents
        self.mask = mask  # [H, B, B] of a caller's pattern
        nseq, T = len(lens), parents.shape[1] if self.tree else 1
        self.nseq, self.T, self.scale = nseq, T, 1.0 / np.sqrt(D)
        self.max_blocks = max_blocks or max(1, -(-(max(lens) + T) // S))
        self.params = B.layout_params(H, self.max_blocks, S, local, stride, base, window, dense)
        self.rule = (local, stride, window, dense)
        self.q, self.kd, self.vd = (synth.normal_bf16(rng, (nseq, H, T, D)) for _ in range(3))
        self.q = synth.round_to_bf16_bits(synth.bf16_bits_to_f32(self.q) * np.float32(spread))
        table = rng.permutation(nseq * H * self.max_blocks + 1)[1:].reshape(nseq, H, self.max_blocks).astype(np.int32)
        self.pools = U.Pools(fmt, nseq * H * self.max_blocks + 1, S, D, gap)
        self.k, self.v = [], []
        for b in range(nseq):
            ks, vs = [], []
            for which, to in ((0, ks), (1, vs)):
                for h in range(H):
                    bits = synth.normal_bf16(rng, (lens[b], D))
                    held, byte, value = U.held_rows(bits, fmt)
                    to.append(value)
                    for j in range(-(-lens[b] // S)):
                        cut = slice(j * S, min((j + 1) * S, lens[b]))
                        self.pools.put(which, table[b, h, j], 0, held[cut], None if byte is None else byte[cut])
            self.k.append(ks)
            self.v.append(vs)
        for b, h, j in evict:  # (not a page: negative, or beyond the last)
            table[b, h, j] = (-1, nseq * H * self.max_blocks + 1, 2 ** 31 - 1)[j % 3]
        self.pages = nseq * H * self.max_blocks + 1
        self.table = table

    def keeps(self, h):
        local, stride, window, dense = self.rule
        if self.mask is not None:
            return lambda i, j: bool(self.mask[h, i, j])
        if dense:
            return lambda i, j: j <= i
        return lambda i, j: bool(orc.block_predicate(i, j, orc.head_offset(self.base + h, stride), local, stride, window))

    def run(self, splits=0, layout=None, strided=False, stream=None):
        cache = self.pools.cache(_ints(self.table))
        lens = _ints(self.lens)
        n, H, T, D = self.nseq, self.H, self.T, self.D
        missing = torch.full((1,), 5, dtype=torch.int32, device="cuda")
        ws_bytes = B.s2_attn_tree_workspace_bytes(n, H, T, D, self.max_blocks * self.S, splits)
        ws = torch.full((ws_bytes,), 0xFF, dtype=torch.uint8, device="cuda")
        lse = torch.full((n, H, T), 9.0, dtype=torch.float32, device="cuda")
        pattern = layout or self.params
        if self.tree:
            q, kd, vd = (G.to_dev(x) for x in (self.q, self.kd, self.vd))
            o = torch.full_like(q, 9.0)
            if strided:
                lay = lambda x: torch.zeros(n, T + 1, H, D + 8, dtype=torch.bfloat16, device="cuda")[:, :T, :, :D].permute(0, 2, 1, 3).copy_(x)  # noqa: E731
                q, o, kd, vd = lay(q), lay(o), lay(kd), lay(vd)
            f = B.s2_attn_tree_paged_layout if layout else B.s2_attn_tree_paged
            f(pattern, cache, q, kd, vd, _ints(self.parents), lens, o, lse, self.scale, ws, missing=missing, num_splits=splits)
        else:
            q = G.to_dev(self.q[:, :, 0])
            o = torch.full_like(q, 9.0)
            if strided:
                lay = lambda x: torch.zeros(H, n, D + 8, dtype=torch.bfloat16, device="cuda")[..., :D].transpose(0, 1).copy_(x)  # noqa: E731
                q, o = lay(q), lay(o)
            f = B.s2_attn_decode_paged_cache_layout if layout else B.s2_attn_decode_paged_cache
            f(pattern, cache, q, lens, o, lse[..., 0].contiguous(), self.scale, ws, missing=missing, num_splits=splits)
            lse1 = torch.full((n, H), 9.0, dtype=torch.float32, device="cuda")
            f(pattern, cache, q, lens, o, lse1, self.scale, ws, num_splits=splits)
            o, lse = o[:, :, None], lse1[:, :, None]
        torch.cuda.synchronize()
        return G.to_f64(o), G.to_f64(lse), int(missing.item()) - 5

    def oracle(self):
        n, H, T, D = self.nseq, self.H, self.T, self.D
        o, lse, weight = np.zeros((n, H, T, D)), np.zeros((n, H, T)), np.zeros((n, H, T, D))
        missing = 0
        q, kd, vd = (G.bits_f64(x) for x in (self.q, self.kd, self.vd))
        for b in range(n):
            L = self.lens[b]
            for h in range(H):
                keeps, held = self.keeps(h), lambda j: 0 <= self.table[b, h, j] < self.pages  # noqa: B023
                if self.tree:
                    o[b, h], lse[b, h], weight[b, h] = orc.tree_attention(q[b, h], self.k[b][h], self.v[b][h], kd[b, h], vd[b, h], self.parents[b], L, keeps,
                                                                          self.S, self.scale, self.max_blocks * self.S, held)
                    rows = {(L + len(c) - 1) // self.S for c in orc.tree_chains(self.parents[b]) if c and L + len(c) - 1 < self.max_blocks * self.S}
                else:
                    rows = {(L - 1) // self.S}
                    seen = [t for t in range(L) if keeps((L - 1) // self.S, t // self.S) and held(t // self.S)]
                    o[b, h, 0], lse[b, h, 0], weight[b, h, 0] = orc.attend(q[b, h, 0], self.k[b][h][seen], self.v[b][h][seen], self.scale)
                missing += sum(any(keeps(r, j) for r in rows) and not held(j) for j in range(-(-L // self.S)))
        return o, lse, weight, missing

    def check(self, **kw):
        o, lse, missing = self.run(**kw)
        want, want_lse, weight, want_missing = self.oracle()
        off = np.abs(o - want) - U.attention_bound(want, weight)
        assert np.all(off <= 0), (float(off.max()), np.argwhere(off > 0)[:5])
        gone = ~np.isfinite(want_lse)
        assert np.array_equal(~np.isfinite(lse), gone) and np.all(o[gone] == 0) and np.all(lse[gone] == -np.inf)
        assert np.all(np.abs(lse[~gone] - want_lse[~gone]) <= U.LSE_BOUND)
        assert missing == want_missing
        return o, lse


# ------------------------------------------------------------------------------------ decode


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("D, S", [(128, 64), (64, 64), (128, 16), (64, 16), (128, 32), (64, 32), (128, 128), (64, 128)])
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_decode(fmt, D, S, splits):
    Case(fmt, D, S, [1, S, S + 1, 5 * S - 3, 9 * S + S // 2], 3, None, seed=splits).check(splits=splits)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
def test_decode_patterns_strides_and_missing_blocks(fmt):
    Case(fmt, 128, 16, [200, 33], 5, None, local=1, stride=4, window=6, base=3).check()
    Case(fmt, 64, 64, [500, 64], 2, None, dense=1).check(strided=True)
    Case(fmt, 128, 32, [300, 97], 2, None, local=3, stride=0, gap=16).check(strided=True)
    c = Case(fmt, 128, 16, [200, 17], 2, None, evict=[(0, 0, 12), (0, 1, 11), (1, 0, 0), (1, 0, 1)])
    o, lse = c.check()
    assert lse[1, 0, 0] == -np.inf  # nothing left


def test_decode_over_bf16_is_the_bf16_call():
    c = Case("bf16", 128, 64, [130, 700, 64], 4, None)
    o, lse, _ = c.run()
    q, lens = G.to_dev(c.q[:, :, 0]), _ints(c.lens)
    want, want_lse = torch.empty_like(q), torch.empty((3, 4), dtype=torch.float32, device="cuda")
    ws = torch.empty(B.s2_attn_decode_workspace_bytes(3, 4, 128, c.max_blocks * 64), dtype=torch.uint8, device="cuda")
    B.s2_attn_decode_paged(c.params, q, c.pools.data[0], c.pools.data[1], _ints(c.table), lens, want, want_lse, c.scale, ws)
    torch.cuda.synchronize()
    assert np.array_equal(o[:, :, 0], G.to_f64(want)) and np.array_equal(lse[:, :, 0], G.to_f64(want_lse))


# ------------------------------------------------------------------------------------ trees


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("D, S", [(128, 64), (64, 64), (128, 16), (64, 16), (128, 32), (64, 128), (128, 128), (64, 32)])
@pytest.mark.parametrize("T", [1, 7, 16, 17, 33, 64])
def test_random_trees(fmt, D, S, T):
    rng = np.random.default_rng([T, S])
    lens = [0, 1, S - 1, 3 * S, 7 * S - 2]
    parents = np.stack([random_tree(rng, T, used) for used in (T, max(1, T // 2), T, T, 1)])
    Case(fmt, D, S, lens, 2, parents, seed=T).check(splits=T % 3)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("S", [16, 32, 64, 128])
def test_chains_across_blocks(fmt, S):
    """64 nodes one below the other: up to five block rows, of which each keeps other blocks, drafted ones among them."""
    T = 64
    parents = np.stack([np.arange(-1, T - 1, dtype=np.int32)] * 3)
    for local, stride, window in ((1, 0, 0), (2, 3, 0), (1, 4, 7), (3, 2, 4)):
        Case(fmt, 64, S, [S - 1, 5 * S + 3, 6 * S], 3, parents, local=local, stride=stride, window=window).check()
    Case(fmt, 128, S, [S - 1, 5 * S + 3, 6 * S], 2, parents, dense=1).check(splits=2)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp4"])
@pytest.mark.parametrize("S", [16, 64])
def test_trees_that_are_no_trees(fmt, S):
    """Nodes whose parent is itself, a later one, out of range, or hangs on such a node; padding; all of it."""
    T = 20
    a = np.arange(-1, T - 1, dtype=np.int32)
    a[5] = 5
    b = random_tree(np.random.default_rng(4), T)
    b[[2, 7, 9]] = [19, -7, 2 ** 31 - 1]
    c = np.full(T, -2, dtype=np.int32)
    d = np.full(T, -1, dtype=np.int32)
    o, lse = Case(fmt, 128, S, [40, 3, 77, 100], 2, np.stack([a, b, c, d])).check()
    assert np.all(lse[2] == -np.inf)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
def test_strides_head_base_splits_and_missing_blocks(fmt):
    rng = np.random.default_rng(8)
    par = np.stack([random_tree(rng, 24), random_tree(rng, 24, 11)])
    Case(fmt, 128, 16, [250, 15], 3, par, base=5, gap=32).check(strided=True, splits=5)
    Case(fmt, 64, 64, [300, 66], 3, par, gap=16, spread=4.0).check(strided=True, splits=64)
    c = Case(fmt, 64, 16, [250, 40], 2, par, evict=[(0, 0, 15), (0, 1, 14), (0, 1, 3), (1, 0, 0), (1, 0, 1), (1, 0, 2)])
    c.check(splits=2)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("T", [1, 5, 16, 40])
def test_missing_blocks_are_counted_once(fmt, T):
    rng = np.random.default_rng(T)
    par = np.stack([random_tree(rng, T), random_tree(rng, T)])
    for S, lens, gone in ((16, [250, 40], [(0, 0, 15), (0, 1, 14), (0, 1, 3), (1, 0, 0), (1, 0, 1), (1, 0, 2)]), (64, [700, 66], [(0, 0, 10), (0, 1, 9), (1, 1, 0)])):
        for splits in (0, 1, 3):
            Case(fmt, 64, S, lens, 2, par, evict=gone, local=4).check(splits=splits)
        if T == 1:
            Case(fmt, 64, S, lens, 2, None, evict=gone, local=4).check(strided=True)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("T", [12, 24, 40])
def test_an_infinity_that_one_wavefront_meets(fmt, T):
    """A token of V that is infinite, in blocks that the first row of the tree keeps and the second does not: the nodes of the first row have the
    infinity, whichever wavefront met it; those of the second stay finite."""
    S, L = 16, 16 * 9 + 15
    par = np.stack([np.arange(-1, T - 1, dtype=np.int32)])
    c = Case(fmt, 64, S, [L], 1, par, local=6, stride=0)
    bits = np.full((S, 64), 0x3F80, dtype=np.uint16)
    bits[3, 5] = 0x7F80
    held, byte, _ = U.held_rows(bits, fmt)
    blk = L // S - 5  # the last that row L // S keeps
    c.pools.put(1, c.table[0, 0, blk], 0, held, None if byte is None else byte)
    o, _, _ = c.run(splits=1)
    first = [i for i in range(T) if (L + i) // S == L // S]
    assert first and len(first) < T
    rest = [i for i in range(T) if i not in first]
    assert np.all(np.isfinite(o[0, 0, rest]))
    if fmt == "bf16":
        assert np.all(o[0, 0, first, 5] == np.inf) and np.all(np.isfinite(np.delete(o[0, 0, first], 5, -1)))
    else:  # (a scale stands for 32 features: none of them is a number)
        assert np.all(np.isnan(o[0, 0, first, :32])) and np.all(np.isfinite(o[0, 0, first, 32:]))


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_no_room_for_the_deeper_nodes(fmt):
    """Nodes at positions that the table has no block for do not exist."""
    par = np.stack([np.arange(-1, 19, dtype=np.int32)] * 2)
    o, lse = Case(fmt, 64, 16, [40, 48], 2, par, max_blocks=3).check()
    assert np.all(np.isfinite(lse[0, :, :8])) and np.all(lse[0, :, 8:] == -np.inf) and np.all(lse[1] == -np.inf)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("S", [16, 64])
def test_a_pattern_of_the_callers_own(fmt, S):
    """Rows that differ from one another at random (and a sink): blocks that one row of a tree keeps and the next does not."""
    H, Bk, T = 3, 12, 40
    rng = np.random.default_rng(S)
    mask = np.tril(rng.random((H, Bk, Bk)) < 0.4)
    mask[:, np.arange(Bk), np.arange(Bk)] = True
    mask[0, :, 0] = True
    row_ptr, col_idx, _, _ = orc.compressed_layout(mask)
    layout = B.s2_layout_from_csr(H, Bk, S, row_ptr, col_idx)
    par = np.stack([np.arange(-1, T - 1, dtype=np.int32), random_tree(rng, T), random_tree(rng, T, 9)])
    lens = [7 * S + 1, 8 * S, 5]
    Case(fmt, 128, S, lens, H, par, max_blocks=Bk, mask=mask).check(layout=layout, splits=2)
    Case(fmt, 64, S, lens, H, par, max_blocks=Bk - 1, mask=mask).check(layout=layout)
    Case(fmt, 64, S, [x + 1 for x in lens], H, None, max_blocks=Bk, mask=mask).check(layout=layout)


# ------------------------------------------------------------------------------------ what is not attended


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("S, local", [(16, 1), (64, 1), (32, 2)])
def test_nothing_of_what_a_node_does_not_attend(fmt, S, local):
    """NaN and infinities in blocks that only another node's row keeps, in siblings, in nodes that do not exist, behind the last token and in
    pages nobody owns: the other nodes' results stay what they are to the last bit."""
    T = 48
    par = np.arange(-1, T - 1, dtype=np.int32)
    par[40:] = [-1, -1, 3, 40, 41, -2, 45, 2]
    clean = Case(fmt, 64, S, [5 * S - 3, 4 * S], 2, np.stack([par, par]), local=local, stride=0)
    o, lse = clean.check()
    dirty = Case(fmt, 64, S, [5 * S - 3, 4 * S], 2, np.stack([par, par]), local=local, stride=0)
    wild = 2
    bits = np.full((S, 64), 0x7FC0, dtype=np.uint16)
    bits[:, ::3] = 0x7F80
    held, byte, value = U.held_rows(bits, fmt)
    sees = np.zeros((2, 2, T), dtype=bool)  # whether a node attends something that is not a number
    for b, L in enumerate(clean.lens):
        j = (L - 1) // S - local + 1  # a block that the first row keeps and later ones do not
        for h in range(2):
            cut = slice(0, min(S, L - j * S))
            dirty.pools.put(1, dirty.table[b, h, j], 0, held[cut], None if byte is None else byte[cut])
            dirty.pools.put(0, dirty.table[b, h, j], 0, held[cut], None if byte is None else byte[cut])
            for i, chain in enumerate(orc.tree_chains(par)):
                if chain:
                    sees[b, h, i] = clean.keeps(h)((L + len(chain) - 1) // S, j)
    for i in (41, 45, 46):  # a sibling with a child, and two nodes that do not exist
        dirty.kd[:, :, i], dirty.vd[:, :, i], dirty.q[:, :, 45:47] = 0x7FC0, 0x7F80, 0x7FC0
    for i, chain in enumerate(orc.tree_chains(par)):
        if chain and 41 in chain:
            sees[:, :, i] = True
    assert sees.any() and not sees.all() and wild
    got, got_lse, _ = dirty.run()
    ok = ~sees
    assert np.array_equal(got[ok], o[ok]) and np.array_equal(got_lse[ok], lse[ok])
    there = np.array([c is not None for c in orc.tree_chains(par)])
    assert np.all(np.isnan(got[sees & there]).any(-1) | np.isinf(got[sees & there]).any(-1))


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("T", [14, 30, 64])
@pytest.mark.parametrize("D, S, splits", [(64, 16, 1), (128, 16, 3), (128, 64, 2), (64, 128, 1)])
def test_who_meets_what_is_no_number(fmt, T, D, S, splits):
    """NaN and infinities in one cached block and in two nodes: whoever attends none of them has what it had, to the last bit."""
    par = np.arange(-1, T - 1, dtype=np.int32)
    par[T - 5:] = [-1, 0, T - 5, 1, -1]
    L = 6 * S + S - 6
    make = lambda: Case(fmt, D, S, [L, L - 2 * S], 2, np.stack([par, par]), local=2, stride=4, window=5)  # noqa: E731
    clean, dirty = make(), make()
    o, lse = clean.check(splits=splits)
    bits = np.full((S, D), 0x7F80, dtype=np.uint16)
    bits[::3], bits[1::3] = 0x7FC0, 0xFF80
    held, byte, _ = U.held_rows(bits, fmt)
    chains = orc.tree_chains(par)
    meets = np.zeros((2, 2, T), dtype=bool)
    for b, n in enumerate(clean.lens):
        blk = n // S - 1  # kept by the row of the first nodes, and not by the next ones (unless it is a stripe of the head's)
        for h in range(2):
            for which in range(2):
                dirty.pools.put(which, dirty.table[b, h, blk], 0, held, byte)
            keeps = clean.keeps(h)
            for i, chain in enumerate(chains):
                row = (n + len(chain) - 1) // S
                meets[b, h, i] = keeps(row, blk) or any(x in chain and keeps(row, (n + len(chains[x]) - 1) // S) for x in (T - 5, T - 2))
    dirty.kd[:, :, T - 5], dirty.vd[:, :, T - 2] = 0x7FC0, 0xFF80
    got, got_lse, _ = dirty.run(splits=splits)
    assert meets.any()
    assert np.array_equal(got[~meets], o[~meets]) and np.array_equal(got_lse[~meets], lse[~meets])
    assert not np.isfinite(got[meets]).all(-1).any()


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
def test_decode_leaves_stale_rows_alone(fmt):
    """Rows behind the last token hold what was there before (the pools are filled with 0xFF: NaN)."""
    o, lse = Case(fmt, 128, 64, [1, 63, 65, 129], 2, None, local=4).check()
    assert np.all(np.isfinite(o))


# ------------------------------------------------------------------------------------ far away


def _attend(cache, H, D, S, L, T, params, splits=1):
    """A decode step and a tree of T nodes (chains of three) over a cache of one sequence."""
    rng = np.random.default_rng([T, D])
    q, kd, vd = (G.to_dev(synth.normal_bf16(rng, (1, H, T, D))) for _ in range(3))
    par = _ints([[i - 1 if i % 3 else -1 for i in range(T)]])
    max_len = cache.tensors[2].shape[2] * S
    ws = torch.empty(B.s2_attn_tree_workspace_bytes(1, H, T, D, max_len, splits), dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), torch.empty((1, H, T), dtype=torch.float32, device="cuda")
    o1, lse1 = torch.empty_like(q[:, :, 0]), torch.empty((1, H), dtype=torch.float32, device="cuda")
    missing = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.s2_attn_tree_paged(params, cache, q, kd, vd, par, _ints([L]), o, lse, 0.125, ws, missing=missing, num_splits=splits)
    B.s2_attn_decode_paged_cache(params, cache, q[:, :, 0], _ints([L]), o1, lse1, 0.125, ws, missing=missing, num_splits=splits)
    torch.cuda.synchronize()
    assert int(missing.item()) == 0
    return [x.clone() for x in (o, lse, o1, lse1)]


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("T", [3, 20, 50])
def test_pages_far_apart(fmt, T):
    """Pages more than 2^32 bytes from the pool's beginning: the same to the last bit as pages side by side."""
    S, D, L = 16, 64, 40
    far = 5 << 30
    rb, e = U.row_bytes(D, fmt), 2 if fmt == "bf16" else 1
    raw = torch.zeros(far + (1 << 20), dtype=torch.uint8, device="cuda")
    make = lambda at: (raw[at:].view(torch.bfloat16) if fmt == "bf16" else raw[at:]).as_strided(  # noqa: E731
        (2, S, rb // e), ((far - 4096) // e, rb // e, 1))
    scale = lambda at: raw[at:].as_strided((2, S, D // 32), (far - 4096, D // 32, 1)) if fmt != "bf16" else None  # noqa: E731
    table = _ints([[[1, 0, 1]]])  # (the third block is the first's page)
    caches = [B.paged_cache(U.FORMATS[fmt], S, make(4096), make(65536), table, scale(131072), scale(196608)), U.Pools(fmt, 2, S, D).cache(table)]
    k, v = (G.to_dev(synth.normal_bf16(np.random.default_rng(x), (2 * S, 1, D))) for x in (1, 2))
    results = []
    for cache in caches:
        B.s2_kv_append_paged(cache, k, v, _ints([0, 2 * S]), _ints([0]), 2 * S)
        results.append(_attend(cache, 1, D, S, L, T, B.layout_params(1, 1, S, 8, 2)))
    for a, b in zip(*results):
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("T", [3, 20, 50])
@pytest.mark.parametrize("S", [16, 64])
def test_a_billion_tokens(fmt, T, S):
    """One sequence of nearly 2^30 tokens, of which the mask keeps twelve blocks: what attention of these side by side gives, to the last bit."""
    D, blocks, every = 64, (1 << 30) // S, (1 << 28) // S
    row = blocks - 3
    kept = [0, every, 2 * every, 3 * every] + list(range(row - 7, row + 1))
    table = np.full((1, 1, blocks), -1, dtype=np.int32)
    table[0, 0, kept] = np.arange(12)
    results = []
    k, v = (G.to_dev(synth.normal_bf16(np.random.default_rng([S, x]), (S, 1, D))) for x in (1, 2))
    for table, at, params in ((table, kept, B.layout_params(1, 1, S, 8, every)),
                              (np.arange(13, dtype=np.int32).reshape(1, 1, 13) % 12, range(12), B.layout_params(1, 1, S, 1, 0, dense=1))):
        cache = U.Pools(fmt, 12, S, D).cache(torch.from_numpy(table).cuda())
        for i, j in enumerate(at):  # (each block other rows: the same in another order)
            B.s2_kv_append_paged(cache, k, v, _ints([0, S]), _ints([j * S]), S, rows=_ints(np.roll(np.arange(S), i)))
        results.append(_attend(cache, 1, D, S, at[-1] * S + 5, T, params))  # (nodes of three to a chain stay in the block row)
    for a, b in zip(*results):
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())


# ------------------------------------------------------------------------------------ as a program uses it


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("T", [0, 9, 24, 45])
def test_workspaces_of_any_size(fmt, T):
    """With the splits left to the library any workspace from the size for one split on will do, and nothing behind it is written."""
    par = np.stack([random_tree(np.random.default_rng(T), T)]) if T else None
    c = Case(fmt, 128, 64, [4000], 2, par, local=30)
    cache, lens, nodes = c.pools.cache(_ints(c.table)), _ints(c.lens), max(T, 1)
    q, kd, vd = (G.to_dev(x) for x in (c.q, c.kd, c.vd))
    size = lambda n: B.s2_attn_tree_workspace_bytes(1, 2, nodes, 128, c.max_blocks * 64, n)  # noqa: E731
    want, _, weight, _ = c.oracle()
    for given in [size(1), size(2), size(3) + 100, size(0)]:
        raw = torch.full((size(0) + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        if T:
            o = torch.empty_like(q)
            B.s2_attn_tree_paged(c.params, cache, q, kd, vd, _ints(par), lens, o, None, c.scale, raw[:given])
        else:
            o = torch.empty_like(q[:, :, 0])
            B.s2_attn_decode_paged_cache(c.params, cache, q[:, :, 0].contiguous(), lens, o, None, c.scale, raw[:given])
            o = o[:, :, None]
        torch.cuda.synchronize()
        assert np.all(np.abs(G.to_f64(o) - want) <= U.attention_bound(want, weight))
        assert bool((raw[given:] == 0xA5).all())
    with pytest.raises(B.S2Error):
        B.s2_attn_decode_paged_cache(c.params, cache, q[:, :, 0].contiguous(), lens, o[:, :, 0].contiguous(), None, c.scale, raw[:size(1) // nodes - 256])


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
def test_prompt_tree_accept_and_decode(fmt):
    """A prompt is written, a tree verified, the nodes accepted written by index, and the next decode step reads them: every
    step against the oracle on the rows as the cache holds them."""
    H, D, S, T, L = 3, 128, 16, 12, 37
    rng = np.random.default_rng(2)
    blocks = 6
    table = np.arange(H * blocks, dtype=np.int32).reshape(1, H, blocks)
    pools = U.Pools(fmt, H * blocks, S, D)
    cache = pools.cache(_ints(table))
    prompt = [synth.normal_bf16(rng, (L, H, D)) for _ in "kv"]
    B.s2_kv_append_paged(cache, G.to_dev(prompt[0]), G.to_dev(prompt[1]), _ints([0, L]), _ints([0]), L)
    par = np.array([[-1, 0, 0, 1, 2, 2, 5, 4, 6, 6, 9, -1]], dtype=np.int32)
    q, kd, vd = (synth.normal_bf16(rng, (1, T, H, D)) for _ in range(3))
    dq, dk, dv = (G.to_dev(x).permute(0, 2, 1, 3) for x in (q, kd, vd))
    o = torch.empty_like(dq)
    lse = torch.empty((1, H, T), dtype=torch.float32, device="cuda")
    ws = torch.empty(B.s2_attn_tree_workspace_bytes(1, H, T, D, blocks * S), dtype=torch.uint8, device="cuda")
    params = B.layout_params(H, 1, S, 2, 2)
    scale = 1 / np.sqrt(D)
    B.s2_attn_tree_paged(params, cache, dq, dk, dv, _ints(par), _ints([L]), o, lse, scale, ws)
    accepted = [0, 2, 5, 6, 9]
    B.s2_kv_append_paged(cache, dk[0].transpose(0, 1), dv[0].transpose(0, 1), _ints([0, 5]), _ints([L]), 5, rows=_ints(accepted))
    q1 = synth.normal_bf16(rng, (1, H, D))
    o1, lse1 = torch.empty((1, H, D), dtype=torch.bfloat16, device="cuda"), torch.empty((1, H), dtype=torch.float32, device="cuda")
    B.s2_attn_decode_paged_cache(params, cache, G.to_dev(q1), _ints([L + 5]), o1, lse1, scale, ws)
    torch.cuda.synchronize()
    k, v = (U.held_rows(np.concatenate([p, d[0, accepted]]), fmt)[2] for p, d in ((prompt[0], kd), (prompt[1], vd)))
    for h in range(H):
        keeps = lambda i, j: bool(orc.block_predicate(i, j, orc.head_offset(h, 2), 2, 2, 0))  # noqa: E731, B023
        want, want_lse, weight = orc.tree_attention(*(G.bits_f64(x)[0, :, h] for x in (q,)), k[:L, h], v[:L, h], G.bits_f64(kd)[0, :, h], G.bits_f64(vd)[0, :, h],
                                                    par[0], L, keeps, S, scale, blocks * S)
        assert np.all(np.abs(G.to_f64(o)[0, h] - want) <= U.attention_bound(want, weight))
        assert np.all(np.abs(G.to_f64(lse)[0, h] - want_lse) <= U.LSE_BOUND)
        seen = [t for t in range(L + 5) if keeps((L + 4) // S, t // S)]
        want, want_lse, weight = orc.attend(G.bits_f64(q1)[0, h], k[seen, h], v[seen, h], scale)
        assert np.all(np.abs(G.to_f64(o1)[0, h] - want) <= U.attention_bound(want, weight))
        assert abs(float(lse1[0, h]) - want_lse) <= U.LSE_BOUND


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
def test_captured_and_on_two_streams_at_once(fmt):
    """A tree step in a graph, replayed beside eager steps on another stream with a workspace of its own: the same bits every time."""
    rng = np.random.default_rng(6)
    c = Case(fmt, 128, 64, [1000, 333, 0], 4, np.stack([random_tree(rng, 30) for _ in range(3)]))
    want, want_lse, _ = c.run(splits=3)
    cache, lens, par = c.pools.cache(_ints(c.table)), _ints(c.lens), _ints(c.parents)
    q, kd, vd = (G.to_dev(x) for x in (c.q, c.kd, c.vd))

    def buffers():
        return (torch.empty_like(q), torch.empty((3, 4, 30), dtype=torch.float32, device="cuda"),
                torch.empty(B.s2_attn_tree_workspace_bytes(3, 4, 30, 128, c.max_blocks * 64, 3), dtype=torch.uint8, device="cuda"))

    def step(o, lse, ws):
        B.s2_attn_tree_paged(c.params, cache, q, kd, vd, par, lens, o, lse, c.scale, ws, num_splits=3)

    one, two = buffers(), buffers()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(*one)
    for _ in range(4):
        one[0].zero_()
        two[0].zero_()
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            step(*two)
        torch.cuda.synchronize()
        for o, lse, _ in (one, two):
            assert np.array_equal(G.to_f64(o), want) and np.array_equal(G.to_f64(lse), want_lse)

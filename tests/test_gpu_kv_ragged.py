"""Rows written into a paged cache and read back for batches whose sequences differ in length, whatever the limit on a sequence's rows is given as."""

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
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()


class Batch:
    """Sequences with `new` tokens from `start` on, a table with blocks that are not held, rows of bf16 bits (and an index of them)."""

    def __init__(self, new, H, D, S, fmt, seed=0, first=0, extra=0, index=False, evicted=0.2):
        rng = np.random.default_rng([seed, len(new), H, D])
        self.new, self.nseq, self.H, self.D, self.S, self.fmt = np.asarray(new), len(new), H, D, S, fmt
        self.cu = first + np.concatenate([[0], np.cumsum(self.new)])
        self.start = rng.integers(0, 2 * S, size=self.nseq)
        blocks = int(-(-(self.start + self.new).max() // S))
        self.table = rng.permutation(self.nseq * H * blocks).reshape(self.nseq, H, blocks)
        self.table[rng.random(self.table.shape) < evicted] = -1
        self.pages = self.nseq * H * blocks
        self.items = int(self.cu[-1]) + extra
        self.index = rng.integers(-2, 42, size=self.items) if index else None
        self.bits = [synth.normal_bf16(rng, (40 if index else self.items, H, D)) for _ in "kv"]
        self.dev = [G.to_dev(x) for x in self.bits]

    def append(self, max_new, skipped=None, rows=None):
        pools = U.Pools(self.fmt, self.pages, self.S, self.D)
        k, v = (x if rows is None else x[:rows] for x in self.dev)
        B.s2_kv_append_paged(pools.cache(_ints(self.table)), k, v, _ints(self.cu), _ints(self.start), max_new,
                             rows=None if self.index is None else _ints(self.index), skipped=skipped)
        torch.cuda.synchronize()
        return pools

    def expect(self, max_new, rows=None):
        """What the pools hold afterwards (as U.Pools.host gives it), and the pairs left out."""
        there = len(self.bits[0]) if rows is None else rows
        pools = U.Pools(self.fmt, self.pages, self.S, self.D)
        out, left = [pools.host(w) for w in range(2)], 0
        held = [U.held_rows(x, self.fmt) for x in self.bits]
        heads = np.arange(self.H)
        for b in range(self.nseq):
            for i in range(min(int(self.new[b]), max_new)):
                item, pos = int(self.cu[b]) + i, int(self.start[b]) + i
                row = item if self.index is None else int(self.index[item]) if item < self.items else -1
                page = self.table[b, :, pos // self.S]
                ok = page >= 0 if 0 <= row < there else np.zeros(self.H, bool)
                left += int((~ok).sum())
                for w in range(2):
                    if ok.any():
                        out[w][0][page[ok], pos % self.S] = held[w][0][row, heads[ok]]
                        if held[w][1] is not None:
                            out[w][1][page[ok], pos % self.S] = held[w][1][row, heads[ok]]
        return out, left

    def check(self, max_new, rows=None):
        skipped = torch.full((1,), 7, dtype=torch.int32, device="cuda")
        want, left = self.expect(max_new, rows)
        for count in (skipped, None):
            pools = self.append(max_new, count, rows)
            for w in range(2):
                for a, b in zip(pools.host(w), want[w]):
                    assert (a is None and b is None) or np.array_equal(a, b)
        assert int(skipped.item()) - 7 == left
        return pools

    def check_read(self, pools, max_rows, margin=3):
        """Rows read back, against the pages; rows that belong to no sequence, or lie behind the limit, stay as they were."""
        outs = [torch.full((self.H, int(self.cu[-1]) + margin, self.D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        B.s2_kv_read_paged(pools.cache(_ints(self.table)), outs[0], outs[1], _ints(self.cu), _ints(self.start), max_rows)
        torch.cuda.synchronize()
        for w in range(2):
            held, byte = pools.host(w)
            want = np.full(outs[w].shape, 7.0)
            for b in range(self.nseq):
                n = min(int(self.new[b]), max_rows)
                if n == 0:
                    continue
                pos = self.start[b] + np.arange(n)
                page = self.table[b][:, pos // self.S]  # [head, row]
                rows = held[np.maximum(page, 0), pos % self.S]
                if self.fmt == "bf16":
                    value = synth.bf16_bits_to_f32(rows).astype(np.float64)
                else:
                    value = orc.mx_values(U.unpack(rows, self.fmt), byte[np.maximum(page, 0), pos % self.S], self.fmt)
                want[:, self.cu[b]:self.cu[b] + n] = np.where((page >= 0)[..., None], value, 0.0)
            assert np.array_equal(G.to_f64(outs[w]), want, equal_nan=True)


MOST = 2 ** 31 - 1


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("D, H", [(64, 3), (128, 5)])
@pytest.mark.parametrize("new", [[1] * 20 + [300], [300] + [1] * 20, [0, 0, 17, 0, 16, 15, 0, 1, 200, 0], [1, 0, 0, 1, 0, 1, 1, 0], [64, 64, 64], [5]])
def test_lengths_that_differ(fmt, D, H, new):
    """The limit as it is, larger, and smaller than the longest sequence."""
    batch = Batch(new, H, D, 16, fmt)
    most = max(new)
    # (with a counter the limit times the pairs has to fit it)
    for limit in (most, most + 1000, MOST // (H * len(new)), max(1, most // 2)):
        pools = batch.check(limit)
        batch.check_read(pools, limit)
    pools = batch.append(MOST)
    batch.check_read(pools, MOST)


@pytest.mark.parametrize("nseq", [63, 64, 65, 130, 4097])
@pytest.mark.parametrize("kind", ["ones", "some", "one"])
def test_many_sequences(nseq, kind):
    """More sequences than a wavefront has lanes, and than it finds in two steps; all with a token, most without, one with many."""
    rng = np.random.default_rng(nseq)
    new = {"ones": np.ones(nseq, int), "some": rng.integers(0, 9, size=nseq) * (rng.random(nseq) < 0.2), "one": np.zeros(nseq, int)}[kind]
    if kind != "ones":
        new[nseq * 2 // 3] = 150
    batch = Batch(new, 1, 64, 64, "bf16", seed=nseq)
    for limit in (int(max(new)), MOST // nseq):
        batch.check_read(batch.check(limit), limit)


@pytest.mark.parametrize("D", [64, 128])
def test_rows_and_items_that_are_not_there(D):
    """Items behind the last row or index are counted, however many a limit allows; numbering may begin behind 0."""
    for new, first in (([5, 0, 4, 91], 0), ([5, 0, 4, 91], 3), ([30, 40], 50), ([1, 1, 300, 1], 0)):
        batch = Batch(new, 2, D, 16, "mxfp8", first=first)
        for rows in (0, 1, 7, 20, len(batch.bits[0])):
            for limit in (3, 50, MOST // 8):
                batch.check(limit, rows=rows)
    for extra in (-30, 0, 9):
        batch = Batch([60, 1, 1, 40], 2, D, 16, "bf16", index=True, extra=extra)
        for limit in (7, 60, MOST // 8):
            batch.check(limit)
            batch.check(limit, rows=11)


def test_a_long_sequence_beside_short_ones():
    """64 sequences of 32 heads, one of 131072 tokens: what is held comes back, everything else is zeros."""
    D, S, H = 64, 128, 32
    lens = np.full(64, 2048)
    lens[37] = 131072
    cu = np.concatenate([[0], np.cumsum(lens)])
    table = torch.full((64, H, 1024), -1, dtype=torch.int32, device="cuda")
    table[37, 3, 1000], table[37, 31, 0], table[0, 0, 15], table[63, 9, 2] = 0, 1, 2, 3
    pools = U.Pools("bf16", 4, S, D)
    for w in range(2):
        pools.data[w].copy_(torch.randn(4, S, D, device="cuda"))
    outs = [torch.full((H, int(cu[-1]) + 1, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    B.s2_kv_read_paged(pools.cache(table), outs[0], outs[1], _ints(cu), _ints(0 * lens), 131072)
    torch.cuda.synchronize()
    for w in range(2):
        for page, (b, h, blk) in enumerate([(37, 3, 1000), (37, 31, 0), (0, 0, 15), (63, 9, 2)]):
            at = outs[w][h, cu[b] + blk * S:cu[b] + (blk + 1) * S]
            assert torch.equal(at, pools.data[w][page])
            at.zero_()
        assert not bool(outs[w][:, :-1].any()) and bool((outs[w][:, -1] == 7).all())


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_captured_with_lengths_that_change(fmt):
    """One graph for every step of a batch: the lengths are read when it runs."""
    nseq, H, D, S, most = 9, 3, 128, 16, 120
    batch = Batch([most] + [3] * (nseq - 1), H, D, S, fmt, evicted=0.0)
    pools, other = (U.Pools(fmt, batch.pages, S, D) for _ in range(2))
    table, cu, start = _ints(batch.table), _ints(batch.cu), _ints(batch.start)
    outs, plain = ([torch.zeros((H, batch.items, D), dtype=torch.bfloat16, device="cuda") for _ in "kv"] for _ in range(2))

    def both(pools, outs):
        B.s2_kv_append_paged(pools.cache(table), *batch.dev, cu, start, MOST)
        B.s2_kv_read_paged(pools.cache(table), *outs, cu, start, MOST)

    both(pools, outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(pools, outs)
    rng = np.random.default_rng(1)
    for _ in range(4):
        new = rng.integers(0, 4, size=nseq)
        new[rng.integers(nseq)] = 100
        start.copy_(_ints(np.minimum(batch.start, batch.table.shape[2] * S - new)))
        cu.copy_(_ints(np.concatenate([[0], np.cumsum(new)])))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in outs]
        both(other, plain)
        torch.cuda.synchronize()
        n = int(new.sum())
        for w in range(2):
            assert torch.equal(got[w][:, :n].view(torch.int16), plain[w][:, :n].view(torch.int16))

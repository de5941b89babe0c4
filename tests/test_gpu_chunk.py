"""Attention of a chunk of new tokens over a paged cache in bf16, 8 and 4 bits against the fp64 oracle on the values the cache stands for."""

import numpy as np
import pytest
import torch

from oracle import s2_oracle as orc
from paper_2407_17678_amd import binding as B
from paper_2407_17678_amd import synth
from tests import cache_util as U
from tests import gpu_util as G
from tests.test_gpu_tree import Case

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(np.asarray(x).tolist(), dtype=torch.int32, device="cuda")


class Chunk:
    """Sequences of `lens` tokens in a cache, of which the last `new` are the chunk; their rows lie from row `first` on, `after` rows beyond them are nobody's."""

    def __init__(self, fmt, D, S, lens, new, H, first=3, after=2, seed=0, start=None, spread=1.0, **kw):
        self.c = Case(fmt, D, S, lens, H, None, seed=seed, **kw)
        rng = np.random.default_rng([seed, D, S, H, 77])
        self.D, self.S, self.H, self.new, self.nseq = D, S, H, list(new), len(lens)
        self.start = [t - n for t, n in zip(lens, new)] if start is None else list(start)
        self.cu = first + np.concatenate([[0], np.cumsum(new)])
        self.rows = int(self.cu[-1]) + after
        self.q = synth.normal_bf16(rng, (self.rows, H, D))
        self.q = synth.round_to_bf16_bits(synth.bf16_bits_to_f32(self.q) * np.float32(spread))

    def run(self, splits=0, layout=None, strided=False, max_new=None, ws=True, in_place=False):
        c = self.c
        cache = c.pools.cache(_ints(c.table))
        missing = torch.full((1,), 5, dtype=torch.int32, device="cuda")
        most = max(self.new) if max_new is None else max_new
        n_bytes = B.s2_attn_chunk_workspace_bytes(c.nseq, self.H, most, self.rows, self.D, c.max_blocks * self.S, splits)
        work = torch.full((max(1, n_bytes),), 0xFF, dtype=torch.uint8, device="cuda") if ws else None
        q = G.to_dev(self.q)
        o = torch.full_like(q, 9.0)
        if strided:
            lay = lambda x: torch.zeros(self.H, self.rows, self.D + 8, dtype=torch.bfloat16, device="cuda")[..., :self.D].transpose(0, 1).copy_(x)  # noqa: E731
            q, o = lay(q), lay(o)
        if in_place:
            o = q
        lse = torch.full((self.H, self.rows), 9.0, dtype=torch.float32, device="cuda")
        f = B.s2_attn_chunk_paged_layout if layout else B.s2_attn_chunk_paged
        f(layout or c.params, cache, q, _ints(self.cu), _ints(self.start), o, lse, c.scale, work, most, missing=missing, num_splits=splits)
        torch.cuda.synchronize()
        return G.to_f64(o), G.to_f64(lse), int(missing.item()) - 5

    def oracle(self):
        c, cap = self.c, self.c.max_blocks * self.S
        o, lse, weight = np.full((self.rows, self.H, self.D), 9.0), np.full((self.H, self.rows), 9.0), np.zeros((self.rows, self.H, self.D))
        q, missing = G.bits_f64(self.q), 0
        for b in range(self.nseq):
            lo, hi = self.cu[b], self.cu[b + 1]
            rows = {(self.start[b] + i) // self.S for i in range(hi - lo) if 0 <= self.start[b] + i < cap}
            for h in range(self.H):
                keeps, held = c.keeps(h), lambda j: 0 <= c.table[b, h, j] < c.pages  # noqa: B023
                o[lo:hi, h], lse[h, lo:hi], weight[lo:hi, h] = orc.chunk_attention(q[lo:hi, h], c.k[b][h], c.v[b][h], self.start[b], keeps, self.S, c.scale,
                                                                                  cap, held)
                missing += sum(any(keeps(r, j) for r in rows if r >= j) and not held(j) for j in range(max(rows, default=-1) + 1))
        return o, lse, weight, missing

    def check(self, exact=None, **kw):
        o, lse, missing = self.run(**kw)
        want, want_lse, weight, want_missing = self.oracle()
        mine = np.zeros(self.rows, bool)
        mine[self.cu[0]:self.cu[-1]] = True
        if not kw.get("in_place"):
            assert np.all(o[~mine] == 9.0)
        assert np.all(lse[:, ~mine] == 9.0)
        want, weight, o = want[mine], weight[mine], o[mine]
        want_lse, lse = want_lse[:, mine], lse[:, mine]
        off = np.abs(o - want) - (exact or U.attention_bound)(want, weight)
        assert np.all(off <= 0), (float(off.max()), np.argwhere(off > 0)[:5], int((off > 0).sum()))
        gone = ~np.isfinite(want_lse)
        assert np.array_equal(~np.isfinite(lse), gone) and np.all(o[gone.T] == 0) and np.all(lse[gone] == -np.inf)
        assert np.all(np.abs(lse[~gone] - want_lse[~gone]) <= U.LSE_BOUND)
        assert missing == want_missing, (missing, want_missing)
        return o, lse


FORMATS = ["bf16", "mxfp8", "mxfp4"]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D, S", [(128, 64), (64, 64), (128, 16), (64, 16), (128, 32), (64, 32), (128, 128), (64, 128)])
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_few_rows(fmt, D, S, splits):
    Chunk(fmt, D, S, [1, S, S + 1, 3 * S + 7, 5 * S - 3], [1, 7, 16, 33, 0], 2, seed=splits).check(splits=splits)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D, S", [(128, 64), (64, 64), (128, 16), (64, 16), (128, 32), (64, 32), (128, 128), (64, 128)])
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_many_rows(fmt, D, S, splits):
    Chunk(fmt, D, S, [130, 270, 2, 401], [130, 65, 1, 150], 2, seed=splits).check(splits=splits)


@pytest.mark.parametrize("new", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257])
def test_a_single_sequence_of_any_length(new):
    for before in (0, 61):
        Chunk("mxfp8", 64, 32, [before + new], [new], 1, local=2, stride=3, seed=new).check()


@pytest.mark.parametrize("new", [[1] * 40 + [300], [0, 0, 5, 0], [70] * 6, [3, 0, 260, 1, 1]])
def test_ragged_batches(new):
    lens = [n + 13 * i % 97 for i, n in enumerate(new)]
    for S in (16, 64):
        Chunk("bf16", 64, S, lens, new, 2, local=1, stride=4, seed=S).check()
        Chunk("mxfp4", 128, S, lens, new, 1, first=0, after=0, local=3, stride=2, seed=S).check(max_new=10 ** 6)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("new", [40, 140])
def test_patterns_and_strides(fmt, new):
    Chunk(fmt, 128, 16, [200, 150], [new, 20], 3, local=1, stride=4, window=6, base=3).check()
    Chunk(fmt, 64, 64, [300, 164], [new, 9], 2, dense=1).check(strided=True)
    Chunk(fmt, 128, 32, [300, 197], [new, 100], 2, local=3, stride=0, gap=16).check(strided=True, splits=2)
    Chunk(fmt, 64, 128, [500, 197], [new, 100], 2, local=1, stride=2).check(in_place=True)


@pytest.mark.parametrize("S, new", [(16, 24), (16, 150), (64, 24), (64, 150), (128, 150)])
def test_blocks_that_are_not_held(S, new):
    lens = [5 * S + 3 + new, new + 2]
    c = Chunk("mxfp8", 64, S, lens, [new, new], 2, local=2, stride=3, seed=S, evict=[(0, 0, 5), (0, 1, 4), (0, 0, 0), (1, 0, 0), (1, 1, 0), (1, 1, 1)][:5 if new < S else 6])
    c.check()
    c.check(splits=4)
    mask = np.tril(np.ones((16, 16), bool))
    mask = np.stack([mask & (np.random.default_rng(h).random((16, 16)) < 0.4) | np.eye(16, dtype=bool) for h in range(2)])
    rp, ci, _, _ = orc.compressed_layout(mask)
    layout = B.s2_layout_from_csr(2, 16, S, rp, ci)
    c = Chunk("bf16", 64, S, [min(16 * S, 5 * S + 3 + new), new + 2], [new, new], 2, seed=S, mask=mask, max_blocks=16,
              evict=[(0, 0, 3), (0, 1, 0), (0, 0, 1), (1, 0, 0), (1, 1, 1)])
    c.check(layout=layout)
    c.check(layout=layout, splits=3)


def test_every_block_of_a_row_missing():
    for new in (5, 130):
        c = Chunk("mxfp4", 128, 64, [new], [new], 1, local=1, stride=0, evict=[(0, 0, j) for j in range(-(-new // 64))])
        o, lse = c.check()
        assert np.all(o == 0) and np.all(lse == -np.inf)


@pytest.mark.parametrize("S", [16, 32, 64, 128])
@pytest.mark.parametrize("new", [30, 200])
def test_layouts(S, new):
    nb = 24
    params = B.layout_params(3, nb, S, 2, 5, 1)
    lens = [min(nb * S, 7 * S + 5 + new), new]
    for fmt in FORMATS:
        c = Chunk(fmt, 128, S, lens, [new, new], 3, local=2, stride=5, base=1, max_blocks=min(nb, -(-max(lens) // S)))
        a = c.run()
        b = c.run(layout=B.s2_layout_build(params))
        c.check(layout=B.s2_layout_build(params))
        assert np.abs(a[0] - b[0])[c.cu[0]:c.cu[-1]].max() < 0.1 and a[2] == b[2]


def test_positions_that_the_cache_has_no_room_for():
    for new in (20, 140):
        for start in (-7, 4 * 32 - 10, 4 * 32, 2 ** 31 - 1, -2 ** 31):
            lens = [4 * 32, 50 + new]
            c = Chunk("bf16", 64, 32, [min(128, x) for x in lens], [new, new], 2, start=[start, 5], max_blocks=4, local=2, stride=2)
            # (all tokens of the cache exist: a row attends those up to its own position)
            c.c.k = [[np.concatenate([k, np.zeros((max(0, 128 - len(k)), 64))]) for k in ks] for ks in c.c.k]
            c.c.v = [[np.concatenate([v, np.zeros((max(0, 128 - len(v)), 64))]) for v in vs] for vs in c.c.v]
            c.check()


def test_offsets_that_leave_the_tensors_or_go_back():
    """Rows outside the tensors are not touched, whatever the array holds; of rows that a sequence has no room for in max_new nothing is written."""
    c = Chunk("bf16", 64, 32, [40, 40, 40], [30, 30, 30], 1)
    for cu in ([-20, 10, 40, 200], [5, 3, 60, 61], [80, 200, 300, 400], [2 ** 31 - 1] * 4, [-2 ** 31, 0, 2 ** 31 - 1, 2 ** 31 - 1]):
        for most in (30, 90):
            q = G.to_dev(c.q)
            o = torch.full_like(q, 9.0)
            ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
            B.s2_attn_chunk_paged(c.c.params, c.c.pools.cache(_ints(c.c.table)), q, _ints(cu), _ints(c.start), o, None, c.c.scale, ws, most)
            torch.cuda.synchronize()
            owned = np.zeros(c.rows, bool)
            for lo, hi in zip(cu, cu[1:]):
                owned[max(0, lo):max(0, min(hi, lo + most))] = True
            if sorted(cu) == list(cu):
                assert np.all(G.to_f64(o)[~owned] == 9.0) and np.all(G.to_f64(o)[owned] != 9.0)


@pytest.mark.parametrize("new", [1, 6, 50])
def test_as_many_decode_steps(new):
    """A chunk's last row is the decode step at its position, up to both roundings; one row is one step."""
    for fmt in FORMATS:
        c = Chunk(fmt, 128, 64, [200, 333], [new, new], 2, seed=new)
        o, _, _ = c.run()
        case, last = c.c, c.cu[1:] - 1
        q = G.to_dev(c.q)[torch.tensor(last)].contiguous()
        od = torch.empty_like(q)
        ws = torch.empty(B.s2_attn_tree_workspace_bytes(2, 2, 1, 128, case.max_blocks * 64), dtype=torch.uint8, device="cuda")
        B.s2_attn_decode_paged_cache(case.params, case.pools.cache(_ints(case.table)), q, _ints([200, 333]), od, None, case.scale, ws)
        _, _, weight, _ = c.oracle()
        got, want = o[last], G.to_f64(od)
        assert np.all(np.abs(got - want) <= 2.0 ** -7 * np.abs(want) * (1 + 2.0 ** -7) + 2.0 ** -12 * weight[last])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("new", [1, 14, 30, 50, 64])
def test_probabilities_of_few_rows_keep_16_bits(fmt, new):
    """As in tests/test_gpu_cache_precision.py: a score is off by D 2^-23 of the sum of its products' magnitudes and by 2^-21 of itself and 2^-21; p_j to 16 bits;
    sums of n values n 2^-23."""
    c = Chunk(fmt, 64, 16, [new + 3, new + 70], [new, new], 3, local=3, seed=new)
    q = np.abs(G.bits_f64(c.q))
    most = max((q[lo:hi, h] @ np.abs(c.c.k[b][h]).T).max() for b, (lo, hi) in enumerate(zip(c.cu, c.cu[1:])) for h in range(3)) * c.c.scale
    eps = 2 * (64 * 2.0 ** -23 * most + 2.0 ** -21 * (most + 1)) + 2.0 ** -16 + 134 * 2.0 ** -23
    assert eps < 2.0 ** -10, eps
    c.check(exact=lambda want, weight: 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -7) + eps * weight)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("S", [16, 64])
@pytest.mark.parametrize("new", [20, 150])
def test_what_is_not_attended_stays_out(fmt, S, new):
    """NaN and infinities in tokens after a row, in blocks that its block row drops, and behind the sequence's end."""
    lens = [4 * S + 5 + new]
    c = Chunk(fmt, 64, S, lens, [new], 2, local=1, stride=3, seed=S)
    clean, clean_lse, _ = c.run()
    case, start = c.c, c.start[0]
    bad = [start + new - 1, start + new // 2, 2 * S + 1]
    values = [np.nan, np.inf, -np.inf]
    for which, rows in ((0, case.k), (1, case.v)):
        for h in range(2):
            for t, x in zip(bad, values):
                held = torch.full((64,), float("nan") if fmt == "bf16" else 0x7F, dtype=torch.bfloat16 if fmt == "bf16" else torch.uint8)
                if fmt == "bf16" and which == 1:
                    held = torch.full((64,), x, dtype=torch.bfloat16)
                case.pools.data[which][case.table[0, h, t // S], t % S] = held.cuda()
                rows[0][h] = rows[0][h].copy()
                rows[0][h][t] = np.nan if fmt != "bf16" or which == 0 else x
    o, lse, _ = c.run()
    touched = 0
    for h in range(2):
        keeps = case.keeps(h)
        for i in range(new):
            at = start + i
            sees = [t for t in bad if t <= at and keeps(at // S, t // S)]
            row = c.cu[0] + i
            if not sees:
                assert np.array_equal(o[row, h], clean[row, h]) and lse[h, row] == clean_lse[h, row], (h, i)
                touched += 1
            else:
                assert np.all(np.isnan(o[row, h])), (h, i, sees)
    assert 0 < touched < 2 * new


@pytest.mark.parametrize("S, new", [(16, 20), (16, 150), (64, 20), (64, 150)])
def test_infinities_of_values_that_are_attended(S, new):
    """V alone: an infinity reaches the rows that attend its token, a NaN or both signs are NaN."""
    c = Chunk("bf16", 64, S, [2 * S + new], [new], 1, local=2, stride=3, seed=S)
    case, start = c.c, c.start[0]
    clean, _, _ = c.run()
    spots = [(start + 3, 0, np.inf), (start + 9, 1, -np.inf), (start + 5, 2, np.inf), (start + 12, 2, -np.inf), (start + 15, 3, np.nan), (0, 4, np.inf)]
    for t, f, x in spots:
        case.pools.data[1][case.table[0, 0, t // S], t % S, f] = x
    o, _, _ = c.run()
    keeps = case.keeps(0)
    for i in range(new):
        at, row = start + i, c.cu[0] + i
        for f in range(64):
            here = [x for t, g, x in spots if g == f and t <= at and keeps(at // S, t // S)]
            got = o[row, 0, f]
            if not here:
                assert got == clean[row, 0, f], (i, f)
            elif any(np.isnan(here)) or len(set(here)) > 1:
                assert np.isnan(got), (i, f)
            else:
                assert got == here[0], (i, f, got)


def test_scores_far_apart_and_of_one_value():
    for new in (20, 140):
        Chunk("bf16", 64, 32, [new + 40], [new], 2, spread=30.0, seed=1, local=2).check(exact=lambda w, a: U.attention_bound(w, a) + 2.0 ** -6 * a)
        c = Chunk("mxfp8", 64, 32, [new + 40], [new], 2, spread=0.0, seed=2, local=2)
        o, lse = c.check()


def test_splits_and_repeats_agree():
    for new in (40, 200):
        c = Chunk("mxfp8", 128, 64, [1500, 700], [new, new - 9], 3, local=8, stride=4)
        first = c.run()
        again = c.run()
        assert all(np.array_equal(a, b) for a, b in zip(first[:2], again[:2]))
        _, _, weight, _ = c.oracle()
        for splits in (1, 2, 7, 64):
            got = c.run(splits=splits)
            lo, hi = c.cu[0], c.cu[-1]
            assert np.all(np.abs(got[0] - first[0])[lo:hi] <= (2.0 ** -7 * np.abs(first[0]) + 2.0 ** -8 * weight)[lo:hi])
        no_room = c.run(ws=False)
        one = c.run(splits=1)
        assert np.array_equal(no_room[0], one[0])


def test_another_stream_and_two_at_once():
    a, b = (Chunk("mxfp8", 128, 64, [900], [140], 4, seed=s) for s in (1, 2))
    want = [x.run()[0] for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in "ab"]
    made = []
    for c, st in zip((a, b), streams):
        case = c.c
        q = G.to_dev(c.q)
        t = dict(cache=case.pools.cache(_ints(case.table)), q=q, o=torch.full_like(q, 9.0), cu=_ints(c.cu), start=_ints(c.start),
                 ws=torch.empty(B.s2_attn_chunk_workspace_bytes(1, 4, 140, c.rows, 128, case.max_blocks * 64), dtype=torch.uint8, device="cuda"))
        made.append(t)
    torch.cuda.synchronize()
    for _ in range(20):
        for c, st, t in zip((a, b), streams, made):
            B.s2_attn_chunk_paged(c.c.params, t["cache"], t["q"], t["cu"], t["start"], t["o"], None, c.c.scale, t["ws"], 140, stream=st)
    torch.cuda.synchronize()
    for t, w in zip(made, want):
        assert np.array_equal(G.to_f64(t["o"]), w)

"""Block tables planned on the GPU against the oracle that keeps them an entry at a time: whole numbers, equal to the last one."""

import numpy as np
import pytest
import torch

from oracle import s2_oracle as orc
from paper_2407_17678_amd import binding as B

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int64).tolist(), dtype=torch.int32, device="cuda")


def rule(local, stride, window=0, dense=0, base=0):
    """attended(h, row, j) of section 4.2's rule, by a scan over rows."""
    far = local + window + max(stride, 1) + 2
    if dense:
        return lambda h, row, j: True
    return lambda h, row, j: any(orc.block_predicate(r, j, orc.head_offset(base + h, stride), local, stride, window) for r in range(max(row, j), max(row, j) + far))


class Plan:
    def __init__(self, S, H, table, lens, new, ring, state, params, attended, query_from=None, rows=None):
        self.S, self.table, self.lens, self.new, self.ring, self.state = S, np.array(table, dtype=np.int64), list(lens), list(new), np.array(ring), list(state)
        self.params, self.attended, self.query_from = params, attended, query_from
        total = int(np.maximum(np.array(new, dtype=np.int64), 0).sum())
        self.rows = total + 3 if rows is None else rows

    def run(self, in_place=False, layout=None, full=True, alias=None, stream=None):
        n = len(self.lens)
        t = dict(table=_ints(self.table), ring=_ints(self.ring), state=_ints(self.state), lens=_ints(self.lens), new=_ints(self.new))
        out = t if in_place else dict(table=torch.full_like(t["table"], 77), ring=torch.full_like(t["ring"], 77), state=torch.full_like(t["state"], 77))
        filled = lambda k: torch.full((k,), 77, dtype=torch.int32, device="cuda")  # noqa: E731
        more = dict(cu_new=filled(n + 1), positions=filled(max(1, self.rows)), seq_lens=t[alias] if alias else filled(n), short=filled(1)) if full else {}
        ws = torch.full((B.s2_kv_plan_workspace_bytes(n, self.table.shape[1]),), 0xFF, dtype=torch.uint8, device="cuda")
        f = B.s2_kv_plan_paged_layout if layout else B.s2_kv_plan_paged
        f(layout or self.params, t["table"], t["lens"], t["new"], t["ring"], t["state"], out["table"], out["ring"], out["state"], ws,
          query_from=None if self.query_from is None else _ints(self.query_from), stream=stream, **more)
        torch.cuda.synchronize()
        got = {k: out[k].cpu().numpy() for k in ("table", "ring", "state")}
        if not in_place:  # what was given is as it was
            assert np.array_equal(t["table"].cpu().numpy(), self.table) and np.array_equal(t["ring"].cpu().numpy(), self.ring)
        got.update({k: v.cpu().numpy() for k, v in more.items()})
        return got

    def oracle(self):
        return orc.plan_tables(self.table, self.lens, self.new, self.ring, self.state, self.attended, self.S, self.query_from)

    def check(self, **kw):
        got, want = self.run(**kw), self.oracle()
        for k in ("table", "ring", "state"):
            assert np.array_equal(got[k], np.array(want[k])), (k, got[k], want[k])
        if "cu_new" in got:
            assert np.array_equal(got["cu_new"], want["cu_new"]) and np.array_equal(got["seq_lens"], want["seq_lens"])
            assert int(got["short"][0]) - 77 == want["short"]
            p = np.full(max(1, self.rows), 77)
            n = min(len(want["positions"]), self.rows)
            p[:n] = want["positions"][:n]
            assert np.array_equal(got["positions"], p)
        return got


def random_plan(seed, S, H, nseq, max_blocks, pages, local=2, stride=3, window=0, dense=0, base=0, with_from=False):
    rng = np.random.default_rng([seed, S, H, nseq])
    cap = S * max_blocks
    lens = rng.integers(0, cap + 1, nseq)
    lens[0] = 0
    new = np.where(rng.random(nseq) < 0.2, -1, np.minimum(rng.integers(0, cap // 2 + 1, nseq), cap - lens))
    order = rng.permutation(pages)
    table = np.full((nseq, H, max_blocks), -1)
    used = 0
    for b in range(nseq):
        for h in range(H):
            for j in range(max_blocks):
                if j * S < lens[b] and rng.random() < 0.6 and used < pages:
                    table[b, h, j] = order[used]
                    used += 1
    free = order[used:]
    first = int(rng.integers(0, pages))
    ring = np.full(pages, -5)
    ring[(first + np.arange(len(free))) % pages] = free
    q = np.clip(lens + rng.integers(-S, 2 * S, nseq), 0, None) if with_from else None
    params = B.layout_params(H, 1, S, local, stride, base, window, dense)
    return Plan(S, H, table, lens, new, ring, [first, len(free)], params, rule(local, stride, window, dense, base), q)


@pytest.mark.parametrize("S", [16, 32, 64, 128])
@pytest.mark.parametrize("nseq, H, max_blocks, pages", [(1, 1, 1, 1), (3, 2, 5, 40), (7, 5, 67, 3000), (2, 3, 130, 500), (300, 2, 3, 900)])
@pytest.mark.parametrize("in_place", [False, True])
def test_random_tables(S, nseq, H, max_blocks, pages, in_place):
    for seed in range(3):
        random_plan(seed, S, H, nseq, max_blocks, pages, with_from=seed == 2).check(in_place=in_place)


@pytest.mark.parametrize("rule_", [dict(local=1, stride=4, window=6, base=3), dict(dense=1), dict(local=3, stride=0), dict(local=1, stride=1), dict(local=40, stride=7)])
def test_patterns(rule_):
    for seed in range(2):
        random_plan(seed, 32, 3, 5, 70, 900, **rule_).check()


def test_pages_run_short_and_the_ring_goes_round():
    for first, count in ((0, 0), (5, 1), (9, 3), (3, 10)):
        ring = np.arange(10) * 1
        p = Plan(16, 1, np.full((2, 1, 8), -1), [0, 5], [40, 30], ring, [first, count], B.layout_params(1, 1, 16, 8, 0), rule(8, 0))
        p.check()
        p.check(in_place=True)


def test_blocks_that_begin_before_the_new_tokens_are_not_made_up():
    """A partly written block that is not held stays so, as does one that was given up."""
    table = np.array([[[-1, -1, 3, -1]]])
    p = Plan(16, 1, table, [40], [20], [0, 1, 2, 3], [0, 3], B.layout_params(1, 1, 16, 4, 0), rule(4, 0))
    got = p.check()
    assert got["table"].tolist() == [[[-1, -1, 3, 0]]]
    p = Plan(16, 1, np.array([[[-1, -1, -7, -1]]]), [40], [20], [0, 1, 2, 3], [0, 4], p.params, p.attended)
    assert p.check()["table"].tolist() == [[[-1, -1, -7, 0]]]


def test_entries_that_are_no_page():
    """Not held: nothing of them goes to the ring; where new tokens come a page takes their place."""
    table = np.array([[[4, 9, -1, 2 ** 31 - 1], [-2 ** 31, 3, 6, 5]]])
    for lens, new in ((0, 64), (0, -1), (64, 0), (33, 9)):
        Plan(16, 2, table, [lens], [new], [0, 1, 2, 0, 0, 0], [0, 3], B.layout_params(2, 1, 16, 2, 0), rule(2, 0)).check()


def test_numbers_that_are_out_of_range():
    big = 2 ** 31 - 1
    for lens, new, q in (([-5, 100, big], [3, 200, big], None), ([big, 0, -2 ** 31], [big, -2 ** 31, 5], [big, -2 ** 31, big]), ([64, 64, 0], [0, 5, 64], [64, 63, 70])):
        p = Plan(16, 2, np.full((3, 2, 4), -1), lens, new, np.arange(30), [0, 30], B.layout_params(2, 1, 16, 2, 3), rule(2, 3), q, rows=6)
        got = p.run()
        with_room = orc.plan_tables(p.table, lens, [min(x, 64) for x in new], p.ring, p.state, p.attended, 16, q)
        assert np.array_equal(got["table"], with_room["table"]) and np.array_equal(got["state"], with_room["state"])
        assert np.array_equal(got["seq_lens"], with_room["seq_lens"])
        cu = np.minimum(np.concatenate([[0], np.cumsum(np.maximum(np.array(new, dtype=np.int64), 0))]), big)
        assert np.array_equal(got["cu_new"], cu)
    for state in ([-1, 5], [30, 31], [7, -3], [big, big]):
        Plan(16, 1, np.full((1, 1, 4), -1), [0], [50], np.arange(30), state, B.layout_params(1, 1, 16, 4, 0), rule(4, 0)).check()


def test_a_page_that_two_entries_name_does_not_overrun_the_ring():
    p = Plan(16, 1, np.zeros((3, 1, 4)), [64, 64, 64], [-1, -1, -1], np.arange(4), [1, 2], B.layout_params(1, 1, 16, 4, 0), rule(4, 0))
    assert p.check()["state"].tolist() == [1, 4]


def test_layouts():
    nb, H, S = 40, 3, 16
    params = B.layout_params(H, nb, S, 2, 5, 1)
    layout = B.s2_layout_build(params)
    mask = np.tril(np.random.default_rng(3).random((H, nb, nb)) < 0.15) | np.eye(nb, dtype=bool)
    rp, ci, _, _ = orc.compressed_layout(mask)
    custom = B.s2_layout_from_csr(H, nb, S, rp, ci)
    by_mask = lambda h, row, j: bool(mask[h, row:, j].any())  # noqa: E731
    m = orc.block_mask(H, nb, 2, 5, 1)
    for seed in range(3):
        p = random_plan(seed, S, H, 4, nb - seed, 700, local=2, stride=5, base=1)
        p.attended = lambda h, row, j: bool(m[h, row:, j].any())
        p.check(layout=layout)
        p.attended = by_mask
        p.check(layout=custom)
        p.check(layout=custom, in_place=True)
    with pytest.raises(B.S2Error, match="SHAPE"):
        random_plan(0, S, H, 2, nb + 1, 100).run(layout=layout)


def test_only_the_tables():
    random_plan(5, 64, 4, 6, 20, 600).check(full=False)
    random_plan(5, 64, 4, 6, 20, 600).check(full=False, in_place=True)


@pytest.mark.parametrize("alias", ["lens", "new"])
def test_lengths_in_place(alias):
    p = random_plan(6, 64, 4, 300, 5, 2000)
    got, want = p.run(alias=alias), p.oracle()
    assert np.array_equal(got["seq_lens"], want["seq_lens"]) and np.array_equal(got["table"], want["table"]) and np.array_equal(got["cu_new"], want["cu_new"])


def test_many_heads_and_sequences():
    """More (sequence, head) pairs than wavefronts of a launch: each takes several."""
    p = random_plan(7, 16, 64, 130, 2, 9000)
    p.check()
    p.check(in_place=True)


def test_a_row_of_steps():
    """Prompts in chunks, then single tokens, in place: a head holds what s2_kv_resident_blocks names, and pages are neither lost nor doubled."""
    S, H, MB, P = 16, 3, 60, 160
    params = B.layout_params(H, 1, S, 2, 4)
    t = dict(table=torch.full((2, H, MB), -1, dtype=torch.int32, device="cuda"), ring=torch.arange(P, dtype=torch.int32, device="cuda"), state=_ints([0, P]),
             lens=_ints([0, 0]))
    ws = torch.empty(B.s2_kv_plan_workspace_bytes(2, H), dtype=torch.uint8, device="cuda")
    short = _ints([0])
    lens = np.zeros(2, dtype=np.int64)
    for new in [(50, 17), (100, 33)] + [(1, 1)] * 40 + [(300, 5), (-1, 1), (1, 0), (40, 200)] + [(1, 1)] * 20 + [(-1, -1)]:
        B.s2_kv_plan_paged(params, t["table"], t["lens"], _ints(new), t["ring"], t["state"], t["table"], t["ring"], t["state"], ws, seq_lens=t["lens"], short=short)
        before, lens = lens, np.where(np.array(new) < 0, 0, lens + np.array(new))
        table, (first, count) = t["table"].cpu().numpy(), t["state"].tolist()
        assert t["lens"].tolist() == lens.tolist() and short.tolist() == [0]
        held = table[table >= 0]
        free = t["ring"].cpu().numpy()[(first + np.arange(count)) % P]
        assert sorted(np.concatenate([held, free]).tolist()) == list(range(P))
        for b in range(2):
            for h in range(H):
                here = np.nonzero(table[b, h] >= 0)[0].tolist()
                if new[b] < 0:
                    assert here == []
                    continue
                wanted = [j for j in B.s2_kv_resident_blocks(params, h, int(before[b]) + 1) if j * S < lens[b]]
                assert here == sorted(set(wanted) | set(range(int(before[b]) // S, -(-int(lens[b]) // S))))


def test_another_stream():
    p = random_plan(8, 64, 8, 20, 30, 6000)
    st = torch.cuda.Stream()
    p.check(stream=st)

"""Pins of the oracle's block tables, of its norm and rotation and of its chunk attention: hand-worked values, closed forms, differences, the decode oracle."""

import numpy as np
import pytest

from oracle import s2_oracle as orc


def test_a_plan_by_hand():
    # one head that attends its own block and block 0; blocks of 4 tokens, ring of 6 pages from entry 4 on with 3 free ones: pages 9, 8, 7 of 10
    attended = lambda h, row, j: j in (0, row) or j > row  # noqa: E731
    table = [[[3, 5, -1, -1, 2]], [[0, -1, -1, -1, -1]], [[1, 4, 6, -1, -1]]]
    ring = [7, 90, 91, 92, 9, 8, 93, 94, 95, 96]
    got = orc.plan_tables(table, [6, 0, 10], [3, 5, -1], ring, [4, 2], attended, 4)
    # sequence 0: blocks 0..2 of 9 tokens, of which 1 is the row that the queries begin in; page 2 of block 4 is given up, block 2 takes page 9
    # sequence 1: block 0 is held, block 1 takes page 8; sequence 2 is over: pages 1, 4, 6 go
    assert got["table"].tolist() == [[[3, 5, 9, -1, -1]], [[0, 8, -1, -1, -1]], [[-1] * 5]]
    assert got["ring"].tolist() == [7, 90, 91, 92, 9, 8, 2, 1, 4, 6] and got["state"] == [6, 4]
    assert got["cu_new"] == [0, 3, 8, 8] and got["positions"] == [6, 7, 8, 0, 1, 2, 3, 4] and got["seq_lens"] == [9, 5, 0] and got["short"] == 0


def test_a_plan_without_pages_by_hand():
    got = orc.plan_tables([[[-1, -1, -1]]], [5], [7], [0, 1], [1, 1], lambda h, row, j: True, 4, query_from=[11])
    # block 0 begins before the 5 tokens, so does block 1 (tokens 4 .. 7): what they held is gone; block 2 takes the page at entry 1
    assert got["table"].tolist() == [[[-1, -1, 1]]] and got["state"] == [0, 0] and got["short"] == 0 and got["seq_lens"] == [12]
    got = orc.plan_tables([[[-1, -1, -1]]], [0], [12], [5, 6, 7], [2, 2], lambda h, row, j: True, 4)
    assert got["table"].tolist() == [[[7, 5, -1]]] and got["state"] == [1, 0] and got["short"] == 1


@pytest.mark.parametrize("seed", range(4))
def test_pages_are_neither_lost_nor_shared(seed):
    rng = np.random.default_rng(seed)
    S, H, n, MB, P = 4, 2, 3, 8, 40
    attended = lambda h, row, j: any(orc.block_predicate(r, j, orc.head_offset(h, 3), 2, 3, 0) for r in range(max(row, j), max(row, j) + 8))  # noqa: E731
    table, ring, state = np.full((n, H, MB), -1), rng.permutation(P), [int(rng.integers(P)), P]
    lens = [0] * n
    for _ in range(12):
        new = [int(rng.integers(0, 7)) if rng.random() > 0.15 else -1 for _ in range(n)]
        got = orc.plan_tables(table, lens, new, ring, state, attended, S)
        table, ring, state, lens = got["table"], got["ring"], got["state"], got["seq_lens"]
        held = table[table >= 0].tolist()
        free = [int(ring[(state[0] + i) % P]) for i in range(state[1])]
        assert sorted(held + free) == list(range(P)) and got["short"] == 0
        for b in range(n):
            for h in range(H):
                for j in range(MB):
                    if j * S >= lens[b]:
                        assert table[b, h, j] == -1
                    elif new[b] > 0 and orc.block_predicate((lens[b] - 1) // S, j, orc.head_offset(h, 3), 2, 3, 0):
                        assert table[b, h, j] >= 0  # (what the step's last query reads is there)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_by_hand(interleaved):
    x = np.arange(1.0, 7.0)[None, :]
    got = orc.rotate_pairs(x, [1], [np.pi / 2, np.pi], interleaved)
    # a quarter turn takes (a, b) to (-b, a), a half turn to (-a, -b); features 4 and 5 stay
    want = [-2, 1, -3, -4, 5, 6] if interleaved else [-3, -2, 1, -4, 5, 6]
    assert np.allclose(got, [want], atol=1e-12)
    assert np.allclose(orc.rotate_pairs(got, [1], [np.pi / 2, np.pi], interleaved, back=True), x, atol=1e-12)


def test_norm_by_hand():
    x = np.array([[[[3.0, -4.0, 0.0, 0.0]]]])
    got = orc.qk_norm_rope(x, [2.0, 1.0, 5.0, 5.0], [[0]], [0.3], 0.0)
    assert np.allclose(got, [[[[2.4, -1.6, 0, 0]]]])  # (the root of the mean square is 2.5)
    assert np.allclose(orc.qk_norm_rope(x, [2.0, 1.0, 5.0, 5.0], [[0]], [0.3], 18.75), got / 2)
    assert np.array_equal(orc.qk_norm_rope(x, None, [[0]], [0.3], 0.0), x)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("with_weight", [False, True])
def test_scores_depend_on_the_distance_alone(interleaved, with_weight):
    rng = np.random.default_rng(2)
    q, k, w = rng.normal(size=(1, 1, 1, 8)), rng.normal(size=(1, 1, 1, 8)), rng.normal(size=8) if with_weight else None
    at = lambda x, p: orc.qk_norm_rope(x, w, [[p]], [1.0, 0.3, 0.01], 1e-6, interleaved)[0, 0, 0]  # noqa: E731
    for p in (5, 1000):
        assert np.isclose(at(q, 17) @ at(k, 4), at(q, 17 + p) @ at(k, 4 + p), rtol=1e-9)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("with_weight", [False, True])
def test_its_gradient_against_differences(interleaved, with_weight):
    rng = np.random.default_rng(3)
    x, g, pos, freq = rng.normal(size=(2, 2, 3, 8)), rng.normal(size=(2, 2, 3, 8)), rng.integers(0, 50, (2, 3)), [1.0, 0.2, 0.05]
    w = rng.normal(size=8) if with_weight else None
    f = lambda x_, w_: float((g * orc.qk_norm_rope(x_, w_, pos, freq, 1e-3, interleaved)).sum())  # noqa: E731
    dx, dw = orc.qk_norm_rope_backward(x, w, pos, freq, 1e-3, g, interleaved)
    # central differences of step e: off by e^2 f''' / 6 and 2^-52 |f| / e, both below 1e-7 of these sizes at e = 1e-5
    e = 1e-5
    for i in rng.permutation(x.size)[:40]:
        y = x.copy()
        y.flat[i] += e
        z = x.copy()
        z.flat[i] -= e
        assert abs((f(y, w) - f(z, w)) / (2 * e) - dx.flat[i]) < 1e-7
    if not with_weight:
        assert dw is None
        return
    for i in range(8):
        d = np.eye(8)[i] * e
        assert abs((f(x, w + d) - f(x, w - d)) / (2 * e) - dw[i]) < 1e-7


def test_a_chunk_is_as_many_decode_steps():
    rng = np.random.default_rng(4)
    S, T, start, D, cap = 4, 9, 6, 8, 16
    q, k, v = rng.normal(size=(T, D)), rng.normal(size=(cap, D)), rng.normal(size=(cap, D))
    for h in (0, 1, 2):
        keeps = lambda r, c: orc.block_predicate(r, c, orc.head_offset(h, 3), 2, 3, 0)  # noqa: E731
        o, lse, weight = orc.chunk_attention(q, k, v, start, keeps, S, 0.4, cap)
        for i in range(T):
            want = orc.decode_row(q[i], k, v, start + i + 1, h, S, 2, 3, 0.4)
            want_o, want_lse = want[0], want[1]
            assert np.allclose(o[i], want_o, atol=1e-13) and np.isclose(lse[i], want_lse)
            assert np.all(weight[i] >= np.abs(o[i]) - 1e-13)


def test_a_chunk_of_rows_that_are_nowhere_or_see_nothing():
    q, kv = np.ones((4, 8)), np.ones((8, 8))
    o, lse, _ = orc.chunk_attention(q, kv, kv, -2, lambda r, c: True, 4, 0.5, 8)
    assert np.all(o[:2] == 0) and np.all(np.isinf(lse[:2])) and np.allclose(o[2:], 1)
    o, lse, _ = orc.chunk_attention(q, kv, kv, 6, lambda r, c: True, 4, 0.5, 8)
    assert np.allclose(o[:2], 1) and np.all(o[2:] == 0) and np.all(lse[2:] == -np.inf)
    o, lse, _ = orc.chunk_attention(q, kv, kv, 2, lambda r, c: c == r, 4, 0.5, 8, resident=lambda c: c == 1)
    assert np.all(o[:2] == 0) and np.all(lse[:2] == -np.inf) and np.isclose(lse[2], 4.0) and np.isclose(lse[3], 4.0 + np.log(2))

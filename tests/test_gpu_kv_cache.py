"""Rows written into a paged cache and read back: codes, scales and values bit for bit as the oracle's search gives them, everything else left as it was."""

import numpy as np
import pytest
import torch

from oracle import s2_oracle as orc
from paper_2407_17678_amd import binding as B
from paper_2407_17678_amd import synth
from tests import cache_util as U
from tests import gpu_util as G

pytestmark = pytest.mark.gpu


def _same(got, want):
    if not np.array_equal(got, want):
        at = np.argwhere(got != want)
        raise AssertionError("%d of %d differ: %s" % (len(at), got.size, [(tuple(int(x) for x in i), got[tuple(i)], want[tuple(i)]) for i in at[:8]]))


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _table(nseq, H, blocks, rng, evicted=0.0):
    order = rng.permutation(nseq * H * blocks + 2)
    table = order[:nseq * H * blocks].reshape(nseq, H, blocks).astype(np.int32)
    table[rng.random(table.shape) < evicted] = -1
    return table, nseq * H * blocks + 2


def _random_bits(rng, shape):
    """bf16 rows of every kind: normal ones at many magnitudes, blocks of zeros, subnormals, the largest, infinities and NaN."""
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-30, 30, size=shape[:-1] + (1,)))
    bits = synth.round_to_bf16_bits(x.astype(np.float32))
    blocks = bits.reshape(-1, 32)
    kind = rng.integers(0, 12, size=len(blocks))
    blocks[kind == 0] = 0
    blocks[kind == 1] = rng.integers(0, 128, size=blocks[kind == 1].shape) | (rng.integers(0, 2, size=blocks[kind == 1].shape) << 15)
    blocks[kind == 2] = rng.integers(0, 0x10000, size=blocks[kind == 2].shape)  # any pattern at all
    blocks[kind == 3, 7] = 0x7F80
    blocks[kind == 4, 31] = 0xFFC1
    blocks[kind == 5, 0] = 0x7F7F
    blocks[kind == 6] = rng.integers(0x8000, 0x8002, size=blocks[kind == 6].shape)
    return bits


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("D, S, gap", [(128, 64, 0), (64, 16, 0), (128, 16, 16), (64, 128, 32), (128, 32, 0), (64, 64, 0), (128, 128, 48)])
def test_written_and_read_back(fmt, D, S, gap):
    rng = np.random.default_rng([D, S, gap])
    nseq, H, blocks = 4, 3, 4
    start, new = [0, S - 3, 2 * S, 5], [S + 1, 2 * S, 0, 1]
    table, pages = _table(nseq, H, blocks, rng, evicted=0.2)
    cu = np.concatenate([[0], np.cumsum(new)])
    bits = [_random_bits(rng, (int(cu[-1]), H, D)) for _ in "kv"]
    pools = U.Pools(fmt, pages, S, D, gap)
    cache = pools.cache(_ints(table.tolist()))
    rows = [G.to_dev(x) for x in bits]
    skipped = torch.zeros(1, dtype=torch.int32, device="cuda")
    # (rows and heads in another order in memory, longer rows)
    wide = [torch.zeros(H, int(cu[-1]), D + 8, dtype=torch.bfloat16, device="cuda")[..., :D].transpose(0, 1) for _ in "kv"]
    for w, r in zip(wide, rows):
        w.copy_(r)
    B.s2_kv_append_paged(cache, wide[0], wide[1], _ints(cu.tolist()), _ints(start), max(new), skipped=skipped)
    torch.cuda.synchronize()

    left_out = 0
    values = []
    for which in range(2):
        held, byte, value = U.held_rows(bits[which], fmt)
        got, got_byte = pools.host(which)
        want, want_byte = np.full_like(got, 0xFFFF if fmt == "bf16" else 0xFF), None if byte is None else np.full_like(got_byte, 0xFF)
        read = np.zeros((H, int(sum(new)) + 0, D))
        for b in range(nseq):
            for i in range(new[b]):
                pos = start[b] + i
                for h in range(H):
                    page = table[b, h, pos // S]
                    if page < 0:
                        left_out += which == 0
                        continue
                    want[page, pos % S] = held[cu[b] + i, h]
                    if byte is not None:
                        want_byte[page, pos % S] = byte[cu[b] + i, h]
                    read[h, cu[b] + i] = value[cu[b] + i, h]
        if byte is not None:
            _same(got_byte, want_byte)
        _same(got, want)
        values.append(read)
    assert int(skipped.item()) == left_out

    # what was written, read back, with rows of the output that belong to no sequence
    extra = 5
    outs = [torch.full((H, int(cu[-1]) + extra, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    B.s2_kv_read_paged(cache, outs[0], outs[1], _ints(cu.tolist()), _ints(start), max(new))
    torch.cuda.synchronize()
    for got, want in zip(outs, values):
        got = G.to_f64(got)
        assert np.all(got[:, int(cu[-1]):] == 7)
        got = got[:, :int(cu[-1])]
        if fmt == "bf16":  # (NaN patterns pass as they are)
            nan = np.isnan(want)
            assert np.array_equal(np.isnan(got), nan) and np.array_equal(got[~nan], want[~nan])
        else:
            assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
def test_every_bf16_number_as_the_largest_and_beside_a_larger(fmt):
    """Each of the 65536 patterns alone in its block, and beside 1.0: two blocks of a row, 65536 rows of one head."""
    bits = np.zeros((65536, 1, 64), dtype=np.uint16)
    bits[:, 0, 3] = np.arange(65536)
    bits[:, 0, 40] = np.arange(65536)
    bits[:, 0, 63] = 0x3F80
    S, blocks = 128, 512
    pools = U.Pools(fmt, blocks, S, 64)
    cache = pools.cache(torch.arange(blocks, dtype=torch.int32, device="cuda").view(1, 1, blocks))
    rows = G.to_dev(bits)
    B.s2_kv_append_paged(cache, rows, rows, _ints([0, 65536]), _ints([0]), 65536)
    torch.cuda.synchronize()
    # (the search is slow: blocks of a row at a time, only the two features that are not zero and the marker)
    x = synth.bf16_bits_to_f32(bits).astype(np.float64).reshape(65536, 2, 32)
    top = np.abs(x).max(-1)
    limit, values = (464.0, orc.mx_code_values(fmt)) if fmt == "mxfp8" else (7.0, orc.mx_code_values(fmt))
    with np.errstate(all="ignore"):
        wild = ~(top < 2.0 ** 127)
        e = np.full(top.shape, -110)
        for t in range(-110, 128):
            e = np.where((top * 2.0 ** -t >= limit) & ~wild, t + 1, e)
        want_byte = np.where(wild, 255, e + 127)
        y = np.where(wild[..., None], 0, x) * np.exp2(-e.astype(np.float64))[..., None]
    half = len(values) // 2
    positive = values[:half][~np.isnan(values[:half])]
    got, got_byte = pools.host(0)
    assert np.array_equal(got_byte.reshape(65536, 2), want_byte)
    codes = U.unpack(got, fmt).reshape(65536, 2, 32)
    for block, f in ((0, 3), (1, 8), (1, 31)):
        a = np.abs(y[:, block, f])
        off = np.abs(a[:, None] - positive[None, :]) - np.where(np.arange(len(positive)) % 2 == 0, 1e-300, 0)[None, :]
        at = np.searchsorted(positive, a)
        lo, hi = np.clip(at - 1, 0, len(positive) - 1), np.clip(at, 0, len(positive) - 1)
        dl, dh = a - positive[lo], positive[hi] - a
        pick = np.where(at == 0, 0, np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi))))
        del off
        want = pick + np.where(np.signbit(y[:, block, f]) & ~wild[:, block], half, 0)
        assert np.array_equal(codes[:, block, f], want)
    other = np.ones((2, 32), bool)
    other[0, 3] = other[1, 8] = other[1, 31] = False
    assert np.all(codes[:, other] == 0)
    outs = [torch.empty((1, 65536, 64), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    B.s2_kv_read_paged(cache, outs[0], outs[1], _ints([0, 65536]), _ints([0]), 65536)
    torch.cuda.synchronize()
    want = orc.mx_values(codes.reshape(65536, 64), want_byte, fmt)
    assert np.array_equal(G.to_f64(outs[1])[0], want, equal_nan=True)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("H", [1, 5, 33])
def test_rows_by_index(fmt, H):
    """Accepted nodes of a batch of trees: any rows in any order, the same row twice, rows that do not exist, positions that do not."""
    D, S, nseq, blocks = 128, 16, 3, 2
    rng = np.random.default_rng(H)
    bits = _random_bits(rng, (20, H, D))
    rows = [3, 3, 19, 20, -1, 0, 7, 2 ** 31 - 1]
    cu, start = [0, 3, 6, 8], [0, 14, 31]
    table, pages = _table(nseq, H, blocks, rng)
    table[1, 0, 1] = pages      # not a page
    pools = U.Pools(fmt, pages, S, D)
    skipped = torch.full((1,), 100, dtype=torch.int32, device="cuda")
    k = G.to_dev(bits)
    B.s2_kv_append_paged(pools.cache(_ints(table.tolist())), k, k, _ints(cu), _ints(start), 3, rows=_ints(rows), skipped=skipped)
    torch.cuda.synchronize()
    held, byte, _ = U.held_rows(bits, fmt)
    got, got_byte = pools.host(1)
    want = np.full_like(got, 0xFFFF if fmt == "bf16" else 0xFF)
    left_out = 0
    for b in range(nseq):
        for i in range(cu[b], cu[b + 1]):
            pos = start[b] + i - cu[b]
            for h in range(H):
                page = table[b, h, pos // S] if pos < blocks * S else -1
                if not 0 <= rows[i] < 20 or not 0 <= page < pages:
                    left_out += 1
                    continue
                want[page, pos % S] = held[rows[i], h]
                if byte is not None:
                    assert np.array_equal(got_byte[page, pos % S], byte[rows[i], h])
    _same(got, want)
    assert int(skipped.item()) == 100 + left_out


def test_more_tokens_than_allowed_and_positions_outside():
    """max_new cuts; negative positions and ones past the table are left out, and read as zeros."""
    S, D, H = 16, 64, 2
    rng = np.random.default_rng(1)
    bits = synth.normal_bf16(rng, (40, H, D))
    pools = U.Pools("mxfp8", 4, S, D)
    cache = pools.cache(_ints([[[0, 1], [2, 3]]]))
    skipped = torch.zeros(1, dtype=torch.int32, device="cuda")
    k = G.to_dev(bits)
    B.s2_kv_append_paged(cache, k, k, _ints([0, 40]), _ints([-3]), 39, skipped=skipped)
    outs = [torch.full((H, 40, D), 3.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    B.s2_kv_read_paged(cache, outs[0], outs[1], _ints([0, 40]), _ints([-3]), 39)
    torch.cuda.synchronize()
    assert int(skipped.item()) == H * (3 + 39 - 35)
    value = U.held_rows(bits, "mxfp8")[2].transpose(1, 0, 2)
    got = G.to_f64(outs[0])
    assert np.array_equal(got[:, 3:35], value[:, 3:35]) and np.all(got[:, :3] == 0) and np.all(got[:, 35:39] == 0) and np.all(got[:, 39] == 3)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp4"])
def test_pages_far_apart(fmt):
    """Pages more than 2^32 bytes from the pool's beginning."""
    S, D = 16, 128
    far = 5 << 30
    raw = torch.zeros(far + (1 << 20), dtype=torch.uint8, device="cuda")
    rb = U.row_bytes(D, fmt)
    make = lambda at: (raw[at:].view(torch.bfloat16) if fmt == "bf16" else raw[at:]).as_strided(  # noqa: E731
        (2, S, rb // (2 if fmt == "bf16" else 1)), (far // (2 if fmt == "bf16" else 1), rb // (2 if fmt == "bf16" else 1), 1))
    scale = lambda at: raw[at:].as_strided((2, S, D // 32), (far, D // 32, 1)) if fmt != "bf16" else None  # noqa: E731
    cache = B.paged_cache(U.FORMATS[fmt], S, make(0), make(65536), _ints([[[1]]]), scale(131072), scale(196608))
    bits = synth.normal_bf16(np.random.default_rng(3), (S, 1, D))
    k = G.to_dev(bits)
    B.s2_kv_append_paged(cache, k, k, _ints([0, S]), _ints([0]), S)
    outs = [torch.empty((1, S, D), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    B.s2_kv_read_paged(cache, outs[0], outs[1], _ints([0, S]), _ints([0]), S)
    torch.cuda.synchronize()
    value = U.held_rows(bits, fmt)[2][:, 0]
    assert np.array_equal(G.to_f64(outs[0])[0], value) and np.array_equal(G.to_f64(outs[1])[0], value)
    assert int(torch.count_nonzero(raw[:1 << 20])) == 0


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_no_limit_on_the_rows(fmt):
    """max_new and max_rows as large as they can be: the rows that there are."""
    S, D, H = 16, 64, 3
    rng = np.random.default_rng(12)
    bits = synth.normal_bf16(rng, (70, H, D))
    table, pages = _table(2, H, 5, rng)
    pools = U.Pools(fmt, pages, S, D)
    cache = pools.cache(_ints(table.tolist()))
    k, cu, start = G.to_dev(bits), _ints([0, 1, 70]), _ints([3, 0])
    most = 2 ** 31 - 1
    B.s2_kv_append_paged(cache, k, k, cu, start, most)
    outs = [torch.full((H, 71, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    B.s2_kv_read_paged(cache, outs[0], outs[1], cu, start, most)
    torch.cuda.synchronize()
    value = U.held_rows(bits, fmt)[2].transpose(1, 0, 2)
    for got in outs:
        got = G.to_f64(got)
        assert np.array_equal(got[:, :70], value) and np.all(got[:, 70] == 5)


def test_nothing_to_write_or_read():
    pools = U.Pools("mxfp8", 2, 16, 64)
    cache = pools.cache(_ints([[[0]], [[1]]]))
    none = torch.empty((0, 1, 64), dtype=torch.bfloat16, device="cuda")
    B.s2_kv_append_paged(cache, none, none, _ints([0, 0, 0]), _ints([0, 0]), 0)
    B.s2_kv_append_paged(cache, none, none, _ints([0, 0, 0]), _ints([0, 0]), 5)
    out = torch.empty((1, 0, 64), dtype=torch.bfloat16, device="cuda")
    B.s2_kv_read_paged(cache, out, out, _ints([0, 0, 0]), _ints([0, 0]), 5)
    torch.cuda.synchronize()
    assert np.all(pools.host(0)[0] == 0xFF)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
def test_captured_on_a_stream_of_its_own(fmt):
    """Written and read in one graph on another stream, replayed with new rows, eager calls in between."""
    S, D, H = 32, 128, 3
    rng = np.random.default_rng(5)
    pools, other = U.Pools(fmt, 6, S, D), U.Pools(fmt, 6, S, D)
    table = _ints([[[4, 0], [1, 5], [2, 3]]])
    cu, start = _ints([0, 40]), _ints([10])
    k = torch.zeros((40, H, D), dtype=torch.bfloat16, device="cuda")
    outs = [torch.zeros((H, 40, D), dtype=torch.bfloat16, device="cuda") for _ in "kv"]

    def both(cache):
        B.s2_kv_append_paged(cache, k, k, cu, start, 40)
        B.s2_kv_read_paged(cache, outs[0], outs[1], cu, start, 40)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(pools.cache(table))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both(pools.cache(table))
    for i in range(3):
        k.copy_(G.to_dev(_random_bits(rng, (40, H, D))))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in outs]
        both(other.cache(table))
        torch.cuda.synchronize()
        for a, b in zip(got, outs):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
        for w in range(2):
            for a, b in zip(pools.host(w), other.host(w)):
                assert a is None or np.array_equal(a, b)

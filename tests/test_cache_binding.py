"""CPU tests of what the binding of the calls over a paged cache checks before anything arrives: types of elements, numbers that do not fit 32 bits."""

import pytest
import torch

from paper_2407_17678_amd import binding as B
from tests.test_cache_host import Stream, _pools, seen  # noqa: F401

D = 128


def _all(cache, st, **kw):
    """Each call once with proper tensors, one of them (kw) put in place of the one of its name."""
    n, H, T = 2, 3, 5
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    t = dict(new=bf(11, H, D), out=bf(H, 13, D), cu=torch.zeros(n + 1, dtype=torch.int32), start=torch.zeros(n, dtype=torch.int32),
             rows=torch.zeros(6, dtype=torch.int32), skipped=torch.zeros(1, dtype=torch.int32), q=bf(n, H, D), lse=torch.zeros(n, H),
             lens=torch.zeros(n, dtype=torch.int32), missing=torch.zeros(1, dtype=torch.int32), t=bf(n, H, T, D), parents=torch.zeros(n, T, dtype=torch.int32),
             tlse=torch.zeros(n, H, T), max_new=5, max_rows=5, splits=0)
    t.update(kw)
    ws, par = torch.zeros(64, dtype=torch.uint8), B.layout_params(H, 1, 64, 2, 4)
    return (lambda: B.s2_kv_append_paged(cache, t["new"], t["new"], t["cu"], t["start"], t["max_new"], rows=t["rows"], skipped=t["skipped"], stream=st),
            lambda: B.s2_kv_read_paged(cache, t["out"], t["out"], t["cu"], t["start"], t["max_rows"], stream=st),
            lambda: B.s2_attn_decode_paged_cache(par, cache, t["q"], t["lens"], t["q"], t["lse"], 0.5, ws, missing=t["missing"], num_splits=t["splits"], stream=st),
            lambda: B.s2_attn_tree_paged(par, cache, t["t"], t["t"], t["t"], t["parents"], t["lens"], t["t"], t["tlse"], 0.5, ws, missing=t["missing"],
                                         num_splits=t["splits"], stream=st))


def _cache(fmt=B.KV_MXFP8):
    k, v, ks, vs = _pools(fmt)
    return B.paged_cache(fmt, 64, k, v, torch.zeros(2, 3, 7, dtype=torch.int32), ks, vs)


# the tensors, another type of the same size, and the calls that take them
TYPES = [("new", torch.float16, [0]), ("new", torch.int16, [0]), ("out", torch.float16, [1]), ("cu", torch.float32, [0, 1]), ("start", torch.float32, [0, 1]),
         ("rows", torch.float32, [0]), ("skipped", torch.float32, [0]), ("q", torch.float16, [2]), ("lse", torch.int32, [2]), ("lens", torch.float32, [2, 3]),
         ("missing", torch.float32, [2, 3]), ("t", torch.float16, [3]), ("t", torch.int16, [3]), ("parents", torch.float32, [3]), ("tlse", torch.int32, [3])]


@pytest.mark.parametrize("name, other, calls", TYPES)
def test_other_types_of_the_same_size_are_refused(seen, name, other, calls):  # noqa: F811
    st, cache = Stream(), _cache()
    right = {"new": (11, 3, D), "out": (3, 13, D), "cu": (3,), "start": (2,), "rows": (6,), "skipped": (1,), "q": (2, 3, D), "lse": (2, 3), "lens": (2,),
             "missing": (1,), "t": (2, 3, 5, D), "parents": (2, 5), "tlse": (2, 3, 5)}[name]
    for f in _all(cache, st):
        f()
    assert len(seen) == 4
    made = _all(cache, st, **{name: torch.zeros(right, dtype=other)})
    for i in range(4):
        if i in calls:
            with pytest.raises(AssertionError):
                made[i]()
        else:
            made[i]()
    assert len(seen) == 8 - len(calls)


def test_pages_and_tables_of_other_types_are_refused():
    k, v, _, _ = _pools(B.KV_BF16)
    table = torch.zeros(2, 3, 7, dtype=torch.int32)
    B.paged_cache(B.KV_BF16, 64, k, v, table)
    for other in (torch.float16, torch.int16):
        with pytest.raises(AssertionError):
            B.paged_cache(B.KV_BF16, 64, k.to(other), v.to(other), table)
    with pytest.raises(AssertionError):
        B.paged_cache(B.KV_BF16, 64, k, v, table.float())
    k, v, ks, vs = _pools(B.KV_MXFP4)
    B.paged_cache(B.KV_MXFP4, 64, k.view(torch.int8), v.view(torch.int8), table, ks, vs)


@pytest.mark.parametrize("name, calls", [("max_new", [0]), ("max_rows", [1]), ("splits", [2, 3])])
@pytest.mark.parametrize("value", [2 ** 32, 2 ** 32 + 3, 2 ** 31, -2 ** 31 - 1, 2 ** 70])
def test_numbers_that_do_not_fit_are_refused(seen, name, calls, value):  # noqa: F811
    made = _all(_cache(), Stream(), **{name: value})
    for i in calls:
        with pytest.raises(OverflowError):
            made[i]()
    assert not seen
    for ok in (0, 2 ** 31 - 1, -1):
        made = _all(_cache(), Stream(), **{name: ok})
        for i in calls:
            made[i]()
    with pytest.raises(TypeError):
        _all(_cache(), Stream(), **{name: 1.5})[calls[0]]()


@pytest.mark.parametrize("value", [2 ** 32 + B.KV_MXFP8, -2 ** 32 + B.KV_MXFP8])
def test_a_format_is_not_taken_modulo_anything(value):
    k, v, ks, vs = _pools(B.KV_MXFP8)
    with pytest.raises(OverflowError):
        B.paged_cache(value, 64, k, v, torch.zeros(2, 3, 7, dtype=torch.int32), ks, vs)


def test_strides_of_a_single_one_are_any(seen):  # noqa: F811
    """One sequence of many, one head, one node, one page: the stride of a size of 1 is nothing that has to agree."""
    k, v, ks, vs = _pools(B.KV_MXFP8)
    one = lambda x, s: x.as_strided((1,) + x.shape[1:], (s,) + x.stride()[1:])  # noqa: E731
    table = torch.zeros(1, 3, 7, dtype=torch.int32)
    cache = B.paged_cache(B.KV_MXFP8, 64, one(k, 7), one(v, 99999), table, one(ks, 3), one(vs, 64))
    q, o = torch.zeros(5, 3, D, dtype=torch.bfloat16)[2:3], torch.empty_strided((1, 3, D), (1, D, 1), dtype=torch.bfloat16)
    lens, ws, par, st = torch.zeros(1, dtype=torch.int32), torch.zeros(64, dtype=torch.uint8), B.layout_params(3, 1, 64, 2, 4), Stream()
    B.s2_attn_decode_paged_cache(par, cache, q, lens, o, None, 0.5, ws, stream=st)
    assert seen[0][1][1]["page_stride"] == seen[0][1][1]["scale_page_stride"] == seen[0][1][2]["q_stride_seq"] == 0
    assert seen[0][1][1]["tok_stride"] == k.stride(1) and seen[0][1][2]["q_stride_head"] == D
    t = torch.zeros(1, 3, 4, 1, D, dtype=torch.bfloat16)
    q = t[:, :, 2]
    o = torch.empty_strided((1, 3, 1, D), (5, q.stride(1), 3, 1), dtype=torch.bfloat16)
    parents = torch.zeros(1, 1, dtype=torch.int32)
    B.s2_attn_tree_paged(par, cache, q, q, o, parents, lens, o, None, 0.5, ws, stream=st)
    assert seen[1][1][2]["q_stride_node"] == seen[1][1][2]["kv_stride_node"] == 0 and seen[1][1][2]["q_stride_head"] == q.stride(1)
    new = torch.zeros(1, 3, D, dtype=torch.bfloat16)
    B.s2_kv_append_paged(cache, new, torch.empty_strided((1, 3, D), (3, D, 1), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), lens, 1, stream=st)
    assert seen[2][1][1]["stride_row"] == 0 and seen[2][1][1]["stride_head"] == D
    with pytest.raises(AssertionError):  # (of the others they do)
        B.s2_attn_decode_paged_cache(par, cache, torch.zeros(1, 3, D, dtype=torch.bfloat16), lens, torch.zeros(1, 3, D + 8, dtype=torch.bfloat16)[..., :D], None, 0.5,
                                     ws, stream=st)

"""CPU tests of the binding of the calls around attention in a step: what arrives at the C entry points, types and sizes that it refuses, numbers beyond 32 bits."""

import ctypes as C

import pytest
import torch

from paper_2407_17678_amd import binding as B
from tests.test_cache_host import Stream, _pools

D = 128


class Handle:
    handle = C.c_void_p(0x7000)


@pytest.fixture()
def step():
    calls, got = B._marshal(), []
    P, F, Z, CP, LP = C.c_void_p, C.c_float, C.c_size_t, C.POINTER(B.PagedCacheStruct), C.POINTER(B.LayoutParams)
    A, K, R = C.POINTER(B.ChunkArgs), C.POINTER(B.KvPlanArgs), C.POINTER(B.QkNormRopeArgs)
    signatures = {"s2_attn_chunk_paged": (LP, CP, A, F, P, Z, P), "s2_attn_chunk_paged_layout": (P, CP, A, F, P, Z, P), "s2_kv_plan_paged": (LP, K, P, Z, P),
                  "s2_kv_plan_paged_layout": (P, K, P, Z, P), "s2_qk_norm_rope_fwd": (R, P), "s2_qk_norm_rope_bwd": (R, P, Z, P)}

    def callback(name):
        def f(*args):
            got.append((name, [{n: getattr(a.contents, n) for n, *_ in a.contents._fields_} if hasattr(a, "contents") else a for a in args]))
            return 0
        return C.CFUNCTYPE(C.c_int, *signatures[name])(f)

    kept = [callback(n) for n in B._STEP_CALLS]
    calls.bind_step(*(C.cast(f, C.c_void_p).value for f in kept))
    yield got
    calls.bind_step(*(C.cast(getattr(B.lib(), n), C.c_void_p).value for n in B._STEP_CALLS))


def _ints(*s):
    return torch.zeros(*s, dtype=torch.int32)


def _bf(*s):
    return torch.zeros(*s, dtype=torch.bfloat16)


def _all(**kw):
    """Each call once with proper tensors, some of them (kw) put in place of those of their names."""
    k, v, ks, vs = _pools(B.KV_MXFP8)
    cache = B.paged_cache(B.KV_MXFP8, 64, k, v, _ints(2, 3, 7), ks, vs)
    t = dict(q=_bf(11, 3, D), o=_bf(11, 3, D), cu=_ints(3), start=_ints(2), lse=torch.zeros(3, 11), missing=_ints(1), ws=torch.zeros(64, dtype=torch.uint8), max_new=8,
             splits=0, table=_ints(2, 3, 7), new_table=_ints(2, 3, 7), lens=_ints(2), new=_ints(2), ring=_ints(9), new_ring=_ints(9), state=_ints(2), new_state=_ints(2),
             plan_cu=_ints(3), positions=_ints(11), seq_lens=_ints(2), query_from=_ints(2), short=_ints(1),
             x=_bf(2, 3, 5, D), y=_bf(2, 3, 5, D), xk=_bf(2, 3, 5, D), yk=_bf(2, 3, 5, D), weight=torch.zeros(D), d_weight=torch.zeros(D), freq=torch.zeros(32),
             at=_ints(2, 5), eps=0.5, g=_bf(2, 3, 5, D), dx=_bf(2, 3, 5, D), dxk=_bf(2, 3, 5, D))
    assert not set(kw) - set(t)
    t.update(kw)
    st, par = Stream(), B.layout_params(3, 1, 64, 2, 4)
    return t, cache, (
        lambda: B.s2_attn_chunk_paged(par, cache, t["q"], t["cu"], t["start"], t["o"], t["lse"], 0.5, t["ws"], t["max_new"], missing=t["missing"],
                                      num_splits=t["splits"], stream=st),
        lambda: B.s2_attn_chunk_paged_layout(Handle(), cache, t["q"], t["cu"], t["start"], t["o"], None, 0.5, None, t["max_new"], stream=st),
        lambda: B.s2_kv_plan_paged(par, t["table"], t["lens"], t["new"], t["ring"], t["state"], t["new_table"], t["new_ring"], t["new_state"], t["ws"],
                                   cu_new=t["plan_cu"], positions=t["positions"], seq_lens=t["seq_lens"], query_from=t["query_from"], short=t["short"], stream=st),
        lambda: B.s2_kv_plan_paged_layout(Handle(), t["table"], t["lens"], t["new"], t["ring"], t["state"], t["new_table"], t["new_ring"], t["new_state"], t["ws"],
                                          stream=st),
        lambda: B.s2_qk_norm_rope_fwd(t["x"], t["xk"], t["y"], t["yk"], t["weight"], t["weight"], t["freq"], t["eps"], positions=t["at"], stream=st),
        lambda: B.s2_qk_norm_rope_bwd(t["x"], t["xk"], t["g"], t["g"], t["dx"], t["dxk"], t["weight"], t["weight"], t["d_weight"], t["d_weight"], t["freq"], t["eps"],
                                      t["ws"], positions=t["at"], interleaved=True, stream=st))


def test_what_arrives(step):
    rows = _bf(3, 11, D + 8)[..., :D].transpose(0, 1)
    across = _bf(2, 5, 3, D).transpose(1, 2)
    t, cache, made = _all(q=rows, o=torch.empty_strided(rows.shape, rows.stride(), dtype=torch.bfloat16), splits=3, x=across, xk=across, dx=across, dxk=across)
    for f in made:
        f()
    assert [n for n, _ in step] == list(B._STEP_CALLS)
    p = {k: v.data_ptr() for k, v in t.items() if isinstance(v, torch.Tensor)}
    chunk = dict(q=p["q"], cu_new=p["cu"], start=p["start"], o=p["o"], lse=p["lse"], missing=p["missing"], num_rows=11, max_new=8, num_splits=3,
                 q_stride_row=D + 8, q_stride_head=11 * (D + 8))
    assert step[0][1][0]["num_heads"] == 3 and step[0][1][1]["num_pages"] == 9 and step[0][1][2:] == [chunk, 0.5, p["ws"], 64, 0x5000]
    assert step[1][1][0] == 0x7000 and step[1][1][2:] == [dict(chunk, lse=None, missing=None, num_splits=0), 0.5, None, 0, 0x5000]
    plan = dict(block_table=p["table"], lens=p["lens"], new_lens=p["new"], query_from=p["query_from"], free_pages=p["ring"], free_state=p["state"],
                new_table=p["new_table"], new_free_pages=p["new_ring"], new_free_state=p["new_state"], cu_new=p["plan_cu"], positions=p["positions"],
                seq_lens=p["seq_lens"], short_of=p["short"], nseq=2, heads=3, max_blocks=7, num_pages=9, num_rows=11)
    assert step[2][1][0]["num_heads"] == 3 and step[2][1][1:] == [plan, p["ws"], 64, 0x5000]
    none = dict(query_from=None, cu_new=None, positions=None, seq_lens=None, short_of=None, num_rows=0)
    assert step[3][1] == [0x7000, dict(plan, **none), p["ws"], 64, 0x5000]
    rope = dict(q=p["x"], k=p["xk"], q_out=p["y"], k_out=p["yk"], q_weight=p["weight"], k_weight=p["weight"], inv_freq=p["freq"], positions=p["at"], d_q_out=None,
                d_k_out=None, dq=None, dk=None, dq_weight=None, dk_weight=None, batch=2, heads=3, seqlen=5, head_dim=D, rotary_dim=64, interleaved=0, eps=0.5,
                in_stride_b=15 * D, in_stride_h=D, in_stride_t=3 * D, out_stride_b=15 * D, out_stride_h=5 * D, out_stride_t=D)
    assert step[4][1] == [rope, 0x5000]
    back = dict(rope, q_out=None, k_out=None, d_q_out=p["g"], d_k_out=p["g"], dq=p["dx"], dk=p["dxk"], dq_weight=p["d_weight"], dk_weight=p["d_weight"], interleaved=1)
    assert step[5][1] == [back, p["ws"], 64, 0x5000]


def test_one_of_queries_and_keys_arrives(step):
    x, y, st = _bf(2, 3, 5, 64), _bf(2, 3, 5, 64), Stream()
    B.s2_qk_norm_rope_fwd(None, x, None, y, None, None, None, 0.0, stream=st)
    B.s2_qk_norm_rope_bwd(x, None, y, None, x, None, None, None, None, None, None, 0.0, None, stream=st)
    a, b = step[0][1][0], step[1][1][0]
    assert (a["q"], a["k"], a["q_out"], a["k_out"], a["rotary_dim"], a["inv_freq"], a["positions"]) == (None, x.data_ptr(), None, y.data_ptr(), 0, None, None)
    assert (b["q"], b["k"], b["d_q_out"], b["dq"], b["dk"]) == (x.data_ptr(), None, y.data_ptr(), x.data_ptr(), None) and step[1][1][1:3] == [None, 0]
    assert a["batch"] == 2 and a["heads"] == 3 and a["seqlen"] == 5 and a["head_dim"] == 64


# the tensors, another type of the same size, and the calls that take them
TYPES = [("q", torch.float16, [0, 1]), ("o", torch.int16, [0, 1]), ("cu", torch.float32, [0, 1]), ("start", torch.float32, [0, 1]), ("lse", torch.int32, [0]),
         ("missing", torch.float32, [0])] + [(n, torch.float32, [2, 3]) for n in ("table", "new_table", "lens", "new", "ring", "new_ring", "state", "new_state")] + \
        [(n, torch.float32, [2]) for n in ("plan_cu", "positions", "seq_lens", "query_from", "short")] + \
        [("x", torch.float16, [4, 5]), ("xk", torch.float16, [4, 5]), ("y", torch.int16, [4]), ("yk", torch.float16, [4]), ("weight", torch.int32, [4, 5]),
         ("d_weight", torch.int32, [5]), ("freq", torch.int32, [4, 5]), ("at", torch.float32, [4, 5]), ("g", torch.float16, [5]), ("dx", torch.float16, [5])]


@pytest.mark.parametrize("name, other, calls", TYPES)
def test_other_types_of_the_same_size_are_refused(step, name, other, calls):
    right, _, made = _all()
    for f in made:
        f()
    assert len(step) == 6
    _, _, made = _all(**{name: torch.zeros(right[name].shape, dtype=other)})
    for i in range(6):
        if i in calls:
            with pytest.raises(AssertionError):
                made[i]()
        else:
            made[i]()
    assert len(step) == 12 - len(calls)


# tensors of other sizes or strides, and the calls that take them
SIZES = [(dict(q=_bf(11, 2, D)), [0, 1]), (dict(q=_bf(11, 3, 64)), [0, 1]), (dict(o=_bf(12, 3, D)), [0, 1]), (dict(o=_bf(3, 11, D).transpose(0, 1)), [0, 1]),
         (dict(cu=_ints(2)), [0, 1]), (dict(start=_ints(3)), [0, 1]), (dict(lse=torch.zeros(3, 10)), [0]), (dict(missing=_ints(0)), [0]),
         (dict(new_table=_ints(2, 3, 6)), [2, 3]), (dict(table=_ints(2, 3, 8)[..., :7]), [2, 3]), (dict(lens=_ints(3)), [2, 3]), (dict(new=_ints(1)), [2, 3]),
         (dict(new_ring=_ints(8)), [2, 3]), (dict(state=_ints(1)), [2, 3]), (dict(new_state=_ints(3)), [2, 3]), (dict(plan_cu=_ints(2)), [2]),
         (dict(seq_lens=_ints(1)), [2]), (dict(query_from=_ints(4)), [2]), (dict(ring=_ints(18)[::2]), [2, 3]),
         (dict(xk=_bf(2, 3, 4, D)), [4, 5]), (dict(xk=_bf(2, 5, 3, D).transpose(1, 2)), [4, 5]), (dict(y=_bf(2, 3, 5, 64)), [4]), (dict(weight=torch.zeros(64)), [4, 5]),
         (dict(d_weight=torch.zeros(D - 1)), [5]), (dict(at=_ints(2, 4)), [4, 5]), (dict(dx=_bf(2, 5, 3, D).transpose(1, 2)), [5]),
         (dict(x=_bf(2, 3, 5, 2 * D)[..., ::2]), [4, 5])]


@pytest.mark.parametrize("kw, calls", SIZES, ids=lambda x: "_".join(x) if isinstance(x, dict) else None)
def test_other_sizes_and_strides_are_refused(step, kw, calls):
    _, _, made = _all(**kw)
    for i in range(6):
        if i in calls:
            with pytest.raises(AssertionError):
                made[i]()
        else:
            made[i]()


@pytest.mark.parametrize("name", ["max_new", "splits"])
@pytest.mark.parametrize("value", [2 ** 32, 2 ** 32 + 3, 2 ** 31, -2 ** 31 - 1, 2 ** 70])
def test_numbers_that_do_not_fit_are_refused(step, name, value):
    with pytest.raises(OverflowError):
        _all(**{name: value})[2][0]()
    assert not step
    for ok in (0, 2 ** 31 - 1, -1):
        _all(**{name: ok})[2][0]()
    with pytest.raises(TypeError):
        _all(**{name: 1.5})[2][0]()


def test_no_rows_of_queries_and_keys(step):
    empty = dict.fromkeys(("x", "xk", "y", "yk", "g", "dx", "dxk"), _bf(2, 3, 0, D))
    _, _, made = _all(at=_ints(2, 0), **empty)
    made[4]()
    made[5]()
    assert step[0][1][0]["seqlen"] == 0 and step[0][1][0]["q"] and step[1][1][0]["dq"]
    _, _, made = _all(q=_bf(0, 3, D), o=_bf(0, 3, D), lse=torch.zeros(3, 0))
    made[0]()
    assert step[2][1][2]["num_rows"] == 0

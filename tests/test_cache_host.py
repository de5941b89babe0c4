"""CPU tests of the calls over a paged cache of any format: what they refuse (nothing is launched then), sizes of workspaces, and what the binding
hands to the C entry points."""

import ctypes as C

import pytest
import torch

from paper_2407_17678_amd import binding as B

NULL, BAD_PARAM, SHAPE, ALIGN, WORKSPACE = -1, -2, -3, -4, -5
INT_MAX = 2 ** 31 - 1


def _cache(fmt=B.KV_MXFP8, **kw):
    c = dict(k_pages=0x1000, v_pages=0x2000, k_scales=0x3000, v_scales=0x4000, block_table=0x5000, format=fmt, nseq=2, heads=3, head_dim=128,
             block_size=64, max_blocks=7, num_pages=9, page_stride=64 * 128, tok_stride=128, scale_page_stride=256, scale_tok_stride=4)
    if fmt == B.KV_BF16:
        c.update(k_scales=None, v_scales=None, scale_page_stride=0, scale_tok_stride=0)
    c.update(kw)
    return B.PagedCacheStruct(**c)


BAD_CACHES = [
    (dict(k_pages=None), NULL), (dict(v_pages=None), NULL), (dict(block_table=None), NULL), (dict(k_scales=None), NULL), (dict(v_scales=None), NULL),
    (dict(format=3), BAD_PARAM), (dict(format=-1), BAD_PARAM), (dict(block_size=48), BAD_PARAM), (dict(block_size=0), BAD_PARAM),
    (dict(nseq=0), SHAPE), (dict(heads=0), SHAPE), (dict(max_blocks=0), SHAPE), (dict(num_pages=0), SHAPE), (dict(head_dim=96), SHAPE),
    (dict(head_dim=256), SHAPE), (dict(nseq=1 << 20, heads=1 << 10), SHAPE), (dict(max_blocks=INT_MAX // 64), SHAPE), (dict(max_blocks=INT_MAX), SHAPE),
    (dict(k_pages=0x1008), ALIGN), (dict(v_pages=0x2004), ALIGN), (dict(block_table=0x5002), ALIGN), (dict(k_scales=0x3002), ALIGN),
    (dict(v_scales=0x4001), ALIGN), (dict(page_stride=8200), ALIGN), (dict(page_stride=-16), ALIGN), (dict(tok_stride=120), ALIGN),
    (dict(tok_stride=112), ALIGN), (dict(tok_stride=-128), ALIGN), (dict(scale_tok_stride=0), ALIGN), (dict(scale_tok_stride=6), ALIGN),
    (dict(scale_page_stride=257), ALIGN), (dict(scale_page_stride=-4), ALIGN), (dict(tok_stride=(1 << 24) + 16), SHAPE),
    (dict(scale_tok_stride=(1 << 24) + 4), SHAPE), (dict(page_stride=1 << 57), SHAPE),
]


def _append(c, **kw):
    a = dict(k=0x6000, v=0x7000, cu_new=0x8000, start=0x9000, rows=None, skipped=None, num_rows=5, num_items=0, max_new=5, stride_row=384, stride_head=128)
    a.update(kw)
    return B.lib().s2_kv_append_paged(C.byref(c), C.byref(B.KvAppendArgs(**a)), None)


def _read(c, **kw):
    a = dict(k=0x6000, v=0x7000, cu_rows=0x8000, start=0x9000, num_rows=5, max_rows=5, stride_row=128, stride_head=640)
    a.update(kw)
    return B.lib().s2_kv_read_paged(C.byref(c), C.byref(B.KvReadArgs(**a)), None)


PARAMS = dict(num_heads=3, head_index_base=0, num_blocks=1, block_size=64, local_blocks=2, stride=4, window_blocks=0, dense=0)


def _decode(c, scale=0.5, ws=0x100000, ws_bytes=1 << 20, params=PARAMS, **kw):
    a = dict(q=0x6000, seq_lens=0x8000, o=0x7000, lse=None, missing=None, num_splits=0, q_stride_seq=384, q_stride_head=128)
    a.update(kw)
    return B.lib().s2_attn_decode_paged_cache(C.byref(B.LayoutParams(**params)), C.byref(c), C.byref(B.CacheDecodeArgs(**a)), scale, ws, ws_bytes, None)


def _tree(c, scale=0.5, ws=0x100000, ws_bytes=1 << 20, params=PARAMS, **kw):
    a = dict(q=0x6000, k=0xa000, v=0xb000, parents=0xc000, seq_lens=0x8000, o=0x7000, lse=None, missing=None, nodes=4, num_splits=0,
             q_stride_seq=1536, q_stride_head=512, q_stride_node=128, kv_stride_seq=1536, kv_stride_head=512, kv_stride_node=128)
    a.update(kw)
    return B.lib().s2_attn_tree_paged(C.byref(B.LayoutParams(**params)), C.byref(c), C.byref(B.TreeArgs(**a)), scale, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_append, _read, _decode, _tree])
@pytest.mark.parametrize("bad, status", BAD_CACHES)
def test_caches_that_are_refused(call, bad, status):
    assert call(_cache(**bad)) == status


def test_bf16_rows_are_counted_in_elements():
    for call in (_append, _read, _tree):
        assert call(_cache(B.KV_BF16, tok_stride=120, page_stride=64 * 128)) == ALIGN
        assert call(_cache(B.KV_BF16, tok_stride=132, page_stride=64 * 256)) == ALIGN
        assert call(_cache(B.KV_BF16, tok_stride=(1 << 23) + 8)) == SHAPE
    assert _tree(_cache(B.KV_MXFP4, tok_stride=48)) == ALIGN
    assert _tree(_cache(B.KV_MXFP4, head_dim=64, tok_stride=24, scale_tok_stride=2, scale_page_stride=128)) == ALIGN


@pytest.mark.parametrize("bad, status", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(cu_new=None), NULL), (dict(start=None), NULL), (dict(num_rows=-1), SHAPE), (dict(max_new=-1), SHAPE),
    (dict(rows=0x1000, num_items=-1), SHAPE), (dict(k=0x6008), ALIGN), (dict(v=0x7002), ALIGN), (dict(cu_new=0x8001), ALIGN), (dict(start=0x9002), ALIGN),
    (dict(rows=0x1002), ALIGN), (dict(skipped=0x1003), ALIGN), (dict(stride_row=4), ALIGN), (dict(stride_row=-8), ALIGN), (dict(stride_head=12), ALIGN),
    (dict(stride_head=-128), ALIGN), (dict(stride_row=1 << 41), SHAPE), (dict(stride_head=1 << 41), SHAPE)])
def test_appends_that_are_refused(bad, status):
    assert _append(_cache(), **bad) == status


@pytest.mark.parametrize("bad, status", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(cu_rows=None), NULL), (dict(start=None), NULL), (dict(num_rows=-1), SHAPE), (dict(max_rows=-1), SHAPE),
    (dict(k=0x6008), ALIGN), (dict(v=0x7002), ALIGN), (dict(cu_rows=0x8001), ALIGN), (dict(start=0x9002), ALIGN), (dict(stride_row=4), ALIGN),
    (dict(stride_head=-8), ALIGN), (dict(stride_row=1 << 41), SHAPE)])
def test_reads_that_are_refused(bad, status):
    assert _read(_cache(), **bad) == status


def test_grids_beyond_int32_are_refused():
    wide = _cache(nseq=4096, heads=8000)
    assert _append(wide, num_rows=INT_MAX, max_new=INT_MAX) == SHAPE
    assert _read(wide, num_rows=INT_MAX, max_rows=INT_MAX) == SHAPE


def test_launches_of_more_than_32_bits_of_threads_are_refused():
    few = _cache(nseq=1, heads=3)
    assert _append(few, skipped=0xd000, max_new=INT_MAX) == SHAPE  # (without a counter it is the rows that there are)
    assert _read(_cache(nseq=64, heads=256), num_rows=1 << 20, max_rows=1 << 20) == SHAPE
    many = dict(nseq=4096, heads=8000)
    for call in (_decode, _tree):
        assert call(_cache(**many), params=dict(PARAMS, num_heads=8000), ws_bytes=1 << 60) == SHAPE
    assert _tree(_cache(nseq=1024, heads=8000), params=dict(PARAMS, num_heads=8000), nodes=64, ws_bytes=1 << 60) == SHAPE


def test_no_rows_need_no_memory():
    assert _append(_cache(), k=None, v=None, num_rows=0, max_new=0) == 0
    assert _read(_cache(), k=None, v=None, num_rows=0, max_rows=7) == 0
    assert _read(_cache(), k=None, v=None, num_rows=0, max_rows=-1) == SHAPE


ATTEND = [
    (dict(q=None), NULL), (dict(seq_lens=None), NULL), (dict(o=None), NULL), (dict(scale=0.0), BAD_PARAM), (dict(scale=-1.0), BAD_PARAM),
    (dict(scale=float("nan")), BAD_PARAM), (dict(scale=float("inf")), BAD_PARAM), (dict(num_splits=-1), BAD_PARAM), (dict(num_splits=65), BAD_PARAM),
    (dict(q=0x6008), ALIGN), (dict(o=0x7008), ALIGN), (dict(seq_lens=0x8002), ALIGN), (dict(lse=0x8002), ALIGN), (dict(missing=0x8001), ALIGN),
    (dict(q_stride_seq=4), ALIGN), (dict(q_stride_head=-8), ALIGN), (dict(q_stride_seq=1 << 41), SHAPE), (dict(ws=None), WORKSPACE),
    (dict(ws=0x100080), WORKSPACE), (dict(ws_bytes=100), WORKSPACE),
    (dict(params=dict(PARAMS, num_heads=4)), SHAPE), (dict(params=dict(PARAMS, block_size=32)), SHAPE), (dict(params=dict(PARAMS, local_blocks=0)), BAD_PARAM),
    (dict(params=dict(PARAMS, stride=-1)), BAD_PARAM), (dict(params=dict(PARAMS, window_blocks=-1)), BAD_PARAM), (dict(params=dict(PARAMS, dense=2)), BAD_PARAM),
    (dict(params=dict(PARAMS, head_index_base=-1)), BAD_PARAM)]


@pytest.mark.parametrize("call", [_decode, _tree])
@pytest.mark.parametrize("bad, status", ATTEND)
def test_attention_that_is_refused(call, bad, status):
    assert call(_cache(), **bad) == status


@pytest.mark.parametrize("bad, status", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(parents=None), NULL), (dict(nodes=0), SHAPE), (dict(nodes=65), SHAPE), (dict(nodes=-3), SHAPE),
    (dict(k=0xa008), ALIGN), (dict(v=0xb008), ALIGN), (dict(parents=0xc002), ALIGN), (dict(q_stride_node=4), ALIGN), (dict(kv_stride_seq=-8), ALIGN),
    (dict(kv_stride_head=2), ALIGN), (dict(kv_stride_node=1), ALIGN), (dict(kv_stride_node=1 << 41), SHAPE)])
def test_trees_that_are_refused(bad, status):
    assert _tree(_cache(), **bad) == status


def test_null_structures():
    L, c, p = B.lib(), _cache(), B.LayoutParams(**PARAMS)
    assert L.s2_kv_append_paged(None, C.byref(B.KvAppendArgs()), None) == NULL and L.s2_kv_append_paged(C.byref(c), None, None) == NULL
    assert L.s2_kv_read_paged(None, C.byref(B.KvReadArgs()), None) == NULL and L.s2_kv_read_paged(C.byref(c), None, None) == NULL
    for call, args in ((L.s2_attn_decode_paged_cache, B.CacheDecodeArgs()), (L.s2_attn_tree_paged, B.TreeArgs())):
        assert call(None, C.byref(c), C.byref(args), 1.0, None, 0, None) == NULL
        assert call(C.byref(p), None, C.byref(args), 1.0, None, 0, None) == NULL
        assert call(C.byref(p), C.byref(c), None, 1.0, None, 0, None) == NULL
    for call, args in ((L.s2_attn_decode_paged_cache_layout, B.CacheDecodeArgs()), (L.s2_attn_tree_paged_layout, B.TreeArgs())):
        assert call(None, C.byref(c), C.byref(args), 1.0, None, 0, None) == NULL


def test_layouts_have_to_cover_the_cache():
    lay = B.s2_layout_build(B.layout_params(3, 6, 64, 2, 4))
    args = B.TreeArgs(q=0x6000, k=0xa000, v=0xb000, parents=0xc000, seq_lens=0x8000, o=0x7000, nodes=4, q_stride_seq=1536, q_stride_head=512,
                      q_stride_node=128, kv_stride_seq=1536, kv_stride_head=512, kv_stride_node=128)
    call = lambda c: B.lib().s2_attn_tree_paged_layout(lay.handle, C.byref(c), C.byref(args), 1.0, 0x100000, 0, None)  # noqa: E731
    assert call(_cache(max_blocks=7)) == SHAPE
    assert call(_cache(max_blocks=6, heads=2)) == SHAPE
    assert call(_cache(max_blocks=6, block_size=32)) == SHAPE
    assert call(_cache(max_blocks=6)) in (WORKSPACE, -7)  # (-7: a layout without a device copy)


def test_workspaces():
    f = B.s2_attn_tree_workspace_bytes
    assert f(2, 3, 4, 128, 448, 5) == (2 * 3 * 4 * 5 * 130 * 4 + 255) // 256 * 256
    assert f(2, 3, 1, 64, 448, 3) == B.s2_attn_decode_workspace_bytes(2, 3, 64, 448, 3)
    assert f(2, 3, 4, 128, 40000, 0) == f(2, 3, 4, 128, 40000, 64) and f(64, 8, 4, 128, 40000, 0) == f(64, 8, 4, 128, 40000, 2)
    assert f(1, 1, 4, 128, 256, 0) == f(1, 1, 4, 128, 256, 2) and f(1000, 8, 4, 128, 256, 0) == f(1000, 8, 4, 128, 256, 1)
    for nseq, heads, length in ((1, 1, 100), (1, 32, 4096), (7, 13, 30000), (300, 40, 1 << 20)):  # enough for the bf16 call as well
        assert f(nseq, heads, 1, 128, length) >= B.s2_attn_decode_workspace_bytes(nseq, heads, 128, length)
    assert f(0, 3, 4, 128, 448, 5) == f(2, 3, 0, 128, 448, 5) == f(2, -1, 4, 128, 448, 5) == 0
    assert f(64, 32, 64, 128, 1 << 20, 64) == 64 * 32 * 64 * 64 * 130 * 4


# ------------------------------------------------------------------------------------ the binding


class Stream:
    cuda_stream = 0x5000


@pytest.fixture()
def seen():
    calls, got = B._marshal(), []
    P, F, Z, CP = C.c_void_p, C.c_float, C.c_size_t, C.POINTER(B.PagedCacheStruct)
    LP, D, T = C.POINTER(B.LayoutParams), C.POINTER(B.CacheDecodeArgs), C.POINTER(B.TreeArgs)
    signatures = {"s2_kv_append_paged": (CP, C.POINTER(B.KvAppendArgs), P), "s2_kv_read_paged": (CP, C.POINTER(B.KvReadArgs), P),
                  "s2_attn_decode_paged_cache": (LP, CP, D, F, P, Z, P), "s2_attn_decode_paged_cache_layout": (P, CP, D, F, P, Z, P),
                  "s2_attn_tree_paged": (LP, CP, T, F, P, Z, P), "s2_attn_tree_paged_layout": (P, CP, T, F, P, Z, P)}

    def callback(name):
        def f(*args):
            got.append((name, [{n: getattr(a.contents, n) for n, *_ in a.contents._fields_} if hasattr(a, "contents") else a for a in args]))
            return 0
        return C.CFUNCTYPE(C.c_int, *signatures[name])(f)

    kept = [callback(n) for n in B._CACHE_CALLS]
    calls.bind_cache(*(C.cast(f, C.c_void_p).value for f in kept))
    yield got
    calls.bind_cache(*(C.cast(getattr(B.lib(), n), C.c_void_p).value for n in B._CACHE_CALLS))


def _pools(fmt, D=128, pages=9, S=64, gap=16):
    rb = {B.KV_BF16: D, B.KV_MXFP8: D, B.KV_MXFP4: D // 2}[fmt]
    dt = torch.bfloat16 if fmt == B.KV_BF16 else torch.uint8
    k, v = (torch.zeros(pages, S, rb + gap, dtype=dt)[..., :rb] for _ in "kv")
    ks, vs = (None if fmt == B.KV_BF16 else torch.zeros(pages, S, D // 32 * 2, dtype=torch.uint8)[..., :D // 32] for _ in "kv")
    return k, v, ks, vs


@pytest.mark.parametrize("fmt", [B.KV_BF16, B.KV_MXFP8, B.KV_MXFP4])
@pytest.mark.parametrize("D", [64, 128])
def test_what_arrives(seen, fmt, D):
    k, v, ks, vs = _pools(fmt, D)
    table = torch.zeros(2, 3, 7, dtype=torch.int32)
    cache = B.paged_cache(fmt, 64, k, v, table, ks, vs)
    if fmt == B.KV_MXFP8:  # any element of one byte
        assert B.paged_cache(fmt, 64, k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), table, ks, vs).raw == cache.raw
    want = dict(k_pages=k.data_ptr(), v_pages=v.data_ptr(), k_scales=ks.data_ptr() if ks is not None else None,
                v_scales=vs.data_ptr() if ks is not None else None, block_table=table.data_ptr(), format=fmt, nseq=2, heads=3, head_dim=D, block_size=64,
                max_blocks=7, num_pages=9, page_stride=k.stride(0), tok_stride=k.stride(1), scale_page_stride=ks.stride(0) if ks is not None else 0,
                scale_tok_stride=ks.stride(1) if ks is not None else 0)
    st = Stream()
    new = [torch.zeros(3, 11, D + 8, dtype=torch.bfloat16)[..., :D].transpose(0, 1) for _ in "kv"]
    cu, start, idx, count = (torch.zeros(n, dtype=torch.int32) for n in (3, 2, 6, 1))
    B.s2_kv_append_paged(cache, *new, cu, start, 8, stream=st)
    B.s2_kv_append_paged(cache, *new, cu, start, 8, rows=idx, skipped=count, stream=st)
    out = [torch.zeros(3, 13, D, dtype=torch.bfloat16) for _ in "kv"]
    B.s2_kv_read_paged(cache, *out, cu, start, 12, stream=st)
    a = dict(k=new[0].data_ptr(), v=new[1].data_ptr(), cu_new=cu.data_ptr(), start=start.data_ptr(), rows=None, skipped=None, num_rows=11, num_items=0,
             max_new=8, stride_row=new[0].stride(0), stride_head=new[0].stride(1))
    assert seen[0] == ("s2_kv_append_paged", [want, a, 0x5000])
    assert seen[1][1][1] == dict(a, rows=idx.data_ptr(), skipped=count.data_ptr(), num_items=6)
    assert seen[2] == ("s2_kv_read_paged", [want, dict(k=out[0].data_ptr(), v=out[1].data_ptr(), cu_rows=cu.data_ptr(), start=start.data_ptr(), num_rows=13,
                                                       max_rows=12, stride_row=D, stride_head=13 * D), 0x5000])
    q, o = (torch.zeros(3, 2, D, dtype=torch.bfloat16).transpose(0, 1) for _ in "qo")
    lse, ws, par = torch.zeros(2, 3), torch.zeros(64, dtype=torch.uint8), B.layout_params(3, 1, 64, 2, 4)

    class Handle:
        handle = C.c_void_p(0x7000)

    B.s2_attn_decode_paged_cache(par, cache, q, start, o, lse, 0.5, ws, missing=count, num_splits=2, stream=st)
    B.s2_attn_decode_paged_cache_layout(Handle(), cache, q, start, o, None, 0.5, ws, stream=st)
    d = dict(q=q.data_ptr(), seq_lens=start.data_ptr(), o=o.data_ptr(), lse=lse.data_ptr(), missing=count.data_ptr(), num_splits=2, q_stride_seq=D,
             q_stride_head=2 * D)
    assert seen[3][1][0]["num_heads"] == 3 and seen[3][1][1:] == [want, d, 0.5, ws.data_ptr(), 64, 0x5000]
    assert seen[4][1] == [0x7000, want, dict(d, lse=None, missing=None, num_splits=0), 0.5, ws.data_ptr(), 64, 0x5000]
    q, o = (torch.zeros(2, 5, 3, D, dtype=torch.bfloat16).permute(0, 2, 1, 3) for _ in "qo")
    kd, vd = (torch.zeros(2, 3, 5, D, dtype=torch.bfloat16) for _ in "kv")
    lse, parents = torch.zeros(2, 3, 5), torch.zeros(2, 5, dtype=torch.int32)
    B.s2_attn_tree_paged(par, cache, q, kd, vd, parents, start, o, lse, 0.5, ws, missing=count, num_splits=2, stream=st)
    B.s2_attn_tree_paged_layout(Handle(), cache, q, kd, vd, parents, start, o, None, 0.5, ws, stream=st)
    t = dict(q=q.data_ptr(), k=kd.data_ptr(), v=vd.data_ptr(), parents=parents.data_ptr(), seq_lens=start.data_ptr(), o=o.data_ptr(), lse=lse.data_ptr(),
             missing=count.data_ptr(), nodes=5, num_splits=2, q_stride_seq=15 * D, q_stride_head=D, q_stride_node=3 * D, kv_stride_seq=15 * D,
             kv_stride_head=5 * D, kv_stride_node=D)
    assert seen[5][1][1:] == [want, t, 0.5, ws.data_ptr(), 64, 0x5000]
    assert seen[6][1] == [0x7000, want, dict(t, lse=None, missing=None, num_splits=0), 0.5, ws.data_ptr(), 64, 0x5000]


def test_what_the_binding_refuses(seen):
    k, v, ks, vs = _pools(B.KV_MXFP8)
    table = torch.zeros(2, 3, 7, dtype=torch.int32)
    for bad in ((k, v[:8], table, ks, vs), (k, v[:, :, :64], table, ks, vs), (k, v.contiguous(), table, ks, vs), (k, v, table.long(), ks, vs),
                (k, v, table.transpose(0, 1), ks, vs), (k, v, table, ks[..., :2], vs[..., :2]), (k, v, table, ks, vs.contiguous()),
                (k[:, :32], v[:, :32], table, ks[:, :32], vs[:, :32]), (k.view(torch.bfloat16), v.view(torch.bfloat16), table, ks, vs),
                (k, v, table, ks.float(), vs.float())):
        with pytest.raises(AssertionError):
            B.paged_cache(B.KV_MXFP8, 64, *bad)
    with pytest.raises((AttributeError, TypeError)):
        B.paged_cache(B.KV_MXFP8, 64, k, v, table)
    with pytest.raises(ValueError):
        B.paged_cache(B.KV_MXFP8, 64, k, v, table[0], ks, vs)
    kb, vb, _, _ = _pools(B.KV_BF16)
    with pytest.raises(AssertionError):
        B.paged_cache(B.KV_BF16, 64, kb, vb, table, ks, vs)
    cache, st = B.paged_cache(B.KV_MXFP8, 64, k, v, table, ks, vs), Stream()
    new, cu, start = torch.zeros(11, 3, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for a, b, c, d in ((new[:, :2], new[:, :2], cu, start), (new[..., :64], new[..., :64], cu, start), (new, new[:5], cu, start), (new.float(), new.float(), cu, start),
                       (new, new, cu[:2], start), (new, new, cu, start[:1]), (new, new, cu.long(), start), (new, new, cu, start.long())):
        with pytest.raises(AssertionError):
            B.s2_kv_append_paged(cache, a, b, c, d, 5, stream=st)
    with pytest.raises(AssertionError):
        B.s2_kv_append_paged(cache, new, new, cu, start, 5, rows=cu[:0], stream=st)
    with pytest.raises(AssertionError):
        B.s2_kv_read_paged(cache, new, new, cu, start, 5, stream=st)  # heads come first
    with pytest.raises(TypeError):
        B._marshal().kv_read(b"short", new, new, cu, start, 5, 0)
    q, lse, ws, par = torch.zeros(2, 3, 128, dtype=torch.bfloat16), torch.zeros(2, 3), torch.zeros(64, dtype=torch.uint8), B.layout_params(3, 1, 64, 2, 4)
    for a, b, l in ((q[:1], q[:1], None), (q, q.transpose(0, 1).contiguous().transpose(0, 1), None), (q, q, lse[:1]), (q, q, lse.double()), (q[..., :64], q[..., :64], None)):
        with pytest.raises(AssertionError):
            B.s2_attn_decode_paged_cache(par, cache, a, start, b, l, 0.5, ws, stream=st)
    t, parents = torch.zeros(2, 3, 5, 128, dtype=torch.bfloat16), torch.zeros(2, 5, dtype=torch.int32)
    for a, b, p in ((t, t[:, :, :4], parents), (t, t, parents[:, :4].contiguous()), (t, t, parents.long()), (t[:1], t[:1], parents[:1])):
        with pytest.raises(AssertionError):
            B.s2_attn_tree_paged(par, cache, a, b, b, p, start, a, None, 0.5, ws, stream=st)
    with pytest.raises((TypeError, C.ArgumentError)):
        B.s2_attn_tree_paged(5, cache, t, t, t, parents, start, t, None, 0.5, ws, stream=st)
    assert not seen

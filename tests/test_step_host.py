"""CPU tests of the calls around attention in a step (block tables, norm and rotation, a chunk of new tokens): what they refuse (nothing is launched then), and
sizes of workspaces."""

import ctypes as C

import pytest

from paper_2407_17678_amd import binding as B
from tests.test_cache_host import ALIGN, BAD_CACHES, BAD_PARAM, INT_MAX, NULL, PARAMS, SHAPE, WORKSPACE, _cache

BIG = 1 << 60


def _chunk(c, scale=0.5, ws=0x100000, ws_bytes=1 << 24, params=PARAMS, **kw):
    a = dict(q=0x6000, cu_new=0x8000, start=0x9000, o=0x7000, lse=None, missing=None, num_rows=5, max_new=5, num_splits=0, q_stride_row=384, q_stride_head=128)
    a.update(kw)
    return B.lib().s2_attn_chunk_paged(C.byref(B.LayoutParams(**params)), C.byref(c), C.byref(B.ChunkArgs(**a)), scale, ws, ws_bytes, None)


def _plan(ws=0x100000, ws_bytes=1 << 24, params=PARAMS, **kw):
    a = dict(block_table=0x1000, lens=0x2000, new_lens=0x3000, query_from=None, free_pages=0x4000, free_state=0x5000, new_table=0x1000, new_free_pages=0x4000,
             new_free_state=0x5000, cu_new=None, positions=None, seq_lens=None, short_of=None, nseq=2, heads=3, max_blocks=7, num_pages=9, num_rows=0)
    a.update(kw)
    return B.lib().s2_kv_plan_paged(C.byref(B.LayoutParams(**params)), C.byref(B.KvPlanArgs(**a)), ws, ws_bytes, None)


def _rope_args(**kw):
    a = dict(q=0x1000, k=0x2000, q_out=0x3000, k_out=0x4000, q_weight=0x5000, k_weight=0x6000, inv_freq=0x7000, positions=None, d_q_out=0x8000, d_k_out=0x9000,
             dq=0xa000, dk=0xb000, dq_weight=0xc000, dk_weight=0xd000, batch=2, heads=3, seqlen=5, head_dim=128, rotary_dim=64, interleaved=0, eps=1e-6,
             in_stride_b=1920, in_stride_h=128, in_stride_t=384, out_stride_b=1920, out_stride_h=640, out_stride_t=128)
    a.update(kw)
    return B.QkNormRopeArgs(**a)


def _fwd(**kw):
    return B.lib().s2_qk_norm_rope_fwd(C.byref(_rope_args(**kw)), None)


def _bwd(ws=0x100000, ws_bytes=1 << 24, **kw):
    return B.lib().s2_qk_norm_rope_bwd(C.byref(_rope_args(**kw)), ws, ws_bytes, None)


# ------------------------------------------------------------------------------------ a chunk


@pytest.mark.parametrize("bad, status", BAD_CACHES)
def test_caches_that_a_chunk_refuses(bad, status):
    assert _chunk(_cache(**bad)) == status


@pytest.mark.parametrize("bad, status", [
    (dict(q=None), NULL), (dict(o=None), NULL), (dict(cu_new=None), NULL), (dict(start=None), NULL), (dict(scale=0.0), BAD_PARAM), (dict(scale=-1.0), BAD_PARAM),
    (dict(scale=float("nan")), BAD_PARAM), (dict(scale=float("inf")), BAD_PARAM), (dict(num_splits=-1), BAD_PARAM), (dict(num_splits=65), BAD_PARAM),
    (dict(num_rows=-1), SHAPE), (dict(max_new=-1), SHAPE), (dict(q=0x6008), ALIGN), (dict(o=0x7002), ALIGN), (dict(cu_new=0x8001), ALIGN),
    (dict(start=0x9002), ALIGN), (dict(lse=0xa001), ALIGN), (dict(missing=0xa002), ALIGN), (dict(q_stride_row=4), ALIGN), (dict(q_stride_row=-8), ALIGN),
    (dict(q_stride_head=12), ALIGN), (dict(q_stride_head=-128), ALIGN), (dict(q_stride_row=1 << 41), SHAPE), (dict(q_stride_head=1 << 41), SHAPE),
    (dict(num_splits=2, ws=None), WORKSPACE), (dict(num_splits=2, ws=0x100080), WORKSPACE), (dict(num_splits=2, ws_bytes=0), WORKSPACE),
    (dict(params=dict(PARAMS, num_heads=2)), SHAPE), (dict(params=dict(PARAMS, block_size=32)), SHAPE), (dict(params=dict(PARAMS, local_blocks=0)), BAD_PARAM),
    (dict(params=dict(PARAMS, stride=-1)), BAD_PARAM)])
def test_chunks_that_are_refused(bad, status):
    assert _chunk(_cache(), **bad) == status
    assert _chunk(_cache(B.KV_BF16), **bad) == status


def test_null_structures():
    L, par = B.lib(), B.LayoutParams(**PARAMS)
    c, a, p = _cache(), B.ChunkArgs(), B.KvPlanArgs()
    for x in ((None, C.byref(c), C.byref(a)), (C.byref(par), None, C.byref(a)), (C.byref(par), C.byref(c), None)):
        assert L.s2_attn_chunk_paged(*x, 0.5, None, 0, None) == NULL
    assert L.s2_attn_chunk_paged_layout(None, C.byref(c), C.byref(a), 0.5, None, 0, None) == NULL
    assert L.s2_kv_plan_paged(None, C.byref(p), None, 0, None) == NULL and L.s2_kv_plan_paged(C.byref(par), None, None, 0, None) == NULL
    assert L.s2_kv_plan_paged_layout(None, C.byref(p), None, 0, None) == NULL
    assert L.s2_qk_norm_rope_fwd(None, None) == NULL and L.s2_qk_norm_rope_bwd(None, None, 0, None) == NULL


def test_nothing_new_is_nothing_to_launch():
    assert _chunk(_cache(), num_rows=0, q=None, o=None, ws=None, ws_bytes=0) == 0
    assert _chunk(_cache(), max_new=0, ws=None, ws_bytes=0) == 0
    assert _fwd(seqlen=0) == 0
    assert _bwd(seqlen=0, q_weight=None, k_weight=None, ws=None, ws_bytes=0) == 0


def test_launches_that_do_not_fit_are_refused():
    many = dict(params=dict(PARAMS, num_heads=8000), ws_bytes=BIG)
    assert _chunk(_cache(nseq=4096, heads=8000), **many) == SHAPE
    assert _chunk(_cache(nseq=64, heads=3), num_rows=INT_MAX, max_new=INT_MAX, ws_bytes=BIG, num_splits=64) == SHAPE
    assert _chunk(_cache(nseq=4096, heads=64), params=dict(PARAMS, num_heads=64), num_rows=INT_MAX, max_new=64, num_splits=64, ws_bytes=BIG) == SHAPE


def test_workspaces_of_chunks():
    f = B.s2_attn_chunk_workspace_bytes
    size = lambda nseq, heads, new, D, splits: (nseq * heads * new * splits * (D + 2) * 4 + 255) // 256 * 256  # noqa: E731
    assert f(2, 3, 40, 100, 128, 4096, 5) == size(2, 3, 40, 128, 5)
    assert f(2, 3, 40, 30, 128, 4096, 5) == size(2, 3, 30, 128, 5)  # (no sequence has more rows than there are)
    assert f(2, 3, 40, 100, 64, 4096, 1) == 0
    # what the library may choose: a workgroup to a compute unit, two of 33 to 64 rows
    assert f(1, 32, 16, 16, 128, 1 << 20, 0) == f(1, 32, 16, 16, 128, 1 << 20, 8) and f(1, 32, 40, 40, 128, 1 << 20, 0) == f(1, 32, 40, 40, 128, 1 << 20, 16)
    assert f(1, 32, 256, 256, 128, 1 << 20, 0) == f(1, 32, 256, 256, 128, 1 << 20, 4) and f(64, 32, 16, 1024, 128, 1 << 20, 0) == 0
    assert f(1, 1, 16, 16, 128, 1 << 20, 0) == f(1, 1, 16, 16, 128, 1 << 20, 64) and f(1, 1, 16, 16, 128, 256, 0) == f(1, 1, 16, 16, 128, 256, 2)
    for bad in ((0, 3, 4, 4), (2, 0, 4, 4), (2, 3, 0, 4), (2, 3, 4, 0), (2, 3, -1, 4)):
        assert f(*bad, 128, 448, 5) == 0
    assert f(2048, 64, 1 << 14, INT_MAX, 128, 1 << 20, 64) == size(2048, 64, 1 << 14, 128, 64)


# ------------------------------------------------------------------------------------ block tables


@pytest.mark.parametrize("bad, status", [(dict([(n, None)]), NULL) for n in (
    "block_table", "lens", "new_lens", "free_pages", "free_state", "new_table", "new_free_pages", "new_free_state")] + [(dict([(n, 0x9002)]), ALIGN) for n in (
        "block_table", "lens", "new_lens", "query_from", "free_pages", "free_state", "new_table", "new_free_pages", "new_free_state", "cu_new", "positions",
        "seq_lens", "short_of")] + [
    (dict(nseq=0), SHAPE), (dict(heads=0), SHAPE), (dict(max_blocks=0), SHAPE), (dict(num_pages=0), SHAPE), (dict(positions=0x9000, num_rows=-1), SHAPE),
    (dict(max_blocks=INT_MAX // 64), SHAPE), (dict(max_blocks=INT_MAX), SHAPE), (dict(nseq=1 << 20, heads=1 << 10, params=dict(PARAMS, num_heads=1 << 10)), SHAPE),
    (dict(nseq=INT_MAX), SHAPE), (dict(params=dict(PARAMS, num_heads=2)), SHAPE), (dict(params=dict(PARAMS, block_size=48)), BAD_PARAM),
    (dict(params=dict(PARAMS, block_size=0)), BAD_PARAM), (dict(params=dict(PARAMS, local_blocks=0)), BAD_PARAM), (dict(params=dict(PARAMS, stride=-1)), BAD_PARAM),
    (dict(ws=None), WORKSPACE), (dict(ws=0x100080), WORKSPACE), (dict(ws_bytes=0), WORKSPACE),
    (dict(ws_bytes=B.s2_kv_plan_workspace_bytes(2, 3) - 1), WORKSPACE)])
def test_plans_that_are_refused(bad, status):
    assert _plan(**bad) == status


def test_workspaces_of_plans():
    f = B.s2_kv_plan_workspace_bytes
    assert f(0, 3) == f(2, 0) == f(-1, 3) == 0
    assert f(1, 1) % 256 == 0 and f(1, 1) > 0
    assert f(1 << 15, 1 << 10) < 64 * (1 << 25)  # (a few words to a sequence and head)
    assert all(f(n, 8) >= f(n - 1, 8) for n in range(2, 400))


# ------------------------------------------------------------------------------------ norm and rotation


ROPE_BAD = [
    (dict(q=None, k=None), NULL), (dict(inv_freq=None), NULL), (dict(eps=-1.0), BAD_PARAM), (dict(eps=float("nan")), BAD_PARAM), (dict(eps=float("inf")), BAD_PARAM),
    (dict(interleaved=2), BAD_PARAM), (dict(interleaved=-1), BAD_PARAM), (dict(batch=0), SHAPE), (dict(heads=0), SHAPE), (dict(seqlen=-1), SHAPE),
    (dict(head_dim=96), SHAPE), (dict(head_dim=256), SHAPE), (dict(rotary_dim=-16), SHAPE), (dict(rotary_dim=144), SHAPE), (dict(rotary_dim=24), SHAPE),
    (dict(batch=1 << 16, seqlen=1 << 16), SHAPE), (dict(batch=1, seqlen=1 << 20, heads=1 << 12), SHAPE), (dict(q=0x1008), ALIGN), (dict(k=0x2002), ALIGN),
    (dict(q_weight=0x5004), ALIGN), (dict(k_weight=0x6008), ALIGN), (dict(inv_freq=0x7002), ALIGN), (dict(positions=0x7001), ALIGN)] + [
    (dict([(n, v)]), s) for n in ("in_stride_b", "in_stride_h", "in_stride_t", "out_stride_b", "out_stride_h", "out_stride_t")
    for v, s in ((-8, ALIGN), (4, ALIGN), (1 << 41, SHAPE))]


@pytest.mark.parametrize("bad, status", ROPE_BAD)
def test_rotations_that_are_refused(bad, status):
    assert _fwd(**bad) == status
    assert _bwd(**bad) == status


@pytest.mark.parametrize("bad, status", [(dict(q_out=None), NULL), (dict(k_out=None), NULL), (dict(q_out=0x3008), ALIGN), (dict(q_out=0x1000), SHAPE),
                                         (dict(k_out=0x2000), SHAPE)])
def test_forward_rotations_that_are_refused(bad, status):
    assert _fwd(**bad) == status  # (0x1000, 0x2000: in place, between strides that are not alike)


@pytest.mark.parametrize("bad, status", [
    (dict(dq=None), NULL), (dict(dk=None), NULL), (dict(d_q_out=None), NULL), (dict(d_k_out=None), NULL), (dict(dq_weight=None), NULL), (dict(dk_weight=None), NULL),
    (dict(d_q_out=0x8008), ALIGN), (dict(dk=0xb004), ALIGN), (dict(dq_weight=0xc002), ALIGN), (dict(dq=0x8000), SHAPE), (dict(dk=0x9000), SHAPE),
    (dict(ws=None), WORKSPACE), (dict(ws=0x100080), WORKSPACE), (dict(ws_bytes=0), WORKSPACE), (dict(q=None, ws=None), WORKSPACE)])
def test_backward_rotations_that_are_refused(bad, status):
    assert _bwd(**bad) == status


@pytest.mark.parametrize("bad", [dict(q_out=0x2000), dict(k_out=0x1000), dict(k_out=0x3000)])
def test_outputs_of_queries_that_are_the_keys_are_refused(bad):
    same = dict(out_stride_b=1920, out_stride_h=128, out_stride_t=384)
    assert _fwd(**bad) == _fwd(**bad, **same) == SHAPE
    assert _fwd(seqlen=0, **bad) == _fwd(seqlen=0, q_out=0x1000) == 0


@pytest.mark.parametrize("bad", [dict(dq=0x2000), dict(dk=0x1000), dict(dq=0x9000), dict(dk=0x8000), dict(dk=0xa000), dict(dk_weight=0xc000)])
def test_gradients_of_queries_that_are_the_keys_are_refused(bad):
    same = dict(out_stride_b=1920, out_stride_h=128, out_stride_t=384)
    assert _bwd(**bad) == _bwd(**bad, **same) == SHAPE
    assert _bwd(seqlen=0, q_weight=None, k_weight=None, ws=None, **bad) == 0


def test_workspaces_of_rotations():
    f = B.s2_qk_norm_rope_bwd_workspace_bytes
    assert f(0, 3, 5, 128) == f(2, 0, 5, 128) == f(2, 3, -1, 128) == f(2, 3, 5, 96) == 0
    assert f(2, 3, 0, 128) > 0 and f(2, 3, 5, 128) % 256 == 0
    assert f(1 << 10, 64, 1 << 12, 128) == f(1, 64, 1 << 20, 128)  # (bounded by what runs at once)

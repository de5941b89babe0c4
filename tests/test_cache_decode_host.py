"""CPU tests of a decode step over a bf16 cache: what it refuses (nothing is launched then), whatever the strides of q and o are."""

import pytest

from paper_2407_17678_amd import binding as B
from tests.test_cache_host import ALIGN, BAD_PARAM, NULL, SHAPE, WORKSPACE, PARAMS, _cache, _decode


@pytest.mark.parametrize("strides", [dict(), dict(q_stride_seq=640), dict(q_stride_seq=128, q_stride_head=256), dict(q_stride_seq=0, q_stride_head=0)])
@pytest.mark.parametrize("bad, status", [
    (dict(q=None), NULL), (dict(o=None), NULL), (dict(seq_lens=None), NULL), (dict(q=0x6008), ALIGN), (dict(o=0x7004), ALIGN), (dict(lse=0x8002), ALIGN),
    (dict(missing=0x8001), ALIGN), (dict(scale=0.0), BAD_PARAM), (dict(num_splits=65), BAD_PARAM), (dict(num_splits=-1), BAD_PARAM), (dict(ws=None), WORKSPACE),
    (dict(ws_bytes=100), WORKSPACE), (dict(ws=0x100080), WORKSPACE), (dict(params=dict(PARAMS, block_size=32)), SHAPE),
    (dict(params=dict(PARAMS, num_heads=4)), SHAPE)])
def test_refused_with_any_strides(strides, bad, status):
    assert _decode(_cache(B.KV_BF16), **{**strides, **bad}) == status


@pytest.mark.parametrize("bad, status", [
    (dict(q_stride_seq=4), ALIGN), (dict(q_stride_head=-8), ALIGN), (dict(q_stride_seq=-128), ALIGN), (dict(q_stride_head=12), ALIGN),
    (dict(q_stride_seq=1 << 41), SHAPE), (dict(q_stride_head=1 << 41), SHAPE)])
def test_strides_that_are_refused(bad, status):
    assert _decode(_cache(B.KV_BF16), **bad) == status


def test_more_pairs_than_there_are_numbers():
    assert _decode(_cache(B.KV_BF16, nseq=1 << 16, heads=1 << 12), params=dict(PARAMS, num_heads=1 << 12), ws_bytes=1 << 60) == SHAPE


def test_the_stride_of_one_sequence_or_head_is_not_looked_at():
    assert _decode(_cache(B.KV_BF16, nseq=1), q_stride_seq=5, ws_bytes=100) == WORKSPACE
    assert _decode(_cache(B.KV_BF16, heads=1), params=dict(PARAMS, num_heads=1), q_stride_head=-3, ws_bytes=100) == WORKSPACE

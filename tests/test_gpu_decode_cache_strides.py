"""A decode step over a paged cache with q and o laid out in other ways than side by side: the same result to the last bit, in every format."""

import numpy as np
import pytest
import torch

from paper_2407_17678_amd import binding as B
from tests import gpu_util as G
from tests.test_gpu_tree import Case, _ints

pytestmark = pytest.mark.gpu


def _step(c, q, o, lse, splits, layout=None):
    ws = torch.empty(B.s2_attn_tree_workspace_bytes(c.nseq, c.H, 1, c.D, c.max_blocks * c.S, splits), dtype=torch.uint8, device="cuda")
    missing = torch.zeros(1, dtype=torch.int32, device="cuda")
    f = B.s2_attn_decode_paged_cache_layout if layout else B.s2_attn_decode_paged_cache
    f(layout or c.params, c.pools.cache(_ints(c.table)), q, _ints(c.lens), o, lse, c.scale, ws, missing=missing, num_splits=splits)
    torch.cuda.synchronize()
    return int(missing.item())


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("D, S, splits", [(128, 64, 1), (64, 16, 1), (128, 16, 3), (64, 64, 0), (128, 32, 2), (64, 128, 0)])
def test_any_layout_of_q_and_o_gives_the_same(fmt, D, S, splits):
    c = Case(fmt, D, S, [1, 3 * S + 5, 9 * S - 1], 4, None, evict=[(1, 2, 2), (2, 0, 8)], local=3)
    q0 = G.to_dev(c.q[:, :, 0])
    o0, lse0 = torch.empty_like(q0), torch.empty((3, 4), dtype=torch.float32, device="cuda")
    gone = _step(c, q0, o0, lse0, splits)
    layouts = (lambda x: torch.full((4, 3, D), 9.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1).copy_(x),          # noqa: E731  heads outside
               lambda x: torch.full((3, 5, 4, D), 9.0, dtype=torch.bfloat16, device="cuda")[:, 2].copy_(x),                 # noqa: E731  of several tokens
               lambda x: torch.full((3, 4, D + 8), 9.0, dtype=torch.bfloat16, device="cuda")[..., :D].copy_(x),             # noqa: E731  with a margin
               lambda x: torch.full((3, 4, 3 * D), 9.0, dtype=torch.bfloat16, device="cuda")[..., D:2 * D].copy_(x))        # noqa: E731  of a joint projection
    for lay in layouts:
        q, o = lay(q0), lay(torch.zeros_like(q0))
        lse = torch.full((3, 4), 9.0, dtype=torch.float32, device="cuda")
        assert not q.is_contiguous()
        assert _step(c, q, o, lse, splits) == gone
        assert torch.equal(o.contiguous().view(torch.int16), o0.view(torch.int16)) and torch.equal(lse, lse0)
        # nothing beside o is written
        o.fill_(9.0)
        assert o._base is None or bool((o._base == 9.0).all())


@pytest.mark.parametrize("S", [16, 64])
def test_after_a_layout(S):
    H, Bk = 4, 12
    lay = B.s2_layout_build(B.layout_params(H, Bk, S, 2, 3))
    c = Case("bf16", 128, S, [5 * S + 1, 8 * S, 5], H, None, max_blocks=Bk)
    q0 = G.to_dev(c.q[:, :, 0])
    o0, lse0 = torch.empty_like(q0), torch.empty((3, H), dtype=torch.float32, device="cuda")
    _step(c, q0, o0, lse0, 2, lay)
    q, o = (torch.zeros(H, 3, 128 + 8, dtype=torch.bfloat16, device="cuda")[..., :128].transpose(0, 1) for _ in "qo")
    q.copy_(q0)
    lse = torch.empty_like(lse0)
    _step(c, q, o, lse, 2, lay)
    assert torch.equal(o.contiguous().view(torch.int16), o0.view(torch.int16)) and torch.equal(lse, lse0)
    assert np.isfinite(G.to_f64(o)).all()


def test_pages_whose_tokens_are_far_apart():
    """Tokens as far apart as a page's rows may lie (the bf16 kernel's 64-bit addresses)."""
    S, D, H = 64, 64, 2
    stride = (1 << 23)  # elements: 64 tokens within 2^30 bytes
    raw = torch.zeros(S * stride + 4 * D, dtype=torch.bfloat16, device="cuda")
    pools = [raw[x * D:].as_strided((1, S, D), (stride * S, stride, 1)) for x in (0, 2)]
    g = torch.Generator(device="cuda").manual_seed(3)
    for p in pools:
        p.copy_(torch.randn(1, S, D, generator=g, device="cuda"))
    table = torch.zeros((1, H, 1), dtype=torch.int32, device="cuda")
    ws = torch.empty(B.s2_attn_tree_workspace_bytes(1, H, 1, D, S, 1), dtype=torch.uint8, device="cuda")
    results = []
    for k, v in (pools, [p.contiguous() for p in pools]):
        cache = B.paged_cache(B.KV_BF16, S, k, v, table)
        q = torch.ones(1, H, 2 * D, dtype=torch.bfloat16, device="cuda")[..., :D]
        q.copy_(torch.arange(D, device="cuda") / D)
        o = torch.zeros(1, H, 2 * D, dtype=torch.bfloat16, device="cuda")[..., :D]
        B.s2_attn_decode_paged_cache(B.layout_params(H, 1, S, 1, 0), cache, q, _ints([S - 1]), o, None, 0.125, ws)
        results.append(o.clone())
    torch.cuda.synchronize()
    assert torch.equal(*results) and bool(results[0].any())

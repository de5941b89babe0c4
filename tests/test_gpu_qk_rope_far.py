"""Norm and rotation, and the gradient, where results are more than 64 MB, so that they go past the caches: to the last bit what calls of a part of the rows
give, whose results do not."""

import numpy as np
import pytest
import torch

from paper_2407_17678_amd import binding as B
from tests.test_gpu_qk_rope import EPS, frequencies

pytestmark = pytest.mark.gpu


def _bits(x):
    return x.contiguous().view(torch.int16)


@pytest.mark.parametrize("D, R, interleaved, size", [(128, 128, False, (2, 15, 4501)), (64, 32, True, (1, 35, 7777)), (128, 64, True, (1, 32, 4097))])
def test_results_beyond_the_caches(D, R, interleaved, size):
    Bt, H, N = size
    assert 4 * Bt * H * N * D > 64 << 20 > 4 * H * 2000 * D
    g = torch.Generator(device="cuda").manual_seed(D + R)
    normal = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(generator=g)  # noqa: E731
    qkv = normal(Bt, N, 3, H, D)
    q, k = (qkv[:, :, i].permute(0, 2, 1, 3) for i in range(2))
    d_q, d_k = normal(Bt, H, N, D), normal(Bt, H, N, D)
    w = [1 + 0.3 * torch.randn(D, generator=g, device="cuda"), None]
    freq = torch.from_numpy(frequencies(R)).cuda()
    at = torch.randint(0, 70000, (Bt, N), generator=g, device="cuda", dtype=torch.int32)
    how = dict(interleaved=interleaved)

    def call(q, k, d_q, d_k, at):
        y = [torch.full(x.shape, 9.0, dtype=torch.bfloat16, device="cuda") for x in (q, k)]
        dx = [torch.full((x.shape[0], x.shape[2], H, D), 9.0, dtype=torch.bfloat16, device="cuda").permute(0, 2, 1, 3) for x in (q, k)]
        x = [torch.empty_like(t).copy_(s) for t, s in zip(dx, (q, k))]
        dw = torch.full((D,), 9.0, device="cuda")
        ws = torch.empty(B.s2_qk_norm_rope_bwd_workspace_bytes(q.shape[0], H, q.shape[2], D), dtype=torch.uint8, device="cuda")
        B.s2_qk_norm_rope_fwd(q, k, *y, *w, freq, EPS, positions=at, **how)
        B.s2_qk_norm_rope_bwd(*x, d_q, d_k, *dx, *w, dw, None, freq, EPS, ws, positions=at, **how)
        return y, dx, dw

    y, dx, dw = call(q, k, d_q, d_k, at)
    in_place = qkv.clone()
    own = [in_place[:, :, i].permute(0, 2, 1, 3) for i in range(2)]
    B.s2_qk_norm_rope_fwd(*own, *own, *w, freq, EPS, positions=at, **how)
    assert torch.equal(_bits(in_place[:, :, 2]), _bits(qkv[:, :, 2]))
    for i in range(2):
        assert torch.equal(_bits(own[i]), _bits(y[i]))
    total = np.zeros(D)
    for b in range(Bt):
        for lo in range(0, N, 2000):
            part = (slice(b, b + 1), slice(None), slice(lo, lo + 2000))
            py, pdx, pdw = call(q[part], k[part], d_q[part].contiguous(), d_k[part].contiguous(), at[b:b + 1, lo:lo + 2000].contiguous())
            for i in range(2):
                assert torch.equal(_bits(y[i][part]), _bits(py[i])) and torch.equal(_bits(dx[i][part]), _bits(pdx[i]))
            total += pdw.double().cpu().numpy()
    # the same terms in other sums: at most Bt N / 4096 + 1 tokens to a lane, with up to nine of a token's heads each, and 29 additions of those, each off by 2^-24 of the
    # sum of magnitudes, which is sqrt(sum g^2 sum xh^2) at most
    depth = (Bt * N // 4096 + 1) * 9 + 29
    both = np.sqrt(float(d_q.double().square().sum()) / D * Bt * H * N) * 2  # (of a feature: sums of squares of g, turned, and of xh, whose mean is 1)
    assert np.all(np.abs(dw.double().cpu().numpy() - total) <= 2 * depth * 2.0 ** -24 * both)
    assert np.abs(total).max() > 20 * 2 * depth * 2.0 ** -24 * both  # (random signs: the sum is of the order of sqrt(rows))

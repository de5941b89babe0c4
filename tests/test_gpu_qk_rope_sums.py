"""Gradients of the weights where a wavefront takes several tokens and the last turn is for some of the wavefronts only: terms of one sign, so that a part that is
left out or counted twice shows, held to the additions that one lane's share, a workgroup and the parts take."""

import numpy as np
import pytest
import torch

from oracle import s2_oracle as orc
from paper_2407_17678_amd import binding as B
from paper_2407_17678_amd import synth
from tests import gpu_util as G
from tests.test_gpu_qk_rope import ARITHMETIC, EPS, Rope

pytestmark = pytest.mark.gpu

WAVEFRONTS = 4096  # 1024 workgroups at most, of four


def depth(Bt, H, N, D):
    """Additions that a term goes through at most: a lane's own (a token's heads 512 / D at a time), three across lanes at most, four wavefronts, a 64th of 1024 parts, then six."""
    rows, steps = Bt * N, -(-H // (512 // D))
    assert rows > WAVEFRONTS  # (all heads of a token to a wavefront)
    return -(-rows // WAVEFRONTS) * steps + 3 + 4 + 16 + 6


def aligned(size, D, R, interleaved, seed):
    """g is the normalised and rotated row, so that a term is the square of a normalised feature."""
    r = Rope(*size, D, R, interleaved, far=5000, seed=seed)
    freq = r.freq if r.freq is not None else np.zeros(0)
    r.g = [synth.round_to_bf16_bits(orc.qk_norm_rope(G.bits_f64(x), np.ones(D), r.at, freq, EPS, interleaved).astype(np.float32)) for x in r.x]
    return r


@pytest.mark.parametrize("D, R, interleaved, size", [(128, 128, False, (3, 4, 5463)), (128, 64, True, (1, 9, 9001)), (64, 32, True, (5, 7, 2501)),
                                                     (64, 64, False, (2, 17, 4099)), (128, 0, False, (1, 1, 20481)), (64, 16, False, (4097, 3, 1))])
def test_several_tokens_to_a_wavefront(D, R, interleaved, size):
    Bt, H, N = size
    assert Bt * N % WAVEFRONTS != 0
    r = aligned(size, D, R, interleaved, seed=3)
    _, dw = r.backward()
    freq = r.freq if r.freq is not None else np.zeros(0)
    for i in range(2):
        x, g = G.bits_f64(r.x[i]), G.bits_f64(r.g[i])
        turned = orc.rotate_pairs(g, np.asarray(r.at)[:, None], freq, interleaved, back=True)
        unit = x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
        want, size_of = (turned * unit).sum((0, 1, 2)), np.abs(turned * unit).sum((0, 1, 2))
        n = len(freq)
        a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
        both = np.abs(g)  # what a turned gradient is made of
        both[..., a] = both[..., b] = both[..., a] + both[..., b]
        # a term is off by what its turned gradient and its normalised feature are, and by its own rounding; then it is added up
        bound = 2 * ARITHMETIC * (both * np.abs(unit)).sum((0, 1, 2)) + (1 + depth(*size, D)) * 2.0 ** -24 * size_of
        # what this can tell apart: less than a token's worth (all of its heads) on average, and less than a hundredth of a workgroup's
        assert np.all(bound < want / (Bt * N)) and np.all(bound < want / 1024 / 20), (bound / want).max()
        off = np.abs(dw[i] - want)
        assert np.all(off <= bound), (i, float((off / bound).max()))


def test_a_whole_is_the_sum_of_its_parts():
    """Parts of so few rows that a wavefront takes one token of them, or some of its heads: every term is the same number there, only the sums differ."""
    Bt, H, N, D = 2, 6, 4500, 128
    r = aligned((Bt, H, N), D, 64, False, seed=5)
    _, dw = r.backward()
    c = r.common()
    total, edges = [np.zeros(D) for _ in "qk"], (0, 1, 300, 1300, 3400, N)
    for b in range(Bt):
        for lo, hi in zip(edges, edges[1:]):
            x, g = ([G.to_dev(np.ascontiguousarray(t[b:b + 1, :, lo:hi])) for t in of] for of in (r.x, r.g))
            at = c["pos"][b:b + 1, lo:hi].contiguous()
            part = [torch.full((D,), 9.0, device="cuda") for _ in "qk"]
            ws = torch.empty(B.s2_qk_norm_rope_bwd_workspace_bytes(1, H, hi - lo, D), dtype=torch.uint8, device="cuda")
            B.s2_qk_norm_rope_bwd(*x, *g, *[torch.empty_like(t) for t in x], *c["w"], *part, c["freq"], EPS, ws, positions=at)
            torch.cuda.synchronize()
            for i in range(2):
                total[i] += part[i].double().cpu().numpy()
    for i in range(2):
        # (all terms are positive or, by the rounding of g to bf16 alone, as good as 0: their magnitudes add up to little more than the sum itself)
        assert np.all(total[i] > 0)
        bound = 2 * depth(Bt, H, N, D) * 2.0 ** -24 * total[i] * 1.01
        assert np.all(np.abs(dw[i] - total[i]) <= bound), float((np.abs(dw[i] - total[i]) / bound).max())

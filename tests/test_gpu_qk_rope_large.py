"""Norm and rotation where results go past the caches (more than 32 MB), and where a wavefront takes many rows: against the fp64 oracle and against parts of it."""

import numpy as np
import pytest
import torch

from paper_2407_17678_amd import binding as B
from tests import gpu_util as G
from tests.test_gpu_qk_rope import EPS, Rope

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D, R, size", [(128, 128, (2, 17, 2001)), (64, 32, (1, 35, 4100))])
def test_many_rows(D, R, size):
    r = Rope(*size, D, R, interleaved=D == 64, far=5000, seed=1)
    assert np.prod(size) * D * 4 > 32 << 20
    r.check_forward()
    r.check_backward()
    got = r.forward(layouts=("heads", "gaps"))
    assert all(np.array_equal(a, b) for a, b in zip(got, r.forward(in_place=True, layouts=("tokens", "tokens"))))


def test_rows_are_as_in_a_call_of_their_own():
    """Stores that go past the caches, and those that do not."""
    r = Rope(2, 16, 2304, 128, 128, weights=(True, False), seed=2)
    y, (dx, _) = r.forward(), r.backward()
    c = r.common()
    for b in range(2):
        for lo in (0, 1100):
            hi = min(lo + 1204, 2304)
            x, g = ([G.to_dev(np.ascontiguousarray(t[b:b + 1, :, lo:hi])) for t in of] for of in (r.x, r.g))
            at = torch.arange(lo, hi, dtype=torch.int32, device="cuda")[None]
            out, back = [torch.empty_like(t) for t in x], [torch.empty_like(t) for t in x]
            B.s2_qk_norm_rope_fwd(*x, *out, *c["w"], c["freq"], EPS, positions=at)
            ws = torch.empty(B.s2_qk_norm_rope_bwd_workspace_bytes(1, 16, hi - lo, 128), dtype=torch.uint8, device="cuda")
            B.s2_qk_norm_rope_bwd(*x, *g, *back, *c["w"], torch.empty(128, device="cuda"), None, c["freq"], EPS, ws, positions=at)
            for i in range(2):
                assert np.array_equal(G.to_f64(out[i])[0], y[i][b, :, lo:hi]) and np.array_equal(G.to_f64(back[i])[0], dx[i][b, :, lo:hi])


def test_no_rows_between_different_strides():
    x = torch.zeros(0, 3, 4, 128, dtype=torch.bfloat16, device="cuda")
    q, k, dq = (x[:, i].transpose(0, 1)[None] for i in range(3))
    out = [torch.zeros(1, 4, 0, 128, dtype=torch.bfloat16, device="cuda") for _ in "qk"]
    w, f = torch.ones(128, device="cuda"), torch.ones(64, device="cuda")
    B.s2_qk_norm_rope_fwd(q, k, *out, w, w, f, EPS)
    dw = [torch.full((128,), 9.0, device="cuda") for _ in "qk"]
    ws = torch.empty(B.s2_qk_norm_rope_bwd_workspace_bytes(1, 4, 0, 128), dtype=torch.uint8, device="cuda")
    B.s2_qk_norm_rope_bwd(q, k, *out, dq, dq, w, w, *dw, f, EPS, ws)
    torch.cuda.synchronize()
    assert all((t == 0).all() for t in dw)

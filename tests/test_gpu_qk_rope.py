"""Norm and rotation of queries and keys, and the gradient, against the fp64 oracle."""

import numpy as np
import pytest
import torch

from oracle import s2_oracle as orc
from paper_2407_17678_amd import binding as B
from paper_2407_17678_amd import synth
from tests import gpu_util as G

pytestmark = pytest.mark.gpu
EPS = 1e-6

# Cosine and sine: of an angle whose turns are rounded to 2^-25 (2^-23 in the angle), and to two units of their last place: 2^-21 together.  r: a sum of squares in
# twelve additions, the mean, eps and an inverse square root of one unit: 2^-20.  A result is two products of three factors, each rounded.
ARITHMETIC = 2.0 ** -21 + 2.0 ** -20 + 4 * 2.0 ** -24
ROUNDED = 2.0 ** -8 * (1 + 2.0 ** -7)  # half a step of bf16


def frequencies(R, base=10000.0):
    return (base ** (-np.arange(0, R, 2) / R)).astype(np.float32)


class Rope:
    def __init__(self, Bt, H, N, D, R, interleaved=False, far=0, weights=(True, True), seed=0, scale=1.0, eps=EPS, base=10000.0):
        rng = np.random.default_rng([seed, Bt, H, N, D, R])
        self.size, self.R, self.interleaved, self.eps = (Bt, H, N, D), R, interleaved, np.float32(eps)
        self.x = [synth.round_to_bf16_bits(synth.bf16_bits_to_f32(synth.normal_bf16(rng, self.size)) * np.float32(scale)) for _ in "qk"]
        self.g = [synth.normal_bf16(rng, self.size) for _ in "qk"]
        self.w = [(1 + 0.3 * rng.standard_normal(D)).astype(np.float32) if w else None for w in weights]
        self.freq = frequencies(R, base) if R else None
        self.positions = rng.integers(0, far + 1, (Bt, N)).astype(np.int32) if far else None

    @property
    def at(self):
        Bt, _, N, _ = self.size
        return np.broadcast_to(np.arange(N), (Bt, N)) if self.positions is None else self.positions

    def tensors(self, layout):
        """layout "heads": [B, H, N, D] side by side; "tokens": [B, N, 3, H, D]'s first two; "gaps": rows further apart than they are long."""
        Bt, H, N, D = self.size
        def make():
            if layout == "heads":
                return [torch.full((Bt, H, N, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "qk"]
            if layout == "tokens":
                qkv = torch.full((Bt, N, 3, H, D), 9.0, dtype=torch.bfloat16, device="cuda")
                return [qkv[:, :, i].permute(0, 2, 1, 3) for i in range(2)]
            return [torch.full((Bt + 1, N + 2, H, D + 8), 9.0, dtype=torch.bfloat16, device="cuda")[:Bt, 1:N + 1, :, :D].permute(0, 2, 1, 3) for _ in "qk"]
        return make

    def common(self):
        w = [None if w is None else torch.from_numpy(w).cuda() for w in self.w]
        return dict(w=w, freq=None if self.freq is None else torch.from_numpy(self.freq).cuda(),
                    pos=None if self.positions is None else torch.from_numpy(self.positions).cuda())

    def forward(self, layouts=("tokens", "heads"), in_place=False, only=None, stream=None):
        c = self.common()
        x = self.tensors(layouts[0])()
        for t, bits in zip(x, self.x):
            t.copy_(G.to_dev(bits))
        y = x if in_place else self.tensors(layouts[1])()
        pick = lambda v, i: v if only in (None, i) else None  # noqa: E731
        B.s2_qk_norm_rope_fwd(pick(x[0], 0), pick(x[1], 1), pick(y[0], 0), pick(y[1], 1), c["w"][0], c["w"][1], c["freq"], float(self.eps), positions=c["pos"],
                              interleaved=self.interleaved, stream=stream)
        torch.cuda.synchronize()
        if not in_place:
            for t, bits in zip(x, self.x):
                assert torch.equal(t.contiguous().view(torch.int16), G.to_dev(bits).view(torch.int16))
        return [G.to_f64(t) for t in y]

    def check_forward(self, **kw):
        for i, got in enumerate(self.forward(**kw)):
            x = G.bits_f64(self.x[i])
            if kw.get("only") not in (None, i):
                assert np.all(got == 9.0)
                continue
            freq = np.zeros(0) if self.freq is None else self.freq
            want = orc.qk_norm_rope(x, self.w[i], self.at, freq, float(self.eps), self.interleaved)
            size = np.abs(x if self.w[i] is None else self.w[i] * x / np.sqrt((x * x).mean(-1, keepdims=True) + self.eps))
            n = len(freq)
            both = size.copy()
            a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if self.interleaved else (slice(0, n), slice(n, 2 * n))
            both[..., a] = both[..., b] = size[..., a] + size[..., b]
            off = np.abs(got - want) - (ROUNDED * np.abs(want) + ARITHMETIC * both)
            assert np.all(off <= 0), (i, float(off.max()), np.argwhere(off > 0)[:4])

    def backward(self, layouts=("tokens", "heads"), in_place=None, only=None, ws_fill=0xFF, stream=None):
        c = self.common()
        Bt, H, N, D = self.size
        x, g = self.tensors(layouts[0])(), self.tensors(layouts[1])()
        for t, u, xb, gb in zip(x, g, self.x, self.g):
            t.copy_(G.to_dev(xb))
            u.copy_(G.to_dev(gb))
        dx = x if in_place == "x" else g if in_place == "g" else self.tensors(layouts[0])()
        dw = [None if w is None else torch.full((D,), 9.0, device="cuda") for w in self.w]
        ws = torch.full((B.s2_qk_norm_rope_bwd_workspace_bytes(Bt, H, N, D),), ws_fill, dtype=torch.uint8, device="cuda")
        pick = lambda v, i: v if only in (None, i) else None  # noqa: E731
        B.s2_qk_norm_rope_bwd(pick(x[0], 0), pick(x[1], 1), pick(g[0], 0), pick(g[1], 1), pick(dx[0], 0), pick(dx[1], 1), c["w"][0], c["w"][1], dw[0], dw[1],
                              c["freq"], float(self.eps), ws, positions=c["pos"], interleaved=self.interleaved, stream=stream)
        torch.cuda.synchronize()
        return [G.to_f64(t) for t in dx], [None if t is None else t.double().cpu().numpy() for t in dw]

    def check_backward(self, **kw):
        dx, dw = self.backward(**kw)
        for i in range(2):
            if kw.get("only") not in (None, i):
                continue
            x, g = G.bits_f64(self.x[i]), G.bits_f64(self.g[i])
            freq = np.zeros(0) if self.freq is None else self.freq
            want, want_w = orc.qk_norm_rope_backward(x, self.w[i], self.at, freq, float(self.eps), g, self.interleaved)
            n = len(freq)
            a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if self.interleaved else (slice(0, n), slice(n, 2 * n))
            both = np.abs(g).copy()  # what a turned gradient is made of
            both[..., a] = both[..., b] = np.abs(g)[..., a] + np.abs(g)[..., b]
            if self.w[i] is None:
                off = np.abs(dx[i] - want) - (ROUNDED * np.abs(want) + ARITHMETIC * both)
                assert np.all(off <= 0), float(off.max())
                continue
            size = np.sqrt((x * x).mean(-1, keepdims=True) + self.eps)
            unit, gw = np.abs(x) / size, both * np.abs(self.w[i])
            parts = (gw + unit * (gw * unit).mean(-1, keepdims=True)) / size
            # (r enters three times, the mean of products is a sum of 12)
            off = np.abs(dx[i] - want) - (ROUNDED * np.abs(want) + (3 * ARITHMETIC + 2.0 ** -20) * parts)
            assert np.all(off <= 0), (i, float(off.max()), np.argwhere(off > 0)[:4])
            # every addition of a sum rounds, at most as many as there are terms
            terms = both * unit
            off = np.abs(dw[i] - want_w) - (2 * ARITHMETIC + terms[..., 0].size * 2.0 ** -24) * terms.sum((0, 1, 2))
            assert np.all(off <= 0), (i, float(off.max()))
        return dx, dw


SIZES = [(1, 1, 1), (1, 3, 5), (2, 5, 33), (3, 9, 17), (1, 32, 4), (5, 16, 130)]


@pytest.mark.parametrize("D, R", [(128, 128), (128, 64), (128, 96), (128, 16), (64, 64), (64, 32), (64, 48), (64, 16), (128, 0), (64, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_forward(D, R, interleaved):
    for i, (Bt, H, N) in enumerate(SIZES):
        r = Rope(Bt, H, N, D, R, interleaved, far=0 if i % 2 else 5000, seed=i)
        r.check_forward(layouts=(("tokens", "heads"), ("heads", "tokens"), ("gaps", "heads"))[i % 3])


@pytest.mark.parametrize("D, R", [(128, 128), (128, 64), (128, 96), (128, 16), (64, 64), (64, 32), (64, 48), (64, 16), (128, 0), (64, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_backward(D, R, interleaved):
    for i, (Bt, H, N) in enumerate(SIZES):
        r = Rope(Bt, H, N, D, R, interleaved, far=0 if i % 2 else 5000, seed=i)
        r.check_backward(layouts=(("tokens", "heads"), ("heads", "tokens"), ("gaps", "heads"))[i % 3])


@pytest.mark.parametrize("weights", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("D, R, interleaved", [(128, 128, False), (64, 32, True), (64, 48, False)])
def test_without_weights(weights, D, R, interleaved):
    r = Rope(2, 5, 21, D, R, interleaved, weights=weights)
    r.check_forward()
    r.check_backward()


@pytest.mark.parametrize("only", [0, 1])
def test_one_of_the_two(only):
    r = Rope(2, 5, 21, 128, 64)
    r.check_forward(only=only)
    r.check_backward(only=only)


@pytest.mark.parametrize("layout", ["heads", "tokens", "gaps"])
def test_in_place(layout):
    for D, R in ((128, 128), (64, 32)):
        r = Rope(2, 5, 37, D, R)
        r.check_forward(layouts=(layout, layout), in_place=True)
        r.check_backward(layouts=(layout, layout), in_place="x")
        r.check_backward(layouts=(layout, layout), in_place="g")


def test_far_positions():
    for far in (1 << 17, 1 << 24, 2 ** 31 - 2):
        r = Rope(1, 2, 60, 128, 128, far=far, seed=1)
        r.check_forward()
        r.check_backward()
        r = Rope(1, 2, 60, 128, 128, far=far, seed=2, base=1.0)  # (every pair a radian to a position)
        r.positions[:, :30] *= -1
        r.check_forward()


def test_rows_of_zeros_and_of_extreme_sizes():
    r = Rope(1, 3, 9, 128, 128)
    for x in r.x:
        x[:, :, :4] = 0
    r.check_forward()
    r.check_backward()
    for scale in (1e-15, 1e-4, 1e4, 1e15):
        r = Rope(1, 3, 9, 64, 64, scale=scale)
        r.check_forward()
    r = Rope(1, 3, 9, 128, 64, eps=0.0)
    r.check_forward()
    r.check_backward()
    r.x[0][0, 1, 3] = 0  # 0 / 0
    y = r.forward()
    assert np.all(np.isnan(y[0][0, 1, 3])) and np.isnan(y[0]).sum() == 128


def test_values_that_are_not_numbers_stay_in_their_row():
    for interleaved in (False, True):
        r = Rope(1, 3, 9, 128, 64, interleaved, weights=(True, False))
        clean = r.forward()
        r.x[0][0, 1, 3, 100] = 0x7FC0
        r.x[1][0, 2, 5, 100] = 0x7F80
        r.x[1][0, 2, 6, 0] = 0x7FC0
        y = r.forward()
        assert np.all(np.isnan(y[0][0, 1, 3]))  # (the norm is of the whole row)
        hit = np.zeros(r.size, bool)
        hit[0, 1, 3] = True
        assert np.array_equal(y[0][~hit], clean[0][~hit])
        assert y[1][0, 2, 5, 100] == np.inf
        hit[:] = False
        hit[0, 2, 5, 100] = hit[0, 2, 6, 0] = hit[0, 2, 6, 1 if interleaved else 32] = True
        assert np.array_equal(y[1][~hit], clean[1][~hit]) and np.isnan(y[1][0, 2, 6, 0]) and np.isnan(y[1][0, 2, 6, 1 if interleaved else 32])


def test_gradients_against_differences():
    """A step along a direction that bf16 holds: the change of sum(g y), in 64 bits from results in bf16, against sum(dx d) and sum(dw d)."""
    r = Rope(1, 4, 64, 128, 128, seed=4)
    dx, dw = r.backward()
    rng = np.random.default_rng(9)
    g = [G.bits_f64(b) for b in r.g]
    for i in range(2):
        d = rng.choice([-1.0, 1.0], r.size)
        x = synth.bf16_bits_to_f32(r.x[i]).astype(np.float64)
        h = 2.0 ** -3
        ends = []
        for sign in (1, -1):
            s = Rope(1, 4, 64, 128, 128, seed=4)
            s.x[i] = synth.round_to_bf16_bits((x + sign * h * d).astype(np.float32))
            moved = synth.bf16_bits_to_f32(s.x[i]).astype(np.float64)
            ends.append((moved, (g[i] * s.forward()[i]).sum()))
        # the middle of the two ends is x but for their rounding: the derivative along (moved+ - moved-) / 2
        along = (ends[0][0] - ends[1][0]) / 2
        slope = (dx[i] * along).sum()
        change = (ends[0][1] - ends[1][1]) / 2
        # the results' rounding is half a step each, as if random: sqrt(n) of them; the third derivative is of the order of h^3 of a value
        n = x.size
        noise = 8 * 2.0 ** -9 * np.sqrt(n) + 4 * h ** 2 * np.sqrt(n) * h
        assert abs(change - slope) <= noise, (change, slope, noise)
        assert abs(slope) > 0
        up, down = Rope(1, 4, 64, 128, 128, seed=4), Rope(1, 4, 64, 128, 128, seed=4)
        dir_w = rng.choice([-1.0, 1.0], 128).astype(np.float32)
        up.w[i], down.w[i] = up.w[i] + np.float32(0.5) * dir_w, down.w[i] - np.float32(0.5) * dir_w
        change = (g[i] * up.forward()[i]).sum() - (g[i] * down.forward()[i]).sum()  # (linear in the weights)
        assert abs(change - (dw[i] * dir_w).sum()) <= 8 * 2.0 ** -9 * np.sqrt(n) * 2


def test_results_do_not_depend_on_the_workspace_or_the_run():
    r = Rope(3, 7, 211, 128, 128)
    a, b = r.backward(), r.backward(ws_fill=0)
    for u, v in zip(a[0] + a[1], b[0] + b[1]):
        assert np.array_equal(u, v)


def test_no_rows():
    for D in (64, 128):
        q, k = (torch.zeros(2, 3, 0, D, dtype=torch.bfloat16, device="cuda") for _ in "qk")
        w, dw = torch.ones(D, device="cuda"), [torch.full((D,), 9.0, device="cuda") for _ in "qk"]
        f = torch.from_numpy(frequencies(D)).cuda()
        B.s2_qk_norm_rope_fwd(q, k, torch.empty_like(q), torch.empty_like(k), w, w, f, EPS)
        ws = torch.empty(B.s2_qk_norm_rope_bwd_workspace_bytes(2, 3, 0, D), dtype=torch.uint8, device="cuda")
        B.s2_qk_norm_rope_bwd(q, k, q.clone(), k.clone(), torch.empty_like(q), torch.empty_like(k), w, w, dw[0], dw[1], f, EPS, ws)
        torch.cuda.synchronize()
        assert all((x == 0).all() for x in dw)


def test_another_stream_and_captured():
    r = Rope(2, 8, 64, 128, 128)
    want, (want_dx, want_dw) = r.forward(), r.backward()
    got = r.forward(stream=torch.cuda.Stream())
    assert all(np.array_equal(a, b) for a, b in zip(want, got))
    c = r.common()
    x, g, y, dx = (r.tensors(k)() for k in ("tokens", "heads", "heads", "tokens"))
    dw = [torch.empty(128, device="cuda") for _ in "qk"]
    ws = torch.empty(B.s2_qk_norm_rope_bwd_workspace_bytes(2, 8, 64, 128), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.s2_qk_norm_rope_fwd(x[0], x[1], y[0], y[1], c["w"][0], c["w"][1], c["freq"], float(r.eps))
        B.s2_qk_norm_rope_bwd(x[0], x[1], g[0], g[1], dx[0], dx[1], c["w"][0], c["w"][1], dw[0], dw[1], c["freq"], float(r.eps), ws)
    for turn in range(3):
        for i in range(2):
            x[i].copy_(G.to_dev(r.x[i]))
            g[i].copy_(G.to_dev(r.g[i]))
            y[i].fill_(turn)
            dx[i].fill_(turn)
            dw[i].fill_(turn)
        ws.fill_(turn)
        graph.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert np.array_equal(G.to_f64(y[i]), want[i]) and np.array_equal(G.to_f64(dx[i]), want_dx[i])
            assert np.array_equal(dw[i].double().cpu().numpy(), want_dw[i])

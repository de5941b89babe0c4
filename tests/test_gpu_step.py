"""The calls of a step together, as they are used: block tables from the requests' lengths, norm and rotation by the planned positions, append, attention of the new
tokens over the cache (and the decode step beside it); and norm and rotation around attention and its gradient."""

import numpy as np
import pytest
import torch

from oracle import s2_oracle as orc
from paper_2407_17678_amd import binding as B
from paper_2407_17678_amd import synth
from tests import cache_util as U
from tests import gpu_util as G
from tests.test_gpu_qk_rope import ARITHMETIC, EPS, ROUNDED, frequencies

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(np.asarray(x).tolist(), dtype=torch.int32, device="cuda")


class Server:
    """A cache, its tables and a batch of requests on the device; a step reads what it adds from `new_lens` and the first rows of `qkv`."""

    def __init__(self, fmt, D, S, nseq=3, H=3, rows=160, tokens=384, local=2, stride=3, seed=0):
        rng = np.random.default_rng([seed, D, S])
        self.fmt, self.D, self.S, self.H, self.nseq, self.rows, self.rule = fmt, D, S, H, nseq, rows, (local, stride)
        self.max_blocks, self.scale = tokens // S, 1 / np.sqrt(D)
        self.params = B.layout_params(H, 1, S, local, stride)
        pages = nseq * H * self.max_blocks
        self.pools = U.Pools(fmt, pages, S, D)
        self.table, self.ring, self.state = _ints(np.full((nseq, H, self.max_blocks), -1)), _ints(rng.permutation(pages)), _ints([pages // 2, pages])
        self.cache = self.pools.cache(self.table)
        self.lens, self.grown, self.new_lens = _ints([0] * nseq), _ints([0] * nseq), _ints([0] * nseq)
        self.cu, self.positions = _ints([0] * (nseq + 1)), _ints([0] * rows)
        self.short, self.missing = _ints([0]), _ints([0])
        self.qkv = torch.zeros(rows, 3, H, D, dtype=torch.bfloat16, device="cuda")
        self.o, self.lse = torch.zeros(rows, 3, H, D, dtype=torch.bfloat16, device="cuda")[:, 0], torch.zeros(H, rows, device="cuda")
        self.w = [(1 + 0.3 * rng.standard_normal(D)).astype(np.float32) for _ in "qk"]
        self.freq = frequencies(D)
        self.d_w, self.d_freq = [torch.from_numpy(w).cuda() for w in self.w], torch.from_numpy(self.freq).cuda()
        self.plan_ws = torch.empty(B.s2_kv_plan_workspace_bytes(nseq, H), dtype=torch.uint8, device="cuda")
        self.ws = torch.empty(B.s2_attn_chunk_workspace_bytes(nseq, H, rows, rows, D, tokens), dtype=torch.uint8, device="cuda")

    def fill(self, new, rng):
        """The next step's tokens; returns their bits."""
        total = int(sum(max(n, 0) for n in new))
        assert total <= self.rows
        bits = synth.normal_bf16(rng, (total, 3, self.H, self.D))
        self.new_lens.copy_(_ints(new))
        self.qkv[:total].copy_(G.to_dev(bits))
        return bits

    def step(self, max_new, stream=None):
        B.s2_kv_plan_paged(self.params, self.table, self.lens, self.new_lens, self.ring, self.state, self.table, self.ring, self.state, self.plan_ws,
                           cu_new=self.cu, positions=self.positions, seq_lens=self.grown, short=self.short, stream=stream)
        q, k, v = (self.qkv[:, i] for i in range(3))
        heads = lambda x: x.transpose(0, 1)[None]  # noqa: E731
        B.s2_qk_norm_rope_fwd(heads(q), heads(k), heads(q), heads(k), *self.d_w, self.d_freq, EPS, positions=self.positions[None], stream=stream)
        B.s2_kv_append_paged(self.cache, k, v, self.cu, self.lens, max_new, stream=stream)
        B.s2_attn_chunk_paged(self.params, self.cache, q, self.cu, self.lens, self.o, self.lse, self.scale, self.ws, max_new, missing=self.missing, stream=stream)

    def done(self):
        self.lens.copy_(self.grown)

    def keeps(self, h):
        local, stride = self.rule
        return lambda i, j: bool(orc.block_predicate(i, j, orc.head_offset(h, stride), local, stride, 0))

    def state_of(self):
        return [t.clone() for t in (self.table, self.ring, self.state, self.cu, self.grown, self.positions, self.qkv, self.o, self.lse, self.short, self.missing)]


STEPS = [(70, 5, 0), (1, 1, 1), (3, -1, 12), (1, 150, 1), (40, 1, 2), (1, 1, 1), (-1, 30, 0), (9, 60, 1)]


@pytest.mark.parametrize("fmt, D, S", [("bf16", 128, 64), ("mxfp8", 64, 32), ("mxfp4", 128, 64), ("bf16", 64, 128), ("mxfp8", 128, 64)])
def test_steps_of_a_batch(fmt, D, S):
    s, rng = Server(fmt, D, S), np.random.default_rng(5)
    held = [[[np.zeros((0, D)) for _ in "kv"] for _ in range(s.H)] for _ in range(s.nseq)]  # what the cache stands for
    lens = np.zeros(s.nseq, dtype=np.int64)
    table, ring, state = (t.cpu().numpy() for t in (s.table, s.ring, s.state))
    for new in STEPS:
        far = lambda h, row, j: any(s.keeps(h)(r, j) for r in range(max(row, j), max(row, j) + 8))  # noqa: E731
        plan = orc.plan_tables(table, lens, new, ring, state, far, S)
        bits = s.fill(new, rng)
        s.o.fill_(9.0)
        s.step(max(max(new), 1))
        torch.cuda.synchronize()
        table, ring, state = (t.cpu().numpy() for t in (s.table, s.ring, s.state))
        assert np.array_equal(table, plan["table"]) and np.array_equal(ring, plan["ring"]) and state.tolist() == plan["state"]
        n = len(plan["positions"])
        assert s.cu.tolist() == plan["cu_new"] and s.positions.tolist()[:n] == plan["positions"] and s.grown.tolist() == plan["seq_lens"]
        assert s.short.tolist() == [plan["short"]] == [0]
        qkv = s.qkv[:n].contiguous()
        turned = G.to_f64(qkv)
        for i in range(2):
            x = G.bits_f64(bits[:, i]).transpose(1, 0, 2)[None]
            want = orc.qk_norm_rope(x, s.w[i], [plan["positions"]], s.freq, EPS)
            size = np.abs(s.w[i] * x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS))
            both = np.tile(size[..., :D // 2] + size[..., D // 2:], 2)
            assert np.all(np.abs(turned[:, i].transpose(1, 0, 2)[None] - want) <= ROUNDED * np.abs(want) + ARITHMETIC * both)
        assert np.array_equal(turned[:, 2], G.bits_f64(bits[:, 2]))
        raw = qkv.view(torch.int16).cpu().numpy().view(np.uint16)
        o, lse, missing = G.to_f64(s.o), s.lse.double().cpu().numpy(), 0
        assert np.all(o[n:] == 9.0)
        for b in range(s.nseq):
            lo, hi = plan["cu_new"][b:b + 2]
            rows = {p // S for p in plan["positions"][lo:hi]}
            for h in range(s.H):
                if new[b] < 0:
                    held[b][h] = [np.zeros((0, D)) for _ in "kv"]
                    continue
                held[b][h] = [np.concatenate([held[b][h][i], U.held_rows(raw[lo:hi, i + 1, h], fmt)[2]]) for i in range(2)]
                resident = lambda j: table[b, h, j] >= 0  # noqa: B023, E731
                missing += sum(any(s.keeps(h)(r, j) for r in rows if r >= j) and not resident(j) for j in range(max(rows, default=-1) + 1))
                want, want_lse, weight = orc.chunk_attention(turned[lo:hi, 0, h], *held[b][h], int(lens[b]), s.keeps(h), S, s.scale, s.max_blocks * S, resident)
                assert np.all(np.abs(o[lo:hi, h] - want) <= U.attention_bound(want, weight)), (new, b, h)
                assert np.all(np.abs(lse[h, lo:hi] - want_lse) <= U.LSE_BOUND)
        assert missing == 0 and s.missing.tolist() == [0]  # (what a step's queries attend is there)
        lens = np.array(plan["seq_lens"])
        # the newest token of every sequence that has one, decoded beside it
        last = [plan["cu_new"][b + 1] - 1 for b in range(s.nseq)]
        if min(new) > 0:
            q = s.qkv[:, 0][torch.tensor(last)].contiguous()
            od = torch.empty_like(q)
            ws = torch.empty(B.s2_attn_tree_workspace_bytes(s.nseq, s.H, 1, D, s.max_blocks * S), dtype=torch.uint8, device="cuda")
            B.s2_attn_decode_paged_cache(s.params, s.cache, q, s.grown, od, None, s.scale, ws)
            weight = np.stack([np.stack([orc.chunk_attention(turned[r:r + 1, 0, h], *held[b][h], int(lens[b]) - 1, s.keeps(h), S, s.scale, s.max_blocks * S)[2][0]
                                         for h in range(s.H)]) for b, r in enumerate(last)])
            want = G.to_f64(od)
            # (rounded once each, and the chunk's probabilities once, half a step of the value)
            assert np.all(np.abs(o[last] - want) <= 2 * U.attention_bound(want, weight))
        s.done()


def test_captured_steps():
    """One graph of a step, replayed with other lengths and tokens, eager steps of the same kind and other work between: as a server without a graph."""
    made = [Server("mxfp8", 128, 64, seed=3) for _ in range(2)]
    graph, eager = made
    recorded = torch.cuda.CUDAGraph()
    with torch.cuda.graph(recorded):
        graph.step(150)
        graph.done()
    for i, new in enumerate(STEPS):
        for s in made:
            s.fill(new, np.random.default_rng([7, i]))
        if i % 3 == 2:
            graph.step(150)
            graph.done()
        else:
            recorded.replay()
        eager.step(150)
        eager.done()
        other = torch.randn(512, 512, device="cuda") @ torch.randn(512, 512, device="cuda")
        torch.cuda.synchronize()
        assert torch.isfinite(other).all()
        for a, b in zip(graph.state_of(), eager.state_of()):
            assert torch.equal(a, b), i


def test_two_servers_on_two_streams():
    """Steps of two batches at once, each on its own stream, as one after the other."""
    pair, one = [Server("bf16", 128, 64, seed=i) for i in range(2)], [Server("bf16", 128, 64, seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in pair]
    for i, new in enumerate(STEPS[:5]):
        for j, s in enumerate(pair + one):
            s.fill(new[j % 2:] + new[:j % 2], np.random.default_rng([9, i, j % 2]))
        torch.cuda.synchronize()
        for s, st in zip(pair, streams):
            s.step(150, stream=st)
        torch.cuda.synchronize()
        for s in one:
            s.step(150)
            s.done()
        for s in pair:
            s.done()
        torch.cuda.synchronize()
        for a, b in zip(pair, one):
            for x, y in zip(a.state_of(), b.state_of()):
                assert torch.equal(x, y)


@pytest.mark.parametrize("cut", [(320,), (64, 256), (1, 100, 64, 27, 128), (33,) * 9 + (23,)])
def test_a_prompt_in_chunks_is_the_whole_prompt(cut):
    """A sequence that comes in pieces against s2_attn_fwd over all of it at once."""
    D, S, N = 128, 64, 320
    s, rng = Server("bf16", D, S, nseq=1, H=4, rows=N), np.random.default_rng(11)
    bits = synth.normal_bf16(rng, (N, 3, s.H, D))
    got, kept = [], []
    for n in cut:
        s.new_lens.fill_(n)
        s.qkv[:n].copy_(G.to_dev(bits[sum(map(len, got)):][:n]))
        s.step(n)
        got.append(s.o[:n].clone())
        kept.append(s.qkv[:n].clone())
        s.done()
    q, k, v = (x.contiguous() for x in torch.cat(kept).permute(1, 2, 0, 3)[:, None])
    o, lse = torch.empty_like(q), torch.empty(1, s.H, N, device="cuda")
    layout = B.s2_layout_build(B.layout_params(s.H, N // S, S, *s.rule))
    B.s2_attn_fwd(layout, q, k, v, o, lse, s.scale)
    got, want = G.to_f64(torch.cat(got)).transpose(1, 0, 2), G.to_f64(o)[0]
    M = orc.block_mask(s.H, N // S, *s.rule)
    weight = orc.attention_forward(G.to_f64(q), G.to_f64(k), np.abs(G.to_f64(v)), M, S, s.scale)[0][0]
    assert np.all(np.abs(got - want) <= 2 * U.attention_bound(want, weight))  # (either may be off by one bound)


@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_and_rotation_around_attention_and_its_gradient(interleaved):
    """From projected queries and keys to attention, and back: gradients of the whole against the formulas' in 64 bits.  Rounded to bf16 on the way are q and k
    (2^-8 each, which shifts scores of a few units by as much), the probabilities, dO's products, dS, dq and dk before and after their way back: ten such
    steps at most, so gradients agree to 16 * 2^-8 of their norm; a term that was missing or of the other sign would be off by the most of it."""
    Bt, H, N, D, S, rng = 2, 3, 256, 64, 64, np.random.default_rng(13)
    bits = [synth.normal_bf16(rng, (Bt, N, 3, H, D)) for _ in range(2)]
    qkv, grad = (G.to_dev(b) for b in bits)
    x = [qkv[:, :, i].permute(0, 2, 1, 3) for i in range(3)]
    g = grad[:, :, 0].permute(0, 2, 1, 3).contiguous()
    w = [(1 + 0.3 * rng.standard_normal(D)).astype(np.float32) for _ in "qk"]
    dev_w, freq = [torch.from_numpy(a).cuda() for a in w], frequencies(D)
    d_freq = torch.from_numpy(freq).cuda()
    q, k = (torch.empty(Bt, H, N, D, dtype=torch.bfloat16, device="cuda") for _ in "qk")
    v = x[2].contiguous()
    o, lse = torch.empty_like(q), torch.empty(Bt, H, N, device="cuda")
    dq, dk, dv = (torch.empty_like(q) for _ in range(3))
    dx = [torch.empty_like(qkv)[:, :, i].permute(0, 2, 1, 3) for i in range(2)]
    dw = [torch.empty(D, device="cuda") for _ in "qk"]
    layout, scale = B.s2_layout_build(B.layout_params(H, N // S, S, 2, 3)), 1 / np.sqrt(D)
    ws = torch.empty(B.s2_attn_bwd_workspace_bytes(Bt, H, N, D), dtype=torch.uint8, device="cuda")
    rope_ws = torch.empty(B.s2_qk_norm_rope_bwd_workspace_bytes(Bt, H, N, D), dtype=torch.uint8, device="cuda")

    def both():
        B.s2_qk_norm_rope_fwd(x[0], x[1], q, k, *dev_w, d_freq, EPS, interleaved=interleaved)
        B.s2_attn_fwd(layout, q, k, v, o, lse, scale)
        B.s2_attn_bwd(layout, q, k, v, o, lse, g, dq, dk, dv, scale, ws)
        B.s2_qk_norm_rope_bwd(x[0], x[1], dq, dk, *dx, *dev_w, *dw, d_freq, EPS, rope_ws, interleaved=interleaved)

    both()
    torch.cuda.synchronize()
    at, M = np.broadcast_to(np.arange(N), (Bt, N)), orc.block_mask(H, N // S, 2, 3)
    x64 = [G.to_f64(t) for t in x]
    q64, k64 = (orc.qk_norm_rope(x64[i], w[i], at, freq, EPS, interleaved) for i in range(2))
    grads = orc.attention_backward(q64, k64, x64[2], G.to_f64(g), M, S, scale)
    assert G.rel_l2(G.to_f64(dv), grads[2]) <= 16 * 2.0 ** -8
    for i in range(2):
        want, want_w = orc.qk_norm_rope_backward(x64[i], w[i], at, freq, EPS, grads[i], interleaved)
        assert G.rel_l2(G.to_f64(dx[i]), want) <= 16 * 2.0 ** -8
        assert G.rel_l2(dw[i].double().cpu().numpy(), want_w) <= 16 * 2.0 ** -8
    # the same, captured, over outputs that hold something else
    kept = [t.clone() for t in (*dx, *dw, dv, o)]
    recorded = torch.cuda.CUDAGraph()
    with torch.cuda.graph(recorded):
        both()
    for turn in range(3):
        for t in (*dx, *dw, dq, dk, dv, o, q, k, lse):
            t.fill_(turn)
        recorded.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, (*dx, *dw, dv, o)))

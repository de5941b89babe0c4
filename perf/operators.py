"""What a serving program asks of a paged KV cache: rows written into it (quantised on the way), rows read back, a decode step over it,
and the attention of a tree of drafted tokens over it.

A cache is a pool of pages for keys and one for values, a page holding the block_size tokens of one block of one (sequence, head), and a
table of page numbers [nseq, heads, max_blocks], negative where a block is not held.  Formats: bf16; mxfp8 (e4m3) and mxfp4 (e2m1, two to a byte,
the even feature in the low half), with one power of two to 32 features of a row, held as a byte (exponent + 127).
"""

import math

import numpy as np
import torch

own = False

SPLITS_BYTES = 256 << 20  # the workspace that a program keeps for its attention calls

# ------------------------------------------------------------------------------------ cases


def _mask(block_size, local_blocks, stride):
    return {"block_size": block_size, "local_blocks": local_blocks, "stride": stride}


def listed():
    return [
        # a serving batch writes the one token of a decode step: a launch's latency
        dict(name="append_step", kind="append", fmt="mxfp8", nseq=64, heads=32, head_dim=128, min_len=8192, max_len=32768, min_new=1, max_new=1,
             len_seed=5, **_mask(64, 16, 16)),
        # prompts of any length go in, of which a head holds what later tokens attend
        dict(name="append_prompts", kind="append", fmt="mxfp8", nseq=8, heads=32, head_dim=128, min_len=0, max_len=0, min_new=1001, max_new=16384,
             len_seed=6, **_mask(64, 16, 16)),
        # a small model's prompts in the finest blocks, not quantised, some sequences without a new token
        dict(name="append_fine", kind="append", fmt="bf16", nseq=11, heads=7, head_dim=64, min_len=0, max_len=1500, min_new=0, max_new=777,
             len_seed=7, **_mask(16, 16, 32)),
        # a chunk of a long prompt in 4 bits: written, and the whole read back for the chunk's attention
        dict(name="chunk_fp4", kind="chunk", fmt="mxfp4", nseq=1, heads=32, head_dim=128, min_len=30720, max_len=30720, min_new=2048, max_new=2048,
             len_seed=5, **_mask(64, 16, 16)),
        # a context that is taken up again: all of it read back
        dict(name="read_32k", kind="read", fmt="mxfp8", nseq=1, heads=32, head_dim=128, min_len=32768, max_len=32768, len_seed=5,
             **_mask(64, 16, 16)),
        # a serving batch's decode step
        dict(name="decode_fp8_64", kind="decode", fmt="mxfp8", nseq=64, heads=32, head_dim=128, min_len=8192, max_len=32768, len_seed=5,
             **_mask(64, 16, 16)),
        # the same with the smallest cache: 4 bits, 16-token blocks
        dict(name="decode_fp4_64", kind="decode", fmt="mxfp4", nseq=64, heads=32, head_dim=128, min_len=8192, max_len=32768, len_seed=5,
             **_mask(16, 64, 64)),
        # a single user's decode step
        dict(name="decode_fp8_one", kind="decode", fmt="mxfp8", nseq=1, heads=32, head_dim=128, min_len=32768, max_len=32768, len_seed=5,
             **_mask(64, 16, 16)),
        # wide trees over a bf16 cache
        dict(name="tree_bf16_64", kind="tree", fmt="bf16", nseq=16, heads=32, head_dim=128, min_len=8192, max_len=32768, nodes=64, len_seed=5,
             **_mask(64, 16, 16)),
        # a serving batch with a tree of ordinary size to each sequence
        dict(name="tree_fp8_24", kind="tree", fmt="mxfp8", nseq=64, heads=32, head_dim=128, min_len=8192, max_len=32768, nodes=24, len_seed=5,
             **_mask(64, 16, 16)),
        # an odd number of everything, short contexts (the first ones empty), 4 bits
        dict(name="tree_fp4_odd", kind="tree", fmt="mxfp4", nseq=7, heads=13, head_dim=64, min_len=0, max_len=5001, nodes=33, len_seed=9,
             **_mask(32, 8, 16)),
        # a single user's few drafted tokens
        dict(name="tree_one", kind="tree", fmt="bf16", nseq=1, heads=32, head_dim=128, min_len=32768, max_len=32768, nodes=8, len_seed=5,
             **_mask(64, 16, 16)),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    while True:
        S = rng.choice([16, 32, 64, 64, 128])
        case = dict(kind=rng.choice(["append", "append", "chunk", "read", "decode", "decode", "tree", "tree", "tree"]),
                    fmt=rng.choice(["bf16", "mxfp8", "mxfp8", "mxfp4", "mxfp4"]), nseq=round(_log_uniform(rng, 1, 64)), heads=rng.randint(1, 32),
                    head_dim=rng.choice([64, 128, 128]), len_seed=rng.randrange(1 << 20),
                    **_mask(S, max(1, round(_log_uniform(rng, 16, 1024) / S)), max(2, round(_log_uniform(rng, 256, 2048) / S))))
        if case["kind"] == "append" and case["fmt"] == "mxfp4":
            case["kind"] = "chunk"  # (what is held in 4 bits comes back as values)
        lo = round(_log_uniform(rng, 1, 32768)) - 1
        hi = min(32768, round((lo + 1) * rng.uniform(1.0, 4.0)))
        if case["kind"] == "append":
            new = round(_log_uniform(rng, 1, 16384)) if rng.random() < 0.7 else 1
            case.update(min_len=lo, max_len=hi, min_new=rng.randint(0, new), max_new=new)
        elif case["kind"] == "chunk":
            new = round(_log_uniform(rng, 1, 4096))
            case.update(min_len=lo, max_len=hi, min_new=rng.randint(0, new), max_new=new)
        elif case["kind"] == "tree":
            case.update(min_len=lo, max_len=hi, nodes=round(_log_uniform(rng, 1, 64)))
        else:
            if case["kind"] == "decode" and case["fmt"] == "bf16":
                case["fmt"] = "mxfp8"  # (a decode step over a bf16 cache is no new operator)
            case.update(min_len=max(1, lo), max_len=max(1, hi))
        w = work(case)
        # no state larger than the listed ones', no pass longer
        held = int(_resident(case).sum()) * S * 2 * (case["head_dim"] * 2 + 4)
        if w["bytes"] > 0 and w["bytes"] < 1.5e9 and w["flops"] < 1e11 and held < 3e9 and _lengths(case)[1].sum() * case["heads"] < 4e6:
            return case


# ------------------------------------------------------------------------------------ what a case holds


def _lengths(case):
    """Tokens cached before the call, and tokens that the call writes or reads, of each sequence: part of the case."""
    rng = np.random.Generator(np.random.PCG64([20240717, case["len_seed"]]))
    lens = rng.integers(case["min_len"], case["max_len"] + 1, size=case["nseq"])
    if case["kind"] in ("append", "chunk"):
        lo, hi = case["min_new"], case["max_new"]
        new = np.exp(rng.uniform(np.log(lo + 1), np.log(hi + 1.999), size=case["nseq"])).astype(np.int64) - 1
        return lens, np.clip(new, lo, hi)
    return lens, lens if case["kind"] == "read" else np.zeros_like(lens)


def _used(case):
    """Nodes of each sequence's tree (the rest of the rows is padding)."""
    rng = np.random.Generator(np.random.PCG64([case["len_seed"], 1]))
    return rng.integers((case["nodes"] + 1) // 2, case["nodes"] + 1, size=case["nseq"])


def _max_blocks(case):
    lens, new = _lengths(case)
    ends = lens + (0 if case["kind"] == "read" else new) + (case["nodes"] if case["kind"] == "tree" else 0)
    return max(1, -(-int(ends.max()) // case["block_size"]))


def _keeps(case, row, col, head):
    """Whether block row `row` of a head's mask keeps block column `col`: the local window, and a stripe every `stride` blocks."""
    back = row - col
    return (back >= 0) & ((back < case["local_blocks"]) | ((col - head) % case["stride"] == 0))


def _resident(case):
    """[nseq, heads, blocks]: the blocks that the cache holds, those that a token from the call on can attend."""
    S, (lens, new) = case["block_size"], _lengths(case)
    end = lens + (new if case["kind"] in ("append", "chunk") else 0)
    col, head = np.arange(_max_blocks(case))[None, None, :], np.arange(case["heads"])[None, :, None]
    exists = col * S < end[:, None, None]
    if case["kind"] == "read":
        return np.broadcast_to(exists, (case["nseq"], case["heads"], col.size)).copy()
    # a chunk's own rows attend too; else the newest token's row is the first that matters
    first = (lens if case["kind"] == "chunk" else np.maximum(end, 1) - 1) // S
    row = first[:, None, None]
    return exists & (_keeps(case, row, col, head) | (col >= row))


def _row_bytes(case):
    D = case["head_dim"]
    return {"bf16": 2 * D, "mxfp8": D + D // 32, "mxfp4": D // 2 + D // 32}[case["fmt"]]


def _attended(case):
    """Cached tokens that the heads of each sequence attend, summed over heads."""
    S, (lens, _) = case["block_size"], _lengths(case)
    col, head = np.arange(_max_blocks(case))[None, None, :], np.arange(case["heads"])[None, :, None]
    at = lens if case["kind"] == "tree" else lens - 1
    kept = _keeps(case, (at // S)[:, None, None], col, head) & (col * S < lens[:, None, None])
    tokens = np.clip(lens[:, None, None] - col * S, 0, S)
    # (as the last cached token's block row goes on: a tree that reaches into the next block reads a block more at most)
    return (kept * tokens).sum((1, 2))


def work(case):
    D, H = case["head_dim"], case["heads"]
    lens, new = _lengths(case)
    if case["kind"] in ("append", "chunk", "read"):
        S, res = case["block_size"], _resident(case)
        col = np.arange(res.shape[2])[None, :]
        tokens = lambda lo, hi: np.clip(np.minimum(hi[:, None], (col + 1) * S) - np.maximum(lo[:, None], col * S), 0, None)  # noqa: E731
        held = lambda lo, hi: int((res.sum(1) * tokens(lo, hi)).sum())  # noqa: E731
        if case["kind"] == "read":
            rows = held(np.zeros_like(lens), lens)
            return {"bytes": 2 * (rows * _row_bytes(case) + int(lens.sum()) * H * 2 * D), "flops": 2 * rows * D}
        rows = held(lens, lens + new)
        b, f = 2 * rows * (2 * D + _row_bytes(case)), 6 * rows * D
        if case["kind"] == "chunk":
            back = held(np.zeros_like(lens), lens + new)
            b, f = b + 2 * (back * _row_bytes(case) + int((lens + new).sum()) * H * 2 * D), f + 2 * back * D
        return {"bytes": b, "flops": f}
    tokens = _attended(case)
    b = 2 * int(tokens.sum()) * _row_bytes(case)
    if case["kind"] == "decode":
        return {"bytes": b + case["nseq"] * H * (4 * D + 4), "flops": 4 * int(tokens.sum()) * D}
    used, T = _used(case), case["nodes"]
    return {"bytes": b + int(used.sum()) * H * 6 * D + case["nseq"] * H * T * (2 * D + 4), "flops": 4 * D * int((tokens * used).sum())}


# ------------------------------------------------------------------------------------ quantised rows, in elementary operations


def _power(e):
    """2^e for whole e in [-126, 127], exactly."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _quantise(x, fmt):
    """x [..., D] -> (codes, scale bytes): per 32 features the smallest power of two 2^e, e >= -110, with max |x| 2^-e below 464 (e4m3: the middle
    between its largest number and the step after it) or 7 (e2m1)."""
    b = x.float().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1)
    m, e = torch.frexp(top)  # top = m 2^e, m in [1/2, 1)
    e = e - 9 + (m >= 464 / 512).int() if fmt == "mxfp8" else e - 3 + (m >= 7 / 8).int()
    wild = ~(top < 2.0 ** 127)
    e = torch.where((top == 0) | wild, -110, e.clamp(min=-110))
    y = torch.where(wild[..., None], torch.zeros_like(b), b) * _power(-e)[..., None]
    byte = torch.where(wild, 255, e + 127).to(torch.uint8)
    if fmt == "mxfp8":
        return y.to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2), byte
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.round(a / step) * step  # (to the even one of two neighbours that are as near)
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    code = code.flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), byte


def _values(codes, byte, fmt):
    """What (codes, scale bytes) stand for, in float32; bf16 rows as they are."""
    if fmt == "bf16":
        return codes.float()
    if fmt == "mxfp8":
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
        table = torch.cat([table, -table])
        v = table[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    return (v.unflatten(-1, (-1, 32)) * (byte.int() << 23).view(torch.float32)[..., None]).flatten(-2)


# ------------------------------------------------------------------------------------ inputs


def _rows(g, shape, spread):
    """Keys or values as a model makes them: normal, with features that are larger than others."""
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    return x.mul_(spread)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, H, D, S, fmt = (case[k] for k in ("nseq", "heads", "head_dim", "block_size", "fmt"))
    lens, new = _lengths(case)
    ints = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(torch.int32).cuda()  # noqa: E731
    res = torch.from_numpy(_resident(case)).cuda()
    pages = int(res.sum()) + 3
    order = torch.randperm(pages, generator=g, device="cuda", dtype=torch.int32)
    table = torch.where(res, order[(res.flatten().cumsum(0) - 1).clamp(min=0).view_as(res)], -1).to(torch.int32)
    spread = torch.exp2(torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16)
    s = {"case": case, "table": table, "lens": ints(lens)}
    for name in ("k", "v"):
        rows = _rows(g, (pages, S, D), spread if name == "k" else 1.0)
        if fmt == "bf16":
            s[name + "_pages"], s[name + "_scales"] = rows, None
        else:
            parts = [_quantise(r, fmt) for r in rows.split(max(1, (1 << 27) // (S * D)))]
            codes = torch.cat([p[0] for p in parts])
            s[name + "_pages"], s[name + "_scales"] = codes.view(torch.float8_e4m3fn) if fmt == "mxfp8" else codes, torch.cat([p[1] for p in parts])
            del parts
        del rows
    if case["kind"] in ("append", "chunk"):
        cu = np.concatenate([[0], np.cumsum(new)])
        s["cu_new"], s["max_new"] = ints(cu), max(1, int(new.max()))
        s["k"], s["v"] = (_rows(g, (int(cu[-1]), H, D), x) for x in (spread, 1.0))
    if case["kind"] in ("chunk", "read"):
        all_ = lens + (new if case["kind"] == "chunk" else 0)
        cu = np.concatenate([[0], np.cumsum(all_)])
        s["cu_read"], s["max_read"], s["from"] = ints(cu), max(1, int(all_.max())), ints(0 * lens)
        s["k_out"], s["v_out"] = (torch.empty((H, int(cu[-1]), D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    if case["kind"] in ("decode", "tree"):
        T = case.get("nodes", 1)
        s["scale"] = 1.0 / math.sqrt(D)
        s["most"] = int((_resident(case).sum(-1)).max())  # blocks that a table row holds at most
        s["workspace"] = torch.empty(SPLITS_BYTES, dtype=torch.uint8, device="cuda")
        # as a model's projections leave them: [sequence, token, head, feature]
        q = _rows(g, (n, T, H, D), 1.0 / spread)
        s["o"] = torch.empty_like(q)
        s["lse"] = torch.empty((n, H, T), dtype=torch.float32, device="cuda")
        if case["kind"] == "decode":
            s["q"], s["o"], s["lse"] = q[:, 0], s["o"][:, 0], s["lse"][..., 0]
        else:
            kd, vd = (_rows(g, (n, T, H, D), x) for x in (spread, 1.0))
            s["q"], s["o"], s["k_draft"], s["v_draft"] = (x.permute(0, 2, 1, 3) for x in (q, s["o"], kd, vd))
            node = torch.arange(T, device="cuda")
            # node i hangs on an earlier one or on the last cached token
            parents = (torch.rand((n, T), generator=g, device="cuda") * (node + 1)).floor().int() - 1
            s["parents"] = torch.where(node < ints(_used(case))[:, None], parents, -2).to(torch.int32)
    return s


# ------------------------------------------------------------------------------------ one pass


def _plain_append(s):
    case, S = s["case"], s["case"]["block_size"]
    H, maxb = s["table"].shape[1:]
    row = torch.arange(s["k"].shape[0], device="cuda")
    seq = torch.searchsorted(s["cu_new"][1:].contiguous(), row, right=True)
    pos = s["lens"][seq] + row - s["cu_new"][seq]
    page = s["table"][seq[:, None], torch.arange(H, device="cuda"), (pos // S)[:, None]]  # [row, head]
    held = page >= 0
    to = (page.long() * S + (pos % S)[:, None])[held]
    for name in ("k", "v"):
        x, pool, scales = s[name][held], s[name + "_pages"], s[name + "_scales"]
        if case["fmt"] == "bf16":
            pool.view(-1, pool.shape[-1])[to] = x
        else:
            codes, byte = _quantise(x, case["fmt"])
            pool.view(torch.uint8).view(-1, codes.shape[-1])[to] = codes
            scales.view(-1, byte.shape[-1])[to] = byte


def _plain_read(s):
    case, S = s["case"], s["case"]["block_size"]
    row = torch.arange(s["k_out"].shape[1], device="cuda")
    seq = torch.searchsorted(s["cu_read"][1:].contiguous(), row, right=True)
    pos = s["from"][seq] + row - s["cu_read"][seq]
    page = s["table"][seq, :, pos // S].T  # [head, row]
    for name in ("k", "v"):
        pool, scales = s[name + "_pages"], s[name + "_scales"]
        at = page.clamp(min=0).long() * S + pos % S
        got = _values(pool.view(-1, pool.shape[-1])[at], None if scales is None else scales.view(-1, scales.shape[-1])[at], case["fmt"])
        s[name + "_out"].copy_(torch.where((page >= 0)[..., None], got, 0.0))


def _plain_attention(s):
    case, S = s["case"], s["case"]["block_size"]
    n, H, maxb = s["table"].shape
    tree = case["kind"] == "tree"
    lens = s["lens"]
    head, col = torch.arange(H, device="cuda"), torch.arange(maxb, device="cuda")
    if tree:
        par = s["parents"].long()
        T = par.shape[1]
        node = torch.arange(T, device="cuda")
        there = par >= -1
        # ancestors, itself among them: the closure of "is the parent of", doubled as often as a chain of all nodes needs
        up = (par[..., None] == node) | torch.eye(T, dtype=torch.bool, device="cuda")
        for _ in range(6):
            up = up.float().matmul(up.float()) > 0
        pos = lens[:, None] + up.sum(-1) - 1
        q = s["q"].float()
    else:
        pos = lens[:, None] - 1
        q = s["q"][:, :, None].float()
    # the blocks that the tables hold, side by side; what a row of the mask keeps of them
    blk = (s["table"] < 0).to(torch.int8).argsort(dim=-1, stable=True)[..., :s["most"]]
    page = s["table"].gather(-1, blk)
    kept = _keeps(case, (pos // S)[:, None, :, None], blk[:, :, None], head[:, None, None]) & (page >= 0)[:, :, None]  # [n, H, T, C]
    tok = blk[..., None] * S + torch.arange(S, device="cuda")
    seen = (kept[..., None] & (tok < lens[:, None, None, None])[:, :, None]).flatten(-2)
    at = page.clamp(min=0).long()

    def held(name):
        pool, scales = s[name + "_pages"], s[name + "_scales"]
        return _values(pool[at], None if scales is None else scales[at], case["fmt"]).flatten(2, 3)

    score = q.matmul(held("k").transpose(-1, -2)) * s["scale"]
    score = torch.where(seen, score, -math.inf)
    if tree:
        ours = _keeps(case, (pos // S)[:, None, :, None], (pos // S)[:, None, None, :], head[:, None, None]) & up[:, None]
        drafted = q.matmul(s["k_draft"].float().transpose(-1, -2)) * s["scale"]
        score = torch.cat([score, torch.where(ours & there[:, None, :, None], drafted, -math.inf)], -1)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    cached = tok.shape[-1] * tok.shape[-2]
    o = p[..., :cached].matmul(held("v"))
    if tree:
        o = o + p[..., cached:].matmul(s["v_draft"].float())
    o = torch.where(total > 0, o / total, 0.0)
    lse = (torch.log(total) + torch.where(total > 0, top, 0.0))[..., 0]
    if tree:
        o, lse = torch.where(there[:, None, :, None], o, 0.0), torch.where(there[:, None], lse, -math.inf)
    s["o"].copy_(o if tree else o[:, :, 0])
    s["lse"].copy_(lse if tree else lse[..., 0])


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        from paper_2407_17678_amd import binding as B
        cache = B.paged_cache({"bf16": B.KV_BF16, "mxfp8": B.KV_MXFP8, "mxfp4": B.KV_MXFP4}[case["fmt"]], case["block_size"], s["k_pages"],
                              s["v_pages"], s["table"], s["k_scales"], s["v_scales"])
        if kind in ("append", "chunk"):
            B.s2_kv_append_paged(cache, s["k"], s["v"], s["cu_new"], s["lens"], s["max_new"])
        if kind in ("chunk", "read"):
            B.s2_kv_read_paged(cache, s["k_out"], s["v_out"], s["cu_read"], s["from"], s["max_read"])
        if kind in ("decode", "tree"):
            mask = B.layout_params(case["heads"], 1, case["block_size"], case["local_blocks"], case["stride"])
            if kind == "decode":
                B.s2_attn_decode_paged_cache(mask, cache, s["q"], s["lens"], s["o"], s["lse"], s["scale"], s["workspace"])
            else:
                B.s2_attn_tree_paged(mask, cache, s["q"], s["k_draft"], s["v_draft"], s["parents"], s["lens"], s["o"], s["lse"], s["scale"],
                                     s["workspace"])
    else:
        if kind in ("append", "chunk"):
            _plain_append(s)
        if kind in ("chunk", "read"):
            _plain_read(s)
        if kind in ("decode", "tree"):
            _plain_attention(s)
    if kind == "append":
        return {x: s[x] for x in ("k_pages", "v_pages", "k_scales", "v_scales") if s[x] is not None}
    return {"k": s["k_out"], "v": s["v_out"]} if kind in ("chunk", "read") else {"o": s["o"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------ the same by definition, in 64 bits


def _nearest(x, digits, least):
    """x to the nearest number of `digits` binary places after the leading one (ties to even), spaced as at 2^least below it."""
    _, e = torch.frexp(x.abs())
    quantum = torch.exp2((torch.clamp(e - 1, min=least) - digits).double())
    return torch.round(x / quantum) * quantum


def _as_held(x, fmt):
    """What rows x read back as once they are written."""
    x = x.double()
    if fmt == "bf16":
        return x, x
    b = x.unflatten(-1, (-1, 32))
    digits, least, limit = (3, -6, 464.0) if fmt == "mxfp8" else (1, 0, 7.0)
    top = b.abs().amax(-1, keepdim=True)
    guess = torch.floor(torch.log2(top.clamp(min=2.0 ** -120)))
    tried = torch.clamp(guess - torch.arange(12, device="cuda"), min=-110.0)  # the smallest that does is among these
    e = torch.where(top / torch.exp2(tried) < limit, tried, math.inf).amin(-1, keepdim=True)
    codes = _nearest(b / torch.exp2(e), digits, least)
    return codes.flatten(-2), (codes * torch.exp2(e)).flatten(-2)


def _decoded(codes, byte, fmt):
    """The values of held rows, bit field by bit field."""
    if fmt == "bf16":
        return codes.double()
    if fmt == "mxfp8":
        c = codes.view(torch.uint8).long()
        ex, m, sign, low, bias, width = (c >> 3) & 15, c & 7, c >> 7, 3, 7, 32
    else:
        c = torch.stack([codes.long() & 15, codes.long() >> 4], -1).flatten(-2)
        ex, m, sign, low, bias, width = (c >> 1) & 3, c & 1, c >> 3, 1, 1, 32
    v = torch.where(ex > 0, (1 + m / 2.0 ** low) * torch.exp2((ex - bias).double()), m.double() * 2.0 ** (1 - bias - low))
    v = v * (1 - 2 * sign)
    return (v.unflatten(-1, (-1, width)) * torch.exp2(byte.double() - 127)[..., None]).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    fmt, S, D, H = case["fmt"], case["block_size"], case["head_dim"], case["heads"]
    table, lens = s["table"].cpu(), s["lens"].tolist()
    result = {}
    if case["kind"] in ("append", "chunk", "read"):
        for name in ("k", "v"):
            pool = s[name + "_pages"]
            values = torch.cat([_decoded(p, None if fmt == "bf16" else q, fmt) for p, q in
                                zip(pool.split(4096), [None] * (1 + len(pool) // 4096) if fmt == "bf16" else s[name + "_scales"].split(4096))])
            codes = pool.double() if fmt != "mxfp4" else None
            for b in range(case["nseq"] if "cu_new" in s else 0):
                lo, hi = s["cu_new"][b:b + 2].tolist()
                for blk in range(lens[b] // S, -(-(lens[b] + hi - lo) // S)):
                    t0, t1 = max(lens[b], blk * S), min(lens[b] + hi - lo, (blk + 1) * S)
                    heads = torch.nonzero(table[b, :, blk] >= 0)[:, 0].cuda()
                    if t1 <= t0 or not len(heads):
                        continue
                    rows = s[name][lo + t0 - lens[b]:lo + t1 - lens[b]].transpose(0, 1)[heads]
                    code, value = _as_held(rows, fmt)
                    pages = s["table"][b, heads, blk].long()
                    values[pages, t0 - blk * S:t1 - blk * S] = value
                    if codes is not None:
                        codes[pages, t0 - blk * S:t1 - blk * S] = code
            if case["kind"] == "append":
                result[name + "_pages"], result[name + "_scales"] = codes, None
                continue
            out = torch.zeros(s[name + "_out"].shape, dtype=torch.float64, device="cuda")
            for b in range(case["nseq"]):
                lo, hi = s["cu_read"][b:b + 2].tolist()
                nb = -(-(hi - lo) // S)
                page = s["table"][b, :, :nb].long()
                got = values[page.clamp(min=0)] * (page >= 0)[..., None, None]
                out[:, lo:hi] = got.flatten(1, 2)[:, :hi - lo]
            result[name] = out
        return {k: v for k, v in result.items() if s.get(k, 0) is not None}
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    head = torch.arange(H, device="cuda")[:, None]
    for b in range(case["nseq"]):
        L = lens[b]
        nb = -(-L // S)
        page = s["table"][b, :, :nb].long().clamp(min=0)
        k, v = (_decoded(s[x + "_pages"][page], None if fmt == "bf16" else s[x + "_scales"][page], fmt).flatten(1, 2)[:, :L] for x in "kv")
        block = torch.arange(L, device="cuda") // S
        chains = [[0]] if case["kind"] == "decode" else []
        if case["kind"] == "tree":
            for p in s["parents"][b].tolist():
                chains.append(None if p < -1 else (chains[p] if p >= 0 else []) + [len(chains)])
        for i, chain in enumerate(chains):
            if chain is None:
                continue
            at = L - 1 if case["kind"] == "decode" else L + len(chain) - 1
            sees = _keeps(case, at // S, block[None], head)
            q = (s["q"][b] if case["kind"] == "decode" else s["q"][b, :, i]).double()
            score = torch.where(sees, (k * q[:, None]).sum(-1) * s["scale"], -math.inf)
            kept_v = [v]
            if case["kind"] == "tree":
                where = torch.tensor([(L + j) // S for j in range(len(chain))], device="cuda")
                sees = _keeps(case, at // S, where[None], head)
                kd, vd = (s[x][b][:, chain].double() for x in ("k_draft", "v_draft"))
                score = torch.cat([score, torch.where(sees, (kd * q[:, None]).sum(-1) * s["scale"], -math.inf)], 1)
                kept_v.append(vd)
            w = torch.softmax(score, -1)
            to = (b, slice(None)) if case["kind"] == "decode" else (b, slice(None), i)
            at_v, total = 0, 0
            for x in kept_v:
                total = total + torch.matmul(w[:, None, at_v:at_v + x.shape[1]], x)[:, 0]
                at_v += x.shape[1]
            o[to], lse[to] = total, torch.logsumexp(score, -1)
    return {"o": o, "lse": lse}

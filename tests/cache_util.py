"""Helpers of the tests of a paged cache in several formats: pools on the device, the bound on attention's errors."""

import numpy as np
import torch

from oracle import s2_oracle as orc
from paper_2407_17678_amd import binding as B
from paper_2407_17678_amd import synth

FORMATS = {"bf16": B.KV_BF16, "mxfp8": B.KV_MXFP8, "mxfp4": B.KV_MXFP4}


def pack(codes, fmt):
    """Codes [..., D] as they lie in a page."""
    return codes if fmt == "mxfp8" else (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(held, fmt):
    return held if fmt == "mxfp8" else np.stack([held & 15, held >> 4], axis=-1).reshape(held.shape[:-1] + (-1,))


def row_bytes(D, fmt):
    return {"bf16": 2 * D, "mxfp8": D, "mxfp4": D // 2}[fmt]


def held_rows(bits, fmt):
    """bf16 rows (bit patterns) -> (what pages hold of them, scale bytes or None, the float64 values they read back as)."""
    if fmt == "bf16":
        return bits, None, synth.bf16_bits_to_f32(bits).astype(np.float64)
    codes, byte = orc.mx_quantise(synth.bf16_bits_to_f32(bits), fmt)
    return pack(codes, fmt), byte, orc.mx_values(codes, byte, fmt)


class Pools:
    """K and V pools with a margin of bytes after every token and page (gap), filled with a byte that is no sensible value."""

    def __init__(self, fmt, pages, S, D, gap=0, fill=0xFF):
        rb = row_bytes(D, fmt)
        self.fmt, self.shape = fmt, (pages, S, D)
        self.data, self.scales = [], []
        for _ in "kv":
            raw = torch.full((pages, S, rb + gap), fill, dtype=torch.uint8, device="cuda")
            x = raw if fmt != "bf16" else raw.view(torch.bfloat16)
            self.data.append(x[..., :D if fmt != "mxfp4" else D // 2])
            s = torch.full((pages, S, D // 32 * (2 if gap else 1)), fill, dtype=torch.uint8, device="cuda")
            self.scales.append(s[..., :D // 32] if fmt != "bf16" else None)

    def cache(self, table):
        return B.paged_cache(FORMATS[self.fmt], self.shape[1], self.data[0], self.data[1], table, *self.scales)

    def host(self, which):
        """(held bytes or bf16 bits, scale bytes) as numpy."""
        x = self.data[which]
        x = x.contiguous().view(torch.int16).cpu().numpy().view(np.uint16) if self.fmt == "bf16" else x.cpu().numpy()
        return x, None if self.fmt == "bf16" else self.scales[which].cpu().numpy()

    def put(self, which, page, token, held, byte):
        """Rows of one page from the host."""
        n = held.shape[0]
        t = torch.from_numpy(np.ascontiguousarray(held))
        if self.fmt == "bf16":
            t = torch.from_numpy(np.ascontiguousarray(held).view(np.int16)).view(torch.bfloat16)
        self.data[which][page, token:token + n] = t.cuda()
        if byte is not None:
            self.scales[which][page, token:token + n] = torch.from_numpy(np.ascontiguousarray(byte)).cuda()


def attention_bound(o, weight):
    """How far a bf16 output may be off.  Its own rounding, and that of each p_j to bf16 before the product with V: half a step, 2^-8 of the
    value, each.  Sums and exponentials in 32 bits: a score is a sum of up to 128 products, off by at most 128 * 2^-24 of the sum of their
    magnitudes, for normal values below 100 after scaling, so p_j by at most 2^-10 with its exponential; weight = sum_j p_j |v_j|."""
    return 2.0 ** -8 * (np.abs(o) + weight) * (1 + 2.0 ** -7) + 2.0 ** -10 * weight + 1e-30


LSE_BOUND = 1e-3

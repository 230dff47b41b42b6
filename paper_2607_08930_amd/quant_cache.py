"""The dual cache of all layers held in 8 bits, for the step and the server.

Codes lie where the bf16 cache has its cells, [layers][R][Hkv][W][D] of one byte;
every T tokens of a head share an fp32 scale, [layers][R][Hkv][S]. Groups run both
ways from a row's first generated token, so a block of L tokens is whole groups
whenever T divides L, and a step's write replaces whole groups.
"""
from __future__ import annotations

import numpy as np
import torch

from . import (BS_BF16, BS_E4M3, BS_F32, BS_I8, REQ_DTYPE, Context, bs_kv_dequantize, bs_kv_quantize,
               bs_kv_scatter_compact, bs_quant_cache_block_attention)

FORMATS = {"e4m3": BS_E4M3, "i8": BS_I8}


def largest_group(L: int) -> int:
    """The largest T that divides L: a power of two, 64 at most."""
    return min(L & -L, 64)


class QuantCache:
    def __init__(self, layers: int, R: int, W: int, Hkv: int, D: int, L: int, fmt: str = "e4m3", T: int = 0,
                 device="cuda", empty: bool = False):
        """empty: leave the memory as it comes (rows are read only after they are written)."""
        if fmt not in FORMATS:
            raise ValueError(f"an 8-bit cache is one of {sorted(FORMATS)}, not {fmt!r}")
        self.layers, self.R, self.W, self.Hkv, self.D, self.L = layers, R, W, Hkv, D, L
        self.name, self.fmt, self.T = fmt, FORMATS[fmt], T or largest_group(L)
        if L < 1 or self.T not in (1, 2, 4, 8, 16, 32, 64) or L % self.T:
            raise ValueError(f"groups of T={self.T} tokens: a power of two up to 64 that divides L={L}")
        # a row of up to W tokens has at most W / T + 2 groups; scale rows move in cells of four
        self.S = -(-(W // self.T + 2) // 4) * 4
        codes, scales = (layers, R, Hkv, W, D), (layers, R, Hkv, self.S)
        self.k, self.v = (torch.empty(codes, dtype=torch.uint8, device=device) for _ in range(2))
        self.k_scale, self.v_scale = (torch.empty(scales, dtype=torch.float32, device=device) for _ in range(2))
        if not empty:
            for x, fill in ((self.k, 0), (self.v, 0), (self.k_scale, 1.0), (self.v_scale, 1.0)):
                x.fill_(fill)

    def write(self, ctx: Context, reqs: np.ndarray, layer: int, k, v, stream=None) -> None:
        """Quantises the rows of ``reqs`` from the bf16 box k, v [R][Hkv][W][D]."""
        bs_kv_quantize(ctx, reqs, self.L, self.R, self.W, self.Hkv, self.D, BS_BF16, self.fmt, self.T, k, v,
                       self.k[layer], self.v[layer], self.k_scale[layer], self.v_scale[layer], self.S, stream=stream)

    def read(self, ctx: Context, reqs: np.ndarray, layer: int, k, v, stream=None) -> None:
        """Writes the numbers that the rows of ``reqs`` hold into the bf16 box k, v."""
        bs_kv_dequantize(ctx, reqs, self.L, self.R, self.W, self.Hkv, self.D, BS_BF16, self.fmt, self.T, self.k[layer],
                         self.v[layer], self.k_scale[layer], self.v_scale[layer], self.S, k, v, stream=stream)

    def attend(self, ctx: Context, reqs: np.ndarray, layer: int, q, k_new, v_new, out, *, Hq: int, scale: float = 0.0,
               write_back: bool = True, ws=None, ws_bytes: int = 0, stream=None) -> None:
        bs_quant_cache_block_attention(ctx, reqs, self.L, Hq, self.Hkv, self.D, self.fmt, self.T, scale, q, k_new, v_new,
                                       self.k[layer], self.v[layer], self.k_scale[layer], self.v_scale[layer], self.S,
                                       self.R, self.W, write_back, out, ws, ws_bytes, stream=stream)

    def admit(self, ctx: Context, segs: np.ndarray, p, g, stg_k, stg_v) -> None:
        """Quantises staged rows and moves them in, on the current stream. stg_k, stg_v: bf16
        [layers][n][Hkv][Ws][D], row a holding a request of prompt length p[a] and generation length g[a]
        from column 0; ``segs`` (SEG_DTYPE) says where the staged rows go, as for a bf16 cache."""
        n, Ws = stg_k.shape[1], stg_k.shape[3]
        stg = QuantCache(self.layers, n, Ws, self.Hkv, self.D, self.L, self.name, self.T, self.k.device, empty=True)
        reqs = np.zeros(n, REQ_DTYPE)
        reqs["p"], reqs["g"], reqs["row"] = p, g, np.arange(n)
        for l in range(self.layers):
            stg.write(ctx, reqs, l, stg_k[l], stg_v[l])
        self.move(ctx, segs, None, stg)

    def move(self, ctx: Context, segs: np.ndarray, src: QuantCache | None, stg: QuantCache | None = None) -> None:
        """Whole rows, one segment each, from the caches ``src`` (src_kind 0, which may be this one) and ``stg``
        (src_kind 1) into this one, every layer, on the current stream: codes as pairs of bytes, scale rows as
        they are (groups belong to the row, not to its column)."""
        for c in (src, stg):
            if c is not None and (c.layers, c.Hkv, c.D, c.fmt, c.T) != (self.layers, self.Hkv, self.D, self.fmt, self.T):
                raise ValueError("rows move between caches of the same layers, heads, format and groups")
        segs = np.asarray(segs)
        rows = segs.copy()
        rows["src_col"] = rows["dst_col"] = 0
        for kind, c in ((0, src), (1, stg)):
            if c is not None:
                rows["len"][(rows["src_kind"] == kind) & (rows["len"] > 0)] = min(c.S, self.S) // 4
        live = rows["dst_row"][rows["len"] > 0]
        if len(np.unique(live)) != len(live):
            raise ValueError("two segments for one row: rows move whole")

        def box(c, k, v, width):
            return (None, None, 0, 1, 1) if c is None else (k, v, k[0].numel() * k.element_size(), c.R, width)

        def codes(c):
            return box(c, *((c.k, c.v, c.W) if c is not None else (None, None, 0)))

        def scales(c, copied=False):
            if c is None:
                return box(None, None, None, 0)
            # rows of one box may change places without their cells meeting, but their scales always start at 0
            return box(c, *((x.clone() if copied else x) for x in (c.k_scale, c.v_scale)), c.S // 4)

        bs_kv_scatter_compact(ctx, segs, self.layers, self.Hkv, self.D // 2, BS_BF16, *codes(src), *codes(stg), *codes(self))
        bs_kv_scatter_compact(ctx, rows, self.layers, self.Hkv, 4, BS_F32, *scales(src, src is self), *scales(stg), *scales(self))

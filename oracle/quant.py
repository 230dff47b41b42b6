"""The dual cache held in 8 bits, and the per-head norm with rotation.

Scale groups: T consecutive tokens of one head share a scale; the grid is laid
from the first generated token (logical position p) both ways, so token t is in
group (t + pad) // T with pad = -p mod T, and an active block is whole groups
whenever T divides the block length. With a = max(max |x|, 2^-64) over a group
and Q = 448 (e4m3) or 127 (int8):
    scale = a / Q,   code = rne(x * (Q / a)),   number held = code * scale.
The quotients, the product and the number read back are fp32 roundings of the
definition, so codes and scales are exact values that a kernel has to meet bit
for bit; they are formed here by NumPy's fp32 arithmetic (round to nearest
even). Attention over the codes is the block attention over the numbers that
they hold, in fp64.

Norm: y = x / sqrt(mean(x^2) + eps) * w per head, then the rotation of the
refresh (rotate-half pairs at the token's position), in fp64.

Test infrastructure: the oracle, not the product path.
"""
from __future__ import annotations

import math

import numpy as np

from .attention import attention_rows
from .geometry import geometry, widen
from .refresh import rope

QMAX = {"e4m3": 448.0, "i8": 127.0}
FLOOR = 2.0 ** -64


def e4m3_value(code) -> np.ndarray:
    """Numbers that e4m3 codes stand for: sign, 4 exponent bits (bias 7), 3
    fraction bits; exponent 0 is subnormal; 0x7f and 0xff are NaN."""
    b = np.asarray(code).astype(np.int64) & 0xFF
    e, f = (b >> 3) & 15, b & 7
    mag = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    return np.where((b & 0x7F) == 0x7F, np.nan, np.where(b >> 7, -mag, mag))


def e4m3_code(x) -> np.ndarray:
    """Codes of finite x, |x| <= 448 after rounding: nearest, ties to the even code."""
    x = np.asarray(x, np.float64)
    tab = e4m3_value(np.arange(0x7F))                       # increasing, 0 .. 448
    a = np.abs(x)
    hi = np.clip(np.searchsorted(tab, a), 1, 0x7E)
    lo = hi - 1
    dl, dh = a - tab[lo], tab[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (c | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def values(codes, fmt: str) -> np.ndarray:
    return e4m3_value(codes) if fmt == "e4m3" else np.asarray(codes).astype(np.uint8).view(np.int8).astype(np.float64)


def group_pad(p: int, T: int) -> int:
    return (-int(p)) % T


def group_count(p: int, g: int, T: int) -> int:
    return -(-int(p) // T) + -(-int(g) // T)


def quantize_tokens(x, first: int, p: int, T: int, fmt: str):
    """x [tokens][D] fp32, token m at logical position first + m. Returns (codes
    uint8 [tokens][D], {group: scale fp32})."""
    x = np.asarray(x, np.float32)
    grp = (first + np.arange(len(x)) + group_pad(p, T)) // T
    q = np.float32(QMAX[fmt])
    codes, scales = np.zeros(x.shape, np.uint8), {}
    for j in np.unique(grp):
        m = grp == j
        a = np.maximum(np.abs(x[m]).max(), np.float32(FLOOR)).astype(np.float32)
        scales[int(j)] = np.float32(a / q)
        y = (x[m] * np.float32(q / a)).astype(np.float32)
        codes[m] = e4m3_code(y) if fmt == "e4m3" else np.rint(y).astype(np.int8).view(np.uint8)
    return codes, scales


def kv_quantize(reqs, box, codes, scales, T: int, fmt: str, dtype: str):
    """Whole rows of one box [R][Hkv][W][D]; codes and scales are copied, then filled."""
    codes, scales = codes.copy(), scales.copy()
    for r in reqs:
        row, off, ln = int(r["row"]), int(r["off"]), int(r["p"]) + int(r["g"])
        for c in range(box.shape[1]):
            cd, sc = quantize_tokens(widen(box[row, c, off:off + ln], dtype), 0, r["p"], T, fmt)
            codes[row, c, off:off + ln] = cd
            for j, v in sc.items():
                scales[row, c, j] = v
    return codes, scales


def row_numbers(r, c: int, codes, scales, T: int, fmt: str) -> np.ndarray:
    """The numbers row r's head c holds, [len][D], fp64 (code times scale, unrounded)."""
    row, off, ln = int(r["row"]), int(r["off"]), int(r["p"]) + int(r["g"])
    grp = (np.arange(ln) + group_pad(r["p"], T)) // T
    return values(codes[row, c, off:off + ln], fmt) * scales[row, c, grp].astype(np.float64)[:, None]


def quant_cache_attention(reqs, L: int, q, k_new, v_new, k8, v8, k_scale, v_scale, T: int, fmt: str, *,
                          scale: float | None = None, only=None):
    """Block attention over the codes; q, k_new, v_new bf16 bit patterns.

    Returns (out [n][L][Hq][D] fp64, spread [n][L][Hq][D]: the weighted mean of
    |value|, which rounding errors of the weights are relative to)."""
    n, _, Hq, D = q.shape
    Hkv = k_new.shape[2]
    G = Hq // Hkv
    if scale is None or scale <= 0:
        scale = 1.0 / math.sqrt(D)
    out, spread = np.zeros((n, L, Hq, D)), np.zeros((n, L, Hq, D))
    for i in range(n) if only is None else only:
        r = reqs[i]
        t = geometry(r, L)
        for c in range(Hkv):
            keys = row_numbers(r, c, k8, k_scale, T, fmt)
            vals = row_numbers(r, c, v8, v_scale, T, fmt)
            keys[t.s:t.e] = widen(k_new[i, :t.B, c], "bf16")
            vals[t.s:t.e] = widen(v_new[i, :t.B, c], "bf16")
            for h in range(c * G, (c + 1) * G):
                x = widen(q[i, :t.B, h], "bf16")
                out[i, :t.B, h] = attention_rows(x, keys, vals, scale)
                spread[i, :t.B, h] = attention_rows(x, keys, np.abs(vals), scale)
    return out, spread


def norm_rope(x, weight, pos, eps: float, base: float) -> np.ndarray:
    """x [..., D] fp64 at positions pos (broadcast against x.shape[:-1])."""
    x = np.asarray(x, np.float64)
    if eps >= 0:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * np.asarray(weight, np.float64)
    return rope(x, pos, base)

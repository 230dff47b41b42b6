"""Pins of oracle.quant: the number formats against torch's, group borders
enumerated by hand, rounding and scales on chosen values, attention over codes
against the pinned block attention, the norm in closed form."""
import numpy as np
import pytest
import torch

import oracle
from oracle import quant


def bits(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def test_e4m3_table_and_rounding():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    ref = codes.view(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(quant.e4m3_value(codes.numpy()), ref)
    rng = np.random.default_rng(1)
    fin = np.sort(np.unique(ref[np.isfinite(ref)]))
    x = np.concatenate([rng.uniform(-448, 448, 4000), rng.normal(0, 0.01, 4000), fin, (fin[1:] + fin[:-1]) / 2, [0.0, -0.0]])
    x = x.astype(np.float32)
    np.testing.assert_array_equal(quant.e4m3_code(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_group_borders():
    # p = 5, T = 4: pad 3; tokens 0 | 1 2 3 4 | 5 6 7 8 | ...: the first generated token opens a group
    assert quant.group_pad(5, 4) == 3 and quant.group_count(5, 6, 4) == 4
    grp = (np.arange(11) + 3) // 4
    assert grp.tolist() == [0, 1, 1, 1, 1, 2, 2, 2, 2, 3, 3]
    assert quant.group_pad(8, 4) == 0 and quant.group_pad(0, 32) == 0 and quant.group_count(0, 1, 64) == 1
    for p in range(0, 70):
        for T in (1, 2, 4, 8, 16, 32, 64):
            assert (p + quant.group_pad(p, T)) % T == 0
            assert (p + 77 - 1 + quant.group_pad(p, T)) // T + 1 == quant.group_count(p, 77, T)


@pytest.mark.parametrize("fmt,q", [("e4m3", 448.0), ("i8", 127.0)])
def test_codes_and_scales(fmt, q):
    x = np.array([[1.0, -2.0], [0.5, 0.25], [0.0, 0.0], [3.0, -3.0]], np.float32)
    codes, sc = quant.quantize_tokens(x, 0, 0, 2, fmt)
    assert sc == {0: np.float32(2.0 / q), 1: np.float32(3.0 / q)}
    v = quant.values(codes, fmt)
    assert v[0, 1] == -q and v[3].tolist() == [q, -q] and v[2].tolist() == [0.0, 0.0]
    # rounding: half a step of the format, relative (e4m3) or of the scale (int8)
    rng = np.random.default_rng(2)
    x = rng.normal(size=(64, 16)).astype(np.float32)
    codes, sc = quant.quantize_tokens(x, 7, 3, 8, fmt)
    s = np.array([sc[(7 + m + quant.group_pad(3, 8)) // 8] for m in range(64)], np.float64)[:, None]
    back = quant.values(codes, fmt) * s
    step = np.maximum(2.0 ** -4 * np.abs(x), s * 2.0 ** -10) if fmt == "e4m3" else s / 2
    assert (np.abs(back - x) <= step * (1 + 1e-5)).all()
    # a group of zeros, and one far below the floor: finite scales, codes of zero
    codes, sc = quant.quantize_tokens(np.array([[0.0], [1e-30]], np.float32), 0, 0, 1, fmt)
    assert sc[0] == sc[1] == np.float32(2.0 ** -64) / np.float32(q) and quant.values(codes, fmt).tolist() == [[0.0], [0.0]]


def test_attention_over_codes_is_the_block_attention_over_their_numbers():
    rng = np.random.default_rng(3)
    reqs = np.array([(5, 16, 1, 1, 2), (0, 6, 0, 0, 17)], [(a, "<i4") for a in ("p", "g", "k", "row", "off")])
    L, Hq, Hkv, D, R, W, T = 8, 4, 2, 16, 2, 23, 4
    box = rng.normal(size=(R, Hkv, W, D)).astype(np.float32)
    codes, scales = quant.kv_quantize(reqs, box, np.zeros(box.shape, np.uint8), np.ones((R, Hkv, 6), np.float32), T, "i8", "f32")
    held = np.zeros(box.shape)
    for r in reqs:
        for c in range(Hkv):
            held[r["row"], c, r["off"]:r["off"] + r["p"] + r["g"]] = quant.row_numbers(r, c, codes, scales, T, "i8")
    assert np.abs(held - box)[1, :, 2:23].max() <= np.abs(box).max() / 127 / 2 * 1.001
    q, kn, vn = (bits(rng.normal(size=(2, L, h, D))) for h in (Hq, Hkv, Hkv))
    out, spread = quant.quant_cache_attention(reqs, L, q, kn, vn, codes, codes, scales, scales, T, "i8")
    wide = [oracle.widen(x, "bf16") for x in (q, kn, vn)]
    ref, _, _ = oracle.dual_cache_block_attention(reqs, L, *wide, held, held, dtype="f64")
    np.testing.assert_allclose(out, ref, rtol=1e-12, atol=1e-12)
    assert (spread >= np.abs(out) - 1e-12).all() and (out[1, 6:] == 0).all()


def test_norm_rope_closed_form():
    x = np.array([[3.0, 4.0, 0.0, 0.0]])
    w = np.array([1.0, 2.0, 1.0, 1.0])
    y = quant.norm_rope(x, w, np.array([0]), 0.0, 100.0)
    np.testing.assert_allclose(y, [[3 / 2.5, 2 * 4 / 2.5, 0, 0]])
    y = quant.norm_rope(x, None, np.array([1]), 0.0, 100.0)            # pairs (0, 2), (1, 3): angles 1 and 1/10
    np.testing.assert_allclose(y, [[1.2 * np.cos(1), 1.6 * np.cos(0.1), 1.2 * np.sin(1), 1.6 * np.sin(0.1)]])
    np.testing.assert_array_equal(quant.norm_rope(x, w, np.array([5]), -1.0, 0.0), x)
    np.testing.assert_allclose(quant.norm_rope(1e-20 * x, None, np.array([0]), 1e-6, 0.0), 1e-17 * x)

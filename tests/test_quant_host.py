"""The 8-bit cache's entry points on the host: what they refuse before any device
work, the group count, the split plan's workspace."""
import numpy as np
import pytest

import paper_2607_08930_amd as bs
from oracle import quant


def test_calls_without_context_fail_before_any_device_work():
    none = None
    for call in (lambda: bs.lib.bs_kv_quantize(none, none, 0, 8, 1, 1, 1, 64, 1, 0, 8, none, none, none, none, none, none, 1, none),
                 lambda: bs.lib.bs_kv_dequantize(none, none, 0, 8, 1, 1, 1, 64, 1, 0, 8, none, none, none, none, 1, none, none, none),
                 lambda: bs.lib.bs_quant_cache_block_attention(none, none, 0, 8, 1, 1, 64, 0, 8, 0.0, none, none, none, none, none,
                                                               none, none, 1, 1, 1, 1, none, none, 0, none),
                 lambda: bs.lib.bs_qk_norm_rope(none, none, 0, 8, 1, 1, 0, 1, 1, 64, 1, none, 64, none, 64, none, none, 1e-6, 1e4,
                                                none, none, none)):
        assert call() == 1
        assert "ctx is NULL" in bs.bs_last_error()


def test_scale_groups_against_the_oracle():
    for T in (1, 2, 4, 8, 16, 32, 64):
        for p in (0, 1, 31, 32, 33, 64, 4095, 4096):
            for g in (1, 5, 64, 65, 1000):
                assert bs.bs_kv_scale_groups(p, g, T) == quant.group_count(p, g, T)
    for bad in ((-1, 5, 8), (5, 0, 8), (5, 5, 0), (5, 5, 3), (5, 5, 128)):
        assert bs.bs_kv_scale_groups(*bad) == 0
    assert bs.bs_kv_scale_groups(2 ** 31 - 1, 2 ** 31 - 1, 1) == 0          # more than an int holds


def rows(n, p, g=64, k=0):
    r = np.zeros(n, bs.REQ_DTYPE)
    r["p"], r["g"], r["k"], r["row"] = p, g, k, np.arange(n)
    return r


def test_workspace_of_the_split_plan():
    query = bs.bs_quant_attention_workspace_bytes
    wave = (32 * 128 + 2 * 64) * 4            # a wave's partial: 32 rows of D, a maximum and a sum per lane
    # one long row of few heads is cut, and the room is whole partials
    need = query(rows(1, 8192), 32, 4, 4, 128)
    assert need > 0 and need % wave == 0
    # grouped heads: seven row tiles are two workgroups of four waves
    need = query(rows(1, 8192), 32, 28, 4, 128)
    assert need > 0 and need % (4 * wave) == 0
    # a full machine of equal rows, and rows of one tile, run whole
    assert query(rows(96, 1000), 32, 32, 32, 128) == 0
    assert query(rows(4, 20, g=32), 32, 4, 4, 128) == 0
    # arguments that the attention refuses
    for bad in ((rows(1, 8192), 0, 4, 4, 128), (rows(1, 8192), 65, 4, 4, 128), (rows(1, 8192), 32, 3, 2, 128),
                (rows(1, 8192), 32, 18, 2, 128), (rows(1, 8192), 32, 4, 4, 96), (rows(0, 0), 32, 4, 4, 128),
                (rows(1, -1), 32, 4, 4, 128), (rows(1, 8192, g=0), 32, 4, 4, 128), (rows(1, 8192, k=2), 32, 4, 4, 128),
                (rows(1, 2 ** 31 - 64), 32, 4, 4, 128)):
        assert query(*bad) == 0


def test_workspace_depends_on_the_rows_not_on_their_order():
    rng = np.random.default_rng(3)
    r = rows(24, rng.integers(20, 300, 24))
    r["p"][7] = 8000
    a = bs.bs_quant_attention_workspace_bytes(r, 32, 28, 4, 128)
    assert a > 0
    for _ in range(4):
        assert bs.bs_quant_attention_workspace_bytes(rng.permutation(r), 32, 28, 4, 128) == a


def test_group_of_a_cache_object():
    from paper_2607_08930_amd.quant_cache import QuantCache, largest_group
    assert [largest_group(x) for x in (1, 7, 8, 24, 32, 48, 64)] == [1, 1, 8, 8, 32, 16, 64]
    c = QuantCache(1, 2, 100, 1, 64, 32, "i8", device="cpu")
    assert c.T == 32 and c.S == 8 and c.fmt == bs.BS_I8
    # no row of that width has more groups than S
    for T in (1, 4, 32):
        c = QuantCache(1, 1, 100, 1, 64, 32, "e4m3", T, device="cpu")
        assert max(bs.bs_kv_scale_groups(p, 100 - p, T) for p in range(100)) <= c.S
    for bad in (dict(fmt="e5m2"), dict(T=64), dict(T=3)):
        with pytest.raises(ValueError):
            QuantCache(1, 2, 100, 1, 64, 32, **{"device": "cpu", **bad})

"""GPU parity of the operators around an 8-bit dual cache against oracle.quant:
quantising and reading back, the block attention over codes with its write of
the block, the per-head norm with rotation, and the four together.

Tolerances. Codes, scales and numbers read back are chains of single fp32
roundings that the oracle repeats, so they match bit for bit. Attention: the
scores are fp32 sums of exact products, the weights are rounded to bf16 (2^-8) and
the output to 2^-8 of its value, so |d| <= 2^-8 |out| + (2^-8 + 2^-9) spread with
the spread of oracle.quant; 2^-9 covers the scores: their error e moves a weight by
the factor exp(e). Of it, e <= 128 * 2^-24 * sum |q k| from the fp32 sums stays under
2^-10 for the sum |q k| scale <= 128 that the inputs keep, as does the hardware
exp2. A query element is off by up to 2^-15 (int8) or, with more than 32 query rows a
KV head, 2^-17 (e4m3) of its row's largest, with either sign: over a key of
deviation s that is a score error of deviation 2^-15 max|q| s / sqrt(3), 2^-14 s for
the normal queries here, and it averages out over the keys of a row.
Norm: fp32 sums of 256 squares at most, one reciprocal square root and two
products (under 16 roundings of 2^-24) and an angle good to 2^-22 turns: 4e-6 of
the rotated pair's size in all, then the output's rounding (2^-8 bf16, 2^-24
fp32); the bf16 form takes the hardware's sine, 2^-16 of the pair."""
import numpy as np
import pytest

import oracle
from gpu_util import lazy, say
from oracle import quant

pytestmark = pytest.mark.gpu

FMT = {"e4m3": 0, "i8": 1}


@pytest.fixture(scope="module")
def ctx():
    torch, bs, _ = lazy()
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    c = bs.Context(0)
    yield c
    c.close()


def batch(rng, lens, L, *, slack=3, extra_rows=1):
    """Requests (p, g, k), shuffled over a box with an unused row and padding on both sides."""
    _, bs, _ = lazy()
    n = len(lens)
    R, W = n + extra_rows, max(p + g for p, g, _ in lens) + slack
    rows = rng.permutation(R)[:n]
    reqs = np.zeros(n, bs.REQ_DTYPE)
    for i, (p, g, k) in enumerate(lens):
        reqs[i] = (p, g, k, rows[i], rng.integers(0, W - p - g + 1))
    bs.bs_validate_requests(reqs, L, R, W)
    return reqs, R, W


def logical(reqs, R, W):
    used = np.zeros((R, W), bool)
    for r in reqs:
        used[r["row"], r["off"]:r["off"] + r["p"] + r["g"]] = True
    return used


def bf16(x):
    torch, _, bstep = lazy()
    return bstep.to_host(torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16))


def numbers(rng, shape, dtype, sigma=1.0):
    x = (rng.normal(size=shape) * sigma).astype(np.float32)
    return bf16(x) if dtype == "bf16" else x


def scale_len(reqs, T, more=1):
    return max(quant.group_count(r["p"], r["g"], T) for r in reqs) + more


def nan_outside(x, used, dtype):
    """x [R][Hkv][W][D] with NaN in every cell that belongs to no row."""
    x = x.copy()
    x.transpose(0, 2, 1, 3)[~used] = np.uint16(0x7FC0) if dtype == "bf16" else np.float32("nan")
    return x


LENS = [(0, 1, 0), (1, 5, 0), (37, 40, 1), (64, 64, 1), (200, 77, 2), (31, 9, 0)]


# ---------------------------------------------------------------- quantising and reading back
@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype,D,T", [("bf16", 128, 32), ("bf16", 128, 1), ("bf16", 64, 64), ("bf16", 128, 64),
                                       ("bf16", 64, 8), ("f32", 128, 16), ("f32", 64, 2), ("f32", 128, 64),
                                       ("bf16", 128, 4), ("bf16", 64, 16)])
def test_quantize_and_read_back(ctx, fmt, dtype, D, T):
    torch, bs, bstep = lazy()
    rng = np.random.default_rng(100 * T + D)
    reqs, R, W = batch(rng, LENS, 32)
    used, Hkv, S = logical(reqs, R, W), 3, scale_len(reqs, T)
    k = numbers(rng, (R, Hkv, W, D), dtype)
    v = numbers(rng, (R, Hkv, W, D), dtype, 1e-3)
    r = reqs[2]
    k[r["row"], 1, r["off"]:r["off"] + 40] = 0                                    # groups of zeros
    v[r["row"], 0, r["off"] + 8, 3] = bf16([3e38])[0] if dtype == "bf16" else np.float32(3.3e38)
    v[r["row"], 2, r["off"]:r["off"] + 70] = bf16([1e-30])[0] if dtype == "bf16" else np.float32(1e-39)
    k, v = nan_outside(k, used, dtype), nan_outside(v, used, dtype)
    c0, s0 = np.full((R, Hkv, W, D), 0x5A, np.uint8), np.full((R, Hkv, S), -7.0, np.float32)
    dc = [torch.from_numpy(c0.copy()).cuda() for _ in range(2)]
    ds = [torch.from_numpy(s0.copy()).cuda() for _ in range(2)]
    dk, dv = bstep.to_device(k, dtype), bstep.to_device(v, dtype)
    dt = bstep.dt_code(dtype)
    bs.bs_kv_quantize(ctx, reqs, 32, R, W, Hkv, D, dt, FMT[fmt], T, dk, dv, dc[0], dc[1], ds[0], ds[1], S)
    torch.cuda.synchronize()
    refs = [quant.kv_quantize(reqs, x, c0, s0, T, fmt, dtype) for x in (k, v)]
    for name, (rc, rs), gc, gs in zip("kv", refs, dc, ds):
        np.testing.assert_array_equal(gs.cpu().numpy(), rs, err_msg=name)
        np.testing.assert_array_equal(gc.cpu().numpy(), rc, err_msg=name)
    # and back, into boxes whose other cells stay as they were
    back = [torch.full((R, Hkv, W, D), 5.0, dtype=bstep.torch_dtype(dtype), device="cuda") for _ in range(2)]
    bs.bs_kv_dequantize(ctx, reqs, 32, R, W, Hkv, D, dt, FMT[fmt], T, dc[0], dc[1], ds[0], ds[1], S, back[0], back[1])
    torch.cuda.synchronize()
    for (rc, rs), g in zip(refs, back):
        want = np.full((R, Hkv, W, D), 5.0, np.float32)
        for r in reqs:
            ln = int(r["p"] + r["g"])
            grp = (np.arange(ln) + quant.group_pad(r["p"], T)) // T
            for c in range(Hkv):
                cells = rc[r["row"], c, r["off"]:r["off"] + ln]
                with np.errstate(over="ignore"):
                    want[r["row"], c, r["off"]:r["off"] + ln] = quant.values(cells, fmt).astype(np.float32) * rs[r["row"], c, grp][:, None]
        if dtype == "bf16":
            np.testing.assert_array_equal(bstep.to_host(g), bf16(want))
        else:
            np.testing.assert_array_equal(g.cpu().numpy(), want)


# ---------------------------------------------------------------- attention
def attention_case(rng, lens, L, Hq, Hkv, D, T, fmt, *, sigma=1.0, q_sigma=1.0):
    reqs, R, W = batch(rng, lens, L)
    S = scale_len(reqs, T)
    boxes = [numbers(rng, (R, Hkv, W, D), "bf16", sigma * np.exp(rng.normal())) for _ in range(2)]
    # garbage outside the rows and in the stale slot: codes of NaN, scales of NaN
    c0 = np.full((R, Hkv, W, D), 0x7F if fmt == "e4m3" else 0x80, np.uint8)
    s0 = np.full((R, Hkv, S), np.nan, np.float32)
    cache = [quant.kv_quantize(reqs, x, c0, s0, T, fmt, "bf16") for x in boxes]
    for r in reqs:
        t = oracle.geometry(r, L)
        for cd, sc in cache:
            cd[t.row, :, t.off + t.s:t.off + t.e] = c0[0, 0, 0, 0]
            g0 = (t.s + quant.group_pad(t.p, T)) // T
            sc[t.row, :, g0:g0 + -(-t.B // T)] = np.nan
    n = len(reqs)
    q = numbers(rng, (n, L, Hq, D), "bf16", q_sigma)
    kn, vn = numbers(rng, (n, L, Hkv, D), "bf16", sigma), numbers(rng, (n, L, Hkv, D), "bf16", sigma)
    for i, r in enumerate(reqs):                         # rows behind a short block are not read
        B = oracle.geometry(r, L).B
        for x in (q, kn, vn):
            x[i, B:] = 0x7FC0
    return dict(reqs=reqs, R=R, W=W, S=S, L=L, Hq=Hq, Hkv=Hkv, D=D, T=T, fmt=fmt, q=q, k_new=kn, v_new=vn,
                k8=cache[0][0], v8=cache[1][0], k_scale=cache[0][1], v_scale=cache[1][1])


def on_device(w):
    torch, _, bstep = lazy()
    d = {x: bstep.to_device(w[x], "bf16") for x in ("q", "k_new", "v_new")}
    d.update({x: torch.from_numpy(w[x].copy()).cuda() for x in ("k8", "v8", "k_scale", "v_scale")})
    d["out"] = torch.full(tuple(d["q"].shape), float("nan"), dtype=torch.bfloat16, device="cuda")
    return d


def attend(ctx, w, d, *, write_back=True, split=True, stream=None, scale=0.0, ws=None):
    torch, bs, _ = lazy()
    need = bs.bs_quant_attention_workspace_bytes(w["reqs"], w["L"], w["Hq"], w["Hkv"], w["D"]) if split else 0
    if ws is None and need:
        ws = torch.full((need,), 0xA5, dtype=torch.uint8, device="cuda")
    bs.bs_quant_cache_block_attention(ctx, w["reqs"], w["L"], w["Hq"], w["Hkv"], w["D"], FMT[w["fmt"]], w["T"], scale,
                                      d["q"], d["k_new"], d["v_new"], d["k8"], d["v8"], d["k_scale"], d["v_scale"],
                                      w["S"], w["R"], w["W"], write_back, d["out"], ws if need else None, need,
                                      stream=stream)
    return need


def check_out(w, d, only=None, scale=None, label=""):
    _, _, bstep = lazy()
    ref, spread = quant.quant_cache_attention(w["reqs"], w["L"], w["q"], w["k_new"], w["v_new"], w["k8"], w["v8"],
                                              w["k_scale"], w["v_scale"], w["T"], w["fmt"], only=only, scale=scale)
    got = oracle.widen(bstep.to_host(d["out"]), "bf16")
    worst = 0.0
    for i in range(len(w["reqs"])) if only is None else only:
        B = oracle.geometry(w["reqs"][i], w["L"]).B
        tol = 2.0 ** -8 * np.abs(ref[i, :B]) + (2.0 ** -8 + 2.0 ** -9) * spread[i, :B] + 1e-30
        assert np.isfinite(got[i, :B]).all(), f"{label}: request {i} has outputs that are not finite"
        worst = max(worst, float((np.abs(got[i, :B] - ref[i, :B]) / tol).max()))
        assert (got[i, B:] == 0).all(), f"{label}: rows behind the block of request {i} are not zero"
    assert worst <= 1.0, f"{label}: {worst:.2f} of the bound"
    return worst


def check_cache(w, d, write_back, label=""):
    """The block's cells and scales as quantised on the host, everything else as it was."""
    for a in "kv":
        codes, scales = w[a + "8"].copy(), w[a + "_scale"].copy()
        if write_back:
            for i, r in enumerate(w["reqs"]):
                t = oracle.geometry(r, w["L"])
                for c in range(w["Hkv"]):
                    cd, sc = quant.quantize_tokens(oracle.widen(w[a + "_new"][i, :t.B, c], "bf16"), t.s, t.p, w["T"], w["fmt"])
                    codes[t.row, c, t.off + t.s:t.off + t.e] = cd
                    for j, v in sc.items():
                        scales[t.row, c, j] = v
        np.testing.assert_array_equal(d[a + "8"].cpu().numpy(), codes, err_msg=label + a)
        np.testing.assert_array_equal(d[a + "_scale"].cpu().numpy(), scales, err_msg=label + a)


SHAPES = [
    # L, Hq, Hkv, D, T: MHA and groups, one and two row tiles a head, single tokens, odd block lengths
    (32, 4, 4, 128, 32), (32, 2, 2, 64, 16), (64, 2, 2, 128, 64), (1, 3, 3, 128, 1), (1, 16, 2, 64, 1),
    (32, 14, 2, 128, 32), (8, 14, 2, 128, 8), (64, 8, 1, 128, 16), (48, 12, 2, 64, 16), (33, 6, 2, 128, 1),
    (7, 4, 4, 128, 1), (24, 5, 1, 128, 8), (64, 7, 1, 64, 32), (62, 3, 1, 128, 2), (12, 8, 4, 64, 4),
]


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("L,Hq,Hkv,D,T", SHAPES)
def test_attention(ctx, L, Hq, Hkv, D, T, fmt):
    torch, _, _ = lazy()
    rng = np.random.default_rng(1000 * L + 10 * Hq + D + T)
    # no prompt and one block; one token; a prompt shorter than a group; several tiles; a
    # short last block; a last block of one token; the first block of many
    lens = [(0, min(L, 5), 0), (1, 1, 0), (3, 2 * L, 1), (130, 3 * L + 1, 1), (77, 2 * L - L // 2, 1), (64, L + 1, 1),
            (97, 4 * L, 0), (320, 64, (64 - 1) // L)]
    w = attention_case(rng, lens, L, Hq, Hkv, D, T, fmt)
    d = on_device(w)
    attend(ctx, w, d)
    torch.cuda.synchronize()
    say(f"L={L} Hq={Hq} Hkv={Hkv} D={D} T={T} {fmt}: {check_out(w, d):.3f} of the bound")
    check_cache(w, d, True)


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("L,Hq,Hkv,T", [(32, 4, 4, 32), (32, 7, 1, 32), (1, 4, 1, 1), (64, 4, 2, 64)])
def test_attention_long_rows(ctx, L, Hq, Hkv, T, fmt):
    # whole rows and the split plan, which has to agree within the bound
    torch, _, _ = lazy()
    rng = np.random.default_rng(L + Hq)
    w = attention_case(rng, [(3000, 2 * L, 1), (5111, 3 * L, 0), (40, L, 0)], L, Hq, Hkv, 128, T, fmt, sigma=2.0)
    for split in (False, True):
        d = on_device(w)
        need = attend(ctx, w, d, split=split)
        torch.cuda.synchronize()
        say(f"split={split} ({need} bytes): {check_out(w, d):.3f} of the bound")
        check_cache(w, d, True)


def test_attention_peaked_scores_and_scale(ctx):
    # scores of hundreds (weights of one key, the running maximum moves often) and a caller's scale
    torch, _, _ = lazy()
    for fmt, T in (("e4m3", 32), ("i8", 8)):
        rng = np.random.default_rng(9)
        w = attention_case(rng, [(400, 64, 1), (33, 96, 2)], 32, 4, 2, 128, T, fmt)
        for scale in (0.25, 0.02):
            d = on_device(w)
            attend(ctx, w, d, scale=scale)
            torch.cuda.synchronize()
            # sum |q k| scale is 128 * 0.64 * scale: 20 at most, so the fp32 scores keep the bound
            say(f"{fmt} scale={scale}: {check_out(w, d, scale=scale):.3f} of the bound")


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
def test_attention_group_sizes_far_apart(ctx, fmt):
    # groups of values from 2^-40 to 2^40 and of zeros in one row, and queries of every size
    torch, _, _ = lazy()
    rng = np.random.default_rng(11)
    w = attention_case(rng, [(256, 64, 0), (100, 64, 1)], 32, 4, 2, 128, 32, fmt)
    for r in w["reqs"]:
        m = quant.group_count(r["p"], r["g"], 32)
        f = np.exp2(rng.integers(-40, 41, size=(w["Hkv"], m))).astype(np.float32)
        w["v_scale"][r["row"], :, :m] *= f
        w["v8"][r["row"], 0, r["off"]:r["off"] + 20] = 0
    w["q"] = numbers(rng, w["q"].shape, "bf16")
    for i, r in enumerate(w["reqs"]):
        B = oracle.geometry(r, 32).B
        w["q"][i, :B] = bf16(oracle.widen(w["q"][i, :B], "bf16") * np.exp2(rng.integers(-30, 1, size=(B, 4, 1))))
    d = on_device(w)
    attend(ctx, w, d)
    torch.cuda.synchronize()
    say(f"{fmt}: {check_out(w, d):.3f} of the bound")


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("Hq,T,scale", [(2, 32, None), (2, 8, None), (8, 32, None), (8, 8, None), (2, 32, 1e-38), (8, 32, 1e-38)])
def test_attention_scores_that_vanish(ctx, fmt, Hq, T, scale):
    """Queries of zero or near nothing against groups of zeros, whose scale is the least there is: every key of
    the row weighs the same, and the keys of its first and last tiles that do not exist weigh nothing."""
    torch, _, _ = lazy()
    rng = np.random.default_rng(31)
    w = attention_case(rng, [(70, 64, 1), (5, 40, 0), (300, 33, 0)], 32, Hq, 2, 128, T, fmt)
    for i, r in enumerate(w["reqs"]):
        t = oracle.geometry(r, 32)
        w["q"][i, :t.B] = bf16(rng.choice([0.0, 1e-38, -1e-38], size=w["q"][i, :t.B].shape))
        for c in range(2):
            for j in range(quant.group_count(r["p"], r["g"], T)):
                if rng.random() < 0.6:
                    w["k_scale"][t.row, c, j] = np.float32(2.0 ** -64) / np.float32(quant.QMAX[fmt])
    w["k8"][:] = np.where(rng.random(w["k8"].shape) < 0.5, 0, w["k8"])
    d = on_device(w)
    attend(ctx, w, d, scale=scale or 0.0)
    torch.cuda.synchronize()
    # all scores are under 2^-20, so the bound's share for the scores is not used up
    say(f"{fmt} Hq={Hq} T={T}: {check_out(w, d, scale=scale):.3f} of the bound")


def test_attention_reads_only(ctx):
    torch, _, _ = lazy()
    rng = np.random.default_rng(4)
    w = attention_case(rng, [(90, 64, 1), (10, 20, 0)], 32, 4, 2, 128, 32, "e4m3")
    d = on_device(w)
    attend(ctx, w, d, write_back=False)
    torch.cuda.synchronize()
    check_out(w, d)
    check_cache(w, d, False)


def test_attention_cache_beyond_32_bits(ctx):
    # the row's cells lie more than 2^31 bytes into each tensor
    torch, bs, _ = lazy()
    rng = np.random.default_rng(5)
    w = attention_case(rng, [(140, 64, 1)], 32, 4, 2, 128, 32, "e4m3")
    d = on_device(w)
    r, W = w["reqs"][0], 1 << 20
    R, ln, off = 10, int(r["p"] + r["g"]), W - 300
    big = dict(d, out=torch.full_like(d["out"], float("nan")))
    for a in ("k8", "v8"):
        big[a] = torch.zeros((R, 2, W, 128), dtype=torch.uint8, device="cuda")
        big[a][9, :, off:off + ln] = d[a][r["row"], :, r["off"]:r["off"] + ln]
    for a in ("k_scale", "v_scale"):
        big[a] = torch.ones((R, 2, w["S"]), dtype=torch.float32, device="cuda")
        big[a][9] = d[a][r["row"]]
    far = w["reqs"].copy()
    far["row"], far["off"] = 9, off
    attend(ctx, dict(w, reqs=far, R=R, W=W), big)
    attend(ctx, w, d)
    torch.cuda.synchronize()
    assert torch.equal(big["out"].view(torch.int16), d["out"].view(torch.int16))
    check_out(w, big)
    for a in ("k8", "v8"):
        assert torch.equal(big[a][9, :, off:off + ln], d[a][r["row"], :, r["off"]:r["off"] + ln])
    back = [torch.empty((R, 2, W, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    bs.bs_kv_dequantize(ctx, far, 32, R, W, 2, 128, bs.BS_BF16, 0, 32, big["k8"], big["v8"], big["k_scale"],
                        big["v_scale"], w["S"], back[0], back[1])
    near = [torch.empty((w["R"], 2, w["W"], 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    bs.bs_kv_dequantize(ctx, w["reqs"], 32, w["R"], w["W"], 2, 128, bs.BS_BF16, 0, 32, d["k8"], d["v8"], d["k_scale"],
                        d["v_scale"], w["S"], near[0], near[1])
    torch.cuda.synchronize()
    for x, y in zip(back, near):
        assert torch.equal(x[9, :, off:off + ln], y[r["row"], :, r["off"]:r["off"] + ln])


# ---------------------------------------------------------------- norm and rotation
@pytest.mark.parametrize("dtype,D,Hq,Hkv,rows,eps,base,weights", [
    ("bf16", 128, 7, 1, False, 1e-6, 1e6, True), ("bf16", 128, 32, 32, True, 1e-6, 5e5, True),
    ("f32", 128, 4, 2, True, 1e-5, 1e4, True), ("f32", 64, 5, 5, False, 1e-6, 1e4, False),
    ("bf16", 64, 9, 3, True, -1.0, 1e4, True), ("f32", 256, 3, 1, False, 1e-6, 0.0, True),
    ("bf16", 80, 4, 1, True, 1e-6, 1e4, True), ("f32", 16, 2, 1, True, 0.0, 100.0, True), ("bf16", 32, 3, 3, False, 1e-6, 1e4, True),
    ("f32", 208, 2, 2, False, 1e-6, 1e4, True),
])
def test_norm_rope(ctx, dtype, D, Hq, Hkv, rows, eps, base, weights):
    torch, bs, bstep = lazy()
    rng = np.random.default_rng(D + Hq)
    L = 24
    reqs, R, W = batch(rng, [(0, 1, 0), (1, 24, 0), (300, 100, 4), (17, 48, 1)], L)
    lead, H = ((R, W) if rows else (len(reqs), L)), Hq + 2 * Hkv
    x = numbers(rng, lead + (H * D + 8,), dtype, 3.0)
    nan = np.uint16(0x7FC0) if dtype == "bf16" else np.float32("nan")
    where = np.zeros(lead, bool)
    pos = np.zeros(lead)
    for i, r in enumerate(reqs):
        t = oracle.geometry(r, L)
        at = (t.row, slice(t.off, t.off + t.len)) if rows else (i, slice(0, t.B))
        where[at] = True
        pos[at] = np.arange(t.len) if rows else t.s + np.arange(t.B)
    x[~where] = nan
    qw, kw = numbers(rng, (D,), dtype), numbers(rng, (D,), dtype)
    dx, dqw, dkw = (bstep.to_device(a, dtype) for a in (x, qw, kw))
    outs = [torch.full(lead + (h, D), 9.0, dtype=bstep.torch_dtype(dtype), device="cuda") for h in (Hq, Hkv)]
    bs.bs_qk_norm_rope(ctx, reqs, L, R, W, rows, Hq, Hkv, D, bstep.dt_code(dtype), dx, H * D + 8, dx[..., Hq * D:], H * D + 8,
                       dqw if weights else None, dkw if weights else None, eps, base, outs[0], outs[1])
    torch.cuda.synchronize()
    for lo, h, w, out in ((0, Hq, qw, outs[0]), (Hq * D, Hkv, kw, outs[1])):
        got = oracle.widen(bstep.to_host(out), dtype)
        assert (got[~where] == 9.0).all(), "a token that is not listed was written"
        y = oracle.widen(x[where][:, lo:lo + h * D], dtype).reshape(-1, h, D)
        ww = oracle.widen(w, dtype) if weights else None
        ref = quant.norm_rope(y, ww, pos[where][:, None], eps, base)
        size = np.hypot(ref[..., :D // 2], ref[..., D // 2:])
        size = np.concatenate([size, size], -1)
        tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(ref) + (2.0 ** -16 if dtype == "bf16" else 4e-6) * size
        worst = float((np.abs(got[where] - ref) / (tol + 1e-30)).max())
        say(f"{dtype} D={D} rows={rows}: {worst:.3f} of the bound")
        assert worst <= 1.0


def test_norm_rope_in_place_and_far_positions(ctx):
    # in place over dense inputs; positions of millions, where an fp32 product alone is off by a turn's tenths
    torch, bs, _ = lazy()
    rng = np.random.default_rng(3)
    p, L, D = 9_999_937, 16, 128
    reqs = np.array([(p, L, 0, 0, 5)], bs.REQ_DTYPE)
    q, k = (rng.normal(size=(1, L, h, D)).astype(np.float32) for h in (2, 1))
    dq, dk = torch.from_numpy(q).cuda(), torch.from_numpy(k).cuda()
    bs.bs_qk_norm_rope(ctx, reqs, L, 1, p + L + 5, False, 2, 1, D, bs.BS_F32, dq, 2 * D, dk, D, None, None, 1e-6, 1e4, dq, dk)
    torch.cuda.synchronize()
    for x, d in ((q, dq), (k, dk)):
        ref = quant.norm_rope(x, None, (p + np.arange(L))[None, :, None], 1e-6, 1e4)
        size = np.hypot(ref[..., :D // 2], ref[..., D // 2:])
        assert (np.abs(d.cpu().numpy() - ref) <= 2.0 ** -24 * np.abs(ref) + 4e-6 * np.concatenate([size, size], -1)).all()


# ---------------------------------------------------------------- streams, capture, refusals
def test_another_stream_and_two_at_once(ctx):
    torch, _, _ = lazy()
    rng = np.random.default_rng(6)
    ws = [attention_case(rng, [(300, 64, 1), (2500, 64, 0)], 32, 4, 4, 128, 32, f) for f in ("e4m3", "i8")]
    ds = [on_device(w) for w in ws]
    streams = [torch.cuda.Stream() for _ in ws]
    need = lazy()[1].bs_quant_attention_workspace_bytes(ws[0]["reqs"], 32, 4, 4, 128)
    rooms = [torch.full((max(need, 16),), 0xA5, dtype=torch.uint8, device="cuda") for _ in ws]
    torch.cuda.synchronize()
    for _ in range(3):
        for w, d, s, room in zip(ws, ds, streams, rooms):
            attend(ctx, w, d, stream=s, ws=room)
    torch.cuda.synchronize()
    for w, d in zip(ws, ds):
        check_out(w, d)
        check_cache(w, d, True)


def test_captured_and_replayed(ctx):
    torch, bs, _ = lazy()
    rng = np.random.default_rng(7)
    w = attention_case(rng, [(300, 64, 1), (4000, 64, 0)], 32, 4, 4, 128, 32, "e4m3")
    d = on_device(w)
    need = bs.bs_quant_attention_workspace_bytes(w["reqs"], 32, 4, 4, 128)
    ws = torch.full((max(need, 16),), 0xA5, dtype=torch.uint8, device="cuda")
    box = torch.zeros((w["R"], 4, w["W"], 128), dtype=torch.bfloat16, device="cuda")
    box2 = torch.zeros_like(box)
    qo, ko = torch.empty_like(d["q"]), torch.empty_like(d["k_new"])

    def calls():
        bs.bs_qk_norm_rope(ctx, w["reqs"], 32, w["R"], w["W"], False, 4, 4, 128, bs.BS_BF16, d["q"], 512, d["k_new"], 512,
                           None, None, 1e-6, 1e4, qo, ko)
        bs.bs_quant_cache_block_attention(ctx, w["reqs"], 32, 4, 4, 128, 0, 32, 0.0, qo, ko, d["v_new"], d["k8"],
                                          d["v8"], d["k_scale"], d["v_scale"], w["S"], w["R"], w["W"], True, d["out"],
                                          ws, need)
        bs.bs_kv_dequantize(ctx, w["reqs"], 32, w["R"], w["W"], 4, 128, bs.BS_BF16, 0, 32, d["k8"], d["v8"], d["k_scale"],
                            d["v_scale"], w["S"], box, box2)

    # lists that a launch cannot carry, and that no call outside a capture has uploaded, are refused
    fresh = bs.Context(0)
    many = np.zeros(80, bs.REQ_DTYPE)
    many["p"], many["g"], many["row"] = 1, 2, np.arange(80)
    small = [torch.zeros(80 * 4 * 3 * 128, dtype=torch.bfloat16, device="cuda") for _ in range(6)]
    for call in (lambda: bs.bs_kv_dequantize(fresh, many, 2, 80, 3, 4, 128, bs.BS_BF16, 0, 2, *small[:2], *small[2:4], 3, *small[4:]),
                 lambda: bs.bs_qk_norm_rope(fresh, w["reqs"], 32, w["R"], w["W"], False, 4, 4, 128, bs.BS_BF16, d["q"], 512, d["k_new"],
                                            512, None, None, 1e-6, 1e4, qo, ko)):
        g = torch.cuda.CUDAGraph()
        with pytest.raises(bs.BlockServeError, match="captured"):
            with torch.cuda.graph(g):
                torch.zeros(1, device="cuda").add_(1)
                call()
    fresh.close()
    calls()
    torch.cuda.synchronize()
    want = [x.clone() for x in (d["out"], box, box2, d["k8"], d["k_scale"])]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for rep in range(4):
        for x in (d["out"], box, box2):
            x.zero_()
        # eager work between the replays, with other descriptors, enough to turn the upload slots over
        for i in range(24):
            other = w["reqs"].copy()
            other["p"] -= i + 1
            bs.bs_kv_dequantize(ctx, other, 32, w["R"], w["W"], 4, 128, bs.BS_BF16, 0, 32, d["k8"], d["v8"], d["k_scale"],
                                d["v_scale"], w["S"], torch.empty_like(box), torch.empty_like(box))
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip((d["out"], box, box2, d["k8"], d["k_scale"]), want):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), f"replay {rep}"


def test_captured_by_a_context_that_never_ran():
    # short lists travel with the launch: nothing has to be there before
    torch, bs, _ = lazy()
    rng = np.random.default_rng(17)
    w = attention_case(rng, [(300, 64, 1), (2100, 64, 0)], 32, 14, 2, 128, 32, "e4m3")
    d = on_device(w)
    need = bs.bs_quant_attention_workspace_bytes(w["reqs"], 32, 14, 2, 128)
    assert need > 0                                # the long row is split: two launches
    ws = torch.full((need,), 0xA5, dtype=torch.uint8, device="cuda")
    box = [torch.zeros((w["R"], 2, w["W"], 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    with bs.Context(0) as ctx:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            attend(ctx, w, d, ws=ws)
            bs.bs_kv_dequantize(ctx, w["reqs"], 32, w["R"], w["W"], 2, 128, bs.BS_BF16, 0, 32, d["k8"], d["v8"], d["k_scale"],
                                d["v_scale"], w["S"], *box)
        for _ in range(3):
            d["out"].fill_(float("nan"))
            for x in box:
                x.zero_()
            g.replay()
            torch.cuda.synchronize()
            check_out(w, d)
            check_cache(w, d, True)
            for i, r in enumerate(w["reqs"]):
                t = oracle.geometry(r, 32)
                for c in range(2):
                    num = quant.row_numbers(r, c, d["v8"].cpu().numpy(), d["v_scale"].cpu().numpy(), 32, "e4m3")
                    got = box[1][t.row, c, t.off:t.off + len(num)].float().cpu().numpy()
                    assert (np.abs(got - num) <= 2.0 ** -8 * np.abs(num)).all()


def test_long_lists_captured_and_replayed(ctx):
    # 80 requests: uploaded by the call before, whose slot then keeps them whatever else is uploaded
    torch, bs, _ = lazy()
    rng = np.random.default_rng(18)
    w = attention_case(rng, [(int(rng.integers(0, 90)), int(rng.integers(1, 40)), 0) for _ in range(80)], 8, 4, 2, 64, 8, "e4m3")
    d = on_device(w)
    box = [torch.zeros((w["R"], 2, w["W"], 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    qo, ko = torch.empty_like(d["q"]), torch.empty_like(d["k_new"])

    def calls():
        bs.bs_qk_norm_rope(ctx, w["reqs"], 8, w["R"], w["W"], False, 4, 2, 64, bs.BS_BF16, d["q"], 256, d["k_new"], 128, None,
                           None, 1e-6, 1e4, qo, ko)
        bs.bs_quant_cache_block_attention(ctx, w["reqs"], 8, 4, 2, 64, 0, 8, 0.0, qo, ko, d["v_new"], d["k8"], d["v8"],
                                          d["k_scale"], d["v_scale"], w["S"], w["R"], w["W"], True, d["out"])
        bs.bs_kv_dequantize(ctx, w["reqs"], 8, w["R"], w["W"], 2, 64, bs.BS_BF16, 0, 8, d["k8"], d["v8"], d["k_scale"],
                            d["v_scale"], w["S"], *box)

    calls()
    torch.cuda.synchronize()
    want = [x.clone() for x in (d["out"], *box, d["k8"], d["k_scale"])]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for rep in range(3):
        for x in (d["out"], *box):
            x.zero_()
        for i in range(24):                        # enough other lists to turn the upload slots over
            other = np.roll(w["reqs"], i + 1)
            bs.bs_kv_dequantize(ctx, other, 8, w["R"], w["W"], 2, 64, bs.BS_BF16, 0, 8, d["k8"], d["v8"], d["k_scale"],
                                d["v_scale"], w["S"], torch.empty_like(box[0]), torch.empty_like(box[0]))
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip((d["out"], *box, d["k8"], d["k_scale"]), want):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), f"replay {rep}"


@pytest.mark.parametrize("n", [64, 65, 130])
def test_lists_that_travel_with_the_launch_and_longer_ones(ctx, n):
    torch, bs, bstep = lazy()
    rng = np.random.default_rng(n)
    lens = [(int(rng.integers(0, 70)), int(rng.integers(1, 40)), 0) for _ in range(n - 1)] + [(1500, 40, 0)]
    w = attention_case(rng, lens, 8, 10, 2, 64, 8, "i8")
    d = on_device(w)
    attend(ctx, w, d)
    torch.cuda.synchronize()
    say(f"n={n}: {check_out(w, d):.3f} of the bound")
    check_cache(w, d, True)
    for dt, tol in (("bf16", 2.0 ** -8), ("f32", 2.0 ** -24)):
        box = [torch.zeros((w["R"], 2, w["W"], 64), dtype=bstep.torch_dtype(dt), device="cuda") for _ in range(2)]
        again = [torch.zeros_like(d["k8"]) for _ in range(2)] + [torch.zeros_like(d["k_scale"]) for _ in range(2)]
        bs.bs_kv_dequantize(ctx, w["reqs"], 8, w["R"], w["W"], 2, 64, bstep.dt_code(dt), 1, 8, d["k8"], d["v8"], d["k_scale"],
                            d["v_scale"], w["S"], *box)
        bs.bs_kv_quantize(ctx, w["reqs"], 8, w["R"], w["W"], 2, 64, bstep.dt_code(dt), 1, 8, *box, *again, w["S"])
        torch.cuda.synchronize()
        codes, scales = d["k8"].cpu().numpy(), d["k_scale"].cpu().numpy()
        rc, rs = quant.kv_quantize(w["reqs"], bstep.to_host(box[0]), np.zeros_like(codes), np.zeros_like(scales), 8, "i8", dt)
        np.testing.assert_array_equal(again[0].cpu().numpy(), rc)
        np.testing.assert_array_equal(again[2].cpu().numpy(), rs)
        for r in w["reqs"]:
            for c in range(2):
                num = quant.row_numbers(r, c, codes, scales, 8, "i8")
                got = box[0][r["row"], c, r["off"]:r["off"] + len(num)].double().cpu().numpy()
                assert (np.abs(got - num) <= tol * np.abs(num)).all()


def test_refusals(ctx):
    torch, bs, _ = lazy()
    rng = np.random.default_rng(8)
    w = attention_case(rng, [(40, 64, 1)], 32, 4, 2, 128, 32, "e4m3")
    d = on_device(w)
    before = {a: x.clone() for a, x in d.items()}

    def att(**kw):
        a = dict(L=32, Hq=4, Hkv=2, D=128, fmt=0, T=32, scale=0.0, q=d["q"], S=w["S"], W=w["W"], k8=d["k8"], ks=d["k_scale"],
                 reqs=w["reqs"])
        a.update(kw)
        bs.bs_quant_cache_block_attention(ctx, a["reqs"], a["L"], a["Hq"], a["Hkv"], a["D"], a["fmt"], a["T"], a["scale"],
                                          a["q"], d["k_new"], d["v_new"], a["k8"], d["v8"], a["ks"], d["v_scale"], a["S"],
                                          w["R"], a["W"], True, d["out"])

    for kw, name, msg in [(dict(T=3), "INVALID_ARG", "power of two"), (dict(T=128), "INVALID_ARG", "power of two"),
                          (dict(T=64), "UNSUPPORTED", "does not divide"), (dict(fmt=2), "INVALID_ARG", "format"),
                          (dict(D=96), "UNSUPPORTED", "D in"), (dict(Hq=3), "UNSUPPORTED", "multiple"),
                          (dict(Hq=18), "UNSUPPORTED", "Hq/Hkv"), (dict(S=3), "INVALID_ARG", "scale groups"),
                          (dict(q=None), "INVALID_ARG", "NULL"), (dict(k8=d["k8"].data_ptr() + 8), "INVALID_ARG", "aligned"),
                          (dict(ks=None), "INVALID_ARG", "NULL"), (dict(scale=float("nan")), "INVALID_ARG", "NaN"),
                          (dict(L=65, T=1, S=200, reqs=np.array([(40, 64, 0, 0, 0)], bs.REQ_DTYPE)), "UNSUPPORTED", "L <= 64"), (dict(W=1 << 25), "UNSUPPORTED", "2^31"),
                          (dict(reqs=np.array([(40, 64, 2, 0, 0)], bs.REQ_DTYPE)), "DESCRIPTOR", "block index")]:
        with pytest.raises(bs.BlockServeError, match=msg.replace("^", r"\^")) as e:
            att(**kw)
        assert e.value.name == "BS_ERR_" + name
    box = torch.zeros((w["R"], 2, w["W"], 128), dtype=torch.bfloat16, device="cuda")
    two = torch.zeros_like(box)

    def qz(**kw):
        a = dict(dt=bs.BS_BF16, k=box, v=two, k8=d["k8"], D=128, S=w["S"], Hkv=2)
        a.update(kw)
        bs.bs_kv_quantize(ctx, w["reqs"], 32, w["R"], w["W"], a["Hkv"], a["D"], a["dt"], 0, 32, a["k"], a["v"], a["k8"], d["v8"],
                          d["k_scale"], d["v_scale"], a["S"])

    for kw, name, msg in [(dict(dt=7), "INVALID_ARG", "dtype"), (dict(k=None), "INVALID_ARG", "NULL"), (dict(k8=box), "OVERLAP", "overlap"),
                          (dict(k8=d["v8"]), "OVERLAP", "overlap"), (dict(D=32), "UNSUPPORTED", "D in"), (dict(S=0), "INVALID_ARG", "S must"),
                          (dict(Hkv=40000), "UNSUPPORTED", "Hkv")]:
        with pytest.raises(bs.BlockServeError, match=msg) as e:
            qz(**kw)
        assert e.value.name == "BS_ERR_" + name
    with pytest.raises(bs.BlockServeError, match="overlap"):
        bs.bs_kv_dequantize(ctx, w["reqs"], 32, w["R"], w["W"], 2, 128, bs.BS_BF16, 0, 32, d["k8"], d["v8"], d["k_scale"],
                            d["v_scale"], w["S"], box, box)

    def nr(**kw):
        a = dict(D=128, dt=bs.BS_BF16, qs=512, eps=1e-6, base=1e4, qo=torch.empty_like(d["q"]), W=w["W"], q=d["q"])
        a.update(kw)
        bs.bs_qk_norm_rope(ctx, w["reqs"], 32, w["R"], a["W"], False, 4, 2, a["D"], a["dt"], a["q"], a["qs"], d["k_new"], 256,
                           None, None, a["eps"], a["base"], a["qo"], torch.empty_like(d["k_new"]))

    for kw, name, msg in [(dict(D=100), "UNSUPPORTED", "D % 16"), (dict(D=272), "UNSUPPORTED", "D % 16"), (dict(qs=504), "INVALID_ARG", "strides"),
                          (dict(qs=516), "INVALID_ARG", "strides"), (dict(eps=float("nan")), "INVALID_ARG", "finite"),
                          (dict(base=float("inf")), "INVALID_ARG", "finite"), (dict(qo=d["q"], qs=520), "OVERLAP", "overlaps"),
                          (dict(qo=d["k_new"]), "OVERLAP", "overlaps"), (dict(W=1 << 24), "UNSUPPORTED", "positions"),
                          (dict(q=None), "INVALID_ARG", "NULL")]:
        with pytest.raises(bs.BlockServeError, match=msg) as e:
            nr(**kw)
        assert e.value.name == "BS_ERR_" + name
    torch.cuda.synchronize()
    for a, x in d.items():
        assert torch.equal(x.view(torch.uint8), before[a].view(torch.uint8)), f"a refused call wrote {a}"
    # nothing to do
    none = np.zeros(0, bs.REQ_DTYPE)
    bs.bs_kv_quantize(ctx, none, 32, 1, 1, 2, 128, bs.BS_BF16, 0, 32, None, None, None, None, None, None, 1)
    bs.bs_qk_norm_rope(ctx, none, 32, 1, 1, False, 4, 2, 128, bs.BS_BF16, None, 512, None, 256, None, None, 1e-6, 1e4, None, None)
    assert [bs.bs_kv_scale_groups(*a) for a in ((5, 6, 4), (0, 1, 64), (5, 6, 3), (-1, 2, 4), (3, 0, 4))] == [4, 1, 0, 0, 0]


def test_refusals_of_overlaps_and_of_lists_too_long(ctx):
    torch, bs, _ = lazy()
    reqs = np.array([(5, 8, 0, 0, 0)], bs.REQ_DTYPE)
    k, v, k8, v8 = (torch.zeros(16 * 128, dtype=t, device="cuda") for t in (torch.bfloat16, torch.bfloat16, torch.uint8, torch.uint8))
    ks, vs = (torch.ones(8, device="cuda") for _ in range(2))
    for name, a in (("k over scales", dict(ks=k)), ("codes over scales", dict(vs=k8)), ("one scale tensor", dict(vs=ks)),
                    ("scales that meet", dict(vs=ks.data_ptr() + 16)), ("one code tensor", dict(v8=k8))):
        x = dict(k=k, v=v, k8=k8, v8=v8, ks=ks, vs=vs)
        x.update(a)
        with pytest.raises(bs.BlockServeError, match="overlap") as e:
            bs.bs_kv_quantize(ctx, reqs, 8, 1, 16, 1, 128, bs.BS_BF16, 0, 8, x["k"], x["v"], x["k8"], x["v8"], x["ks"], x["vs"], 8)
        assert e.value.name == "BS_ERR_OVERLAP", name
    for name, a in (("k over scales", dict(ks=k)), ("v over codes", dict(v8=v)), ("one box", dict(v=k))):
        x = dict(k=k, v=v, k8=k8, v8=v8, ks=ks, vs=vs)
        x.update(a)
        with pytest.raises(bs.BlockServeError, match="overlap") as e:
            bs.bs_kv_dequantize(ctx, reqs, 8, 1, 16, 1, 128, bs.BS_BF16, 0, 8, x["k8"], x["v8"], x["ks"], x["vs"], 8, x["k"], x["v"])
        assert e.value.name == "BS_ERR_OVERLAP", name
    many = np.zeros(64, bs.REQ_DTYPE)
    many["p"], many["g"], many["row"] = 5, 8, np.arange(64)
    with pytest.raises(bs.BlockServeError, match="n . Hkv") as e:
        bs.bs_quant_cache_block_attention(ctx, many, 8, 20000, 20000, 64, 0, 8, 0.0, k, k, v, k8, v8, ks, vs, 8, 64, 16, True, k)
    assert e.value.name == "BS_ERR_UNSUPPORTED"
    assert bs.bs_quant_attention_workspace_bytes(many, 8, 20000, 20000, 64) == 0


# ---------------------------------------------------------------- as a serving program uses them
def test_a_layer_from_projection_to_read_back(ctx):
    """Whole rows are normalised, rotated, written and quantised; the block's
    projections follow; attention writes the block; the rows are moved to other
    places of another box and read back there."""
    torch, bs, bstep = lazy()
    rng = np.random.default_rng(12)
    L, Hq, Hkv, D, T, base = 32, 8, 2, 128, 32, 1e4
    reqs, R, W = batch(rng, [(75, 64, 1), (200, 96, 0), (0, 40, 1)], L)
    n, H = len(reqs), Hq + 2 * Hkv
    S = -(-scale_len(reqs, T) // 4) * 4
    x = numbers(rng, (R, W, H * D), "bf16")
    dx = bstep.to_device(x, "bf16")
    qw, kw = bstep.to_device(numbers(rng, (D,), "bf16"), "bf16"), bstep.to_device(numbers(rng, (D,), "bf16"), "bf16")
    q, k = (torch.zeros((R, W, h, D), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv))
    bs.bs_qk_norm_rope(ctx, reqs, L, R, W, True, Hq, Hkv, D, bs.BS_BF16, dx, H * D, dx[..., Hq * D:], H * D, qw, kw, 1e-6, base, q, k)
    v = dx[..., (Hq + Hkv) * D:].reshape(R, W, Hkv, D).contiguous()
    kc, vc, ro = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((R, Hkv, W, D), (R, Hkv, W, D), (R, W, Hq, D)))
    bs.bs_dual_cache_refresh(ctx, reqs, L, Hq, Hkv, D, bs.BS_BF16, 0.0, 0.0, q, k, v, R, W, kc, vc, ro)
    k8, v8 = (torch.zeros((R, Hkv, W, D), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.ones((R, Hkv, S), device="cuda") for _ in range(2))
    bs.bs_kv_quantize(ctx, reqs, L, R, W, Hkv, D, bs.BS_BF16, bs.BS_E4M3, T, kc, vc, k8, v8, ks, vs, S)
    # the block: fresh projections of its tokens
    xb = bstep.to_device(numbers(rng, (n, L, H * D), "bf16"), "bf16")
    qb, kb = (torch.zeros((n, L, h, D), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv))
    bs.bs_qk_norm_rope(ctx, reqs, L, R, W, False, Hq, Hkv, D, bs.BS_BF16, xb, H * D, xb[..., Hq * D:], H * D, qw, kw, 1e-6, base, qb, kb)
    vb = xb[..., (Hq + Hkv) * D:].reshape(n, L, Hkv, D).contiguous()
    host = lambda t: bstep.to_host(t)  # noqa: E731
    w = dict(reqs=reqs, R=R, W=W, S=S, L=L, Hq=Hq, Hkv=Hkv, D=D, T=T, fmt="e4m3", q=host(qb), k_new=host(kb), v_new=host(vb),
             k8=k8.cpu().numpy(), v8=v8.cpu().numpy(), k_scale=ks.cpu().numpy(), v_scale=vs.cpu().numpy())
    d = dict(q=qb, k_new=kb, v_new=vb, k8=k8, v8=v8, k_scale=ks, v_scale=vs, out=torch.empty_like(qb))
    attend(ctx, w, d)
    torch.cuda.synchronize()
    check_out(w, d)
    check_cache(w, d, True)
    # against the bf16 cache: the codes' rounding is what is left (e4m3: 2^-4 of a key or value at most)
    ob, kc2, vc2 = torch.empty_like(qb), kc.clone(), vc.clone()
    bs.bs_dual_cache_block_attention(ctx, reqs, L, Hq, Hkv, D, bs.BS_BF16, 0.0, qb, kb, vb, kc2, vc2, R, W, True, ob)
    torch.cuda.synchronize()
    for i, r in enumerate(reqs):
        B = oracle.geometry(r, L).B
        diff = (ob[i, :B].float() - d["out"][i, :B].float()).norm() / ob[i, :B].float().norm()
        assert diff < 2.0 ** -4, float(diff)
    # move the rows (codes, then scales) and read them back at their new places
    W2, R2 = W + 21, R + 2
    seg, seg_s = np.zeros(n, bs.SEG_DTYPE), np.zeros(n, bs.SEG_DTYPE)
    moved = reqs.copy()
    for i, r in enumerate(reqs):
        ln = int(r["p"] + r["g"])
        moved[i]["row"], moved[i]["off"] = R2 - 1 - i, W2 - ln
        seg[i] = (0, r["row"], r["off"], moved[i]["row"], moved[i]["off"], ln)
        seg_s[i] = (0, r["row"], 0, moved[i]["row"], 0, -(-bs.bs_kv_scale_groups(int(r["p"]), int(r["g"]), T) // 4))
    n8 = [torch.zeros((R2, Hkv, W2, D), dtype=torch.uint8, device="cuda") for _ in range(2)]
    ns = [torch.ones((R2, Hkv, S), device="cuda") for _ in range(2)]
    bs.bs_kv_scatter_compact(ctx, seg, 1, Hkv, D // 2, bs.BS_BF16, k8, v8, k8.numel(), R, W, None, None, 0, 1, 1, n8[0], n8[1],
                             n8[0].numel(), R2, W2)
    bs.bs_kv_scatter_compact(ctx, seg_s, 1, Hkv, 4, bs.BS_F32, ks, vs, ks.numel() * 4, R, S // 4, None, None, 0, 1, 1, ns[0], ns[1],
                             ns[0].numel() * 4, R2, S // 4)
    here = [torch.zeros((R, Hkv, W, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    there = [torch.zeros((R2, Hkv, W2, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    bs.bs_kv_dequantize(ctx, reqs, L, R, W, Hkv, D, bs.BS_BF16, bs.BS_E4M3, T, k8, v8, ks, vs, S, *here)
    bs.bs_kv_dequantize(ctx, moved, L, R2, W2, Hkv, D, bs.BS_BF16, bs.BS_E4M3, T, n8[0], n8[1], ns[0], ns[1], S, *there)
    torch.cuda.synchronize()
    for a, b in zip(here, there):
        for r, m in zip(reqs, moved):
            ln = int(r["p"] + r["g"])
            assert torch.equal(a[r["row"], :, r["off"]:r["off"] + ln], b[m["row"], :, m["off"]:m["off"] + ln])
            assert a[r["row"], :, r["off"]:r["off"] + ln].any()

"""The operators of a cache held in 8 bits, measured call by call.

A serving program that keeps its dual cache in 8 bits normalises and rotates the
projections of a block (or of whole rows, at a refresh), attends the block
against the cache (which quantises the block's own keys and values into it), and
quantises whole rows or reads them back when rows are admitted, refreshed or
inspected. A case is one such call: its request lengths, head shape, format and
number of tokens that share a scale belong to the case; which box row a request
takes and every tensor value come from the seed. With ``own`` the calls go to
the library; without, the same is computed by elementary torch operations in 32
bits (angles in 64).

The scale groups of a row are laid from its first generated token outwards:
token t of a request with prompt length p is in group (t + pad) // T with
pad = -p mod T, so that a block of L tokens is whole groups whenever T divides L.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

# head shapes of the repository's two model configurations, and a small generic one
LLADA = dict(Hq=32, Hkv=32, D=128, base=500000.0)
DREAM = dict(Hq=28, Hkv=4, D=128, base=1000000.0)
SMALL = dict(Hq=8, Hkv=2, D=64, base=10000.0)

QMAX = {"e4m3": 448.0, "i8": 127.0}
FLOOR = 2.0 ** -64      # least group maximum: a group of zeros gets a scale that is not zero


def _case(name, kind, shape, n, p, g, L=32, T=32, fmt="e4m3", dtype="bf16", batch=0):
    c = dict(kind=kind, n=n, p_lo=p[0], p_hi=p[1], g=g, L=L, T=T, fmt=fmt, dtype=dtype, batch=batch, **shape)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's block against its cache: the latency of a call
        _case("attention-llada-e4m3-n1", "attention", LLADA, 1, (64, 512), 256),
        # an ordinary MHA batch: the cache is what is read
        _case("attention-llada-e4m3-n32", "attention", LLADA, 32, (64, 512), 256),
        # an ordinary GQA batch: the matrix products weigh as much as the cache
        _case("attention-dream-e4m3-n64", "attention", DREAM, 64, (128, 1024), 512),
        # short blocks with a ragged last one, int8, prompts of any length
        _case("attention-llada-i8-n24-L16", "attention", LLADA, 24, (1, 700), 200, L=16, T=16, fmt="i8"),
        # single tokens against long rows, a scale for each token
        _case("attention-dream-i8-tokens-n16", "attention", DREAM, 16, (2000, 8000), 512, L=1, T=1, fmt="i8"),
        # queries and keys of every request's block, out of the fused projection
        _case("norm-rope-llada-blocks-n32", "norm_blocks", LLADA, 32, (64, 512), 256),
        # the same for whole rows, at a refresh
        _case("norm-rope-dream-rows-n64", "norm_rows", DREAM, 64, (128, 1024), 512),
        # whole rows into the cache, at admission or after a refresh
        _case("quantize-llada-e4m3-n32", "quantize", LLADA, 32, (64, 512), 256),
        _case("quantize-small-i8-f32-n5", "quantize", SMALL, 5, (1, 300), 77, L=8, T=8, fmt="i8", dtype="f32"),
        # rows read back in the type of the other calls
        _case("dequantize-llada-e4m3-n32", "dequantize", LLADA, 32, (64, 512), 256),
        _case("dequantize-dream-i8-n64", "dequantize", DREAM, 64, (128, 1024), 512, T=16, fmt="i8"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attention", "attention", "attention", "norm_blocks", "norm_rows", "quantize", "dequantize"))
    shape = dict(rng.choice((LLADA, LLADA, DREAM, DREAM, SMALL)))
    if rng.random() < 0.25:
        Hkv = rng.choice((1, 2, 4, 8))
        shape.update(Hq=Hkv * rng.randint(1, 8), Hkv=Hkv, D=rng.choice((64, 128)))
    L = rng.choice((1, 8, 16, 24, 32, 32, 32, 48, 64, rng.randint(1, 64)))
    T = rng.choice([t for t in (1, 2, 4, 8, 16, 32, 64) if L % t == 0])
    g = rng.choice((128, 256, 512, rng.randint(1, 512)))
    p_hi = _log(rng, 16, 8000)
    p_lo = rng.randint(0, p_hi)
    # at most 24576 tokens, a box of as many rows as requests
    n = _log(rng, 1, max(1, min(128, 24576 // (p_hi + g))))
    dtype = rng.choice(("bf16", "bf16", "f32")) if kind != "attention" else "bf16"
    return _case(None, kind, shape, n, (p_lo, p_hi), g, L=L, T=T, fmt=rng.choice(("e4m3", "e4m3", "i8")), dtype=dtype,
                 batch=rng.randint(1, 1 << 20))


# ---------------------------------------------------------------- geometry of a case
def _lengths(c):
    """(p, k) of each request: the case's own, not the seed's."""
    rng = random.Random("%d %d %d %d %d %d" % (c["n"], c["p_lo"], c["p_hi"], c["g"], c["L"], c["batch"]))
    return [(rng.randint(c["p_lo"], c["p_hi"]), rng.randrange(-(-c["g"] // c["L"]))) for _ in range(c["n"])]


def _geometry(c, seed):
    """Requests as a structured array (rows shuffled by the seed, cells at the right end of the box)."""
    rng = random.Random("%d %s" % (seed, sorted((k, v) for k, v in c.items() if k != "name")))
    rows = _lengths(c)
    rng.shuffle(rows)
    place = list(range(c["n"]))
    rng.shuffle(place)
    p = np.array([r[0] for r in rows], np.int64)
    W = int(p.max()) + c["g"]
    reqs = np.zeros(c["n"], [("p", "<i4"), ("g", "<i4"), ("k", "<i4"), ("row", "<i4"), ("off", "<i4")])
    reqs["p"], reqs["g"], reqs["k"] = p, c["g"], [r[1] for r in rows]
    reqs["row"], reqs["off"] = place, W - p - c["g"]
    return reqs, W


def _groups(c, reqs):
    """Scale groups of the longest row."""
    T = c["T"]
    return int((-(-reqs["p"].astype(np.int64) // T) + -(-reqs["g"].astype(np.int64) // T)).max())


def _plan(c, reqs, whole):
    """Flat lists of the cells a call works on: request, place in the request's list, box row, column, position, group."""
    p, g, k = (reqs[x].astype(np.int64) for x in ("p", "g", "k"))
    s = np.zeros_like(p) if whole else p + k * c["L"]
    count = p + g if whole else np.minimum(c["L"], g - k * c["L"])
    i = np.repeat(np.arange(len(reqs)), count)
    j = np.arange(int(count.sum())) - np.repeat(np.cumsum(count) - count, count)
    t = s[i] + j
    grp = (t + (-p[i]) % c["T"]) // c["T"]
    dev = torch.device("cuda")
    return {a: torch.from_numpy(np.ascontiguousarray(b, dtype=np.int64)).to(dev) for a, b in
            dict(i=i, j=j, row=reqs["row"][i], col=reqs["off"][i] + t, pos=t, grp=grp).items()}


def _cached_plan(c, reqs):
    """Cells outside the active block, padded to the longest request's number of them: [n][M] columns, groups, validity."""
    p, g, k, off = (reqs[x].astype(np.int64)[:, None] for x in ("p", "g", "k", "off"))
    s = p + k * c["L"]
    B = np.minimum(c["L"], g - k * c["L"])
    m = np.arange(max(1, int((p + g - B).max())))[None]
    t = np.minimum(m + np.where(m >= s, B, 0), p + g - 1)
    dev = torch.device("cuda")
    return {a: torch.from_numpy(np.ascontiguousarray(b)).to(dev) for a, b in
            dict(col=off + t, grp=(t + (-p) % c["T"]) // c["T"], ok=m < p + g - B,
                 own=np.arange(c["L"])[None] < B).items()}


# ---------------------------------------------------------------- inputs
def _code_type(fmt):
    return torch.float8_e4m3fn if fmt == "e4m3" else torch.int8


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _tensors(c, seed):
    reqs, W = _geometry(c, seed)
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 17)
    td, n, L, Hq, Hkv, D = _dtype(c), c["n"], c["L"], c["Hq"], c["Hkv"], c["D"]

    def normal(shape):
        return torch.empty(shape, dtype=td, device=dev).normal_(generator=gen)

    # a few features of the keys are several times larger than the rest, and heads
    # differ in size, as in trained models
    kf = (1.0 + 3.0 * (torch.rand(Hkv, D, device=dev, generator=gen) < 0.04).float()).to(td)
    vf = torch.exp(torch.empty(Hkv, 1, device=dev).normal_(generator=gen)).to(td)
    t = dict(reqs=reqs, W=W, S=_groups(c, reqs))
    if c["kind"] in ("norm_blocks", "norm_rows"):
        lead = (n, L) if c["kind"] == "norm_blocks" else (n, W)
        # the fused projection: queries, keys and values of a token side by side
        t["qkv"] = normal(lead + ((Hq + 2 * Hkv) * D,))
        t["qw"], t["kw"] = (1.0 + 0.2 * normal((D,))).to(td), (1.0 + 0.2 * normal((D,))).to(td)
        t["plan"] = _plan(c, reqs, c["kind"] == "norm_rows")
        return t
    t["k"], t["v"] = normal((n, Hkv, W, D)) * kf[:, None], normal((n, Hkv, W, D)) * vf[:, None]
    t["plan"] = _plan(c, reqs, True)
    if c["kind"] == "attention":
        t["q"] = normal((n, L, Hq, D))
        t["k_new"], t["v_new"] = normal((n, L, Hkv, D)) * kf, normal((n, L, Hkv, D)) * vf
        t["block"], t["cached"] = _plan(c, reqs, False), _cached_plan(c, reqs)
    return t


class _State:
    pass


def _empty_cache(c, t):
    dev = torch.device("cuda")
    box = (c["n"], c["Hkv"], t["W"], c["D"])
    sc = (c["n"], c["Hkv"], t["S"])
    return dict(k8=torch.zeros(box, dtype=torch.uint8, device=dev).view(_code_type(c["fmt"])),
                v8=torch.zeros(box, dtype=torch.uint8, device=dev).view(_code_type(c["fmt"])),
                k_scale=torch.ones(sc, dtype=torch.float32, device=dev),
                v_scale=torch.ones(sc, dtype=torch.float32, device=dev))


def prepare(case, seed):
    c, t = case, _tensors(case, seed)
    s = _State()
    s.c, s.t = c, t
    dev, td = torch.device("cuda"), _dtype(c)
    n, W, L, Hq, Hkv, D = c["n"], t["W"], c["L"], c["Hq"], c["Hkv"], c["D"]
    if c["kind"] in ("norm_blocks", "norm_rows"):
        lead = (n, L) if c["kind"] == "norm_blocks" else (n, W)
        s.q_out = torch.zeros(lead + (Hq, D), dtype=td, device=dev)
        s.k_out = torch.zeros(lead + (Hkv, D), dtype=td, device=dev)
        return s
    s.cache = _empty_cache(c, t)
    if c["kind"] in ("attention", "dequantize"):
        _plain_quantize(c, t, s.cache)
    if c["kind"] == "dequantize":
        s.k_box = torch.zeros((n, Hkv, W, D), dtype=td, device=dev)
        s.v_box = torch.zeros_like(s.k_box)
    if c["kind"] != "quantize":
        del t["k"], t["v"]
    if c["kind"] == "attention":
        s.out = torch.zeros((n, L, Hq, D), dtype=td, device=dev)
    s.ws = {}
    return s


# ---------------------------------------------------------------- the plain forms
def _plain_norm_rope(c, t, q_out, k_out):
    D, Hq, Hkv, pl = c["D"], c["Hq"], c["Hkv"], t["plan"]
    a, b = (pl["i"], pl["j"]) if c["kind"] == "norm_blocks" else (pl["row"], pl["col"])
    x = t["qkv"][a, b].float()
    f = torch.arange(D // 2, dtype=torch.float64, device=x.device)
    ang = pl["pos"].double()[:, None] * torch.exp(f * (-2.0 * math.log(c["base"]) / D))
    cs, sn = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]

    def one(y, w, out):
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        y1, y2 = y[..., : D // 2], y[..., D // 2:]
        out[a, b] = torch.cat([y1 * cs - y2 * sn, y2 * cs + y1 * sn], dim=-1).to(out.dtype)

    one(x[:, : Hq * D].view(-1, Hq, D), t["qw"], q_out)
    one(x[:, Hq * D: (Hq + Hkv) * D].view(-1, Hkv, D), t["kw"], k_out)
    return dict(q=q_out, k=k_out)


def _plain_codes(c, pl, x, R, S, codes, scales):
    """x [N][Hkv][D]: the cells listed in pl, into the boxes of codes and scales."""
    Hkv, at = c["Hkv"], pl["row"] * S + pl["grp"]
    x = x.float()
    top = torch.zeros((R * S, Hkv), dtype=torch.float32, device=x.device).index_reduce_(0, at, x.abs().amax(-1), "amax")
    top = top.clamp_min(FLOOR)
    qmax = torch.full_like(top, QMAX[c["fmt"]])
    y = x * torch.div(qmax, top)[at][..., None]
    y = y.to(torch.float8_e4m3fn) if c["fmt"] == "e4m3" else torch.round(y).to(torch.int8)
    codes.view(torch.uint8)[pl["row"], :, pl["col"]] = y.view(torch.uint8)
    scales[pl["row"], :, pl["grp"]] = torch.div(top, qmax)[at]


def _plain_quantize(c, t, cache):
    """Whole rows of the boxes t["k"], t["v"]."""
    pl = t["plan"]
    _plain_codes(c, pl, t["k"][pl["row"], :, pl["col"]], c["n"], t["S"], cache["k8"], cache["k_scale"])
    _plain_codes(c, pl, t["v"][pl["row"], :, pl["col"]], c["n"], t["S"], cache["v8"], cache["v_scale"])
    return cache


def _plain_dequantize(c, t, cache, k_box, v_box):
    pl = t["plan"]

    def one(codes, scales, out):
        y = codes.view(torch.uint8)[pl["row"], :, pl["col"]].view(codes.dtype).float()
        out[pl["row"], :, pl["col"]] = (y * scales[pl["row"], :, pl["grp"]][..., None]).to(out.dtype)

    one(cache["k8"], cache["k_scale"], k_box)
    one(cache["v8"], cache["v_scale"], v_box)
    return dict(k=k_box, v=v_box)


def _plain_attention(c, t, cache, out):
    n, L, Hq, Hkv, D = c["n"], c["L"], c["Hq"], c["Hkv"], c["D"]
    G, cp = Hq // Hkv, t["cached"]
    row = torch.from_numpy(t["reqs"]["row"].astype(np.int64)).to(out.device)[:, None]

    def keys(codes, scales, new):
        x = codes.view(torch.uint8)[row, :, cp["col"]].view(codes.dtype).float() * scales[row, :, cp["grp"]][..., None]
        return torch.cat([torch.where(cp["ok"][..., None, None], x, 0.0),
                          torch.where(cp["own"][..., None, None], new.float(), 0.0)], dim=1).transpose(1, 2).contiguous()

    K, V = keys(cache["k8"], cache["k_scale"], t["k_new"]), keys(cache["v8"], cache["v_scale"], t["v_new"])
    q = t["q"].float().view(n, L, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * L, D)
    sc = torch.matmul(q, K.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(D))
    sc = sc.masked_fill(~torch.cat([cp["ok"], cp["own"]], dim=1)[:, None, None], -math.inf)
    e = torch.exp(sc - sc.amax(-1, keepdim=True))
    o = torch.matmul(e, V) / e.sum(-1, keepdim=True)
    o = o.view(n, Hkv, G, L, D).permute(0, 3, 1, 2, 4).reshape(n, L, Hq, D)
    out.copy_(torch.where(cp["own"][..., None, None], o, 0.0))
    pl = t["block"]
    _plain_codes(c, pl, t["k_new"][pl["i"], pl["j"]], n, t["S"], cache["k8"], cache["k_scale"])
    _plain_codes(c, pl, t["v_new"][pl["i"], pl["j"]], n, t["S"], cache["v8"], cache["v_scale"])
    return dict(out=out, **cache)


# ---------------------------------------------------------------- the library's calls
_contexts = {}


def _context(bs):
    """One library context per process, as a serving program keeps it."""
    if "ctx" not in _contexts:
        _contexts["ctx"] = bs.Context(0)
    return _contexts["ctx"]


def _own(s):
    import paper_2607_08930_amd as bs
    c, t, ctx = s.c, s.t, _context(bs)
    reqs, W, S, n = t["reqs"], t["W"], t["S"], c["n"]
    L, T, Hq, Hkv, D = c["L"], c["T"], c["Hq"], c["Hkv"], c["D"]
    dt = bs.BS_BF16 if c["dtype"] == "bf16" else bs.BS_F32
    if c["kind"] in ("norm_blocks", "norm_rows"):
        qkv, stride = t["qkv"], (Hq + 2 * Hkv) * D
        bs.bs_qk_norm_rope(ctx, reqs, L, n, W, c["kind"] == "norm_rows", Hq, Hkv, D, dt, qkv, stride,
                           qkv[..., Hq * D:], stride, t["qw"], t["kw"], 1e-6, c["base"], s.q_out, s.k_out)
        return dict(q=s.q_out, k=s.k_out)
    fmt = bs.BS_E4M3 if c["fmt"] == "e4m3" else bs.BS_I8
    x = s.cache
    if c["kind"] == "quantize":
        bs.bs_kv_quantize(ctx, reqs, L, n, W, Hkv, D, dt, fmt, T, t["k"], t["v"], x["k8"], x["v8"], x["k_scale"],
                          x["v_scale"], S)
        return x
    if c["kind"] == "dequantize":
        bs.bs_kv_dequantize(ctx, reqs, L, n, W, Hkv, D, dt, fmt, T, x["k8"], x["v8"], x["k_scale"], x["v_scale"], S,
                            s.k_box, s.v_box)
        return dict(k=s.k_box, v=s.v_box)
    if not s.ws:    # the workspace of this batch, kept from pass to pass
        need = bs.bs_quant_attention_workspace_bytes(reqs, L, Hq, Hkv, D)
        s.ws["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        s.ws["bytes"] = need
    bs.bs_quant_cache_block_attention(ctx, reqs, L, Hq, Hkv, D, fmt, T, 0.0, t["q"], t["k_new"], t["v_new"], x["k8"],
                                      x["v8"], x["k_scale"], x["v_scale"], S, n, W, True, s.out, s.ws["ws"],
                                      s.ws["bytes"])
    return dict(out=s.out, **x)


def run(s):
    if own:
        return _own(s)
    c, t = s.c, s.t
    if c["kind"] in ("norm_blocks", "norm_rows"):
        return _plain_norm_rope(c, t, s.q_out, s.k_out)
    if c["kind"] == "quantize":
        return _plain_quantize(c, t, s.cache)
    if c["kind"] == "dequantize":
        return _plain_dequantize(c, t, s.cache, s.k_box, s.v_box)
    return _plain_attention(c, t, s.cache, s.out)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    eb = 4 if c["dtype"] == "f32" else 2
    L, T, Hq, Hkv, D = c["L"], c["T"], c["Hq"], c["Hkv"], c["D"]
    by = fl = 0
    for p, k in _lengths(c):
        ln = p + c["g"]
        B = min(L, c["g"] - k * L)
        groups = -(-p // T) + -(-c["g"] // T)
        if c["kind"] == "attention":
            # cached codes and scales, queries and outputs, the block's keys and
            # values read once, and their codes and scales written
            by += 2 * (ln * Hkv * D + groups * Hkv * 4) + (2 * B * Hq + 2 * B * Hkv) * D * eb
            fl += 4 * B * ln * Hq * D
        elif c["kind"] in ("norm_blocks", "norm_rows"):
            m = ln if c["kind"] == "norm_rows" else B
            by += 2 * m * (Hq + Hkv) * D * eb
            fl += 9 * m * (Hq + Hkv) * D
        else:
            by += 2 * (ln * Hkv * D * (eb + 1) + groups * Hkv * 4)
            fl += 2 * 2 * ln * Hkv * D
    return {"bytes": by, "flops": fl}


# ---------------------------------------------------------------- the same in 64 bits
def _exact_group(fmt, x):
    """Codes (the values they stand for) and scale of one group, x [Hkv][tokens][D] in 64 bits."""
    top = x.abs().amax(dim=(1, 2)).clamp_min(FLOOR)
    scale = top / QMAX[fmt]
    y = x / scale[:, None, None]
    if fmt == "i8":
        return torch.round(y), scale
    # e4m3: three bits after the leading one, exponents down to -6
    e = torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(y / step) * step, scale


def _exact_norm_rope(c, t):
    D, Hq, Hkv = c["D"], c["Hq"], c["Hkv"]
    lead = tuple(t["qkv"].shape[:2])
    dev = t["qkv"].device
    res = {}
    f = torch.arange(D // 2, dtype=torch.float64, device=dev)
    for name, w, lo, H in (("q", t["qw"], 0, Hq), ("k", t["kw"], Hq * D, Hkv)):
        out = torch.zeros(lead + (H, D), dtype=torch.float64, device=dev)
        for i, r in enumerate(t["reqs"]):
            p, g, k, row, off = (int(r[a]) for a in ("p", "g", "k", "row", "off"))
            if c["kind"] == "norm_rows":
                at, first, m = (row, slice(off, off + p + g)), 0, p + g
            else:
                m = min(c["L"], g - k * c["L"])
                at, first = (i, slice(0, m)), p + k * c["L"]
            x = t["qkv"][at][:, lo:lo + H * D].double().view(m, H, D)
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + 1e-6) * w.double()
            ang = (first + torch.arange(m, dtype=torch.float64, device=dev))[:, None] * c["base"] ** (-2.0 * f / D)
            z = torch.complex(x[..., : D // 2], x[..., D // 2:]) * torch.polar(torch.ones_like(ang), ang)[:, None]
            out[at] = torch.cat([z.real, z.imag], dim=-1)
        res[name] = out
    return res


def exact(case, seed):
    c, t = case, _tensors(case, seed)
    if c["kind"] in ("norm_blocks", "norm_rows"):
        return _exact_norm_rope(c, t)
    n, L, T, Hq, Hkv, D, fmt = c["n"], c["L"], c["T"], c["Hq"], c["Hkv"], c["D"], c["fmt"]
    dev = torch.device("cuda")
    cache = _empty_cache(c, t)
    s8, f8 = {}, {}
    if c["kind"] == "quantize":
        for a in "kv":
            s8[a] = torch.ones((n, Hkv, t["S"]), dtype=torch.float64, device=dev)
            f8[a] = torch.zeros((n, Hkv, t["W"], D), dtype=torch.float64, device=dev)
            for r in t["reqs"]:
                p, g, row, off = (int(r[b]) for b in ("p", "g", "row", "off"))
                pad = (-p) % T
                for j in range(-(-(p + g + pad) // T)):
                    cells = slice(off + max(0, j * T - pad), off + min(p + g, (j + 1) * T - pad))
                    f8[a][row, :, cells], s8[a][row, :, j] = _exact_group(fmt, t[a][row, :, cells].double())
        return dict(k8=f8["k"] if fmt == "e4m3" else None, v8=f8["v"] if fmt == "e4m3" else None,
                    k_scale=s8["k"], v_scale=s8["v"])
    _plain_quantize(c, t, cache)     # the inputs of the call, not its result
    for a in "kv":
        full = torch.zeros((n, Hkv, t["W"], D), dtype=torch.float64, device=dev)
        for r in t["reqs"]:
            p, g, row, off = (int(r[b]) for b in ("p", "g", "row", "off"))
            at = (torch.arange(p + g, device=dev) + (-p) % T) // T
            cells = slice(off, off + p + g)
            full[row, :, cells] = cache[a + "8"][row, :, cells].double() * cache[a + "_scale"][row][:, at].double()[..., None]
        f8[a] = full
    if c["kind"] == "dequantize":
        return dict(k=f8["k"], v=f8["v"])
    out = torch.zeros((n, L, Hq, D), dtype=torch.float64, device=dev)
    sk, sv = cache["k_scale"].double(), cache["v_scale"].double()
    for i, r in enumerate(t["reqs"]):
        p, g, k, row, off = (int(r[b]) for b in ("p", "g", "k", "row", "off"))
        s, B = p + k * L, min(L, g - k * L)
        kk, vv = (f8[a][row, :, off:off + p + g].clone() for a in "kv")
        kk[:, s:s + B] = t["k_new"][i, :B].double().transpose(0, 1)
        vv[:, s:s + B] = t["v_new"][i, :B].double().transpose(0, 1)
        q = t["q"][i, :B].double().view(B, Hkv, Hq // Hkv, D).permute(1, 2, 0, 3).reshape(Hkv, -1, D)
        w = torch.softmax(torch.bmm(q, kk.transpose(1, 2).contiguous()) / math.sqrt(D), dim=2)
        o = torch.bmm(w, vv).view(Hkv, Hq // Hkv, B, D).permute(2, 0, 1, 3)
        out[i, :B] = o.reshape(B, Hq, D)
        for j in range(-(-B // T)):
            at = (s + j * T + (-p) % T) // T
            cells = slice(j * T, min(B, (j + 1) * T))
            sk[row, :, at] = _exact_group(fmt, t["k_new"][i, cells].double().transpose(0, 1))[1]
            sv[row, :, at] = _exact_group(fmt, t["v_new"][i, cells].double().transpose(0, 1))[1]
    return dict(out=out, k8=None, v8=None, k_scale=sk, v_scale=sv)

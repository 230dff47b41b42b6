"""The 8-bit dual cache and the per-head norms where the step and the server use
them: closed-loop serving against the same run with a bf16 cache, the state's step
against the oracle, rows moved between caches.

The providers draw queries, keys and values from a seeded generator that nothing
else touches, so two runs of one stream see the same numbers, and the decisions
come from the logits alone. A block of L tokens is whole scale groups, so what the
8-bit cache holds after any history of admissions, refreshes and steps is the
quantised form of what the bf16 cache holds, bit for bit."""
import numpy as np
import pytest

import oracle
import synth
from gpu_util import lazy, say
from oracle import quant
from oracle import schedule as osch
from test_gpu_quant import batch, bf16, check_out, logical, nan_outside, numbers
from test_gpu_serve import EOS_ID, L, MASK_ID, TAU, V, RefreshProvider, eos_blocks

pytestmark = pytest.mark.gpu

ROWS, WIDTH, HQ, HKV, D, LAYERS, BASE = 5, 80, 6, 2, 128, 2, 1e4


class Provider(RefreshProvider):
    """Keeps the last step's projections; weights of the norms when asked for."""

    def __init__(self, eos_block):
        super().__init__(LAYERS, eos_block, HQ, HKV, D, ROWS, WIDTH)
        self.last_step = None
        rng = np.random.default_rng(5)
        self.weights = [bf16(1 + 0.1 * rng.normal(size=(2, D))) for _ in range(LAYERS)]

    def step(self, ids, descs, cycle, step):
        layers, logits = super().step(ids, descs, cycle, step)
        self.last_step, self.last_descs = layers, descs.copy()
        return layers, logits

    def qk_weights(self, layer):
        _, _, bstep = lazy()
        return [bstep.to_device(x, "bf16") for x in self.weights[layer]]


def serve_once(max_cycles=1_000_000, **cfg):
    torch, bs, _ = lazy()
    from paper_2607_08930_amd import serve
    stream = synth.serve_stream(12, L)
    with bs.Context(0) as ctx:
        sc = serve.ServeConfig(L=L, layers=LAYERS, Hq=HQ, Hkv=HKV, D=D, V=V, dtype="bf16", rows=ROWS, width=WIDTH,
                               policy=osch.BUDGET, budget=220, order=osch.ASCENDING, tau=TAU, eos_id=EOS_ID,
                               mask_id=MASK_ID, rope_base=BASE, **cfg)
        prov = Provider(eos_blocks(stream))
        srv = serve.Server(ctx, sc, prov)
        res = srv.run(stream, max_cycles=max_cycles)
        torch.cuda.synchronize()
    return res, srv, prov


@pytest.mark.parametrize("refresh", [False, True])
@pytest.mark.parametrize("cache,group,qk_eps", [("e4m3", 0, -1.0), ("i8", 2, -1.0), ("e4m3", 4, 1e-6)])
def test_serving_with_an_8_bit_cache(cache, group, qk_eps, refresh):
    _, bs, bstep = lazy()
    say(f"cache={cache} group={group} eps={qk_eps} refresh={refresh}")
    plain, _, _ = serve_once(refresh=refresh, qk_eps=qk_eps)
    res, _, _ = serve_once(refresh=refresh, qk_eps=qk_eps, cache=cache, cache_group=group)
    assert res.admitted == plain.admitted and res.evicted == plain.evicted and res.steps == plain.steps
    assert res.refreshes == plain.refreshes == (LAYERS * res.cycles if refresh else 0)
    assert sorted(res.outputs) == sorted(plain.outputs)
    for rid, toks in plain.outputs.items():
        np.testing.assert_array_equal(res.outputs[rid], toks, err_msg=f"request {rid}")
    # after some cycles: the cache is the quantised bf16 cache, the outputs the attention over it
    for cycles in (1, 4):
        _, want, _ = serve_once(cycles, refresh=refresh, qk_eps=qk_eps)
        _, got, prov = serve_once(cycles, refresh=refresh, qk_eps=qk_eps, cache=cache, cache_group=group)
        T, descs = got.quant.T, prov.last_descs
        assert T == (group or L) and len(descs) > 0
        used = logical(descs, ROWS, WIDTH)
        for l in range(LAYERS):
            w = dict(reqs=descs, L=L, T=T, fmt=cache)
            for x, box, codes, scales in (("k", want.k_box, got.quant.k, got.quant.k_scale),
                                          ("v", want.v_box, got.quant.v, got.quant.v_scale)):
                cd, sc = codes[l].cpu().numpy(), scales[l].cpu().numpy()
                rc, rs = quant.kv_quantize(descs, bstep.to_host(box[l]), cd, sc, T, cache, "bf16")
                np.testing.assert_array_equal(cd.transpose(0, 2, 1, 3)[used], rc.transpose(0, 2, 1, 3)[used])
                np.testing.assert_array_equal(sc, rs)
                w[x + "8"], w[x + "_scale"] = cd, sc
            q, kn, vn = prov.last_step[l]
            if qk_eps >= 0:       # the server's own norms and rotation
                with bs.Context(0) as got.ctx:
                    q, kn = got._ready(l, descs, q, kn, False)
            w.update(q=bstep.to_host(q), k_new=bstep.to_host(kn), v_new=bstep.to_host(vn))
            say(f"  cycles={cycles} layer {l}: {check_out(w, dict(out=got.out[l][:len(descs)])):.3f} of the bound")


def test_served_norms_are_the_formula_s():
    # the block's keys as the cache holds them after a cycle
    _, _, bstep = lazy()
    _, srv, prov = serve_once(1, qk_eps=1e-6)
    for l in range(LAYERS):
        raw = oracle.widen(bstep.to_host(prov.last_step[l][1]), "bf16")
        weight = oracle.widen(prov.weights[l][1], "bf16")
        box = oracle.widen(bstep.to_host(srv.k_box[l]), "bf16")
        for i, r in enumerate(prov.last_descs):
            t = oracle.geometry(r, L)
            ref = quant.norm_rope(raw[i, :t.B], weight, (t.s + np.arange(t.B))[:, None], 1e-6, BASE)
            size = np.hypot(ref[..., :D // 2], ref[..., D // 2:])
            got = box[t.row, :, t.off + t.s:t.off + t.e].transpose(1, 0, 2)
            assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -16 * np.concatenate([size, size], -1)).all()


@pytest.mark.parametrize("fused,split", [(True, True), (False, True), (True, False)])
def test_step_with_an_8_bit_cache(fused, split):
    """One step of the state: attention and write per layer, then the decode on the dense boxes."""
    torch, bs, bstep = lazy()
    from paper_2607_08930_amd.quant_cache import QuantCache
    rng = np.random.default_rng(21)
    blk, heads, kv, vocab = 32, 4, 4, 1000
    with bs.Context(0) as ctx:
        reqs, R, W = batch(rng, [(70, 64, 1), (2300, 96, 0), (0, 40, 1)], blk)
        n, used = len(reqs), logical(reqs, R, W)
        cache = QuantCache(2, R, W, kv, D, blk, "e4m3")
        lays, host = [], []
        for l in range(2):
            kc, vc = (nan_outside(numbers(rng, (R, kv, W, D), "bf16"), used, "bf16") for _ in range(2))
            cache.write(ctx, reqs, l, bstep.to_device(kc, "bf16"), bstep.to_device(vc, "bf16"))
            q, kn, vn = (numbers(rng, (n, blk, h, D), "bf16") for h in (heads, kv, kv))
            lays.append(bstep.Layer(*(bstep.to_device(x, "bf16") for x in (q, kn, vn)), None, None,
                                    torch.empty((n, blk, heads, D), dtype=torch.bfloat16, device="cuda")))
            host.append(dict(reqs=reqs, L=blk, T=32, fmt="e4m3", q=q, k_new=kn, v_new=vn))
        logits = numbers(rng, (n, blk, vocab), "bf16", 4.0)
        tok, msk = np.full((R, W), 7, np.int32), np.ones((R, W), np.uint8)
        st = bstep.StepState(L=blk, Hq=heads, Hkv=kv, D=D, V=vocab, dtype="bf16", R=R, W=W,
                             tokens=torch.from_numpy(tok).cuda(), mask=torch.from_numpy(msk).cuda(), layers=lays,
                             logits=bstep.to_device(logits, "bf16"), n_max=n, tau=0.5, cache=cache).alloc()
        bstep.run_step(ctx, st, reqs, fused=fused, split=split)
        torch.cuda.synchronize()
        for l, w in enumerate(host):
            w.update(k8=cache.k[l].cpu().numpy(), v8=cache.v[l].cpu().numpy(), k_scale=cache.k_scale[l].cpu().numpy(),
                     v_scale=cache.v_scale[l].cpu().numpy())
            say(f"layer {l}: {check_out(w, dict(out=lays[l].out)):.3f} of the bound")
            for i, r in enumerate(reqs):
                t = oracle.geometry(r, blk)
                for c in range(kv):
                    cd, _ = quant.quantize_tokens(oracle.widen(w["v_new"][i, :t.B, c], "bf16"), t.s, t.p, 32, "e4m3")
                    np.testing.assert_array_equal(w["v8"][t.row, c, t.off + t.s:t.off + t.e], cd)
        # the decode is the bf16 state's, with no layers
        plain = bstep.StepState(L=blk, Hq=heads, Hkv=kv, D=D, V=vocab, dtype="bf16", R=R, W=W,
                                tokens=torch.from_numpy(tok).cuda(), mask=torch.from_numpy(msk).cuda(), layers=[],
                                logits=st.logits, n_max=n, tau=0.5).alloc()
        bstep.run_step(ctx, plain, reqs)
        torch.cuda.synchronize()
        assert torch.equal(st.tokens, plain.tokens) and torch.equal(st.mask, plain.mask)
        assert (plain.mask.cpu().numpy() != msk).any()


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
def test_rows_move_between_caches(fmt):
    """A row that changes its column, one that changes its row, one that is admitted, one whose box grows."""
    torch, bs, bstep = lazy()
    from paper_2607_08930_amd.quant_cache import QuantCache
    rng = np.random.default_rng(22)
    R, W, blk, kv, T = 6, 120, 16, 2, 8
    reqs = np.array([(21, 32, 0, 0, 5), (40, 16, 0, 2, 60), (9, 30, 1, 4, 70)], bs.REQ_DTYPE)
    k, v = (numbers(rng, (2, R, kv, W, D), "bf16") for _ in range(2))
    sk, sv = (numbers(rng, (2, 1, kv, 50, D), "bf16") for _ in range(2))
    with bs.Context(0) as ctx:
        def read(c, q, l):
            o = [torch.zeros((c.R, kv, c.W, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            c.read(ctx, q, l, *o)
            torch.cuda.synchronize()
            return [[x[r["row"], :, r["off"]:r["off"] + r["p"] + r["g"]].clone() for r in q] for x in o]

        a = QuantCache(2, R, W, kv, D, blk, fmt, T)
        for l in range(2):
            a.write(ctx, reqs, l, bstep.to_device(k[l], "bf16"), bstep.to_device(v[l], "bf16"))
        before = [read(a, reqs, l) for l in range(2)]
        # within the box: row 0 to another column, row 2 to row 3, row 4 stays
        moved = reqs.copy()
        moved[0]["off"], moved[1]["row"], moved[1]["off"] = 66, 3, 1
        a.move(ctx, np.array([(0, 0, 5, 0, 66, 53), (0, 2, 60, 3, 1, 56)], bs.SEG_DTYPE), a)
        # a request of 13 + 37 tokens into row 1
        a.admit(ctx, np.array([(1, 0, 0, 1, 60, 50)], bs.SEG_DTYPE), [13], [37], bstep.to_device(sk, "bf16"),
                bstep.to_device(sv, "bf16"))
        new = np.array([(13, 37, 0, 1, 60)], bs.REQ_DTYPE)
        for l in range(2):
            for x, y in zip(read(a, moved, l), before[l]):
                assert all(torch.equal(p, q) for p, q in zip(x, y))
            for x, box, codes, scales in zip(read(a, new, l), (sk, sv), (a.k, a.v), (a.k_scale, a.v_scale)):
                for c in range(kv):
                    cd, sc = quant.quantize_tokens(oracle.widen(box[l, 0, c], "bf16"), 0, 13, T, fmt)
                    np.testing.assert_array_equal(codes[l, 1, c, 60:110].cpu().numpy(), cd)
                    assert all(scales[l, 1, c, j].item() == s for j, s in sc.items())
        # into a larger box, with another number of scales a row
        b = QuantCache(2, 4, 400, kv, D, blk, fmt, T)
        there = moved.copy()
        there["row"], there["off"] = [3, 0, 1], [300, 0, 77]
        b.move(ctx, np.array([(0, m["row"], m["off"], t["row"], t["off"], m["p"] + m["g"]) for m, t in zip(moved, there)],
                             bs.SEG_DTYPE), a)
        for l in range(2):
            for x, y in zip(read(b, there, l), before[l]):
                assert all(torch.equal(p, q) for p, q in zip(x, y))
        # two rows change places inside a box, at columns where their cells do not meet
        c = QuantCache(2, 2, 300, kv, D, blk, fmt, T)
        pair = moved[:2].copy()
        pair["row"], pair["off"] = [0, 1], [0, 60]
        c.move(ctx, np.array([(0, m["row"], m["off"], t["row"], t["off"], m["p"] + m["g"]) for m, t in zip(moved, pair)],
                             bs.SEG_DTYPE), a)
        swapped = pair.copy()
        swapped["row"], swapped["off"] = [1, 0], [200, 200]
        c.move(ctx, np.array([(0, m["row"], m["off"], t["row"], t["off"], m["p"] + m["g"]) for m, t in zip(pair, swapped)],
                             bs.SEG_DTYPE), c)
        for l in range(2):
            for x, y in zip(read(c, swapped, l), before[l]):
                assert all(torch.equal(p, q) for p, q in zip(x, y[:2]))
        with pytest.raises(ValueError, match="rows move whole"):
            c.move(ctx, np.array([(0, 0, 0, 1, 0, 10), (0, 1, 0, 1, 20, 10)], bs.SEG_DTYPE), a)
        with pytest.raises(ValueError, match="same layers"):
            QuantCache(2, 4, 50, kv, D, blk, fmt, 16).move(ctx, np.zeros(0, bs.SEG_DTYPE), a)

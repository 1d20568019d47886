"""Model calls on 4-bit KV caches against the oracle: the verify step and the decoder layer, and a serving loop of
prefill, draft head, verify step and replay recompute.

The oracle keeps decoded caches and takes, for the rows that a call writes, the values that the GPU stored, after
checking them against its own quantisation: a row that differs by rounding (f32: 2^-20, bf16: a step of 2^-8) may
land on the next code, which is one unit of its group, so a small share of elements may differ and none by more
than two units. With the same cache contents the outputs then agree as they do on the other caches."""
import numpy as np
import pytest
import torch

import workloads
from oracle import kvq, model as omodel, mtp as omtp, sampler as osamp
from oracle.prefix import prefill_logits
from helpers import dev, host, layer_host, max_abs, model_from, oracle_cfg
from test_gpu_verify import _route_sets_agree, _tiny_setup

pytestmark = pytest.mark.gpu


class Forced(np.ndarray):
    """A decoded cache whose rows take the GPU's values when written (forced: the GPU's cache, decoded)."""

    def __setitem__(self, idx, val):
        got = self.forced[idx]
        codes, scales = kvq.encode(val)
        unit = np.repeat(2.0 ** (scales.astype(int) - 127.0), 32, axis=-1)
        assert (np.abs(val - got) <= 2 * unit).all()
        self.differ += int((got != kvq.decode(codes, scales)).sum())
        self.written += got.size
        super().__setitem__(idx, got)


class Quantised(np.ndarray):
    """A decoded cache that quantises the rows written to it."""

    def __setitem__(self, idx, val):
        super().__setitem__(idx, kvq.decode(*kvq.encode(val)))


def _decoded(kc, vc, D):
    """GPU caches as [nb, Hkv, 16, D] and [nb, Hkv, D, 16] float64."""
    out = []
    for c, value in ((host(kc), False), (host(vc), True)):
        x = np.stack([np.stack([kvq.read(c, b, s, D, value) for s in range(16)]) for b in range(len(c))])
        out.append(x.transpose(0, 2, 3, 1) if value else x.transpose(0, 2, 1, 3))
    return [np.ascontiguousarray(x) for x in out]


def _forced(before, after):
    f = before.copy().view(Forced)
    f.forced, f.differ, f.written = after, 0, 0
    return f


def _fill(molt, caches, kc, vc, layout, D):
    """The oracle's contexts (float64 caches) written into 4-bit caches."""
    B, n = len(layout.context_lens), int(max(layout.context_lens))
    table = dev(torch.from_numpy(layout.block_tables))
    lens = dev(torch.from_numpy(layout.context_lens.astype(np.int32)))
    rows = []
    for c, value in ((caches[0], False), (caches[1], True)):
        x = np.zeros((B * n, c.shape[1], D), np.float32)
        for b in range(B):
            for p in range(int(layout.context_lens[b])):
                blk = layout.block_tables[b][p // 16]
                x[b * n + p] = c[blk, :, :, p % 16] if value else c[blk, :, p % 16]
        rows.append(torch.from_numpy(x).cuda())
    molt.kvq_write(rows[0], rows[1], kc, vc, table, torch.zeros_like(lens), n, lens=lens)


def _share(caches, most):
    differ, written = (sum(getattr(x, k) for c in caches for x in c) for k in ("differ", "written"))
    print(f"{differ} of {written} stored values differ from the oracle's own", flush=True)
    assert written > 0 and differ <= most * written


def test_tiny_verify_step(molt_lib):
    w, cfg, layout, layers, head, lh, hh, caches = _tiny_setup()
    D, nb = w.head_dim, caches[0][0].shape[0]
    pairs = [molt_lib.kvq_cache(nb, w.n_kv_heads, D) for _ in range(w.n_layers)]
    for c, (kc, vc) in zip(caches, pairs):
        _fill(molt_lib, c, kc, vc, layout, D)
    before = [_decoded(kc, vc, D) for kc, vc in pairs]
    toks = workloads.make_step_tokens(w, 1)
    q = workloads.make_softmax_q(w.batch, w.k, w.vocab, 2)
    u = workloads.make_uniforms(w.batch, w.k, 3)
    dtoks = dev(torch.from_numpy(toks))
    model = model_from(w, layers, head, molt_lib)
    kv = molt_lib.KVCache([p[0] for p in pairs], [p[1] for p in pairs], dev(torch.from_numpy(layout.block_tables)),
                          dev(torch.from_numpy(layout.context_lens)))
    r = molt_lib.verify_step(model, kv, dtoks, dev(u), dev(q), want_routes=True)
    again = molt_lib.verify_step(model, kv, dtoks, dev(u), dev(q))
    assert torch.equal(r["logits"], again["logits"])
    assert torch.equal(r["logprobs"].nan_to_num(), again["logprobs"].nan_to_num())     # NaN past the emitted tokens
    after = [_decoded(kc, vc, D) for kc, vc in pairs]
    oc = [tuple(_forced(b, a) for b, a in zip(*x)) for x in zip(before, after)]
    o = omodel.verify_step(toks, lambda l: lh[l], hh, oc, layout.block_tables, layout.context_lens, cfg, host(q),
                           host(u))
    _share(oc, 1e-3)
    err = max_abs(r["logits"].cpu().numpy(), o["logits"])
    print("logits", err, flush=True)
    assert err <= 1e-4
    assert np.array_equal(r["n_accepted"].cpu().numpy(), o["n_accepted"])
    assert np.array_equal(r["tokens"].cpu().numpy(), o["tokens"])
    # the actor's recompute on the recorded routes gives the recorded log-probs
    s = molt_lib.score_tokens(model, kv, dtoks, r["tokens"].clamp(min=0), replay_routes=r["routes"])
    live = r["tokens"] >= 0
    assert torch.equal(s["logprobs"][live], r["logprobs"][live])


@pytest.mark.parametrize("B,k,Hq,Hkv,D,lo,hi", [
    (3, 4, 32, 4, 128, 5, 400),          # the RoPE-fused projection's head layout, splits of the attention's keys
    (2, 8, 8, 1, 128, 0, 60),            # 72 rows: two row groups
    (2, 20, 8, 4, 64, 30, 47),
    (1, 2, 8, 2, 128, 1400, 1400),       # a long key range
    (1, 2, 8, 2, 128, 2200, 2200),       # a cut one
    (2, 6, 16, 2, 64, 30, 2100),         # one of two cut, 56 rows
])
def test_bf16_layer(molt_lib, B, k, Hq, Hkv, D, lo, hi):
    w = workloads.LAYER_BF16.scaled(batch=B, k=k, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, ctx_lo=lo, ctx_hi=hi,
                                    d_model=512, n_experts=16, top_k=4, d_ff=256)
    cfg = oracle_cfg(w)
    layout = workloads.make_kv_layout(w, 5)
    rng = np.random.default_rng(5)
    lw = workloads.make_layer_weights(w, 5, 0)
    lh = layer_host(lw)
    nb = int(layout.block_tables.max()) + 1
    kc, vc = molt_lib.kvq_cache(nb, Hkv, D)
    shape = (nb, Hkv, 16, D)
    _fill(molt_lib, (rng.standard_normal(shape), rng.standard_normal((nb, Hkv, D, 16))), kc, vc, layout, D)
    before = _decoded(kc, vc, D)
    model = molt_lib.Model([{n: dev(v) for n, v in lw.items()}], None, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D,
                           top_k=w.top_k, rms_eps=w.rms_eps, rope_theta=w.rope_theta)
    kv = molt_lib.KVCache([kc], [vc], dev(torch.from_numpy(layout.block_tables)),
                          dev(torch.from_numpy(layout.context_lens)))
    x = torch.from_numpy(rng.standard_normal((B * (k + 1), w.d_model)).astype(np.float32))
    xd = x.cuda()
    routes = molt_lib.decoder_forward(model, kv, B, k, xd, want_routes=True)
    oc = [tuple(_forced(b, a) for b, a in zip(before, _decoded(kc, vc, D)))]
    want, orr = omodel.decoder_forward(x.numpy(), lambda l: lh, oc, layout.block_tables, layout.context_lens, k, cfg)
    _share(oc, 2e-2)
    same = _route_sets_agree(routes[0].cpu().numpy(), orr[0]["ids"], orr[0]["margin"], max_frac=0.1)
    err = np.abs(xd.cpu().numpy() - want)[same].max()
    print("residual", err, flush=True)
    assert err <= 2e-2


def test_captured_layer(molt_lib):
    """A captured call replayed on other inputs and contexts, eager calls between: the same bits as eager calls."""
    B, k, Hq, Hkv, D = 2, 3, 8, 2, 128
    w = workloads.LAYER_BF16.scaled(batch=B, k=k, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, ctx_lo=2200, ctx_hi=2300,
                                    d_model=512, n_experts=16, top_k=4, d_ff=256)
    layout = workloads.make_kv_layout(w, 5)
    model = molt_lib.Model([{n: dev(v) for n, v in workloads.make_layer_weights(w, 5, 0).items()}], None, n_q_heads=Hq,
                           n_kv_heads=Hkv, head_dim=D, top_k=w.top_k, rms_eps=w.rms_eps, rope_theta=w.rope_theta)
    gen = torch.Generator(device="cuda").manual_seed(7)
    draw = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    kc, vc = molt_lib.kvq_cache(int(layout.block_tables.max()) + 1, Hkv, D)
    tables = dev(torch.from_numpy(layout.block_tables))
    molt_lib.kvq_write(draw(B * 2300, Hkv, D), draw(B * 2300, Hkv, D), kc, vc, tables,
                       torch.zeros(B, dtype=torch.int32, device="cuda"), 2300)
    ctx = torch.tensor([2200, 40], dtype=torch.int32, device="cuda")
    kv = molt_lib.KVCache([kc], [vc], tables, ctx)
    size = molt_lib.decoder_workspace_size(model, B, k, tables.shape[1]) + kv.extra(model, B, k)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    x = torch.zeros(B * (k + 1), w.d_model, device="cuda")
    inputs = [draw(B * (k + 1), w.d_model) for _ in range(4)]
    contexts = [torch.tensor(c, dtype=torch.int32, device="cuda") for c in ([2200, 40], [100, 2290], [2250, -4], [0, 7])]

    def step(own=None):
        molt_lib.decoder_forward(model, kv, B, k, x, workspace=own)

    step(ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ws)
    for xi, ci in zip(inputs, contexts):
        before = kc.clone(), vc.clone()
        ctx.copy_(ci)
        x.copy_(xi)
        step()
        want = x.clone(), kc.clone(), vc.clone()
        kc.copy_(before[0])
        vc.copy_(before[1])
        x.copy_(xi)
        graph.replay()
        torch.cuda.synchronize()
        for got, expected in zip((x, kc, vc), want):
            assert torch.equal(got, expected)


def test_serving_loop(molt_lib):
    """Prefill, first token, drafts, verify steps on 4-bit caches of the target and the draft head, each call against
    the oracle on the caches that the GPU holds."""
    molt, seed = molt_lib, 61
    w = workloads.TINY_FP32.scaled(batch=2, k=3, ctx_lo=0, ctx_hi=0)
    B, k, V, D, Hkv = w.batch, w.k, w.vocab, w.head_dim, w.n_kv_heads
    cfg = oracle_cfg(w)
    layers = [workloads.make_layer_weights(w, seed, l) for l in range(w.n_layers)]
    head, mt = workloads.make_head_weights(w, seed), workloads.make_mtp_weights(w, seed)
    model = model_from(w, layers, head, molt)
    mtp = molt.Mtp(dev(mt["enorm"]), dev(mt["hnorm"]), dev(mt["eh_proj"]), {n: dev(v) for n, v in mt["layer"].items()},
                   dev(mt["final_norm"]), n_q_heads=w.n_q_heads, n_kv_heads=Hkv, head_dim=D, top_k=w.top_k,
                   rms_eps=w.rms_eps, rope_theta=w.rope_theta)
    lh, hh = [layer_host(lw) for lw in layers], layer_host(head)
    mh = {n: host(v) for n, v in mt.items() if n != "layer"}
    mh["layer"] = layer_host(mt["layer"])
    nbps, nb = 8, 16
    bt = np.arange(nb, dtype=np.int32).reshape(B, nbps)
    target = [molt.kvq_cache(nb, Hkv, D) for _ in range(w.n_layers)]
    drafter = [molt.kvq_cache(nb, Hkv, D)]
    btd = dev(torch.from_numpy(bt))

    def kvs(ctx):
        c = dev(torch.from_numpy(ctx.astype(np.int32)))
        return tuple(molt.KVCache([p[0] for p in x], [p[1] for p in x], btd, c) for x in (target, drafter))

    def state(x):
        torch.cuda.synchronize()
        return [_decoded(kc, vc, D) for kc, vc in x]

    def forced(before, after):
        return [tuple(_forced(b, a) for b, a in zip(*x)) for x in zip(before, after)]

    g = np.random.default_rng(seed)
    n, lens = 40, np.array([40, 27], np.int32)
    prompt = g.integers(0, V, (B, n)).astype(np.int32)
    ctx = np.zeros(B, np.int64)
    kv, hkv = kvs(ctx)
    t0, h0 = state(target), state(drafter)
    pf = molt.prefill(model, kv, dev(torch.from_numpy(prompt)), dev(torch.from_numpy(lens)), want_hidden=True)
    t1 = state(target)
    oc = forced(t0, t1)
    olog, _, _ = prefill_logits(prompt, lens, lambda l: lh[l], hh, oc, bt, ctx, cfg)
    _share(oc, 1e-3)
    assert max_abs(pf["logits"].cpu().numpy(), olog) <= 1e-4
    u0 = workloads.make_uniforms(B, 0, seed + 1)
    first = molt.spec_accept(pf["logits"][:, None, :].contiguous(), None, dev(u0))[0][:, 0].contiguous()
    ud = workloads.make_uniforms(B, k - 1, seed + 2, tag="mtp_u")
    last, hidden, toks, n_acc = first.cpu().numpy(), pf["hidden"], prompt, lens - 1
    for it in range(3):
        dr = molt.mtp_draft(model, mtp, hkv, hidden, dev(torch.from_numpy(toks)), dev(torch.from_numpy(n_acc.astype(np.int32))),
                            dev(torch.from_numpy(last.astype(np.int32))), dev(ud), k=k)
        h1 = state(drafter)               # drafting rows overwrite catch-up rows within the call
        oh = [tuple(x.copy().view(Quantised) for x in c) for c in h0]
        drafts, q = dr["drafts"].cpu().numpy(), dr["draft_probs"]
        od = omtp.mtp_draft(host(hidden), toks, n_acc, last, mh, hh, oh[0][0], oh[0][1], bt, ctx, cfg,
                            uniforms=host(ud), forced=drafts, k=k)
        assert np.abs(q.cpu().numpy() - od["q"]).max() <= 1e-5 * od["q"].max() + 1e-9
        assert np.array_equal(drafts, od["drafts"])
        assert all((np.asarray(a) != b).sum() <= 1e-3 * b.size for a, b in zip(oh[0], h1[0]))
        h0 = h1
        ctx = ctx + (lens if it == 0 else n_acc + 1)
        toks = np.concatenate([last[:, None], drafts], axis=1).astype(np.int32)
        u = workloads.make_uniforms(B, k, seed + 10 + it)
        kv, hkv = kvs(ctx)
        t0 = t1
        vs = molt.verify_step(model, kv, dev(torch.from_numpy(toks)), dev(u), q, want_hidden=True)
        t1 = state(target)
        oc = forced(t0, t1)
        ov = omodel.verify_step(toks, lambda l: lh[l], hh, oc, bt, ctx, cfg, host(q), host(u))
        _share(oc, 1e-3)
        assert max_abs(vs["logits"].cpu().numpy(), ov["logits"]) <= 1e-4
        n_acc = vs["n_accepted"].cpu().numpy()
        assert np.array_equal(n_acc, ov["n_accepted"])
        assert np.array_equal(vs["tokens"].cpu().numpy(), ov["tokens"])
        last = ov["tokens"][np.arange(B), n_acc].astype(np.int32)
        hidden = vs["hidden"]
        ud = workloads.make_uniforms(B, k - 1, seed + 20 + it, tag="mtp_u")


def test_refusals(molt_lib):
    w, cfg, layout, layers, head, *_ = _tiny_setup()
    model = model_from(w, layers, head, molt_lib)
    nb, H, D = 64, w.n_kv_heads, w.head_dim
    bt, ctx = dev(torch.from_numpy(layout.block_tables)), dev(torch.from_numpy(layout.context_lens))
    good = [molt_lib.kvq_cache(nb, H, D) for _ in range(w.n_layers)]
    plain = torch.zeros(nb, H, 16, D, device="cuda")
    with pytest.raises(molt_lib.MoltError, match="4-bit"):
        molt_lib.KVCache([good[0][0], plain], [good[0][1], plain], bt, ctx)
    bad = [molt_lib.kvq_cache(nb, H + 1, D) for _ in range(w.n_layers)]
    x = torch.zeros(w.batch * (w.k + 1), w.d_model, device="cuda")
    kv = molt_lib.KVCache([p[0] for p in bad], [p[1] for p in bad], bt, ctx)
    with pytest.raises(molt_lib.MoltError, match="shape"):
        molt_lib.decoder_forward(model, kv, w.batch, w.k, x)
    flat = torch.zeros(good[0][0].numel() + 8, dtype=torch.uint8, device="cuda")
    kv = molt_lib.KVCache([flat[8:].view(good[0][0].shape)] * w.n_layers, [p[1] for p in good], bt, ctx)
    with pytest.raises(molt_lib.MoltError, match="16 bytes"):
        molt_lib.decoder_forward(model, kv, w.batch, w.k, x)

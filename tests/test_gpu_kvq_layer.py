"""GPU tests of what a decoder layer does with its 4-bit caches: the bytes that it writes are those of kvq_write, and a
layer whose output hangs on its cached keys and values, each block of them."""
import numpy as np
import pytest
import torch

import workloads
from helpers import dev, host, layer_host, oracle_cfg
from oracle import model as omodel
from oracle.attention import apply_rope
from test_gpu_kvq_model import _decoded, _fill, _forced, _share
from test_gpu_verify import _route_sets_agree

pytestmark = pytest.mark.gpu


def _scaled(dtype, **kw):
    return workloads.LAYER_BF16.scaled(dtype=dtype, expert_dtype=dtype, n_experts=16, top_k=4, d_ff=256, d_model=512, **kw)


@pytest.mark.parametrize("dtype,D", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("B,k,Hq,Hkv,ctx", [(1, 0, 4, 4, [0]), (3, 4, 8, 2, [0, 14, 301]), (2, 36, 5, 5, [3, 16]),
                                            (3, 2, 8, 1, [-2, 62, 5])])
def test_written_bytes(molt_lib, dtype, D, B, k, Hq, Hkv, ctx):
    """A layer on a residual stream of +-1 (its norm is itself) with weights that are multiples of 1/64, so that every sum
    of the QKV product is exact in f32: the caches hold the bytes that kvq_write makes of the rows, keys after RoPE, and
    every other byte as it was; rows before the sequence, past the table and of a block outside the pool are not written."""
    w = _scaled(dtype, batch=B, k=k, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D)
    gen = torch.Generator().manual_seed(71)
    lw = workloads.make_layer_weights(w, 7, 0)
    lw["w_qkv"] = (torch.randint(-8, 9, lw["w_qkv"].shape, generator=gen) / 64.0).to(lw["w_qkv"].dtype)
    lw["attn_norm"] = torch.ones_like(lw["attn_norm"])
    model = molt_lib.Model([{n: dev(v) for n, v in lw.items()}], None, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D,
                           top_k=w.top_k, rms_eps=0.0, rope_theta=w.rope_theta)
    n, maxb = k + 1, 20
    nb = B * maxb + 1
    tables = torch.randperm(nb, generator=gen)[:B * maxb].view(B, maxb).to(torch.int32)
    if B == 3 and ctx[0] < 0:
        tables[1], tables[2, 0] = tables[1].roll(1), nb          # the third sequence's rows have no place
        tables = tables[:, :4].contiguous()                      # and the second's end past the table
    x = (torch.randint(0, 2, (B * n, w.d_model), generator=gen) * 2 - 1).float()
    kc, vc = (torch.randint(0, 256, (nb, Hkv, 17 * D // 2), generator=gen, dtype=torch.uint8).cuda() for _ in range(2))
    wk, wv = kc.clone(), vc.clone()
    gt, gc = tables.cuda(), torch.tensor(ctx, dtype=torch.int32, device="cuda")
    kv = molt_lib.KVCache([kc], [vc], gt, gc)
    molt_lib.decoder_forward(model, kv, B, k, x.cuda())
    qkv = (x.double() @ lw["w_qkv"].double().t()).numpy().reshape(B * n, Hq + 2 * Hkv, D)
    assert np.array_equal(qkv, qkv.astype(np.float32))
    pos = (np.array(ctx)[:, None] + np.arange(n)).reshape(-1)
    rows = []
    for r in (apply_rope(qkv[:, Hq:Hq + Hkv], pos, w.rope_theta), qkv[:, Hq + Hkv:]):
        rows.append(torch.from_numpy(np.ascontiguousarray(r).astype(np.float32)).to(lw["w_qkv"].dtype).cuda())
    molt_lib.kvq_write(*rows, wk, wv, gt, gc, n)
    assert torch.equal(vc, wv)
    assert torch.equal(kc, wk)


@pytest.mark.parametrize("B,k,Hq,Hkv,D,lo,hi", [
    (3, 4, 32, 4, 128, 150, 400),
    (1, 2, 8, 2, 128, 1400, 1400),       # a long key range
    (1, 2, 8, 2, 128, 2200, 2200),       # a cut one
    (2, 6, 16, 2, 64, 150, 2100),        # one of two cut
])
def test_layer_that_hangs_on_its_cache(molt_lib, B, k, Hq, Hkv, D, lo, hi):
    """Values so large, and softmaxes so uneven, that a layer's output moves by 0.1 and more where one block is taken for
    another or a quarter of the keys is lost (asserted on the oracle); the bar is under a sixth of that. Outputs of the
    attention are of rms 2 at most (values of rms 8, a tenth of 150 keys and more count), off by 2^-9 / sqrt(3) of that
    rms (their rounding to bf16); the O projection sums up to 4096 of them times weights of rms 0.02:
    2 * 1.13e-3 * 0.02 * 64 = 2.9e-3, 1.45e-2 at five sigma; the experts' inputs, and with them their outputs (under a
    tenth of the residual), move by less than the residual does."""
    w = _scaled("bf16", batch=B, k=k, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, ctx_lo=lo, ctx_hi=hi)
    cfg = oracle_cfg(w)
    layout = workloads.make_kv_layout(w, 5)
    rng = np.random.default_rng(5)
    lw = workloads.make_layer_weights(w, 5, 0)
    lh = layer_host(lw)
    nb = int(layout.block_tables.max()) + 1
    kc, vc = molt_lib.kvq_cache(nb, Hkv, D)
    _fill(molt_lib, (3.3 * rng.standard_normal((nb, Hkv, 16, D)), 8.0 * rng.standard_normal((nb, Hkv, D, 16))), kc, vc,
          layout, D)
    before = _decoded(kc, vc, D)
    model = molt_lib.Model([{n: dev(v) for n, v in lw.items()}], None, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D,
                           top_k=w.top_k, rms_eps=w.rms_eps, rope_theta=w.rope_theta)
    kv = molt_lib.KVCache([kc], [vc], dev(torch.from_numpy(layout.block_tables)),
                          dev(torch.from_numpy(layout.context_lens)))
    x = rng.standard_normal((B * (k + 1), w.d_model)).astype(np.float32)
    xd = torch.from_numpy(x).cuda()
    routes = molt_lib.decoder_forward(model, kv, B, k, xd, want_routes=True)
    oc = [tuple(_forced(b, a) for b, a in zip(before, _decoded(kc, vc, D)))]

    def forward(K, V):
        return omodel.decoder_forward(x, lambda l: lh, [(K, V)], layout.block_tables, layout.context_lens, k, cfg)

    want, orr = forward(*oc[0])
    _share(oc, 2e-2)
    same = _route_sets_agree(routes[0].cpu().numpy(), orr[0]["ids"], orr[0]["margin"], max_frac=0.1)
    err = np.abs(xd.cpu().numpy() - want)[same].max()
    print("residual", err, flush=True)
    assert err <= 1.5e-2
    K, V = (np.array(c) for c in oc[0])
    for b in range(B):
        table, blocks = layout.block_tables[b], int(layout.context_lens[b]) // 16
        rows = np.zeros(B * (k + 1), bool)
        rows[b * (k + 1):(b + 1) * (k + 1)] = True
        if blocks < 4:
            continue
        moved = []
        for i in (0, blocks // 2, blocks - 1):
            for which in (0, 1):
                other = [K.copy(), V.copy()]
                other[which][table[i]] = other[which][table[(i + 2) % blocks]]
                moved.append(other)
        lost = V.copy()
        lost[table[blocks // 4:blocks // 2]] = 0.0
        for other in moved + [[K.copy(), lost]]:
            assert np.abs(forward(*other)[0] - want)[same & rows].max() >= 0.1

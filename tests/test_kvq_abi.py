"""Host-side checks of the 4-bit KV cache's C entries: bad arguments are refused before anything is
enqueued (the pointers here are never followed)."""
import ctypes

import pytest

import paper_2607_21653_amd as molt

INVALID, WORKSPACE = -1, -3
P, P2 = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000)


@pytest.fixture(scope="module")
def L():
    return molt.load()


def _write(L, k=P, v=P, ks=512, vs=512, kc=P, vc=P2, bt=P, ctx=P, lens=None, B=2, n=5, H=4, D=128, mb=4, nb=9, dt=1):
    return L.molt_kvq_write(k, v, ks, vs, kc, vc, bt, ctx, lens, B, n, H, D, mb, nb, dt, None)


def _read(L, kc=P, vc=P, bt=P, st=P, lens=None, B=2, n=5, H=4, D=128, mb=4, nb=9, dt=1, k=P, v=P):
    return L.molt_kvq_read(kc, vc, bt, st, lens, B, n, H, D, mb, nb, dt, k, v, None)


def _attend(L, q=P, kc=P, vc=P, bt=P, ctx=P, B=2, k=4, Hq=32, H=4, D=128, mb=4, nb=9, dt=1, out=P, ws=P, wsb=1 << 30):
    return L.molt_paged_attention_kvq(q, kc, vc, bt, ctx, B, k, Hq, H, D, mb, nb, dt, out, ws, wsb, None)


BAD = [dict(B=0), dict(H=0), dict(D=96), dict(D=256), dict(mb=0), dict(nb=0), dict(dt=2), dict(dt=7), dict(kc=None),
       dict(vc=None), dict(bt=None), dict(kc=ctypes.c_void_p(0x1008)), dict(vc=ctypes.c_void_p(0x1001))]


@pytest.mark.parametrize("bad", BAD + [dict(n=0), dict(n=-1), dict(k=None), dict(v=None), dict(ctx=None), dict(ks=511),
                                       dict(vs=0), dict(B=2 ** 20, n=2 ** 20), dict(kc=P2),
                                       dict(B=2 ** 26, n=1)])
def test_write(L, bad):
    assert _write(L, **bad) == INVALID and L.molt_last_error()


@pytest.mark.parametrize("bad", BAD + [dict(n=0), dict(k=None), dict(v=None), dict(st=None), dict(B=2 ** 20, n=2 ** 20)])
def test_read(L, bad):
    assert _read(L, **bad) == INVALID and L.molt_last_error()


@pytest.mark.parametrize("bad", BAD + [dict(k=-1), dict(k=2 ** 31 - 1), dict(q=None), dict(out=None), dict(ctx=None),
                                       dict(Hq=30), dict(Hq=2), dict(B=2 ** 20, k=2 ** 9), dict(mb=2 ** 27),
                                       dict(B=2 ** 22, k=0, D=64)])
def test_attention(L, bad):
    assert _attend(L, **bad) == INVALID and L.molt_last_error()


def test_attention_workspace(L):
    size = L.molt_paged_attention_kvq_workspace_size
    assert size(2, 4, 32, 4, 128, 600) > 0                  # split key range
    assert size(0, 4, 32, 4, 128, 600) == size(2, 4, 30, 4, 128, 600) == 0
    assert _attend(L, mb=600, wsb=size(2, 4, 32, 4, 128, 600) - 1) == WORKSPACE
    assert _attend(L, mb=600, ws=None) == WORKSPACE
    assert b"workspace" in L.molt_last_error()


def test_model_calls(L):
    """4-bit caches of model calls: the flag of block_size, alignment, and the workspace besides."""
    from paper_2607_21653_amd import _lib
    m, kv = _lib.MoltModel(), _lib.MoltKV()
    keep = []

    def arr(v):
        keep.append((ctypes.c_void_p * 1)(v))
        return ctypes.cast(keep[-1], ctypes.c_void_p)

    m.n_layers, m.d_model, m.n_q_heads, m.n_kv_heads, m.head_dim = 1, 256, 8, 2, 128
    m.n_experts, m.top_k, m.d_ff, m.rms_eps, m.rope_theta = 4, 2, 128, 1e-6, 1e6
    m.dtype = m.expert_dtype = _lib.MOLT_BF16
    for key in ("attn_norm", "w_qkv", "w_o", "moe_norm", "w_router", "w_gate_up", "w_down"):
        setattr(m, key, arr(0x4000))
    kv.k_cache, kv.v_cache = arr(0x8000), arr(0x9008)
    kv.block_tables = kv.context_lens = ctypes.c_void_p(0x1000)
    kv.max_blocks_per_seq, kv.num_blocks = 40, 99

    def call(block_size, ws, nb):
        kv.block_size = block_size
        return L.molt_decoder_forward(ctypes.byref(m), ctypes.byref(kv), 2, 4, P, None, ws, nb, None)

    size = L.molt_decoder_workspace_size(ctypes.byref(m), 2, 4, 40)
    extra = L.molt_kvq_workspace_extra(ctypes.byref(m), 2, 4, 40)
    assert extra >= 2 * 5 * (8 + 2 * 2) * 128 * 4                     # the projection's f32 rows
    assert L.molt_kvq_workspace_extra(None, 2, 4, 40) == L.molt_kvq_workspace_extra(ctypes.byref(m), 0, 4, 40) == 0
    for bad in (32, 16 | 0x200, 0x100, 17):
        assert call(bad, P, size + extra) == INVALID
    assert call(16 | _lib.MOLT_KV_MX, P, size + extra) == INVALID and b"16 bytes" in L.molt_last_error()
    kv.v_cache = arr(0x9000)
    assert call(16 | _lib.MOLT_KV_MX, P, extra) == WORKSPACE          # nothing left for the call itself
    assert call(16 | _lib.MOLT_KV_MX, None, 0) == WORKSPACE


def test_python_checks_need_a_gpu_tensor():
    import torch
    kc = torch.zeros(4, 2, 1088, dtype=torch.uint8)
    tables, ctx = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    rows = torch.zeros(2, 2, 128)
    for call in (lambda: molt.kvq_write(rows, rows, kc, kc, tables, ctx, 1),
                 lambda: molt.kvq_read(kc, kc, tables, ctx, 1),
                 lambda: molt.paged_attention_kvq(rows, kc, kc, tables, ctx, 0)):
        with pytest.raises(molt.MoltError, match="GPU"):
            call()

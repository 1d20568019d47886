"""Host-side checks of sizes at and past the limits of the 4-bit KV cache: size functions answer 0 for what no call takes,
and calls refuse it before anything is enqueued (the pointers here are never followed)."""
import ctypes

import pytest

import paper_2607_21653_amd as molt
from paper_2607_21653_amd import _lib

INVALID, WORKSPACE = -1, -3
BIG = 2 ** 31 - 1


@pytest.fixture(scope="module")
def L():
    return molt.load()


def _model(dtype=_lib.MOLT_BF16, **kw):
    m = _lib.MoltModel()
    m.n_layers, m.d_model, m.n_q_heads, m.n_kv_heads, m.head_dim = 1, 256, 8, 2, 128
    m.n_experts, m.top_k, m.d_ff, m.rms_eps, m.rope_theta = 4, 2, 128, 1e-6, 1e6
    m.dtype = m.expert_dtype = dtype
    for key, v in kw.items():
        setattr(m, key, v)
    return m


@pytest.mark.parametrize("B,k,Hq,Hkv,D,mb", [
    (1, BIG, 4, 1, 128, 1),              # 1 + k past an int
    (1, BIG - 1, 4, 1, 128, 1),          # rows of a kv head past an int
    (BIG, BIG - 1, 64, 1, 128, BIG), (1, 4, BIG, 1, 128, 100), (BIG, 0, BIG, BIG, 128, 1),
    (1, 0, 4, 1, 128, 2 ** 26 + 1), (1, 0, 4, 1, 96, 100), (1, 0, 4, 1, 0, 100), (1, 0, 4, 1, BIG, 100),
    (1, -1, 4, 1, 128, 100), (1, 0, 4, 0, 128, 100), (1, 0, 0, 1, 128, 100)])
def test_no_workspace_for_what_no_call_takes(L, B, k, Hq, Hkv, D, mb):
    assert L.molt_paged_attention_kvq_workspace_size(B, k, Hq, Hkv, D, mb) == 0
    for dtype in (_lib.MOLT_F32, _lib.MOLT_BF16):
        m = _model(dtype, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D)
        assert L.molt_kvq_workspace_extra(ctypes.byref(m), B, k, mb) == 0


def test_extra_of_the_largest_sizes(L):
    """The largest numbers of positions and blocks: the QKV product's rows, counted in 64 bits."""
    m = _model()
    k = 8_000_000 - 1
    want = (k + 1) * (8 + 2 * 2) * 128 * 4
    assert want <= L.molt_kvq_workspace_extra(ctypes.byref(m), 1, k, 2 ** 26) <= want + (1 << 20)
    for bad in (dict(n_experts=0), dict(top_k=0), dict(d_model=0)):      # not what the extra goes by
        m = _model(**bad)
        assert L.molt_kvq_workspace_extra(ctypes.byref(m), 2, 4, 40) >= 2 * 5 * (8 + 2 * 2) * 128 * 4


@pytest.mark.parametrize("name", ["decoder", "verify", "prefill", "score", "draft"])
@pytest.mark.parametrize("dtype", [_lib.MOLT_F32, _lib.MOLT_BF16])
def test_model_calls_at_the_limits(L, name, dtype):
    """Calls on a model refuse the sizes that the attention over 4-bit caches refuses, and take those just within."""
    keep = []

    def arr(v):
        keep.append((ctypes.c_void_p * 1)(v))
        return ctypes.cast(keep[-1], ctypes.c_void_p)

    P = ctypes.c_void_p(0x1000)

    def call(B, k, mb, Hq=8, Hkv=2, kind=16 | _lib.MOLT_KV_MX, d=64):
        m = _model(dtype, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=64, d_model=d, d_ff=64, vocab=64, top_k=1)
        for key in ("attn_norm", "w_qkv", "w_o", "moe_norm", "w_router", "w_gate_up", "w_down"):
            setattr(m, key, arr(0x4000))
        m.embed, m.lm_head, m.final_norm = P, P, P
        kv = _lib.MoltKV()
        kv.k_cache, kv.v_cache = arr(0x8000), arr(0x9000)
        kv.block_tables = kv.context_lens = P
        kv.max_blocks_per_seq, kv.num_blocks, kv.block_size = mb, 99, kind
        mr, kr = ctypes.byref(m), ctypes.byref(kv)
        if name == "decoder":
            return L.molt_decoder_forward(mr, kr, B, k, P, None, None, 0, None)
        if name == "verify":
            return L.molt_verify_step(mr, kr, B, k, P, None, P, None, P, P, None, None, None, None, 0, None)
        if name == "prefill":
            return L.molt_prefill(mr, kr, B, k + 1, P, P, P, None, None, None, 0, None)
        if name == "score":
            return L.molt_score_tokens(mr, kr, B, k, P, P, None, P, None, None, None, 0, None)
        mtp = _lib.MoltMtp()
        mtp.enorm = mtp.hnorm = mtp.eh_proj = mtp.final_norm = P
        mtp.layer = ctypes.pointer(m)
        return L.molt_mtp_draft_window(mr, ctypes.byref(mtp), kr, B, k + 1, 1, P, P, P, P, P, P, P, None, 0, None)

    assert call(2, 4, 2 ** 26) == WORKSPACE
    assert call(2, 4, 2 ** 26, kind=16) == WORKSPACE
    assert call(2, 4, 2 ** 26 + 1) == INVALID and b"2^26" in L.molt_last_error()
    assert call(2, 4, 2 ** 26 + 1, kind=16) == WORKSPACE               # other caches keep their own limits
    rows = 16 if dtype == _lib.MOLT_F32 else 48
    n = int(1.4e7 / 8 * rows / 64)                                     # 64 query heads a kv head, 8 kv heads
    assert call(1, n, 4, Hq=512, Hkv=8) == INVALID and b"4-bit" in L.molt_last_error()
    assert call(1, n - 2 * rows, 4, Hq=512, Hkv=8) == WORKSPACE
    assert call(1, 16_000_000, 4, Hq=1, Hkv=1) == INVALID

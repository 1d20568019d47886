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

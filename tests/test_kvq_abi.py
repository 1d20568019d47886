"""Host-side checks of the 4-bit KV cache's C entries: bad arguments are refused before anything is
enqueued (the pointers here are never followed)."""
import ctypes

import pytest

import paper_2607_21653_amd as molt

INVALID, WORKSPACE = -1, -3
P = ctypes.c_void_p(0x1000)


@pytest.fixture(scope="module")
def L():
    return molt.load()


def _write(L, k=P, v=P, ks=512, vs=512, kc=P, vc=P, bt=P, ctx=P, lens=None, B=2, n=5, H=4, D=128, mb=4, nb=9, dt=1):
    return L.molt_kvq_write(k, v, ks, vs, kc, vc, bt, ctx, lens, B, n, H, D, mb, nb, dt, None)


def _read(L, kc=P, vc=P, bt=P, st=P, lens=None, B=2, n=5, H=4, D=128, mb=4, nb=9, dt=1, k=P, v=P):
    return L.molt_kvq_read(kc, vc, bt, st, lens, B, n, H, D, mb, nb, dt, k, v, None)


def _attend(L, q=P, kc=P, vc=P, bt=P, ctx=P, B=2, k=4, Hq=32, H=4, D=128, mb=4, nb=9, dt=1, out=P, ws=P, wsb=1 << 30):
    return L.molt_paged_attention_kvq(q, kc, vc, bt, ctx, B, k, Hq, H, D, mb, nb, dt, out, ws, wsb, None)


BAD = [dict(B=0), dict(H=0), dict(D=96), dict(D=256), dict(mb=0), dict(nb=0), dict(dt=2), dict(dt=7), dict(kc=None),
       dict(vc=None), dict(bt=None), dict(kc=ctypes.c_void_p(0x1008)), dict(vc=ctypes.c_void_p(0x1001))]


@pytest.mark.parametrize("bad", BAD + [dict(n=0), dict(n=-1), dict(k=None), dict(v=None), dict(ctx=None), dict(ks=511),
                                       dict(vs=0), dict(B=2 ** 20, n=2 ** 20)])
def test_write(L, bad):
    assert _write(L, **bad) == INVALID and L.molt_last_error()


@pytest.mark.parametrize("bad", BAD + [dict(n=0), dict(k=None), dict(v=None), dict(st=None), dict(B=2 ** 20, n=2 ** 20)])
def test_read(L, bad):
    assert _read(L, **bad) == INVALID and L.molt_last_error()


@pytest.mark.parametrize("bad", BAD + [dict(k=-1), dict(k=2 ** 31 - 1), dict(q=None), dict(out=None), dict(ctx=None),
                                       dict(Hq=30), dict(Hq=2), dict(B=2 ** 20, k=2 ** 9), dict(mb=2 ** 27)])
def test_attention(L, bad):
    assert _attend(L, **bad) == INVALID and L.molt_last_error()


def test_attention_workspace(L):
    size = L.molt_paged_attention_kvq_workspace_size
    assert size(2, 4, 32, 4, 128, 600) > 0                  # split key range
    assert size(0, 4, 32, 4, 128, 600) == size(2, 4, 30, 4, 128, 600) == 0
    assert _attend(L, mb=600, wsb=size(2, 4, 32, 4, 128, 600) - 1) == WORKSPACE
    assert _attend(L, mb=600, ws=None) == WORKSPACE
    assert b"workspace" in L.molt_last_error()


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

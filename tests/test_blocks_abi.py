"""Host-side checks of the C entries of sparse attention over listed blocks and of their Python calls: bad arguments
are refused before anything is enqueued (the pointers here are never followed)."""
import ctypes

import pytest
import torch

import paper_2607_21653_amd as molt

INVALID, WORKSPACE = -1, -3
P, P2, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000), ctypes.c_void_p(0x1008)
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    return molt.load()


def _plan(L, bt=P, nb=P, ctx=P, new=P, pool=P, shared=None, B=2, n=5, mb=4, cap=9, slots=P, placed=P, ws=P, wsb=BIG):
    return L.molt_plan_blocks(bt, nb, ctx, new, pool, shared, B, n, mb, cap, slots, placed, ws, wsb, None)


def _write(L, k=P, v=P, ks=512, vs=512, slots=P, rows=5, H=4, D=128, nb=9, dt=1, kc=P, vc=P2):
    return L.molt_kv_write(k, v, ks, vs, slots, rows, H, D, nb, dt, kc, vc, None)


def _update(L, kc=P, bounds=P, bt=P, st=P, lens=None, B=2, n=5, H=4, D=128, mb=4, nb=9, dt=1):
    return L.molt_key_bounds_update(kc, bounds, bt, st, lens, B, n, H, D, mb, nb, dt, None)


def _read(L, bounds=P, ids=P, M=3, H=4, D=128, nb=9, hi=P, lo=P):
    return L.molt_key_bounds_read(bounds, ids, M, H, D, nb, hi, lo, None)


def _select(L, q=P, bounds=P, bt=P, ctx=P, lens=None, B=2, k=4, Hq=32, H=4, D=128, mb=4, nb=9, N=8, first=1, last=2,
            dt=1, out=P, ws=P, wsb=BIG):
    return L.molt_select_blocks(q, bounds, bt, ctx, lens, B, k, Hq, H, D, mb, nb, N, first, last, dt, out, ws, wsb, None)


def _attend(L, q=P, kc=P, vc=P, bt=P, ctx=P, blocks=P, B=2, k=4, Hq=32, H=4, D=128, mb=4, nb=9, N=8, dt=1, out=P, ws=P,
            wsb=BIG):
    return L.molt_paged_attention_blocks(q, kc, vc, bt, ctx, blocks, B, k, Hq, H, D, mb, nb, N, dt, out, ws, wsb, None)


def _refused(L, status):
    assert status == INVALID and L.molt_last_error()


@pytest.mark.parametrize("bad", [dict(B=0), dict(n=0), dict(B=2 ** 20, n=2 ** 12), dict(B=2 ** 25, n=1), dict(mb=0),
                                 dict(mb=2 ** 26 + 1), dict(cap=0), dict(cap=2 ** 27), dict(bt=None), dict(nb=None),
                                 dict(ctx=None), dict(new=None), dict(pool=None), dict(slots=None), dict(placed=None)])
def test_plan(L, bad):
    _refused(L, _plan(L, **bad))


CACHE = [dict(H=0), dict(D=96), dict(D=256), dict(nb=0), dict(nb=2 ** 27), dict(H=2 ** 20)]


@pytest.mark.parametrize("bad", CACHE + [dict(rows=0), dict(rows=2 ** 31 - 1), dict(dt=2), dict(dt=-1), dict(k=None),
                                         dict(v=None), dict(slots=None), dict(kc=None), dict(vc=None), dict(kc=ODD),
                                         dict(vc=ODD), dict(kc=P2), dict(ks=511), dict(vs=-512)])
def test_write(L, bad):
    _refused(L, _write(L, **bad))


@pytest.mark.parametrize("bad", CACHE + [dict(B=0), dict(n=0), dict(mb=0), dict(mb=2 ** 27), dict(B=2 ** 26, n=1),
                                         dict(dt=2), dict(kc=None), dict(bounds=None), dict(bt=None), dict(st=None),
                                         dict(bounds=ODD), dict(kc=ODD), dict(B=2 ** 20, n=2 ** 20)])
def test_bounds_update(L, bad):
    _refused(L, _update(L, **bad))


@pytest.mark.parametrize("bad", CACHE + [dict(M=0), dict(M=2 ** 30), dict(bounds=None), dict(ids=None), dict(hi=None),
                                         dict(lo=None), dict(bounds=ODD), dict(hi=ODD)])
def test_bounds_read(L, bad):
    _refused(L, _read(L, **bad))


HEADS = CACHE + [dict(B=0), dict(k=-1), dict(k=2 ** 31 - 1), dict(Hq=30), dict(Hq=2), dict(B=2 ** 24, k=0),
                 dict(B=2 ** 20, k=2 ** 9), dict(mb=0), dict(mb=2 ** 27), dict(dt=2), dict(N=0), dict(N=2 ** 27),
                 dict(q=None), dict(bt=None), dict(ctx=None), dict(out=None), dict(q=ODD)]


@pytest.mark.parametrize("bad", HEADS + [dict(bounds=None), dict(bounds=ODD), dict(first=-1), dict(last=0),
                                         dict(first=7), dict(N=2), dict(first=2 ** 31 - 1)])
def test_select(L, bad):
    _refused(L, _select(L, **bad))


@pytest.mark.parametrize("bad", HEADS + [dict(kc=None), dict(vc=None), dict(blocks=None), dict(kc=ODD), dict(vc=ODD),
                                         dict(out=ODD)])
def test_attention(L, bad):
    _refused(L, _attend(L, **bad))


def test_workspaces(L):
    plan, pick, attend = (L.molt_plan_blocks_workspace_size, L.molt_select_blocks_workspace_size,
                          L.molt_paged_attention_blocks_workspace_size)
    assert plan(0, 5) == plan(5, 0) == plan(128, 5) == 0 and plan(3000, 5) > 0
    assert _plan(L, B=3000, ws=None) == WORKSPACE and _plan(L, B=3000, wsb=plan(3000, 5) - 1) == WORKSPACE
    size = pick(2, 4, 32, 4, 128, 6000)
    assert size > 0 and _select(L, mb=6000, wsb=size - 1) == WORKSPACE and _select(L, mb=6000, ws=None) == WORKSPACE
    assert pick(0, 4, 32, 4, 128, 600) == pick(2, 4, 30, 4, 128, 600) == pick(2, 4, 32, 4, 96, 600) == 0
    size = attend(1, 0, 32, 4, 128, 256)
    assert size > 0 and _attend(L, B=1, k=0, N=256, wsb=size - 1) == WORKSPACE
    assert _attend(L, B=1, k=0, N=256, ws=None) == WORKSPACE and b"workspace" in L.molt_last_error()
    assert attend(1, 0, 32, 4, 128, 0) == attend(1, -1, 32, 4, 128, 8) == 0


def test_a_size_function_leaves_the_last_message(L):
    _refused(L, _plan(L, B=0))
    said = L.molt_last_error()
    assert L.molt_select_blocks_workspace_size(0, 4, 32, 4, 128, 600) == 0 and L.molt_last_error() == said


def test_python_calls_need_gpu_tensors():
    kc, vc, bounds = torch.zeros(4, 2, 16, 128), torch.zeros(4, 2, 128, 16), molt.key_bounds(4, 2, 128, device="cpu")
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    pool = molt.block_pool(5, device="cpu")
    assert pool.tolist() == [0, 5, 0, 1, 2, 3, 4]
    rows = torch.zeros(2, 2, 128)
    for call in (lambda: molt.plan_blocks(i(2, 2), i(2), i(2), i(2), pool, 1),
                 lambda: molt.kv_write(rows, rows, kc, vc, i(2)),
                 lambda: molt.key_bounds_update(kc, bounds, i(2, 2), i(2), 1),
                 lambda: molt.key_bounds_read(bounds, i(3)),
                 lambda: molt.select_blocks(rows, bounds, i(2, 2), i(2), 0, 4),
                 lambda: molt.paged_attention_blocks(rows, kc, vc, i(2, 2), i(2), 0, i(2, 2, 4))):
        with pytest.raises(molt.MoltError, match="GPU"):
            call()

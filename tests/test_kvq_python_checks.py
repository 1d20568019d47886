"""KVCache of 4-bit caches: what a model call would read as something else is refused (host tensors will do here)."""
import os
import subprocess
import sys
import types

import pytest
import torch

import paper_2607_21653_amd as molt
from paper_2607_21653_amd import _lib

L, NB, H, D, B, MAXB = 3, 8, 2, 64, 2, 4


def _model(layers=L, heads=H):
    m = _lib.MoltModel()
    m.n_layers, m.n_q_heads, m.n_kv_heads, m.head_dim = layers, 4 * heads, heads, D
    return types.SimpleNamespace(struct=m)


def _kv(ks=None, vs=None, tables=None, ctx=None):
    pairs = [molt.kvq_cache(NB, H, D, device="cpu") for _ in range(L)]
    ks, vs = (given or [p[i] for p in pairs] for i, given in ((0, ks), (1, vs)))
    tables = torch.zeros(B, MAXB, dtype=torch.int32) if tables is None else tables
    ctx = torch.zeros(B, dtype=torch.int32) if ctx is None else ctx
    return molt.KVCache(ks, vs, tables, ctx)


def test_layers_of_one_pool():
    """pool[:, l] has the shape of a cache and starts at a multiple of 16 bytes, but its blocks are not next to each
    other: a call would write other layers' records. pool[l] is a cache."""
    pool = torch.zeros(NB, L, H, 17 * D // 2, dtype=torch.uint8)
    for kw in (dict(ks=[pool[:, l] for l in range(L)]), dict(vs=[pool[:, l] for l in range(L)])):
        with pytest.raises(molt.MoltError, match="contiguous"):
            _kv(**kw)
    pool = torch.zeros(L, NB, H, 17 * D // 2, dtype=torch.uint8)
    with pytest.raises(molt.MoltError, match="GPU"):             # (all else is right)
        _kv(ks=[pool[l] for l in range(L)]).check(_model(), B)


@pytest.mark.parametrize("word,kw", [
    ("block_tables must be contiguous", dict(tables=torch.zeros(B, 2 * MAXB, dtype=torch.int32)[:, :MAXB])),
    ("context_lens must be contiguous", dict(ctx=torch.zeros(2 * B, dtype=torch.int32)[::2])),
    ("block_tables must be int32", dict(tables=torch.zeros(B, MAXB, dtype=torch.int64))),
    ("context_lens must be int32", dict(ctx=torch.zeros(B, 1, dtype=torch.int32)))])
def test_tables(word, kw):
    with pytest.raises(molt.MoltError, match=word):
        _kv(**kw)


@pytest.mark.parametrize("word,model,batch", [
    ("layers", _model(layers=L + 1), B), ("layers", _model(layers=L - 1), B), ("shape", _model(heads=H + 1), B),
    ("sequences", _model(), B + 1), ("GPU", _model(), B), ("GPU", _model(), B - 1)])
def test_model(word, model, batch):
    with pytest.raises(molt.MoltError, match=word):
        _kv().extra(model, batch, 0)


def test_other_caches_are_as_before():
    """Only 4-bit caches are looked over."""
    k = torch.zeros(NB, L, H, 16, D)
    kv = molt.KVCache([k[:, l] for l in range(L)], [k[:, l] for l in range(L)], torch.zeros(B, MAXB, dtype=torch.int32),
                      torch.zeros(B, dtype=torch.int32))
    kv.check(_model(), B)
    assert kv.extra(_model(), B, 0) == 0


def test_import_without_gpu_support():
    """torch without its GPU functions: the package imports, its prefix cache works, GPU calls refuse host tensors."""
    code = """
import torch
for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
import paper_2607_21653_amd as molt
molt.PrefixCache(8)
cache = molt.kvq_cache(4, 2, 64, device="cpu")
try:
    molt.kvq_read(*cache, torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 1)
except molt.MoltError as e:
    assert "GPU" in str(e), e
else:
    raise SystemExit("not refused")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr

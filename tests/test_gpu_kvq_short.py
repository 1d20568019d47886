"""GPU tests of attention over the 4-bit KV cache by workgroups of one wavefront, which many sequences with short tables
get: key ranges of 1 to 15 pairs of blocks (its ring holds 3), one to three tiles of rows, one and several row groups."""
import numpy as np
import pytest
import torch

import plans
from oracle import kvq
from test_gpu_kvq import _rows
from test_gpu_kvq_weights import _caches, _check

pytestmark = pytest.mark.gpu

# sequences, positions, query heads, kv heads, shortest and longest context
SHAPES = [
    (600, 1, 8, 8, 0, 200),              # one row
    (250, 6, 16, 4, 33, 330),            # 24 rows: two tiles
    (300, 5, 16, 2, 100, 280),           # 40 rows: three tiles
    (300, 9, 16, 2, 3, 400),             # 72 rows: two row groups, the second a tile less
    (60, 40, 16, 2, 0, 290),             # windows of 320 rows
    (150, 20, 14, 7, 190, 430),          # 40 rows, 7 kv heads
    (400, 4, 40, 4, 120, 300),           # 40 rows
]


def _one_wavefront(B, n, Hq, Hkv, D, ctx, dtype):
    maxb = (max(ctx) + n + 15) // 16 + 1                 # (as _caches makes tables)
    plan = plans.kvq_plan(B, n, Hq, Hkv, D, maxb, dtype == "f32")
    assert plan.waves == 1 and plan.slots == B
    return plan


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,n,Hq,Hkv,lo,hi", SHAPES)
def test_against_dense_softmax(molt_lib, B, n, Hq, Hkv, lo, hi, D, dtype):
    """Slots past each sequence's last position, and blocks of no sequence, hold NaN."""
    rng = np.random.default_rng(61)
    ctx = [int(c) for c in rng.permutation(np.linspace(lo, hi, B).astype(int))]
    if (B, n, D, dtype) == (300, 9, 64, "f32"):
        ctx = [c * 2 // 3 for c in ctx]                  # (longer tables get 4 wavefronts there)
    plan = _one_wavefront(B, n, Hq, Hkv, D, ctx, dtype)
    print(f"row groups {plan.row_groups} of {plan.group_rows} rows, up to {(max(ctx) + n + 31) // 32} pairs", flush=True)
    caches, K, V = _caches(molt_lib, rng, ctx, n, Hkv, D)
    q, q64 = _rows(rng, B * n, Hq, D, dtype)
    _check(molt_lib, q, q64, caches, K, V, ctx, n, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_values_beyond_f16(molt_lib, D, dtype):
    """From a first, middle or last pair on values that f16 does not hold."""
    B, n, Hq, Hkv = 300, 5, 16, 2
    rng = np.random.default_rng(63)
    ctx = [int(c) for c in np.linspace(100, 280, B)]
    _one_wavefront(B, n, Hq, Hkv, D, ctx, dtype)
    exps = [np.zeros((c + n, D // 32), int) for c in ctx]
    for b, e in enumerate(exps):
        at = (0, len(e) // 2, len(e) - 1)[b % 3]
        e[at:at + 1 + b % 40, b % (D // 32)] = (60, -60, -90, 90)[b % 4]
    caches, K, V = _caches(molt_lib, rng, ctx, n, Hkv, D, exps)
    q, q64 = _rows(rng, B * n, Hq, D, dtype)
    _check(molt_lib, q, q64, caches, K, V, ctx, n, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where", ["key", "value"])
def test_nan_in_a_later_pair(molt_lib, D, dtype, where):
    """A NaN group of a position of the window: the rows before it are the same bits as without it, the rows from it on
    are NaN, in its group's dims only where it is a value."""
    B, n, Hq, Hkv = 300, 5, 16, 2
    rng = np.random.default_rng(65)
    ctx = [int(c) for c in np.linspace(100, 280, B)]
    _one_wavefront(B, n, Hq, Hkv, D, ctx, dtype)
    (gk, gv, gt, gc), _, _ = _caches(molt_lib, rng, ctx, n, Hkv, D)
    q = _rows(rng, B * n, Hq, D, dtype)[0].cuda()
    clean = molt_lib.paged_attention_kvq(q, gk, gv, gt, gc, n - 1).view(B, n, Hkv, Hq // Hkv, D)
    tables, group, kv_head = gt.cpu().numpy(), D // 32 - 1, 1
    cache = gk if where == "key" else gv
    blocks, offsets = [], []
    for b, c in enumerate(ctx):
        blk, slot = kvq.place(tables[b], c + 2, len(gk))
        blocks.append(blk)
        offsets.append(int(kvq.offsets(slot, D, where == "value")[1][group]))
    cache[torch.tensor(blocks).cuda(), kv_head, torch.tensor(offsets).cuda()] = 255
    out = molt_lib.paged_attention_kvq(q, gk, gv, gt, gc, n - 1).view(clean.shape)
    hit = torch.zeros(clean.shape, dtype=torch.bool, device="cuda")
    hit[:, 2:, kv_head, :, (0 if where == "key" else 32 * group):(D if where == "key" else 32 * group + 32)] = True
    assert torch.isnan(out[hit]).all()
    assert torch.equal(out[~hit], clean[~hit])

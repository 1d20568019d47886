"""GPU parity of sparse attention over listed blocks and of the cache's upkeep against the float64 oracle: plan_blocks,
kv_write, key bounds and select_blocks exactly (every byte of caches and tables, written or not), attention within the
tolerance derived below."""
import numpy as np
import pytest
import torch

from oracle import blocks as ob

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _tol(out, mag, dtype):
    """The output's rounding: half a step, 2^-8 |o| in bf16, 2^-24 |o| in f32. The weights: scores are f32 sums of D
    products, off by at most D 2^-24 sum |q k| / sqrt(D), with unit normals 2^-14 for D = 128; a weight and the sum
    of weights move by that each, 2^-13 in all, and by 2^-19 for the exponential's argument (up to 2^5 in f32). The
    bf16 weights have 16 bits: 2^-17 each. Sums over N keys add at most the number of steps of one lane, 2^7, times
    2^-24. Together under 2^-12 of sum w |v|."""
    return (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(out) + 2.0 ** -12 * mag + 1e-30


def _t(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _i32(a):
    return _t(np.asarray(a, np.int32))


def _val(t):
    return t.double().cpu().numpy()


# ---------------------------------------------------------------- plan

def _plan_both(molt, tables, n_blocks, ctx, new, pool, n, shared=None):
    gt, gn, gp = _t(tables), _t(n_blocks), _t(pool)
    slots, placed = molt.plan_blocks(gt, gn, _i32(ctx), _i32(new), gp, n, n_shared=None if shared is None else _i32(shared))
    want = ob.plan(tables, n_blocks, ctx, new, pool, n, shared)
    for got, w, name in ((slots, want[0], "slots"), (placed, want[1], "placed"), (gt, tables, "tables"),
                         (gn, n_blocks, "n_blocks"), (gp, pool, "pool")):
        assert np.array_equal(got.cpu().numpy(), w), name


@pytest.mark.parametrize("B,n,maxb,cap", [(1, 1, 1, 1), (5, 3, 4, 30), (64, 5, 20, 700), (1024, 8, 3, 2000),
                                          (1025, 2, 4, 3000), (3, 3000, 400, 500), (40, 300, 30, 400), (2500, 1, 2, 3000)])
def test_plan_over_a_session(molt_lib, B, n, maxb, cap):
    """Steps of a session on one state: sequences grow, finish, start again; the pool runs dry at times."""
    rng = np.random.default_rng(B + n)
    tables, n_blocks = np.full((B, maxb), -7, np.int32), np.zeros(B, np.int32)
    pool = np.concatenate([[rng.integers(cap), cap], rng.permutation(cap)]).astype(np.int32)
    ctx = np.zeros(B, np.int32)
    for step in range(8):
        new = rng.integers(0, n + 1, B).astype(np.int32)
        new[rng.random(B) < 0.2] = -1
        before = n_blocks.copy()
        _plan_both(molt_lib, tables, n_blocks, ctx, new, pool, n)
        ctx = np.where(new < 0, 0, np.where((new > 0) & (n_blocks * 16 >= ctx + new), ctx + new, ctx)).astype(np.int32)
        held = np.concatenate([tables[b, :n_blocks[b]] for b in range(B)])
        free = pool[2 + (pool[0] + np.arange(pool[1])) % cap]
        assert sorted([*held, *free]) == list(range(cap)), (step, before.sum())


def test_plan_of_numbers_out_of_range(molt_lib):
    tables = np.arange(60, dtype=np.int32).reshape(10, 6) + 40
    n_blocks = np.array([-1, 7, 2, 2, 2, 0, 6, 3, 2, 2], np.int32)
    ctx = np.array([5, 5, -1, 90, 20, 50, 80, 33, 2 ** 31 - 1, 32], np.int32)
    new = np.array([3, 3, 3, 7, 9, 2, -2 ** 31, 0, 3, 1], np.int32)   # row 5 lacks blocks of its cached tokens
    pool = np.concatenate([[95, 8], np.arange(100)]).astype(np.int32)
    pool[2 + 95] = 100                                               # an id outside the pool: its rows get no slot
    for n in (7, 3000):
        _plan_both(molt_lib, tables.copy(), n_blocks.copy(), ctx, new, pool.copy(), n)
    pool[:2] = -3, 1000                                              # a head and a count that no call leaves
    _plan_both(molt_lib, tables.copy(), n_blocks.copy(), ctx, new, pool.copy(), 7)
    pool[:2] = 3, 97                                                 # gives back more than the ring has room for
    _plan_both(molt_lib, tables.copy(), n_blocks.copy(), ctx, new, pool.copy(), 7)


@pytest.mark.parametrize("n", [5, 5000])
def test_plan_keeps_shared_blocks(molt_lib, n):
    tables = np.arange(24, dtype=np.int32).reshape(4, 6)
    n_blocks, shared = np.array([4, 4, 2, 6], np.int32), np.array([2, 9, 0, -4], np.int32)
    pool = np.concatenate([[28, 3], np.full(30, 29)]).astype(np.int32)
    _plan_both(molt_lib, tables, n_blocks, [64, 64, 32, 96], np.array([-1, -1, 2, -5], np.int32), pool, n, shared)


# ---------------------------------------------------------------- rows by slot

def _cache(rng, nb, H, D, dtype, fill=None):
    shape = (nb, H, 16, D), (nb, H, D, 16)
    return [torch.full(s, fill, dtype=DT[dtype]) if fill is not None
            else torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(DT[dtype]) for s in shape]


def _runs(rng, nb):
    """Slots: runs of all lengths from all offsets, holes, and numbers outside the cache; no slot twice."""
    out, order = [], rng.permutation(nb)
    for i, block in enumerate(order[:nb - 2]):
        first = 0 if i % 3 == 0 else int(rng.integers(16))
        length = 16 - first if i % 3 != 1 else int(rng.integers(1, 17 - first))
        out += [block * 16 + first + t for t in range(length)]
        if i % 4 == 0:
            out += [-1] * int(rng.integers(1, 9))
    a, b = order[nb - 2:] * 16
    return out + [16 * nb, -2 ** 31, 2 ** 31 - 1, a + 3, a + 2, a + 1, a + 7, a + 8, b + 15, b, b + 1, b + 5]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,D", [(4, 128), (1, 128), (3, 64), (1, 64)])
def test_write(molt_lib, dtype, H, D):
    rng = np.random.default_rng(D + H)
    nb = 30
    kc, vc = _cache(rng, nb, H, D, dtype)
    slots = _runs(rng, nb)
    T = len(slots)
    rows = torch.from_numpy(rng.standard_normal((T, 3 * H + 1, D)).astype(np.float32)).to(DT[dtype])
    gk, gv, grows = kc.cuda(), vc.cuda(), rows.cuda()
    k, v = grows[:, H:2 * H], grows[:, 2 * H:3 * H]
    molt_lib.kv_write(k, v, gk, gv, _i32(slots))
    wk, wv = _val(kc), _val(vc)
    ob.write_rows(_val(k), _val(v), wk, wv, slots)
    assert np.array_equal(_val(gk), wk) and np.array_equal(_val(gv), wv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,D", [(4, 128), (3, 64)])
def test_write_of_many_rows(molt_lib, dtype, H, D):
    """Whole and partial blocks, single rows, runs of two to four, holes among them, and changes between these at any
    row of a tile of 16."""
    rng = np.random.default_rng(7 * D + H)
    nb = 700
    order, slots, at = rng.permutation(nb), [], 0
    while at + 20 < nb:
        kind = int(rng.integers(5))
        if kind == 0:                                     # blocks in a row, the first from its middle
            slots += [int(order[at]) * 16 + t for t in range(int(rng.integers(16)), 16)]
            slots += [int(b) * 16 + t for b in order[at + 1:at + 3] for t in range(16)]
            at += 3
        else:
            longest = (1, 1, 4, 16)[kind - 1]
            for b in order[at:at + 20]:
                first = int(rng.integers(16))
                slots += [int(b) * 16 + t for t in range(first, min(16, first + int(rng.integers(1, longest + 1))))]
                if kind == 2 and rng.integers(3) == 0:
                    slots += [-1] * int(rng.integers(1, 4))
            at += 20
    slots += [-1] * (12000 // H - len(slots))  # enough rows for the kernel of many
    T = len(slots)
    kc, vc = _cache(rng, nb, H, D, dtype)
    k, v = (torch.from_numpy(rng.standard_normal((T, H, D)).astype(np.float32)).to(DT[dtype]) for _ in range(2))
    gk, gv = kc.cuda(), vc.cuda()
    molt_lib.kv_write(k.cuda(), v.cuda(), gk, gv, _i32(slots))
    wk, wv = _val(kc), _val(vc)
    ob.write_rows(_val(k), _val(v), wk, wv, slots)
    assert np.array_equal(_val(gk), wk) and np.array_equal(_val(gv), wv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_write_of_rows_at_any_element(molt_lib, dtype):
    rng = np.random.default_rng(5)
    H, D, T = 2, 64, 21
    kc, vc = _cache(rng, 4, H, D, dtype)
    flat = torch.from_numpy(rng.standard_normal(T * 211 + 9).astype(np.float32)).to(DT[dtype]).cuda()
    k = torch.as_strided(flat, (T, H, D), (211, D, 1), 1)
    v = torch.as_strided(flat, (T, H, D), (211, D, 1), 7)
    slots = np.arange(T) + 19
    gk, gv = kc.cuda(), vc.cuda()
    molt_lib.kv_write(k, v, gk, gv, _i32(slots))
    wk, wv = _val(kc), _val(vc)
    ob.write_rows(_val(k), _val(v), wk, wv, slots)
    assert np.array_equal(_val(gk), wk) and np.array_equal(_val(gv), wv)


def test_write_of_a_slot_twice_leaves_one_of_the_rows(molt_lib):
    H, D = 1, 128
    kc, vc = torch.zeros(2, H, 16, D, device="cuda"), torch.zeros(2, H, D, 16, device="cuda")
    rows = torch.arange(1.0, 5.0, device="cuda").view(4, 1, 1).expand(4, H, D).contiguous()
    molt_lib.kv_write(rows, rows, kc, vc, _i32([5, 5, 6, 5]))
    assert set(kc[0, 0, 5].unique().tolist()) <= {1.0, 2.0, 4.0} and set(vc[0, 0, :, 5].unique().tolist()) <= {1.0, 2.0, 4.0}
    assert (kc[0, 0, 6] == 3).all() and (vc[0, 0, :, 6] == 3).all()
    assert kc.count_nonzero() == vc.count_nonzero() == 2 * D


# ---------------------------------------------------------------- bounds

def _special_keys(kc):
    """Blocks that decide: zeros, one sign, the border of a unit, tiny, subnormal, huge, infinities, NaN."""
    kc[0] = 0
    kc[1] = kc[1].abs()
    kc[2] = -kc[2].abs()
    kc[3] = 127.0
    kc[4] = 127.5
    kc[4, 0, 3] = -127.5
    kc[5] *= 2.0 ** -110
    kc[6] *= 2.0 ** -135
    kc[7] *= 2.0 ** 120
    kc[8, 0, 5, 7] = float("inf")
    kc[9, 0, 15, 9] = float("nan")
    kc[10, -1, 0, 0] = float("-inf")
    kc[11, 0, 9] = 3.3e38
    return kc


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,H,D,hi,ragged", [(1, 1, 1, 64, 0, False), (6, 5, 3, 128, 90, True), (5, 70, 2, 64, 40, True),
                                               (3, 16, 4, 128, 33, False), (2, 129, 1, 128, 0, False)])
def test_bounds(molt_lib, dtype, B, n, H, D, hi, ragged):
    rng = np.random.default_rng(B * n)
    maxb = (hi + n + 15) // 16 + 1
    nb = max(B * maxb, 12) + 2
    kc = _special_keys(_cache(rng, nb, H, D, dtype)[0])
    tables = rng.permutation(nb)[:B * maxb].reshape(B, maxb).astype(np.int32)
    ctx = rng.integers(0, hi + 1, B).astype(np.int32)
    lens = rng.integers(0, n + 1, B).astype(np.int32) if ragged else None
    if ragged:
        lens[0], lens[-1] = 0, n + 9
        ctx[-2] = -3                                                 # positions before the table
        tables[1, 0], tables[2, 1] = nb, -1                          # places outside the cache
    start = rng.integers(0, 256, (nb, H, 2 * D + 16)).astype(np.uint8)
    gb = _t(start)
    molt_lib.key_bounds_update(kc.cuda(), gb, _t(tables), _t(ctx), n, lens=None if lens is None else _t(lens))
    want = start.copy()
    ob.update_bounds(_val(kc), want, tables, ctx, n, lens)
    assert np.array_equal(gb.cpu().numpy(), want)


@pytest.mark.parametrize("D", [64, 128])
def test_bounds_of_special_blocks_and_back(molt_lib, D):
    rng = np.random.default_rng(D)
    kc = _special_keys(_cache(rng, 14, 3, D, "f32")[0])
    bounds = molt_lib.key_bounds(14, 3, D)
    molt_lib.key_bounds_update(kc.cuda(), bounds, _i32(np.arange(14)[None]), _i32([0]), 14 * 16)
    for i in range(14):
        for h in range(3):
            assert np.array_equal(bounds[i, h].cpu().numpy(), ob.record(_val(kc[i, h]))), (i, h)
    ids = [3, 8, 14, -1, 0, 5, 3, 7]
    hi, lo = molt_lib.key_bounds_read(bounds, _i32(ids))
    assert hi.shape == lo.shape == (8, 3, D)
    for i, block in enumerate(ids):
        if not 0 <= block < 14:
            assert hi[i].isnan().all() and lo[i].isnan().all()
            continue
        for h in range(3):
            a, b, e = ob.bounds_of(_val(kc[block, h]))
            if e == ob.NOT_FINITE:
                assert (hi[i, h] == float("inf")).all() and (lo[i, h] == float("-inf")).all()
            else:
                assert np.array_equal(_val(hi[i, h]), np.ldexp(a, e)) and np.array_equal(_val(lo[i, h]), np.ldexp(b, e))


# ---------------------------------------------------------------- selection

def _random_bounds(rng, nb, H, D, spread):
    rec = rng.integers(-127, 128, (nb, H, 2 * D + 16)).astype(np.int8)
    rec[..., :D], rec[..., D:2 * D] = np.maximum(rec[..., :D], rec[..., D:2 * D]), np.minimum(rec[..., :D], rec[..., D:2 * D])
    rec[..., 2 * D] = rng.integers(-spread, spread + 1, (nb, H))
    return rec.view(np.uint8)


def _select_both(molt, q, bounds, tables, ctx, n, N, first, last, lens=None):
    got = molt.select_blocks(q.cuda(), _t(bounds), _t(tables), _i32(ctx), n - 1, N, n_first=first, n_last=last,
                             lens=None if lens is None else _i32(lens))
    want = ob.select(_val(q), bounds, tables, ctx, n, N, first, last, lens)
    assert got.dtype == torch.int32 and np.array_equal(got.cpu().numpy(), want)


def _queries(rng, B, n, Hq, D, dtype):
    return torch.from_numpy(rng.standard_normal((B * n, Hq, D)).astype(np.float32)).to(DT[dtype])


@pytest.mark.parametrize("G", [1, 2, 3, 5, 8, 12, 16, 17, 40, 70])
@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "f32")])
def test_select_of_head_layouts(molt_lib, G, D, dtype):
    rng = np.random.default_rng(G)
    H, B, n, maxb = 2, 2, 3, 20
    bounds = _random_bounds(rng, B * maxb + 1, H, D, 1)
    tables = rng.permutation(B * maxb).reshape(B, maxb).astype(np.int32)
    _select_both(molt_lib, _queries(rng, B, n, G * H, D, dtype), bounds, tables, [250, 318 - n], n, 6, 1, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,maxb,N,first,last", [(1, 1, 1, 1, 0, 1), (3, 1, 9, 4, 1, 2), (2, 37, 40, 9, 0, 1),
                                                   (4, 70, 12, 16, 3, 2), (1, 5, 700, 64, 1, 2), (2, 2, 300, 299, 1, 2),
                                                   (1, 2, 200, 210, 2, 3)])
def test_select_of_lengths(molt_lib, dtype, B, n, maxb, N, first, last):
    rng = np.random.default_rng(maxb)
    bounds = _random_bounds(rng, B * maxb + 3, 2, 64, 3)
    tables = rng.permutation(B * maxb).reshape(B, maxb).astype(np.int32)
    ctx = np.linspace(max(0, 16 * maxb - n), 0, B).astype(np.int32)
    lens = [n - b * n // B for b in range(B)]
    _select_both(molt_lib, _queries(rng, B, n, 4, 64, dtype), bounds, tables, ctx, n, N, first, last)
    _select_both(molt_lib, _queries(rng, B, n, 4, 64, dtype), bounds, tables, ctx, n, N, first, last, lens)


@pytest.mark.parametrize("G", [1, 3, 8, 16])
@pytest.mark.parametrize("B,n,maxb,N", [(150, 1, 60, 9), (70, 9, 20, 5), (260, 1, 130, 40), (9, 130, 33, 7), (17, 3, 500, 30)])
def test_select_of_many_sequences(molt_lib, G, B, n, maxb, N):
    """Launches of many workgroups, also by XCD with a number of sequences that 8 does not divide; a sample is checked
    against the oracle, all rows against the same sequences in calls of their own."""
    rng = np.random.default_rng(B)
    H, D = 2, 64
    bounds = _random_bounds(rng, B * maxb + 1, H, D, 2)
    tables = rng.permutation(B * maxb).reshape(B, maxb).astype(np.int32)
    ctx = rng.integers(0, 16 * maxb - n, B).astype(np.int32)
    q = _queries(rng, B, n, G * H, D, "bf16")
    gq, gb, gt, gc = q.cuda(), _t(bounds), _t(tables), _i32(ctx)
    got = molt_lib.select_blocks(gq, gb, gt, gc, n - 1, N)
    for b in range(0, B, 7):
        one = molt_lib.select_blocks(gq[b * n:(b + 1) * n], gb, gt[b:b + 1], gc[b:b + 1], n - 1, N)
        assert torch.equal(got[b * n:(b + 1) * n], one), b
    b, j = B - 1, n - 1
    want = ob.select(_val(q)[b * n + j:b * n + j + 1], bounds, tables[b:], [int(ctx[b]) + j], 1, N, 1, 2)
    assert np.array_equal(got[b * n + j:].cpu().numpy(), want)


@pytest.mark.parametrize("B,H,maxb", [(260, 1, 1100), (2, 130, 2100), (260, 4, 2060), (260, 4, 4100), (1, 2, 4000), (1, 2, 5000)])
def test_select_of_long_tables(molt_lib, B, H, maxb):
    """One launch or two, many lists or few: against a sort of the scores, which are those of one dim here."""
    rng = np.random.default_rng(maxb)
    D, N = 64, 33
    rec = np.zeros((maxb, H, 2 * D + 16), np.int8)
    rec[:, :, 0] = rng.integers(-120, 121, (maxb, H))
    rec[:, :, D] = rec[:, :, 0]
    rec[:, :, 2 * D] = rng.integers(-3, 4, (maxb, H))
    bounds = torch.from_numpy(rec.view(np.uint8)).cuda()
    table = torch.randperm(maxb, dtype=torch.int32).cuda()
    q = torch.zeros(B, H, D)
    q[:, :, 0] = torch.from_numpy(rng.choice([-1.0, 1.0], (B, H)).astype(np.float32))
    ctx = rng.integers(16 * 64, 16 * maxb, B).astype(np.int32)
    got = molt_lib.select_blocks(q.cuda(), bounds, table.expand(B, maxb).contiguous(), _i32(ctx), 0, N).cpu().numpy()
    value = (rec[:, :, 0].astype(float) * 2.0 ** rec[:, :, 2 * D])[table.cpu().numpy()]
    for b in range(0, B, 13):
        last = ctx[b] // 16
        for h in range(H):
            s = q[b, h, 0].item() * value[:last + 1, h]
            s[0], s[last - 1:] = np.inf, np.inf
            order = np.lexsort((np.arange(last + 1), -s))[:N]
            assert np.array_equal(got[b, h], np.sort(order)), (b, h)


@pytest.mark.parametrize("maxb", [30, 1500, 5000, 17000])
def test_select_of_equal_scores(molt_lib, maxb):
    """Few different scores, many ties, all equal ones, zeros: the lowest blocks of them."""
    rng = np.random.default_rng(maxb)
    bounds = np.zeros((maxb, 3, 2 * 64 + 16), np.uint8)
    bounds[:, 0, 0] = rng.integers(0, 3, maxb)
    bounds[:, 1, 0] = 5
    q = torch.zeros(2, 3, 64)
    q[:, :, 0] = 1.0
    tables = rng.permutation(maxb).astype(np.int32)[None]
    for N in (3, 24, 1200):
        _select_both(molt_lib, q, bounds, tables, [16 * maxb - 2], 2, N, 1, 1)


def test_select_of_what_is_not_finite_and_has_no_place(molt_lib):
    rng = np.random.default_rng(9)
    B, n, H, D, maxb = 3, 2, 2, 128, 50
    nb = B * maxb
    bounds = _random_bounds(rng, nb, H, D, 100)
    bounds[rng.permutation(nb)[:40], :, 2 * D] = 127                 # blocks with an infinity or NaN come first
    bounds[3, 0, 2 * D] = 121
    tables = rng.permutation(nb).reshape(B, maxb).astype(np.int32)
    tables[0, ::3], tables[1, -4:], tables[2] = nb, -1, -9
    tables[2, 7] = 4
    q = _queries(rng, B, n, 3 * H, D, "f32")
    q[0, 0, 5], q[0, 4, 0], q[2, :3, 1] = float("nan"), float("inf"), float("-inf")
    q[1, 1] = 0.0
    q[1, 2] *= 2.0 ** 120
    q[3] *= 2.0 ** -120
    for N in (4, 30, 60):
        _select_both(molt_lib, q, bounds, tables, [700, 799 - n, 500], n, N, 1, 2)
    _select_both(molt_lib, q, bounds, tables, [-1, -5, 16 * maxb + 40], n, 6, 1, 2)


def test_select_by_bounds_of_keys(molt_lib):
    """The whole way from keys: what is left out has no larger product than the list's least score."""
    rng = np.random.default_rng(4)
    nb, H, D = 64, 2, 128
    kc = _cache(rng, nb, H, D, "bf16")[0].cuda()
    bounds, table, zero = molt_lib.key_bounds(nb, H, D), _i32(rng.permutation(nb)[None]), _i32([0])
    molt_lib.key_bounds_update(kc, bounds, table, zero, nb * 16)
    q = _queries(rng, 1, 1, 8, D, "bf16")
    q = (q * 0 + torch.round(q * 16) / 16).to(torch.bfloat16)        # (rows that 8 bits hold: |q| < 127 / 16)
    got = molt_lib.select_blocks(q.cuda(), bounds, table, _i32([nb * 16 - 1]), 0, 9, n_first=0, n_last=1)
    k, t = _val(kc), table[0].cpu().numpy()
    rec = bounds.cpu().numpy()
    for h in range(H):
        rows = _val(q)[0, 4 * h:4 * h + 4]
        scores = [ob.score(rows, rec[t[i], h]) for i in range(nb)]
        picked = got[0, h].tolist()
        least = min(scores[i] for i in picked[:-1])
        assert picked[-1] == nb - 1
        assert max((rows @ k[t[i], h].T).max() for i in range(nb) if i not in picked) <= least


# ---------------------------------------------------------------- attention

def _attend_both(molt, q, kc, vc, tables, ctx, n, lists, dtype, **kw):
    got = molt.paged_attention_blocks(q.cuda(), kc.cuda(), vc.cuda(), _t(tables), _i32(ctx), n - 1, _t(lists), **kw)
    clean = [np.nan_to_num(_val(x), nan=1e9, posinf=1e9, neginf=1e9) for x in (kc, vc)]
    want, mag = ob.attend(_val(q), *clean, tables, ctx, n, lists)
    T, Hq, D = q.shape
    assert got.dtype == q.dtype and got.shape == (T, Hq * D)
    err = np.abs(_val(got).reshape(T, Hq, D) - want) - _tol(want, mag, dtype)
    assert err.max() <= 0, err.max()
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,H,G,D,N,maxb", [(1, 1, 1, 1, 64, 1, 1), (2, 3, 2, 4, 128, 5, 9), (3, 1, 4, 8, 128, 16, 30),
                                              (1, 2, 2, 7, 64, 33, 60), (2, 5, 1, 16, 128, 8, 20), (1, 1, 2, 17, 64, 12, 20),
                                              (1, 3, 1, 80, 128, 7, 10), (1, 1, 1, 8, 128, 300, 400), (1, 2, 4, 2, 64, 130, 200),
                                              (7, 9, 3, 2, 64, 12, 20), (33, 3, 3, 8, 128, 24, 30), (20, 5, 3, 1, 64, 130, 140),
                                              (90, 1, 3, 2, 128, 9, 12)])
def test_attention(molt_lib, dtype, B, n, H, G, D, N, maxb):
    rng = np.random.default_rng(N)
    nb = B * maxb + 2
    kc, vc = _cache(rng, nb, H, D, dtype)
    tables = rng.permutation(nb)[:B * maxb].reshape(B, maxb).astype(np.int32)
    ctx = np.linspace(16 * maxb - n, 0, B).astype(np.int32)
    for b in range(B):                                               # slots past the last row, and free blocks: NaN
        for i in range(maxb):
            m = min(max(int(ctx[b]) + n - 16 * i, 0), 16)
            kc[tables[b, i], :, m:], vc[tables[b, i], :, :, m:] = float("nan"), float("nan")
    lists = np.stack([np.stack([rng.permutation(max(maxb, N))[:N] for _ in range(H)]) for _ in range(B * n)]).astype(np.int32)
    lists[lists >= maxb] = -1
    q = _queries(rng, B, n, G * H, D, dtype)
    got = _attend_both(molt_lib, q, kc, vc, tables, ctx, n, lists, dtype)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    again = molt_lib.paged_attention_blocks(q.cuda(), kc.cuda(), vc.cuda(), _t(tables), _i32(ctx), n - 1, _t(lists),
                                            workspace=ws[1:])
    assert torch.equal(again, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_over_odd_lists(molt_lib, dtype):
    """Empty lists, lists of one key, the same block twice, numbers outside the table, places outside the cache,
    blocks past the position, sequences that see nothing."""
    rng = np.random.default_rng(2)
    B, n, H, G, D, maxb, N = 4, 3, 2, 4, 128, 12, 10
    nb = B * maxb
    kc, vc = _cache(rng, nb, H, D, dtype)
    tables = rng.permutation(nb).reshape(B, maxb).astype(np.int32)
    tables[1, 3], tables[1, 5], tables[1, 6] = nb, -1, 2 ** 31 - 1
    ctx = [0, 100, -2, 189]
    lists = rng.integers(0, maxb, (B * n, H, N)).astype(np.int32)     # with repetitions
    lists[0, 0], lists[0, 1] = -1, [-1, -1, -1, -1, 0, -1, -1, -1, -1, -1]
    lists[4, :, ::2] = [-2, maxb, 2 ** 31 - 1, -2 ** 31, maxb + 7]
    lists[9, 0, 1:], lists[10, 0, :9] = 11, -1
    q = _queries(rng, B, n, H * G, D, dtype)
    got = _attend_both(molt_lib, q, kc, vc, tables, ctx, n, lists, dtype)
    assert (got[0, :G * D] == 0).all() and (got[6:8] == 0).all()


def _ascending(lists):
    """The lists as select_blocks leaves them: each block once, ascending, then -1."""
    out = np.full_like(lists, -1)
    for i in np.ndindex(lists.shape[:2]):
        row = np.unique(lists[i][lists[i] >= 0])
        out[i][:len(row)] = row
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,H,G,D,N,maxb", [(1, 2, 1, 8, 128, 1, 3), (2, 5, 2, 8, 128, 24, 40), (3, 4, 1, 7, 64, 63, 70),
                                              (1, 2, 3, 1, 64, 9, 12), (1, 9, 1, 5, 128, 130, 300), (2, 3, 2, 2, 128, 512, 520),
                                              (1, 2, 1, 4, 64, 513, 520)])
def test_attention_over_ascending_lists(molt_lib, dtype, B, n, H, G, D, N, maxb):
    """What neighbouring positions list in common, and what they do not: no block, a few, all."""
    rng = np.random.default_rng(maxb)
    nb = B * maxb
    kc, vc = _cache(rng, nb, H, D, dtype)
    tables = rng.permutation(nb).reshape(B, maxb).astype(np.int32)
    ctx = np.linspace(16 * maxb - n, 30, B).astype(np.int32)
    common = rng.permutation(maxb)
    lists = np.empty((B * n, H, N), np.int32)
    for t in range(B * n):
        for h in range(H):
            own = rng.permutation(maxb)[:N]
            keep = [N, N // 2, 0][(t + h) % 3]
            lists[t, h] = np.concatenate([common[:keep], own[keep:], np.full(N, -1)])[:N]
    _attend_both(molt_lib, _queries(rng, B, n, H * G, D, dtype), kc, vc, tables, ctx, n, _ascending(lists), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [5, 200])
def test_attention_where_only_a_neighbour_sees_nan(molt_lib, dtype, N):
    """A NaN or infinity in a block that the next position lists, or at its own token, leaves a row as it is."""
    rng = np.random.default_rng(12)
    H, G, D, maxb, n = 2, 8, 128, 220, 5
    kc, vc = _cache(rng, maxb, H, D, dtype)
    tables = rng.permutation(maxb).astype(np.int32)[None]
    q = _queries(rng, 1, n, H * G, D, dtype)
    lists = np.tile(np.arange(10, 10 + N, dtype=np.int32), (n, H, 1))
    lists[:, :, 0], lists[:, :, -1] = 3, 219
    ctx = [16 * 219 + 4]
    clean = molt_lib.paged_attention_blocks(q.cuda(), kc.cuda(), vc.cuda(), _t(tables), _i32(ctx), n - 1, _t(lists))
    lists[1, 0, 0], lists[4, 1, 0] = 4, 5                            # others list block 3, or nothing of 4 and 5
    vc[tables[0, 4], 0, 7, 3], kc[tables[0, 5], 1, 2, 8] = float("nan"), float("inf")
    vc[tables[0, 219], 1, 100, 7] = float("-inf")                    # the token of position 3
    got = molt_lib.paged_attention_blocks(q.cuda(), kc.cuda(), vc.cuda(), _t(tables), _i32(ctx), n - 1, _t(lists))
    got, clean = got.view(n, H, G, D), clean.view(n, H, G, D)
    for j, h in ((0, 0), (2, 0), (3, 0), (4, 0), (0, 1), (1, 1), (2, 1)):
        err = (got[j, h].double() - clean[j, h].double()).abs().max().item()
        assert err <= 2.0 ** -7 * clean[j, h].abs().max().item(), (j, h, err)
    assert got[1, 0, :, 7].isnan().all() and not got[1, 0, :, 8:].isnan().any()
    # (bf16 weights go in as two parts, the smaller of any sign or 0: an infinite value gives an infinity or NaN)
    assert not got[3, 1, :, 100].isfinite().any() and not got[3, 1, :, :100].isnan().any()
    assert not got[3, 1, :, 101:].isnan().any()
    up = q.view(n, H, G, D)[4, 1, :, 8].float() > 0                  # heads whose score of the infinite key is +inf
    assert got[4, 1][up].isnan().all() and up.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [3, 200])
def test_attention_of_values_that_are_not_finite(molt_lib, dtype, N):
    """A NaN or infinite key or value that a row sees makes its outputs NaN, as a softmax over them is; others stay."""
    rng = np.random.default_rng(3)
    H, G, D, maxb = 1, 4, 64, 220
    kc, vc = _cache(rng, maxb, H, D, dtype)
    kc[5, 0, 3, 0], kc[9, 0, 1, 2] = float("nan"), float("inf")
    vc[7, 0, 11, 4], vc[2, 0, 9, 15] = float("nan"), float("nan")
    tables = np.arange(maxb, dtype=np.int32)[None]
    q = _queries(rng, 1, 4, G, D, dtype).abs() + 0.1
    lists = np.tile(np.arange(10, 10 + N, dtype=np.int32), (4, 1, 1))
    lists[0, 0, -1], lists[1, 0, 0], lists[2, 0, 1], lists[3, 0, 0] = 5, 9, 7, 2
    ctx = [16 * maxb - 4]
    got = molt_lib.paged_attention_blocks(q.cuda(), kc.cuda(), vc.cuda(), _t(tables), _i32(ctx), 3, _t(lists)).view(4, G, D)
    assert got[0].isnan().all() and got[1].isnan().all()
    assert got[2, :, 11].isnan().all() and not got[2, :, :11].isnan().any() and not got[2, :, 12:].isnan().any()
    assert got[3, :, 9].isnan().all() and not got[3, :, 10:].isnan().any()
    lists[:, 0, :] = -1
    lists[3, 0, 0] = 2
    got = molt_lib.paged_attention_blocks(q.cuda(), kc.cuda(), vc.cuda(), _t(tables), _i32([43]), 3, _t(lists))
    assert not got[3].isnan().any()                                  # position 46: the NaN is at 47


def test_caches_past_2_to_31_elements(molt_lib):
    """Blocks at the end of a pool whose caches have over 2^31 elements, through all of the calls."""
    rng = np.random.default_rng(8)
    H, D = 4, 128
    nb = 2 ** 31 // (H * 16 * D) + 70
    kc = torch.zeros(nb, H, 16, D, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros(nb, H, D, 16, dtype=torch.bfloat16, device="cuda")
    bounds = molt_lib.key_bounds(nb, H, D)
    table, n_blocks = torch.full((1, 64), -1, dtype=torch.int32, device="cuda"), _i32([0])
    pool = torch.zeros(2 + nb, dtype=torch.int32, device="cuda")
    pool[:66] = _i32([0, 64, *range(nb - 1, nb - 65, -1)])
    T = 1000
    slots, placed = molt_lib.plan_blocks(table, n_blocks, _i32([0]), _i32([T]), pool, T)
    assert placed.item() == T and int(slots[0]) == (nb - 1) * 16 and pool[:2].tolist() == [63, 1]
    rows = _queries(rng, 1, T, 2 * H, D, "bf16")
    k, v = rows[:, :H].cuda().contiguous(), rows[:, H:].cuda().contiguous()
    molt_lib.kv_write(k, v, kc, vc, slots)
    molt_lib.key_bounds_update(kc, bounds, table, _i32([0]), T)
    ids = table[0, :63]
    small = [kc[ids.long()], vc[ids.long()], bounds[ids.long()]]
    near = _i32(np.arange(63)[None])
    q, ctx = _queries(rng, 1, 1, 4 * H, D, "bf16").cuda(), _i32([T - 1])
    lists = molt_lib.select_blocks(q, bounds, table, ctx, 0, 9)
    assert torch.equal(lists, molt_lib.select_blocks(q, small[2], near, ctx, 0, 9))
    out = molt_lib.paged_attention_blocks(q, kc, vc, table, ctx, 0, lists)
    assert torch.equal(out, molt_lib.paged_attention_blocks(q, small[0], small[1], near, ctx, 0, lists))
    want, mag = ob.attend(_val(q), _val(small[0]), _val(small[1]), near.cpu().numpy(), [T - 1], 1, lists.cpu().numpy())
    assert (np.abs(_val(out).reshape(want.shape) - want) <= _tol(want, mag, "bf16")).all()

"""GPU parity of the 4-bit KV cache against the float64 oracle: kvq_write bit for bit (every byte of the
caches, written or not), kvq_read exactly, paged_attention_kvq within the tolerance derived below; ragged
and empty contexts, windows of one to many positions, odd head layouts, head dims 64 and 128, slots that
hold NaN where a row must not see them, NaN that it does see, block ids and positions outside the table,
strided and unaligned rows, caches past 2^31 bytes, other streams, graph replays."""
import numpy as np
import pytest
import torch

from helpers import host
from oracle import kvq

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _tol(out, mag, dtype):
    """bf16: the output's rounding, 2^-8 |o|. The weights enter the product rounded to bf16, w (1 + d) with
    |d| <= 2^-8, and so does their sum: the result is off by sum w d (v - o) / (1 + sum w d), at most
    2^-8 (1 + 2^-7) (sum w |v| + |o|). f32 sums, and scores whose f32 sums and hardware exp2 move a weight by
    well under 2^-10: 2^-10 sum w |v|, which also covers the 2^-7 of the line before.
    f32: sums of D products per score and of up to 2^12 keys, each at most 2^-24 of its terms' magnitudes
    with partial sums over 32 keys: under 2^-15 of sum w |v| for scores of magnitude up to ~2^5."""
    if dtype == "bf16":
        return 2.0 ** -7 * np.abs(out) + (2.0 ** -8 + 2.0 ** -10) * mag + 1e-30
    return 2.0 ** -15 * mag + 1e-30


def _caches(molt, rng, B, maxb, Hkv, D, spare=3, fill=0xFF):
    """Zeroed caches' numpy twins filled with `fill`, and a table of distinct blocks."""
    nb = B * maxb + spare
    tables = rng.permutation(nb)[:B * maxb].reshape(B, maxb).astype(np.int32)
    kc = np.full((nb, Hkv, 17 * D // 2), fill, np.uint8)
    return kc, kc.copy(), tables


def _fill(rng, kc, vc, tables, lens, D, scale=1.0):
    """Positions 0 .. lens[b] - 1 of every sequence: quantised normal rows (whole caches at once)."""
    B, Hkv = len(lens), kc.shape[1]
    n = max(max(lens), 1)
    if not any(lens):
        return
    rows = scale * rng.standard_normal((2, B * n, Hkv, D))
    kvq.write_rows(rows[0], rows[1], kc, vc, tables, [0] * B, n, lens)


def _t(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _rows(rng, T, H, D, dtype):
    x = torch.from_numpy(rng.standard_normal((T, H, D)).astype(np.float32)).to(DT[dtype])
    return x, x.double().numpy()


def _special(x):
    """Groups of x [T, H, D] with values where the format decides: ties, zeros, tiny, huge, infinite, NaN."""
    ties = [0.25, -0.25, 0.75, 1.25, -1.25, 1.75, 2.5, -2.5, 3.5, 5.0, -5.0, 6.0]
    x[0, 0, :12] = torch.tensor(ties)
    x[0, 0, 12:32] = 0.0
    x[0, 0, 32:64] = 0.0
    x[0, -1, 0:32] *= 2.0 ** -126
    x[0, -1, 32:64] *= 2.0 ** 124
    x[0, -1, 33] = 3.3e38
    x[-1, 0, 5] = float("inf")
    x[-1, 0, 40] = float("nan")
    x[-1, -1, 32:64] = 7.0
    x[-1, -1, 33] = -6.96875
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,Hkv,D,lo,hi,ragged", [
    (1, 1, 1, 64, 0, 0, False),
    (3, 5, 4, 128, 0, 100, False),
    (2, 1, 2, 128, 15, 16, False),
    (4, 37, 3, 64, 0, 50, True),
    (2, 130, 2, 128, 3, 9, True),
    (5, 16, 5, 128, 0, 16, True),
])
def test_write_and_read(molt_lib, dtype, B, n, Hkv, D, lo, hi, ragged):
    rng = np.random.default_rng(11)
    ctx = np.linspace(lo, hi, B).astype(np.int32)
    lens = (n - np.arange(B) * n // B).astype(np.int32) if ragged else None
    if ragged:
        lens[-1] = 0                               # a sequence without rows
    kc, vc, tables = _caches(molt_lib, rng, B, (hi + n + 15) // 16 + 1, Hkv, D)
    _fill(rng, kc, vc, tables, ctx.tolist(), D)
    k, v = (_special(_rows(rng, B * n, Hkv, D, dtype)[0]) for _ in range(2))
    gk, gv, gt, gc = _t(kc), _t(vc), _t(tables), _t(ctx)
    molt_lib.kvq_write(k.cuda(), v.cuda(), gk, gv, gt, gc, n, lens=None if lens is None else _t(lens))
    kvq.write_rows(k.double().numpy(), v.double().numpy(), kc, vc, tables, ctx, n, lens)
    assert np.array_equal(host(gk), kc) and np.array_equal(host(gv), vc)
    for start, m, ln in ((np.zeros(B, np.int32), hi + n, None), (ctx, n, lens)):
        for out in ("bf16", "f32"):
            got = molt_lib.kvq_read(gk, gv, gt, _t(start), m, lens=None if ln is None else _t(ln), dtype=DT[out])
            want = kvq.read_rows(kc, vc, tables, start, m, D, ln)
            for g, w in zip(got, want):
                assert g.shape == (B * m, Hkv, D) and g.dtype == DT[out]
                assert np.array_equal(g.double().cpu().numpy(), w, equal_nan=True)


def test_every_bf16_value(molt_lib):
    """Every finite bf16 value, each in a group of its own magnitude, against the oracle's nearest value."""
    bits = np.arange(65536, dtype=np.uint32) << 16
    x = bits.view(np.float32)
    x = x[np.isfinite(x)]
    x = np.sort(np.abs(x)) * np.where(np.arange(x.size) % 2, -1, 1)
    x = np.concatenate([x, np.zeros(-x.size % 128)]).reshape(-1, 1, 128)
    n = x.shape[0]
    rng = np.random.default_rng(2)
    kc, vc, tables = _caches(molt_lib, rng, 1, (n + 15) // 16, 1, 128)
    gk, gv, gt, gz = _t(kc), _t(vc), _t(tables), torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = torch.from_numpy(x.astype(np.float32)).cuda().bfloat16()
    molt_lib.kvq_write(rows, rows.flip(2).contiguous(), gk, gv, gt, gz, n)
    kvq.write_rows(x, x[..., ::-1], kc, vc, tables, [0], n)
    assert np.array_equal(host(gk), kc) and np.array_equal(host(gv), vc)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (64, 3), (129, 5)])
def test_strided_and_unaligned_rows(molt_lib, dtype, pad, shift):
    """Rows that are slices of wider ones, from addresses aligned to an element only."""
    rng = np.random.default_rng(7)
    B, n, Hkv, D = 2, 9, 2, 128
    ctx = np.array([3, 14], np.int32)
    kc, vc, tables = _caches(molt_lib, rng, B, 3, Hkv, D)
    wide = 2 * Hkv * D + pad
    buf = torch.from_numpy(rng.standard_normal(B * n * wide + shift).astype(np.float32)).to(DT[dtype]).cuda()
    view = lambda off: buf[shift + off:].as_strided((B * n, Hkv, D), (wide, D, 1))
    k, v = view(0), view(Hkv * D)
    gk, gv = _t(kc), _t(vc)
    molt_lib.kvq_write(k, v, gk, gv, _t(tables), _t(ctx), n)
    kvq.write_rows(k.double().cpu().numpy(), v.double().cpu().numpy(), kc, vc, tables, ctx, n)
    assert np.array_equal(host(gk), kc) and np.array_equal(host(gv), vc)


def test_rows_without_a_place(molt_lib):
    """Negative positions, positions past the table and block ids outside the pool: nothing is written, the
    rows read as zeros, and no query row sees them."""
    rng = np.random.default_rng(9)
    B, n, Hq, Hkv, D, maxb = 5, 6, 4, 2, 64, 3
    kc, vc, tables = _caches(molt_lib, rng, B, maxb, Hkv, D)
    ctx = np.array([-3, 45, 14, -6, 20], np.int32)
    tables[2, 1], tables[4, 0], tables[4, 1] = -1, len(kc), 2 ** 31 - 1
    _fill(rng, kc, vc, tables, [0, 45, 14, 0, 20], D)
    k, v = (_rows(rng, B * n, Hkv, D, "f32")[0] for _ in range(2))
    gk, gv, gt, gc = _t(kc), _t(vc), _t(tables), _t(ctx)
    molt_lib.kvq_write(k.cuda(), v.cuda(), gk, gv, gt, gc, n)
    kvq.write_rows(k.double().numpy(), v.double().numpy(), kc, vc, tables, ctx, n)
    assert np.array_equal(host(gk), kc) and np.array_equal(host(gv), vc)
    got = molt_lib.kvq_read(gk, gv, gt, gc, n, dtype=torch.float32)
    for g, w in zip(got, kvq.read_rows(kc, vc, tables, ctx, n, D)):
        assert np.array_equal(g.double().cpu().numpy(), w)
    for dtype in ("bf16", "f32"):
        q, q64 = _rows(rng, B * n, Hq, D, dtype)
        out = molt_lib.paged_attention_kvq(q.cuda(), gk, gv, gt, gc, n - 1).double().cpu().numpy()
        want, mag = kvq.attention(q64, kc, vc, tables, ctx, n - 1)
        want, mag = want.reshape(out.shape), mag.reshape(out.shape)
        assert (np.abs(out - want) <= _tol(want, mag, dtype)).all()
        assert (out.reshape(B, n, -1)[0, :3] == 0).all() and (out.reshape(B, n, -1)[3] == 0).all()


def test_context_past_the_table(molt_lib):
    """Contexts past the table's end, up to the largest: the rows see the whole table."""
    rng = np.random.default_rng(10)
    B, k, Hq, Hkv, D, maxb = 3, 2, 4, 2, 128, 4
    kc, vc, tables = _caches(molt_lib, rng, B, maxb, Hkv, D)
    _fill(rng, kc, vc, tables, [64] * B, D)
    ctx = np.array([63, 5000, 2 ** 31 - 1], np.int32)
    for dtype in ("bf16", "f32"):
        q, q64 = _rows(rng, B * (k + 1), Hq, D, dtype)
        out = molt_lib.paged_attention_kvq(q.cuda(), _t(kc), _t(vc), _t(tables), _t(ctx), k).double().cpu().numpy()
        want, mag = (x.reshape(out.shape) for x in kvq.attention(q64, kc, vc, tables, np.minimum(ctx, 63), k))
        assert (np.abs(out - want) <= _tol(want, mag, dtype)).all()
    rows = _rows(rng, B * 2, Hkv, D, "f32")[0].cuda()
    gk, gv = _t(kc), _t(vc)
    molt_lib.kvq_write(rows, rows, gk, gv, _t(tables), _t(ctx), 2)     # row 0 of the first sequence only
    kvq.write_rows(rows.double().cpu().numpy(), rows.double().cpu().numpy(), kc, vc, tables, ctx.astype(np.int64), 2)
    assert np.array_equal(host(gk), kc) and np.array_equal(host(gv), vc)


CASES = [
    # B, k, Hq, Hkv, D, lo, hi
    (1, 0, 1, 1, 128, 0, 0),            # one key
    (1, 0, 32, 4, 128, 700, 700),
    (4, 0, 32, 4, 128, 0, 40),          # plain decode, empty contexts
    (3, 4, 32, 4, 128, 1, 1500),        # 40 rows, ragged, splits
    (2, 8, 32, 4, 128, 300, 1100),      # 72 rows: two row groups
    (4, 3, 4, 4, 64, 64, 128),          # the tiny decoder
    (2, 2, 14, 2, 64, 15, 500),         # 7 query heads per kv head
    (3, 1, 5, 1, 128, 30, 33),
    (1, 2, 128, 1, 64, 90, 90),         # 384 rows of one kv head
    (2, 40, 8, 2, 128, 0, 300),         # windows: 164 rows
    (1, 256, 8, 2, 64, 100, 100),       # a window of 257 positions
    (1, 15, 8, 8, 128, 2500, 2500),     # 16 positions of one head
    (33, 1, 2, 1, 64, 0, 129),
    (300, 0, 2, 1, 64, 0, 20),          # more sequences than a cut looks at
    (2, 7, 16, 1, 128, 1000, 2600),     # 128 rows, three row groups with a smaller last, cut
    (5, 2, 4, 4, 128, 0, 1900),         # uneven lengths, cut
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,k,Hq,Hkv,D,lo,hi", CASES)
def test_attention(molt_lib, dtype, B, k, Hq, Hkv, D, lo, hi):
    """Slots past each sequence's last position, and every block of no sequence, hold NaN."""
    print(f"case B={B} k={k} Hq={Hq} Hkv={Hkv} D={D} ctx=[{lo},{hi}] {dtype}", flush=True)
    rng = np.random.default_rng(13)
    ctx = np.linspace(lo, hi, B).astype(np.int32)
    kc, vc, tables = _caches(molt_lib, rng, B, (hi + k + 1 + 15) // 16 + 2, Hkv, D)
    _fill(rng, kc, vc, tables, (ctx + k + 1).tolist(), D)
    q, q64 = _rows(rng, B * (k + 1), Hq, D, dtype)
    args = (_t(kc), _t(vc), _t(tables), _t(ctx), k)
    got = molt_lib.paged_attention_kvq(q.cuda(), *args)
    again = molt_lib.paged_attention_kvq(q.cuda(), *args)
    assert torch.equal(got, again)
    out = got.double().cpu().numpy()
    want, mag = (x.reshape(out.shape) for x in kvq.attention(q64, kc, vc, tables, ctx, k))
    err = np.abs(out - want)
    print("max error / tolerance", (err / _tol(want, mag, dtype)).max(), "rms", np.sqrt((err ** 2).sum() / (want ** 2).sum()))
    assert (err <= _tol(want, mag, dtype)).all()


def _dense_check(molt, rng, ctx, k, Hq, Hkv, D, dtype):
    """Sequences of random rows written and attended over, against a dense softmax of the rows read back. Blocks and
    slots of no row hold NaN."""
    B, n = len(ctx), k + 1
    maxb = (max(ctx) + n + 15) // 16 + 1
    tables = _t(rng.permutation(B * maxb + 3)[:B * maxb].reshape(B, maxb).astype(np.int32))
    gk = torch.full((B * maxb + 3, Hkv, 17 * D // 2), 0xFF, dtype=torch.uint8, device="cuda")
    gv = gk.clone()
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    K, V = [], []
    for b in range(B):
        L, row = int(ctx[b]) + n, tables[b:b + 1]
        molt.kvq_write(*(torch.from_numpy(rng.standard_normal((L, Hkv, D), np.float32)).cuda() for _ in range(2)),
                       gk, gv, row, zero, L)
        for x, to in zip(molt.kvq_read(gk, gv, row, zero, L, dtype=torch.float32), (K, V)):
            to.append(x.double().cpu().numpy())
    q, q64 = _rows(rng, B * n, Hq, D, dtype)
    out = molt.paged_attention_kvq(q.cuda(), gk, gv, tables, _t(np.array(ctx, np.int32)), k).double().cpu().numpy()
    out = out.reshape(B, n, Hkv, Hq // Hkv, D)
    q64 = q64.reshape(out.shape)
    for b in range(B):
        score = np.einsum("jhgd,phd->jhgp", q64[b], K[b]) / np.sqrt(D)
        seen = np.arange(len(K[b]))[None] <= ctx[b] + np.arange(n)[:, None]
        w = np.where(seen[:, None, None], np.exp(score - score.max(axis=-1, keepdims=True)), 0.0)
        w /= w.sum(axis=-1, keepdims=True)
        want, mag = (np.einsum("jhgp,phd->jhgd", w, x) for x in (V[b], np.abs(V[b])))
        assert (np.abs(out[b] - want) <= _tol(want, mag, dtype)).all()


@pytest.mark.parametrize("lo,hi", [(0, 7), (33, 60), (150, 280), (2500, 3000)])
@pytest.mark.parametrize("Hq,k", [(4, 0), (10, 3), (8, 9), (24, 4), (30, 4)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_every_size(molt_lib, dtype, D, Hq, k, lo, hi):
    """2, 20, 40, 60 and 75 rows of a kv head over short, middling and long key ranges and ones that are cut."""
    _dense_check(molt_lib, np.random.default_rng(41), [lo, (lo + hi) // 2, hi], k, Hq, 2, D, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_two_long_sequences_among_many(molt_lib, dtype, D):
    """70 sequences of which two are cut: few parts for most, joined by a thread each."""
    ctx = [i % 90 for i in range(70)]
    ctx[13] = ctx[69] = 3900
    _dense_check(molt_lib, np.random.default_rng(43), ctx, 1, 6, 2, D, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_large_scores(molt_lib, dtype, D):
    """Scores far apart and far from zero (magnitudes up to ~1e8): the largest key of a row takes all."""
    rng = np.random.default_rng(17)
    B, k, Hq, Hkv = 2, 2, 6, 2
    ctx = np.array([40, 77], np.int32)
    kc, vc, tables = _caches(molt_lib, rng, B, 6, Hkv, D)
    _fill(rng, kc, vc, tables, (ctx + k + 1).tolist(), D, scale=64.0)
    q, _ = _rows(rng, B * (k + 1), Hq, D, dtype)
    q = q * 2.0 ** 20 * torch.where(torch.arange(Hq) % 2 == 0, 1.0, -1.0).view(1, Hq, 1).to(q.dtype)
    out = molt_lib.paged_attention_kvq(q.cuda(), _t(kc), _t(vc), _t(tables), _t(ctx), k).double().cpu().numpy()
    want, _ = kvq.attention(q.double().numpy(), kc, vc, tables, ctx, k)
    want = want.reshape(out.shape)
    assert (np.abs(out - want) <= 2.0 ** -8 * np.abs(want) + 1e-30).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where", ["key", "value"])
def test_nan_reaches_the_rows_that_see_it(molt_lib, dtype, D, where):
    """A NaN group of one position of the window (and of one cached position of another sequence): the rows
    before it are as without it, the rows from it on are NaN, in its group's dims only where it is a value."""
    rng = np.random.default_rng(19)
    B, k, Hq, Hkv = 2, 9, 4, 2
    ctx = np.array([25, 70], np.int32)
    kc, vc, tables = _caches(molt_lib, rng, B, 6, Hkv, D)
    _fill(rng, kc, vc, tables, (ctx + k + 1).tolist(), D)
    q, q64 = _rows(rng, B * (k + 1), Hq, D, dtype)
    clean, mag = kvq.attention(q64, kc, vc, tables, ctx, k)
    group, kv_head, first = D // 32 - 1, 1, {0: ctx[0] + 4, 1: 33}
    for b, pos in first.items():
        blk, slot = kvq.place(tables[b], int(pos), len(kc))
        cache = kc if where == "key" else vc
        cache[blk, kv_head, kvq.offsets(slot, D, where == "value")[1][group]] = 255
    out = molt_lib.paged_attention_kvq(q.cuda(), _t(kc), _t(vc), _t(tables), _t(ctx), k)
    out = out.double().cpu().numpy().reshape(B, k + 1, Hq, D)
    clean, mag = clean.reshape(out.shape), mag.reshape(out.shape)
    for b in range(B):
        for j in range(k + 1):
            hit = ctx[b] + j >= first[b]
            for h in range(Hq):
                dims = np.zeros(D, bool)
                if hit and h // (Hq // Hkv) == kv_head:
                    dims[:] = where == "key"
                    dims[32 * group:32 * group + 32] = True
                assert np.isnan(out[b, j, h][dims]).all()
                err = np.abs(out[b, j, h] - clean[b, j, h])[~dims]
                assert (err <= _tol(clean[b, j, h], mag[b, j, h], dtype)[~dims]).all()


def test_infinite_query(molt_lib):
    """An infinite query element gives NaN in its row and head, and nothing in the others."""
    rng = np.random.default_rng(21)
    kc, vc, tables = _caches(molt_lib, rng, 1, 4, 1, 128)
    _fill(rng, kc, vc, tables, [40], 128)
    ctx = _t(np.array([38], np.int32))
    q, _ = _rows(rng, 2, 3, 128, "bf16")
    base = molt_lib.paged_attention_kvq(q.cuda(), _t(kc), _t(vc), _t(tables), ctx, 1).view(2, 3, 128)
    q[1, 2, 77] = float("inf")
    out = molt_lib.paged_attention_kvq(q.cuda(), _t(kc), _t(vc), _t(tables), ctx, 1).view(2, 3, 128)
    assert torch.isnan(out[1, 2]).all()
    keep = torch.ones(2, 3, dtype=torch.bool)
    keep[1, 2] = False
    assert torch.equal(out[keep], base[keep])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_query_of_a_cut_sequence(molt_lib, dtype):
    """A row of NaN scores has no maximum in any part of its keys: the parts joined are NaN, not zeros."""
    rng = np.random.default_rng(31)
    kc, vc, tables = _caches(molt_lib, rng, 1, 200, 1, 128)
    _fill(rng, kc, vc, tables, [902], 128)
    args = (_t(kc), _t(vc), _t(tables), _t(np.array([900], np.int32)), 1)
    assert molt_lib.paged_attention_kvq_workspace_size(1, 1, 3, 1, 128, 200) > 0
    q, _ = _rows(rng, 2, 3, 128, dtype)
    base = molt_lib.paged_attention_kvq(q.cuda(), *args).view(2, 3, 128)
    q[0, 1, 3] = float("nan")
    q[1, 2, 77] = float("inf")
    out = molt_lib.paged_attention_kvq(q.cuda(), *args).view(2, 3, 128)
    bad = torch.zeros(2, 3, dtype=torch.bool)
    bad[0, 1] = bad[1, 2] = True
    assert torch.isnan(out[0, 1]).all() and torch.isnan(out[1, 2]).all()
    assert torch.equal(out[~bad], base[~bad])


@pytest.mark.parametrize("pairs", [24, 47, 1535])
def test_equal_lengths_with_few_spare_slots(molt_lib, pairs):
    """200 sequences of one length (and table, and query), which the workgroups that fit cannot all cut in
    two: none is lost. 1535: the hardware reciprocal is above 1 / 1535."""
    rng = np.random.default_rng(33)
    B, Hq, Hkv, D = 200, 2, 2, 128
    n, maxb = 32 * pairs, 2 * pairs + 10
    gk, gv = molt_lib.kvq_cache(maxb, Hkv, D)
    table = _t(rng.permutation(maxb).astype(np.int32)[None])
    rows = [torch.from_numpy(rng.standard_normal((n, Hkv, D), np.float32)).cuda() for _ in range(2)]
    start = torch.zeros(1, dtype=torch.int32, device="cuda")
    molt_lib.kvq_write(*rows, gk, gv, table, start, n)
    k, v = (x.double().cpu().numpy() for x in molt_lib.kvq_read(gk, gv, table, start, n, dtype=torch.float32))
    q, q64 = _rows(rng, 1, Hq, D, "bf16")
    out = molt_lib.paged_attention_kvq(q.cuda().repeat(B, 1, 1), gk, gv, table.repeat(B, 1), start.repeat(B) + n - 1, 0)
    assert torch.equal(out, out[:1].expand_as(out))
    score = np.einsum("hd,nhd->hn", q64[0], k) / np.sqrt(D)
    w = np.exp(score - score.max(axis=1, keepdims=True))
    w /= w.sum(axis=1, keepdims=True)
    want, mag = (np.einsum("hn,nhd->hd", w, x).reshape(1, -1) for x in (v, np.abs(v)))
    assert (np.abs(out[:1].double().cpu().numpy() - want) <= _tol(want, mag, "bf16")).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padded_batch_of_cut_sequences(molt_lib, dtype):
    """Sequences that sit the step out (no row sees a key) beside one long enough to be cut; a workspace of
    just the size asked for, from an odd address, the bytes around it as they were; a smaller one."""
    rng = np.random.default_rng(35)
    B, k, Hq, Hkv, D, maxb = 4, 4, 8, 2, 64, 130
    ctx = np.array([-(k + 1), 2000, -2 ** 31, -2], np.int32)
    kc, vc, tables = _caches(molt_lib, rng, B, maxb, Hkv, D)
    _fill(rng, kc, vc, tables, [0, 2000 + k + 1, 0, k - 1], D)
    q, q64 = _rows(rng, B * (k + 1), Hq, D, dtype)
    args = (q.cuda(), _t(kc), _t(vc), _t(tables), _t(ctx), k)
    size = molt_lib.paged_attention_kvq_workspace_size(B, k, Hq, Hkv, D, maxb)
    assert size > 0
    buf = torch.full((size + 512,), 0xAB, dtype=torch.uint8, device="cuda")
    got = molt_lib.paged_attention_kvq(*args, workspace=buf[255:255 + size])
    assert (buf[:255] == 0xAB).all() and (buf[255 + size:] == 0xAB).all()
    assert torch.equal(got, molt_lib.paged_attention_kvq(*args))
    assert torch.equal(got, molt_lib.paged_attention_kvq(*args, workspace=buf[:16]))
    out = got.double().cpu().numpy()
    want, mag = (x.reshape(out.shape) for x in kvq.attention(q64, kc, vc, tables, ctx.astype(np.int64), k))
    assert (np.abs(out - want) <= _tol(want, mag, dtype)).all()
    assert (out.reshape(B, k + 1, -1)[[0, 2]] == 0).all()


def test_lens_of_any_value(molt_lib):
    """Negative lens count as 0, lens above n as n, in blocks that begin before, with and behind row 0."""
    rng = np.random.default_rng(37)
    B, n, Hkv, D = 6, 40, 2, 128
    ctx = np.array([0, 7, 7, 7, 16, 3], np.int32)
    lens = np.array([-2 ** 31, -2 ** 31, 2 ** 31 - 1, 41, -1, 2 ** 31 - 1], np.int32)
    kc, vc, tables = _caches(molt_lib, rng, B, 4, Hkv, D)
    k, v = (_rows(rng, B * n, Hkv, D, "bf16")[0] for _ in range(2))
    gk, gv, gt, gc = _t(kc), _t(vc), _t(tables), _t(ctx)
    molt_lib.kvq_write(k.cuda(), v.cuda(), gk, gv, gt, gc, n, lens=_t(lens))
    kvq.write_rows(k.double().numpy(), v.double().numpy(), kc, vc, tables, ctx, n, lens)
    assert np.array_equal(host(gk), kc) and np.array_equal(host(gv), vc)
    got = molt_lib.kvq_read(gk, gv, gt, gc, n, lens=_t(lens))
    for g, w in zip(got, kvq.read_rows(kc, vc, tables, ctx, n, D, lens)):
        assert np.array_equal(g.double().cpu().numpy(), w, equal_nan=True)


def test_zeroed_cache(molt_lib):
    """Slots of kvq_cache that were never written are zeros to the calls that see them."""
    for D in (64, 128):
        kc, vc = molt_lib.kvq_cache(60, 2, D)
        tables = torch.arange(60, dtype=torch.int32, device="cuda").view(1, 60)
        ctx = torch.tensor([900], dtype=torch.int32, device="cuda")
        assert all((t == 0).all() for t in molt_lib.kvq_read(kc, vc, tables, ctx * 0, 900))
        for dt in DT.values():
            assert (molt_lib.paged_attention_kvq(torch.ones(2, 4, D, dtype=dt, device="cuda"), kc, vc, tables, ctx, 1) == 0).all()


def test_two_streams_at_once(molt_lib):
    """Calls of other sizes on two streams beside each other, each with a workspace of its own."""
    rng = np.random.default_rng(39)
    runs = []
    for B, k, Hq, Hkv, D, L in ((2, 1, 16, 2, 128, 2000), (3, 3, 8, 4, 64, 1500)):
        kc, vc, tables = _caches(molt_lib, rng, B, 130, Hkv, D)
        ctx = np.full(B, L, np.int32)
        _fill(rng, kc, vc, tables, [L + k + 1] * B, D)
        args = (_rows(rng, B * (k + 1), Hq, D, "bf16")[0].cuda(), _t(kc), _t(vc), _t(tables), _t(ctx), k)
        runs.append((args, molt_lib.paged_attention_kvq(*args), torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(5):
        for i, (args, _, stream) in enumerate(runs):
            with torch.cuda.stream(stream):
                outs[i].append(molt_lib.paged_attention_kvq(*args))
    torch.cuda.synchronize()
    for (_, want, _), got in zip(runs, outs):
        assert all(torch.equal(want, g) for g in got)


def test_unaligned_rows_of_queries(molt_lib):
    rng = np.random.default_rng(23)
    for dtype in ("bf16", "f32"):
        kc, vc, tables = _caches(molt_lib, rng, 2, 5, 2, 128)
        ctx = np.array([33, 60], np.int32)
        _fill(rng, kc, vc, tables, (ctx + 3).tolist(), 128)
        q, _ = _rows(rng, 6, 6, 128, dtype)
        args = (_t(kc), _t(vc), _t(tables), _t(ctx), 2)
        a = molt_lib.paged_attention_kvq(q.cuda(), *args)
        buf = torch.empty(q.numel() + 1, dtype=q.dtype, device="cuda")
        b = molt_lib.paged_attention_kvq(buf[1:].view(q.shape).copy_(q), *args)
        assert torch.equal(a, b)


def test_offsets_past_32_bits(molt_lib):
    """Blocks that start past 2^31 (and 2^32) bytes of the cache."""
    rng = np.random.default_rng(25)
    Hkv, D, nb = 8, 128, 500_000                       # 4.35 GB per cache
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB of device memory")
    gk, gv = molt_lib.kvq_cache(nb, Hkv, D)
    tables = np.array([[nb - 1, 3, 250_000, nb - 2, 495_000]], np.int32)
    small = np.arange(5, dtype=np.int32)[None]
    kc = np.zeros((5, Hkv, 17 * D // 2), np.uint8)
    vc = kc.copy()
    k, v = (_rows(rng, 70, Hkv, D, "bf16")[0] for _ in range(2))
    start = np.zeros(1, np.int32)
    molt_lib.kvq_write(k.cuda(), v.cuda(), gk, gv, _t(tables), _t(start), 70)
    kvq.write_rows(k.double().numpy(), v.double().numpy(), kc, vc, small, start, 70)
    ids = torch.from_numpy(tables[0]).long().cuda()
    assert np.array_equal(host(gk[ids]), kc) and np.array_equal(host(gv[ids]), vc)
    got = molt_lib.kvq_read(gk, gv, _t(tables), _t(start), 70, dtype=torch.float32)
    for g, w in zip(got, kvq.read_rows(kc, vc, small, start, 70, D)):
        assert np.array_equal(g.double().cpu().numpy(), w)
    q, q64 = _rows(rng, 3, 16, D, "bf16")
    ctx = np.array([67], np.int32)
    out = molt_lib.paged_attention_kvq(q.cuda(), gk, gv, _t(tables), _t(ctx), 2).double().cpu().numpy()
    want, mag = (x.reshape(out.shape) for x in kvq.attention(q64, kc, vc, small, ctx, 2))
    assert (np.abs(out - want) <= _tol(want, mag, "bf16")).all()


def _session(molt, steps, q, k, v, gk, gv, gt, ctx, n):
    outs = []
    for i in range(steps):
        molt.kvq_write(k[i], v[i], gk, gv, gt, ctx, n)
        outs.append(molt.paged_attention_kvq(q[i], gk, gv, gt, ctx, n - 1))
        ctx += n
    return outs


def test_a_session(molt_lib):
    """Decode steps as a serving loop makes them: write the step's rows, attend, advance; then everything
    read back. Each step against the oracle, which does the same; the same bits on a stream of its own."""
    rng = np.random.default_rng(27)
    B, n, Hq, Hkv, D, steps = 3, 3, 8, 2, 128, 6
    kc, vc, tables = _caches(molt_lib, rng, B, 5, Hkv, D)
    ctx = np.array([0, 11, 40], np.int32)
    _fill(rng, kc, vc, tables, ctx.tolist(), D)
    q, k, v = ([_rows(rng, B * n, H, D, "bf16")[0] for _ in range(steps)] for H in (Hq, Hkv, Hkv))
    dq, dk, dv = ([x.cuda() for x in t] for t in (q, k, v))
    gk, gv, gt, gc = _t(kc), _t(vc), _t(tables), _t(ctx)
    side = torch.cuda.Stream()
    gk2, gv2, gc2 = gk.clone(), gv.clone(), gc.clone()
    side.wait_stream(torch.cuda.current_stream())
    outs = _session(molt_lib, steps, dq, dk, dv, gk, gv, gt, gc, n)
    with torch.cuda.stream(side):
        outs2 = _session(molt_lib, steps, dq, dk, dv, gk2, gv2, gt, gc2, n)
    torch.cuda.synchronize()
    for i in range(steps):
        kvq.write_rows(k[i].double().numpy(), v[i].double().numpy(), kc, vc, tables, ctx, n)
        out = outs[i].double().cpu().numpy()
        want, mag = (x.reshape(out.shape) for x in kvq.attention(q[i].double().numpy(), kc, vc, tables, ctx, n - 1))
        assert (np.abs(out - want) <= _tol(want, mag, "bf16")).all()
        assert torch.equal(outs[i], outs2[i])
        ctx = ctx + n
    assert np.array_equal(host(gk), kc) and np.array_equal(host(gv), vc)
    start = np.zeros(B, np.int32)
    got = molt_lib.kvq_read(gk, gv, gt, _t(start), 64, lens=gc)
    for g, w in zip(got, kvq.read_rows(kc, vc, tables, start, 64, D, ctx)):
        assert np.array_equal(g.double().cpu().numpy(), w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graph_replays(molt_lib, dtype):
    """A captured step (write, attend with splits, read back) replayed with other inputs between eager work."""
    rng = np.random.default_rng(29)
    B, n, Hq, Hkv, D = 2, 2, 8, 2, 128
    kc, vc, tables = _caches(molt_lib, rng, B, 200, Hkv, D)
    ctx = np.array([200, 900], np.int32)
    _fill(rng, kc, vc, tables, ctx.tolist(), D)
    gk, gv, gt, gc = _t(kc), _t(vc), _t(tables), _t(ctx)
    draw = lambda H: _rows(rng, B * n, H, D, dtype)[0].cuda()
    q, k, v = draw(Hq), draw(Hkv), draw(Hkv)
    ws = torch.empty(molt_lib.paged_attention_kvq_workspace_size(B, n - 1, Hq, Hkv, D, 200), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0

    def step(gk, gv, ws=None):
        molt_lib.kvq_write(k, v, gk, gv, gt, gc, n)
        out = molt_lib.paged_attention_kvq(q, gk, gv, gt, gc, n - 1, workspace=ws)
        return (out,) + molt_lib.kvq_read(gk, gv, gt, gc, n, dtype=DT[dtype])

    step(gk, gv, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(gk, gv, ws)
    for _ in range(4):
        for t, H in ((q, Hq), (k, Hkv), (v, Hkv)):
            t.copy_(draw(H))
        gc += n
        want = step(gk.clone(), gv.clone())
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)


def test_refusals(molt_lib):
    B, n, Hq, Hkv, D, maxb = 2, 2, 4, 2, 128, 3
    kc, vc = molt_lib.kvq_cache(6, Hkv, D)
    tables = torch.arange(6, dtype=torch.int32, device="cuda").view(B, maxb)
    ctx = torch.zeros(B, dtype=torch.int32, device="cuda")
    rows = torch.zeros(B * n, Hkv, D, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(B * n, Hq, D, dtype=torch.bfloat16, device="cuda")

    def refused(word, call):
        with pytest.raises(molt_lib.MoltError, match=word):
            call()

    W = lambda k=rows, v=rows, kc=kc, vc=vc, t=tables, c=ctx, n=n, **kw: molt_lib.kvq_write(k, v, kc, vc, t, c, n, **kw)
    refused("dtype", lambda: W(k=rows.half()))
    refused("dtype", lambda: W(v=rows.float()))
    refused("shape", lambda: W(n=3))
    refused("shape", lambda: W(k=rows[:, :, :64]))
    refused("heads", lambda: W(k=rows.transpose(1, 2).contiguous().transpose(1, 2)))
    refused("heads", lambda: W(v=rows[:1].expand(B * n, Hkv, D)))
    refused("GPU", lambda: W(k=rows.cpu()))
    refused("dtype", lambda: W(kc=kc.view(torch.int8)))
    refused("shape", lambda: W(vc=vc[:5]))
    refused("shape", lambda: W(kc=kc[:, :, :1000].contiguous()))
    refused("contiguous", lambda: W(t=tables.t().contiguous().t()))
    refused("block_tables", lambda: W(t=tables[:1].contiguous()))
    refused("dtype", lambda: W(c=ctx.long()))
    refused("lens", lambda: W(lens=ctx[:1]))
    flat = torch.empty(kc.numel() + 8, dtype=torch.uint8, device="cuda")
    refused("16 bytes", lambda: W(kc=flat[8:].view(kc.shape)))
    odd = torch.zeros(6, Hkv, 17 * 96 // 2, dtype=torch.uint8, device="cuda")
    refused("head_dim", lambda: W(k=rows[..., :96].contiguous(), v=rows[..., :96].contiguous(), kc=odd, vc=odd))
    R = lambda kc=kc, vc=vc, t=tables, c=ctx, n=n, **kw: molt_lib.kvq_read(kc, vc, t, c, n, **kw)
    refused("dtype", lambda: R(dtype=torch.float16))
    refused("n = 0", lambda: R(n=0))
    refused("16 bytes", lambda: R(vc=flat[8:].view(kc.shape)))
    A = lambda q=q, kc=kc, vc=vc, t=tables, c=ctx, k=n - 1, **kw: molt_lib.paged_attention_kvq(q, kc, vc, t, c, k, **kw)
    refused("dtype", lambda: A(q=q.half()))
    refused("multiple", lambda: A(q=q[:, :3].contiguous()))
    refused("shape", lambda: A(k=3))
    flat_ws = torch.empty(1, dtype=torch.uint8, device="cuda")
    refused("workspace", lambda: A(workspace=flat_ws.expand(1 << 20)))
    refused("workspace", lambda: A(workspace=flat_ws.cpu()))
    refused("n = -1", lambda: R(n=-1))
    refused("k = -1", lambda: A(q=q[:0], k=-1))
    refused("contiguous", lambda: A(q=q.transpose(0, 1).contiguous().transpose(0, 1)))

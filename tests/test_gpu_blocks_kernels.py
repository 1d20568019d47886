"""Sparse attention over listed blocks: the kernels that calls of certain sizes take, each on what decides in it.
select_blocks in two launches, by tables and numbers of lists, with scores that differ; kv_write of many rows with slots of
all kinds and rows at any element; attention's f32 weights within a bound of their own."""
import numpy as np
import pytest
import torch

from oracle import blocks as ob

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _i32(a):
    return torch.as_tensor(np.asarray(a, np.int32), device="cuda")


def _val(t):
    return t.double().cpu().numpy()


# ---------------------------------------------------------------- selection in two launches

def _scores(rows, bounds):
    """Scores of query rows [G, D] for blocks of records [nb, 2 D + 16], as ob.score gives them one by one."""
    rec = bounds.view(np.int8).astype(np.int64)
    D = (rec.shape[1] - ob.BLOCK) // 2
    hi, lo, e = rec[:, :D], rec[:, D:2 * D], rec[:, 2 * D]
    best = np.full(len(rec), -np.inf)
    for q in rows:
        f = ob.exponent(np.abs(q).max())
        c = np.rint(np.ldexp(q, -f)).astype(np.int64)
        s = np.maximum(c * hi, c * lo).sum(1).astype(float)
        best = np.maximum(best, np.ldexp(s, np.clip(e + f, -100, 100)))
    return best


def _picked(scores, seen, N, first, last):
    s = scores[:seen].copy()
    s[:first], s[max(0, seen - last):] = np.inf, np.inf
    out = np.full(N, -1)
    best = np.sort(np.lexsort((np.arange(seen), -s))[:N])
    out[:len(best)] = best
    return out


@pytest.mark.parametrize("B,n,G,H,maxb,N,ties", [
    (16, 5, 1, 4, 600, 64, False), (16, 5, 1, 4, 2048, 128, False), (16, 5, 3, 4, 449, 24, True), (64, 2, 2, 2, 1700, 33, True),
    (9, 7, 1, 5, 2000, 1500, False),                                     # many lists: 2 wavefronts each
    (1, 2, 1, 2, 9000, 33, False), (2, 1, 3, 2, 17000, 100, False), (1, 1, 1, 3, 8193, 5, False), (1, 2, 1, 2, 17000, 4000, False),
    (1, 3, 2, 2, 9000, 40, True),                                        # tables past 8192 blocks: keys from memory
    (90, 1, 1, 3, 8300, 17, False),                                      # many lists of these
    (1, 5, 2, 4, 2100, 33, False), (2, 3, 1, 2, 4600, 64, True), (1, 2, 1, 2, 8192, 65, False)])   # few lists
def test_select_in_two_launches(molt_lib, B, n, G, H, maxb, N, ties):
    """Scores of 64 dims, nearly all of them different (or a few hundred values, many times each) and close together at the
    list's border, and rows that see all, some and few of the blocks."""
    assert molt_lib.select_blocks_workspace_size(B, n - 1, G * H, H, 64, maxb) > 0
    rng = np.random.default_rng(maxb + N)
    D = 64
    rec = np.zeros((maxb, H, 2 * D + 16), np.int8)
    if ties:
        rec[..., 0] = rng.integers(-127, 128, (maxb, H))
        rec[..., D] = rec[..., 0]
    else:
        a = rng.integers(-127, 128, (2, maxb, H, D))
        rec[..., :D], rec[..., D:2 * D] = a.max(0), a.min(0)
        rec[..., 2 * D] = rng.integers(-1, 2, (maxb, H))
    bounds = rec.view(np.uint8)
    tables = np.stack([rng.permutation(maxb) for _ in range(B)]).astype(np.int32)
    ctx = rng.integers(0, 16 * maxb - n + 1, B)
    ctx[0], ctx[-1] = 16 * maxb - n, 16 * maxb - 1 - 16 * (maxb // 3) if B > 1 else 16 * maxb - n
    q = torch.from_numpy(rng.standard_normal((B * n, G * H, D)).astype(np.float32))
    first, last = min(2, N - 2), 2
    got = molt_lib.select_blocks(q.cuda(), torch.from_numpy(bounds).cuda(), _i32(tables), _i32(ctx), n - 1, N, n_first=first,
                                 n_last=last).cpu().numpy()
    rows = _val(q)
    for t in range(0, B * n, max(1, B * n * H * maxb // 400000)):        # all, or some of the lists
        b = t // n
        seen = min((int(ctx[b]) + t % n) // 16 + 1, maxb)
        for h in range(H):
            s = _scores(rows[t, h * G:(h + 1) * G], bounds[tables[b], h])
            if t == 0 and not ties:
                assert len(np.unique(s)) > maxb // 2
            assert np.array_equal(got[t, h], _picked(s, seen, N, first, last)), (t, h)


# ---------------------------------------------------------------- many rows by slot

def _hard_slots(rng, nb, T):
    """T slots and the blocks that hold slots of more than one row: runs up and down, from any token, broken by holes and by
    numbers outside the cache, and slots named again, close by and far away."""
    order, at, slots, again = rng.permutation(nb), 0, [], set()
    outside = [-1, 16 * nb, 16 * nb + 5, -2 ** 31, 2 ** 31 - 1, -17]
    while len(slots) < T:
        base, kind = int(order[at % nb]) * 16, int(rng.integers(7))
        at += 1
        assert at < nb
        a, b = sorted(int(x) for x in rng.integers(0, 16, 2))
        run = [base + t for t in range(a, b + 1)]
        if kind == 0:
            run = [base + t for t in range(16)]
        elif kind == 1:
            run = run[::-1]
        elif kind == 2:
            run.insert(int(rng.integers(len(run) + 1)), outside[int(rng.integers(len(outside)))])
        elif kind == 3:
            run = [outside[int(x)] for x in rng.integers(0, len(outside), int(rng.integers(1, 20)))]
        elif kind == 4:                                                  # the same slots once more
            run += run[int(rng.integers(len(run))):]
            again.add(base // 16)
        elif kind == 5:                                                  # one slot many times
            run = [base + a] * int(rng.integers(2, 18))
            again.add(base // 16)
        slots += run
    slots = slots[:T]
    far = [s for s in slots[:T // 3] if 0 <= s < 16 * nb][::9][:40]      # and some of the first rows' at the end
    slots[T - len(far):] = far
    again |= {s // 16 for s in far}
    return np.array(slots, np.int64), again


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,D,T,odd", [(4, 128, 2500, False), (4, 128, 2501, True), (3, 64, 4100, True), (1, 64, 9001, True),
                                       (1, 128, 4500, False)])
def test_write_of_many_rows_with_slots_of_all_kinds(molt_lib, dtype, H, D, T, odd):
    assert T * -(-H * D // 128) > 4096                                   # past the kernel of few rows
    rng = np.random.default_rng(T)
    nb = T // 3
    slots, again = _hard_slots(rng, nb, T)
    row = H * D + (83 if odd else 0)
    flat = torch.from_numpy(rng.standard_normal(2 * T * row + 9).astype(np.float32)).to(DT[dtype]).cuda()
    k = torch.as_strided(flat, (T, H, D), (row, D, 1), 1 if odd else 0)
    v = torch.as_strided(flat, (T, H, D), (row, D, 1), T * row + (7 if odd else 0))
    kc = torch.from_numpy(rng.standard_normal((nb, H, 16, D)).astype(np.float32)).to(DT[dtype]).cuda()
    vc = torch.from_numpy(rng.standard_normal((nb, H, D, 16)).astype(np.float32)).to(DT[dtype]).cuda()
    wk, wv, hk, hv = _val(kc), _val(vc), _val(k), _val(v)
    molt_lib.kv_write(k, v, kc, vc, _i32(slots))
    ob.write_rows(hk, hv, wk, wv, slots)
    gk, gv = _val(kc), _val(vc)
    only = np.array([block not in again for block in range(nb)])
    assert np.array_equal(gk[only], wk[only]) and np.array_equal(gv[only], wv[only])
    named = {}
    for r, s in enumerate(slots):
        named.setdefault(int(s), []).append(r)
    for block in again:
        for t in range(16):
            rows = named.get(16 * block + t, [])
            for got, want, src in ((gk[block, :, t], wk[block, :, t], hk), (gv[block, :, :, t], wv[block, :, :, t], hv)):
                if len(rows) < 2:
                    assert np.array_equal(got, want)
                else:                                                    # of rows with the same slot one stays
                    assert (got[None] == src[rows]).any(0).all(), (block, t)


# ---------------------------------------------------------------- f32 weights

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,lists_cut", [(8, False), (40, True)])
def test_weights_of_f32_calls_have_24_bits(molt_lib, D, N, lists_cut):
    """Values that are 1 in a dim of their key's own and 0 else, so that an output is a weight over the sum of weights, and its
    relative error theirs. Queries and keys are multiples of 2^-6, so that scores are exact; they are within 2 / c of each other,
    c = log2(e) / sqrt(D). In steps of 2^-24: an exponent (s - m) c of up to 2 is off by 3 for c (two constants and
    their quotient) and 1 for the product, times 2 ln 2 in the power, under 6, and the power itself by 2: a weight by 8. Its
    wavefront's factor, and its part's, by 8 each and 1 for the product: 26 at most. The sum of weights as much, and
    its own additions: 4 a block and lane, at most 3 blocks, 2 over lanes, 2 (product and sum) for each of 8 wavefronts,
    2 for each of at most 2 parts: 34. The reciprocal, its product and the output's rounding 1 each. Together
    26 + 26 + 34 + 3 = 89. Weights of 16 bits, as bf16 calls have, would be past it."""
    assert (molt_lib.paged_attention_blocks_workspace_size(1, 1, 6, 2, D, N) > 0) == lists_cut
    rng = np.random.default_rng(N + D)
    H, G, n, maxb = 2, 3, 2, 50
    q = np.zeros((n, H * G, D), np.float32)
    q[:, :, :8] = rng.integers(-64, 65, (n, H * G, 8)) / 64.0
    k = rng.integers(-1, 2, (maxb, H, 16, D)).astype(np.float32)
    k[:, :, :, :8] = rng.choice([0, 1], (maxb, H, 16, 8)) * rng.choice([-1, 1], (maxb, H, 1, 8))
    v = np.zeros((maxb, H, D, 16), np.float32)
    order = rng.permutation(maxb)[:N]
    for i in range(D):                                                   # the list's first D keys
        v[order[i // 16], :, i, i % 16] = 1.0
    scores = np.einsum("nhgd,bhtd->nhgbt", q.reshape(n, H, G, D), k[order]).astype(np.float64)
    spread = (scores.max((3, 4)) - scores.min((3, 4))).max() * np.log2(np.e) / np.sqrt(D)
    assert spread <= 2.0, spread
    got = molt_lib.paged_attention_blocks(*(torch.from_numpy(x).cuda() for x in (q, k, v)), _i32(np.arange(maxb)[None]),
                                          _i32([16 * maxb]), n - 1, _i32(np.tile(order, (n, H, 1))))
    w = np.exp((scores - scores.max((3, 4), keepdims=True)) / np.sqrt(D)).reshape(n, H * G, -1)
    want = w[..., :D] / w.sum(-1, keepdims=True)
    tol = 89 * 2.0 ** -24 * want
    assert (np.abs(_val(got).reshape(n, H * G, D) - want) <= tol).all()
    high = torch.from_numpy(w).float().bfloat16()
    coarse = (high.double() + (torch.from_numpy(w).float() - high.float()).bfloat16().double()).numpy()[..., :D]
    assert (np.abs(coarse / w.sum(-1, keepdims=True) - want) > tol).any()

"""GPU tests of how exactly attention over the 4-bit KV cache holds its softmax weights: in bf16 calls they have 11
significant bits (f16) beside values that f16 holds and 16 (two bf16 parts) beside others, so that the output's own
rounding is what is left of the error; small weights beside a large one; values of any scale, whichever pair of
blocks, wavefront or part of the keys they are in."""
import numpy as np
import pytest
import torch

from test_gpu_kvq import DT, _rows, _t

pytestmark = pytest.mark.gpu


def _tol(out, mag, sum_v, dtype):
    """bf16: the output's rounding, 2^-8 |o| (of the computed value: 1 + 2^-8). A weight is w (1 + d), |d| <= 2^-11,
    and so is the sum of the weights: the result is off by sum w d (v - o) / (1 + sum w d), at most
    2^-11 (1 + 2^-10) (sum w |v| + |o|) <= (2^-10 + 2^-20) sum w |v|. A weight under 2^-24 of the largest is an f16
    subnormal times 2^10: off by 2^-25 / 2^10 of the largest, 2^-35 sum |v|. Scores: their f32 sums, and what the
    queries' fp8 parts lose (2^-22 of a row's largest element times sum |k| / sqrt(D), here under 2^4 * 2^4 * 2^-22),
    move a weight by under 2^-13: 2^-12 sum w |v| with that of |o|.
    f32: as in test_gpu_kvq, 2^-15 sum w |v|."""
    if dtype == "bf16":
        return 2.0 ** -8 * (1 + 2.0 ** -8) * np.abs(out) + (2.0 ** -10 + 2.0 ** -12 + 2.0 ** -20) * mag + 2.0 ** -35 * sum_v
    return 2.0 ** -15 * mag


def _caches(molt, rng, ctx, n, Hkv, D, value_exponents=None, key_rows=None):
    """4-bit caches of random rows, the values times 2^value_exponents[b] ([positions, D / 32]); returns the call's
    caches, tables and contexts, and the rows read back (f64, per sequence)."""
    B = len(ctx)
    maxb = (max(ctx) + n + 15) // 16 + 1
    tables = _t(rng.permutation(B * maxb + 3)[:B * maxb].reshape(B, maxb).astype(np.int32))
    gk = torch.full((B * maxb + 3, Hkv, 17 * D // 2), 0xFF, dtype=torch.uint8, device="cuda")
    gv = gk.clone()
    zero, lens = (_t(np.array(x, np.int32)) for x in ([0] * B, [c + n for c in ctx]))
    most = max(ctx) + n
    k, v = (rng.standard_normal((B, most, Hkv, D), np.float32) for _ in range(2))
    for b, c in enumerate(ctx):
        if key_rows is not None:
            k[b, :c + n] = key_rows[b]
        if value_exponents is not None:
            v[b, :c + n] = np.ldexp(v[b, :c + n], np.repeat(value_exponents[b], 32, axis=-1)[:, None])
    molt.kvq_write(*(_t(x.reshape(B * most, Hkv, D)) for x in (k, v)), gk, gv, tables, zero, most, lens=lens)
    K, V = ([x[b, :c + n] for b, c in enumerate(ctx)]
            for x in (r.double().cpu().numpy().reshape(B, most, Hkv, D)
                      for r in molt.kvq_read(gk, gv, tables, zero, most, lens=lens, dtype=torch.float32)))
    return (gk, gv, tables, _t(np.array(ctx, np.int32))), K, V


def _check(molt, q, q64, caches, K, V, ctx, n, dtype):
    out = molt.paged_attention_kvq(q.cuda(), *caches, n - 1).double().cpu().numpy()
    Hkv, D = K[0].shape[1:]
    q64 = q64.reshape(len(ctx), n, Hkv, -1, D)
    out = out.reshape(q64.shape)
    worst = 0.0
    for b in range(len(ctx)):
        rows = q64[b].transpose(1, 0, 2, 3).reshape(Hkv, -1, D)          # of a kv head: position, query head
        k, v = (x[b].transpose(1, 0, 2) for x in (K, V))
        score = rows @ k.transpose(0, 2, 1) / np.sqrt(D)
        seen = np.arange(k.shape[1])[None] <= ctx[b] + np.arange(n)[:, None]
        seen = np.repeat(seen, rows.shape[1] // n, axis=0)
        w = np.where(seen, np.exp(score - np.where(seen, score, -np.inf).max(axis=-1, keepdims=True)), 0.0)
        w /= w.sum(axis=-1, keepdims=True)
        back = lambda x: x.reshape(Hkv, n, -1, D).transpose(1, 0, 2, 3)
        want, mag, sum_v = back(w @ v), back(w @ np.abs(v)), back((w > 0).astype(float) @ np.abs(v))
        tol = _tol(want, mag, sum_v, dtype)
        err = np.abs(out[b] - want)
        assert np.isfinite(out[b]).all()
        worst = max(worst, (err / np.maximum(tol, 1e-300)).max())
        assert (err <= tol).all(), (b, (err / tol).max())
    print("max error / tolerance", worst, flush=True)


# B sequences, query heads of 2 kv heads, positions, longest context: few and many rows (1 to 3 tiles, one or more row
# groups), keys of one wavefront, of several, and cut ones
SHAPES = [(3, 4, 1, 40), (40, 16, 9, 90), (4, 10, 3, 300), (3, 24, 4, 700), (2, 30, 5, 900), (2, 8, 2, 3000), (900, 4, 5, 20)]


@pytest.mark.parametrize("B,Hq,n,hi", SHAPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sharp", [1.0, 4.0])
def test_error_of_the_weights(molt_lib, sharp, D, B, Hq, n, hi):
    """Outputs that are small against their terms: the error is that of the weights."""
    rng = np.random.default_rng(51)
    ctx = [int(c) for c in np.linspace(hi // 2, hi, B)]
    caches, K, V = _caches(molt_lib, rng, ctx, n, 2, D)
    q, _ = _rows(rng, B * n, Hq, D, "bf16")
    q = q * sharp
    _check(molt_lib, q, q.double().numpy(), caches, K, V, ctx, n, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_small_weights_beside_a_large_one(molt_lib, dtype, D):
    """4000 keys of weights about 2^-28 .. 2^-17 of one key's, in dims where that key's value is 0."""
    rng = np.random.default_rng(53)
    ctx, n, Hq = [4000], 1, 6
    keys = rng.standard_normal((4001, 2, D), np.float32) * 0.125
    keys[:, :, :32] = 0.0
    keys[1234, :, :32] = 6.0
    exps = np.zeros((4001, D // 32), int)
    exps[1234, 1] = -140                               # flushed to 0 by the format
    caches, K, V = _caches(molt_lib, rng, ctx, n, 2, D, [exps], [keys])
    assert (V[0][1234, :, 32:64] == 0).all()
    q = torch.ones(1, Hq, D) * 0.0625
    q[..., :32] = (torch.arange(Hq) * 0.0625 + 0.5).view(1, Hq, 1) * (D / 64) ** 0.5
    q = q.to(DT[dtype])
    _check(molt_lib, q, q.double().numpy(), caches, K, V, ctx, n, dtype)


def _exponents(rng, where, L, groups):
    e = np.zeros((L, groups), int)
    if where == "first":                               # the first key's, one group
        e[0, -1] = 60
    elif where == "last":                              # the last key's
        e[-1, 0] = -60
    elif where == "one late":                          # one pair of the second half
        e[L * 2 // 3, 0] = 30
    elif where == "edges":                             # around the border of what f16 holds, both ends
        e = rng.integers(-26, 14, (L, groups))
        e[: L // 4] = rng.integers(-18, 8, (L // 4, groups))
    elif where == "all":
        e = rng.integers(-100, 100, (L, groups))
    elif where == "groups":                            # each group its own far scale
        e[:] = np.array([-90, 100, 0, -30])[:groups]
    elif where == "zeros":                             # groups of zeros (scale byte 2)
        e[::3, 0] = -200
    return e


@pytest.mark.parametrize("where,dtype", [(w, "bf16") for w in ("first", "last", "one late", "edges", "all", "groups",
                                                               "zeros")] + [("all", "f32")])
@pytest.mark.parametrize("B,Hq,n,hi", SHAPES[1:])
@pytest.mark.parametrize("D", [64, 128])
def test_values_of_any_scale(molt_lib, D, B, Hq, n, hi, where, dtype):
    rng = np.random.default_rng(55)
    ctx = [int(c) for c in np.linspace(hi // 2, hi, B)]
    exps = [_exponents(rng, where if b % 3 != 1 else "none", c + n, D // 32) for b, c in enumerate(ctx)]
    caches, K, V = _caches(molt_lib, rng, ctx, n, 2, D, exps)
    q, q64 = _rows(rng, B * n, Hq, D, dtype)
    _check(molt_lib, q, q64, caches, K, V, ctx, n, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_largest_values(molt_lib, dtype, D):
    """A key's values near the largest that the format holds come out as they are, alone and beside small ones."""
    rng = np.random.default_rng(57)
    for L in (1, 40, 700):
        exps = np.zeros((L, D // 32), int)
        exps[L // 2] = 125
        k = np.zeros((L, 1, D), np.float32)
        k[L // 2] = 6.0                                # and the weight is 1: the other scores are 6 sqrt(D) less
        caches, K, V = _caches(molt_lib, rng, [L - 1], 1, 1, D, [exps], [k])
        # the largest of standard normal values is under 6: no value past 6 * 2^125
        assert np.abs(V[0]).max() > 2.0 ** 124
        q = torch.ones(1, 3, D, dtype=DT[dtype])
        out = molt_lib.paged_attention_kvq(q.cuda(), *caches, 0).double().cpu().numpy().reshape(3, D)
        # f32 sums and the reciprocal: under 2^-20; then the output's rounding; and in dims where the key is 0 the other
        # keys: under 2^10 of them, weights of at most e^-48 < 2^-69, values under 2^3
        want = V[0][L // 2, 0]
        assert (np.abs(out - want) <= 2.0 ** (-8 if dtype == "bf16" else -20) * np.abs(want) + 2.0 ** -56).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_largest_queries(molt_lib, dtype, D):
    """The largest finite query elements, on keys so small there that the scores are ordinary ones."""
    rng = np.random.default_rng(59)
    ctx, n, Hq = [90, 700], 2, 6
    keys = [rng.standard_normal((c + n, 2, D), np.float32) for c in ctx]
    for k in keys:
        k[..., :32] = np.ldexp(k[..., :32], -124)      # times up to 2^128: terms of up to 2^7 / sqrt(D)
    caches, K, V = _caches(molt_lib, rng, ctx, n, 2, D, key_rows=keys)
    q, _ = _rows(rng, len(ctx) * n, Hq, D, dtype)
    big = torch.finfo(DT[dtype]).max
    q[:, :, 3] = big
    q[:, 1::2, 30] = -big
    if dtype == "f32":
        q[0, :, 17], q[1, :, 17] = 3.3961e38, -3.3962e38   # either side of where bf16 rounds to infinity
    # (a bf16 row's other elements are under 2^-22 of its largest: what is lost of them is under the row's bound)
    tail = q[:, :, 32:]
    if dtype == "bf16":
        tail.zero_()
    _check(molt_lib, q, q.double().numpy(), caches, K, V, ctx, n, dtype)

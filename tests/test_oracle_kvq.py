"""Pins of the 4-bit KV cache's oracle: the formats' fixed points, nearest values by brute force, the
scale rule at its edges, the record layout as a one-to-one map of a block's bytes, and the attention
against the dense oracle on the decoded values."""
import numpy as np
import pytest

from oracle import attention as oattn, kvq


def test_fixed_points():
    codes, scales = kvq.encode(np.array([6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.25, -0.75, -6.0] + [0.0] * 21))
    assert scales.tolist() == [127]
    assert codes.tolist()[:11] == [7, 6, 6, 4, 4, 2, 2, 0, 8, 10, 15]
    assert np.array_equal(kvq.decode(np.arange(32, dtype=np.uint8) % 16, np.array([128], np.uint8))[:8], 2 * kvq.GRID)


@pytest.mark.parametrize("a,scale", [(3.5, 127), (6.99, 127), (7.0, 128), (3.49, 126), (0.0, 2), (1e-45, 2),
                                     (3.3e38, 252), (2.0 ** -122, 3), (np.inf, 255), (np.nan, 255)])
def test_scale_rule(a, scale):
    x = np.zeros(64)
    x[7], x[40] = -a, 1.0
    codes, scales = kvq.encode(x)
    assert scales.tolist() == [scale, 125]        # 1 = 4 * 2^-2
    v = kvq.decode(codes, scales)
    assert v[40] == 1.0
    if scale == 255:
        assert np.isnan(v[:32]).all() and np.isfinite(v[32:]).all()
    else:
        assert abs(v[7] + a) <= 2.0 ** (scale - 127.0) * (2 if scale == 252 else 1)


def test_nearest():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((200, 64)) * np.exp2(rng.integers(-20, 20, (200, 1)))
    codes, scales = kvq.encode(x)
    v = kvq.decode(codes, scales)
    unit = np.repeat(2.0 ** (scales.astype(int) - 127.0), 32, axis=-1)
    every = np.concatenate([kvq.GRID, -kvq.GRID]) * unit[..., None]
    assert np.array_equal(np.abs(x - v), np.abs(x[..., None] - every).min(-1))
    a = np.abs(x.reshape(200, 2, 32)).max(-1) / unit[:, ::32]
    assert ((a >= 3.5) & (a < 7)).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [False, True])
def test_layout_covers_the_record(D, value):
    seen = np.zeros(17 * D // 2, int)
    for slot in range(16):
        at, sc = kvq.offsets(slot, D, value)
        np.add.at(seen, at, 1)
        np.add.at(seen, sc, 2)
    assert (seen == 2).all()


@pytest.mark.parametrize("D", [64, 128])
def test_attention_on_the_decoded_values(D):
    rng = np.random.default_rng(5)
    B, k, Hq, Hkv, nb = 2, 2, 6, 2, 9
    kc, vc = (np.zeros((nb, Hkv, 17 * D // 2), np.uint8) for _ in range(2))
    tables, ctx = rng.permutation(nb)[:8].reshape(B, 4), [17, 40]
    starts, n = [0, 0], 43
    rows = rng.standard_normal((2, B * n, Hkv, D))
    kvq.write_rows(rows[0], rows[1], kc, vc, tables, starts, n)
    got = kvq.read_rows(kc, vc, tables, starts, n, D)
    assert all(np.array_equal(g, kvq.decode(*kvq.encode(r))) for g, r in zip(got, rows))
    q = rng.standard_normal((B * (k + 1), Hq, D))
    out, mag = kvq.attention(q, kc, vc, tables, ctx, k)
    for b in range(B):
        for h in range(Hq):
            m = ctx[b] + k + 1
            want = oattn.dense_causal_attention(q[b * (k + 1):(b + 1) * (k + 1), h][:, None],
                                                got[0][b * n:b * n + m, h // 3], got[1][b * n:b * n + m, h // 3], ctx[b], k)
            assert np.abs(out[b * (k + 1):(b + 1) * (k + 1), h] - want[:, 0]).max() < 1e-12
    assert (mag >= np.abs(out)).all()

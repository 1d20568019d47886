"""Pins of the oracle of sparse attention: hand-made plans, the bounds' property, selection by brute force, attention
over all blocks as a dense softmax."""
import numpy as np
import pytest

from oracle import blocks


def test_plan_by_hand():
    tables = np.array([[7, 9, -5], [3, -5, -5], [4, 6, -5], [-5, -5, -5]], np.int32)
    n_blocks, ctx = np.array([1, 1, 2, 0], np.int32), np.array([14, 16, 32, 0], np.int32)
    pool = np.array([10, 4] + [0] * 12, np.int32)
    pool[2 + 10], pool[2 + 11], pool[2], pool[3] = 11, 2, 8, 1       # the ring goes on at its start
    slots, placed = blocks.plan(tables, n_blocks, ctx, np.array([3, 2, -1, 1], np.int32), pool, 3)
    assert tables[0].tolist() == [7, 11, -5] and tables[1].tolist() == [3, 2, -5] and tables[3, 0] == 8
    assert slots.reshape(4, 3).tolist() == [[7 * 16 + 14, 7 * 16 + 15, 11 * 16], [32, 33, -1], [-1] * 3, [128, -1, -1]]
    assert placed.tolist() == [3, 2, 0, 1] and n_blocks.tolist() == [2, 2, 0, 1]
    assert pool[:2].tolist() == [1, 3] and pool[3:6].tolist() == [1, 4, 6]


def test_plan_runs_dry_in_order():
    tables, n_blocks = np.full((4, 4), -1, np.int32), np.zeros(4, np.int32)
    pool = np.array([0, 3, 5, 6, 7, 0], np.int32)
    slots, placed = blocks.plan(tables, n_blocks, np.zeros(4, np.int32), np.array([17, 40, 16, 0], np.int32), pool, 40)
    assert placed.tolist() == [17, 0, 0, 0] and n_blocks.tolist() == [2, 0, 0, 0]
    assert pool[:2].tolist() == [2, 1] and tables[0, :2].tolist() == [5, 6]


@pytest.mark.parametrize("scale", [1.0, 2.0 ** -120, 2.0 ** 100])
def test_no_key_left_out_has_a_larger_product(scale):
    rng = np.random.default_rng(0)
    D, q = 64, rng.standard_normal((3, 64))
    f = [blocks.exponent(np.abs(x).max()) for x in q]
    rounded = np.array([np.ldexp(np.rint(np.ldexp(x, -e)), e) for x, e in zip(q, f)])
    for _ in range(20):
        keys = rng.standard_normal((16, D)) * np.exp(rng.standard_normal(D)) * scale
        hi, lo, e = blocks.bounds_of(keys)
        assert (np.abs(hi) <= 127).all() and (np.abs(lo) <= 127).all()
        assert (np.ldexp(hi, e) >= keys.max(0)).all() and (np.ldexp(lo, e) <= keys.min(0)).all()
        if scale >= 1:
            s = blocks.score(q, blocks.record(keys))
            x = min(max(e + f[0], -100), 100)
            assert x != e + f[0] or s >= (rounded @ keys.T).max() * (1 - 1e-12)
    assert blocks.exponent(0.0) == -100 and blocks.exponent(127.0) == 0 and blocks.exponent(127.0000001) == 1
    assert blocks.exponent(63.5) == -1


def test_select_takes_the_largest_and_the_lowest_of_equal_ones():
    bounds = np.zeros((8, 1, 2 * 64 + 16), np.uint8)
    tables = np.arange(8, dtype=np.int32)[None]
    for blk, a in enumerate([1, 5, 3, 5, 2, 9, 5, 0]):
        bounds[blk, 0, 0] = a                                        # largest key in dim 0
    q = np.zeros((1, 1, 64))
    q[0, 0, 0] = 1.0
    pick = lambda N, first, last, ctx=127, **kw: blocks.select(q, bounds, tables, [ctx], 1, N, first, last, **kw)[0, 0].tolist()  # noqa: E731
    assert pick(3, 0, 1) == [1, 5, 7] and pick(4, 1, 1) == [0, 1, 5, 7] and pick(5, 0, 1) == [1, 3, 5, 6, 7]
    assert pick(4, 1, 2, ctx=40) == [0, 1, 2, -1] and pick(2, 0, 1, ctx=85) == [1, 5]
    assert pick(2, 0, 1, lens=[0]) == [-1, -1]
    tables[0, 5] = 8
    assert pick(3, 0, 1) == [1, 3, 7]


def test_all_blocks_is_dense_attention():
    rng = np.random.default_rng(1)
    B, n, H, G, D, mb = 2, 3, 2, 3, 64, 4
    kc, vc = rng.standard_normal((9, H, 16, D)), rng.standard_normal((9, H, D, 16))
    tables, ctx = rng.permutation(9)[:8].reshape(2, 4).astype(np.int32), np.array([37, 0], np.int32)
    q = rng.standard_normal((B * n, H * G, D))
    lists = np.tile(np.array([2, 0, -1, 3, 1, 9], np.int32), (B * n, H, 1))
    out, _ = blocks.attend(q, kc, vc, tables, ctx, n, lists)
    for t in range(B * n):
        b, keys = t // n, ctx[t // n] + t % n + 1
        k = np.concatenate([kc[i] for i in tables[b]], 1)[:, :keys]
        v = np.concatenate([vc[i] for i in tables[b]], 2)[:, :, :keys]
        for h in range(H * G):
            s = k[h // G] @ q[t, h] / 8.0
            w = np.exp(s - s.max())
            assert np.allclose(out[t, h], v[h // G] @ w / w.sum(), atol=1e-12)

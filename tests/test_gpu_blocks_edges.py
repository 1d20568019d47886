"""Sparse attention over listed blocks and the cache's upkeep at the ends of what their types hold."""
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


# ---------------------------------------------------------------- bounds

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,D", [(2, 64), (1, 128)])
def test_bounds_of_the_largest_keys_and_back(molt_lib, dtype, H, D):
    """Keys above 127 * 2^121 have e = 122: the bounds are the codes times 2^122 in f32, infinite from code 64 on, and lie
    around the keys. 127 * 2^121 itself, and less, have e = 121."""
    rng = np.random.default_rng(D)
    big, border = torch.finfo(DT[dtype]).max, 127.0 * 2.0 ** 121
    kc = torch.from_numpy(rng.standard_normal((9, H, 16, D)).astype(np.float32)).to(DT[dtype])
    kc[0, 0, 3, 5], kc[0, 0, 9, 6] = big, 2.0 ** 125 + 2.0 ** 119
    kc[1, 0, 15, 0] = -big
    kc[2] = big
    kc[3] = -big
    kc[4, -1, 7, D - 1] = border                                     # e = 121
    kc[5, -1, 0, 1], kc[5, -1, 1, 1] = border * (1 + 2.0 ** (-7 if dtype == "bf16" else -23)), -border   # (bf16: infinite)
    kc[6, 0, :, ::2], kc[6, 0, 2, 1] = 2.0 ** 127, -(2.0 ** 127)     # e = 121
    kc[7] *= 2.0 ** 124
    kc[8, 0, 4, 3] = border + 2.0 ** (120 if dtype == "bf16" else 104)   # the next one
    bounds = molt_lib.key_bounds(9, H, D)
    molt_lib.key_bounds_update(kc.cuda(), bounds, _i32(np.arange(9)[None]), _i32([0]), 9 * 16)
    exponents = bounds.view(torch.int8)[..., 2 * D].tolist()
    assert exponents[0][0] == exponents[1][0] == exponents[2][0] == exponents[3][0] == exponents[8][0] == 122
    assert exponents[5][-1] == (127 if dtype == "bf16" else 122)
    assert exponents[4][-1] == exponents[6][0] == 121
    hi, lo = molt_lib.key_bounds_read(bounds, _i32(np.arange(9)))
    for i in range(9):
        for h in range(H):
            keys = _val(kc[i, h])
            a, b, e = ob.bounds_of(keys)
            with np.errstate(over="ignore"):
                want = np.ldexp(a, e).astype(np.float32), np.ldexp(b, e).astype(np.float32)
            if e == ob.NOT_FINITE:
                want = np.full(D, np.inf, np.float32), np.full(D, -np.inf, np.float32)
            got = hi[i, h].cpu().numpy(), lo[i, h].cpu().numpy()
            assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1]), (i, h)
            assert (got[0] >= keys.max(0)).all() and (got[1] <= keys.min(0)).all(), (i, h)
    assert hi[0, 0, 5].item() == float("inf") and hi[0, 0, 6].item() == 9 * 2.0 ** 122 and lo[1, 0, 0].item() == -float("inf")


# ---------------------------------------------------------------- attention

def _attend(molt, q, kc, vc, ctx, n, lists):
    table = np.arange(len(kc), dtype=np.int32)[None]
    got = molt.paged_attention_blocks(q.cuda(), kc.cuda(), vc.cuda(), _i32(table), _i32(ctx), n - 1, _i32(lists))
    want, mag = ob.attend(_val(q), _val(kc), _val(vc), table, ctx, n, lists)
    return _val(got).reshape(want.shape), want, mag


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N", [3, 200])
@pytest.mark.parametrize("scale", [2.0 ** 16, 2.0 ** 24, 2.0 ** 34, 2.0 ** 54])
def test_attention_of_far_scores(molt_lib, dtype, D, N, scale):
    """Scores up to 2^112: the largest has all the weight, 1, however coarse the steps of f32 are at its size. Queries and
    keys are whole numbers in -2 .. 2 times a power of two, so that every score is exact and two that differ do so by scale^2
    at least: the output is the mean of the values of the keys with the largest score, up to N * 16 of them, whose
    weights are 1 and whose sum is exact. A value is rounded half a step, and f32 sums of at most 2^12 values of |v| < 8 and
    their product with the reciprocal are off by 2^12 * 2^-24 of sum w |v| at most."""
    rng = np.random.default_rng(N)
    H, G, n, maxb = 2, 5, 3, 220
    kc = torch.from_numpy(rng.integers(-2, 3, (maxb, H, 16, D)) * np.float32(scale)).to(DT[dtype])
    vc = torch.from_numpy(rng.standard_normal((maxb, H, D, 16)).astype(np.float32)).to(DT[dtype])
    q = torch.from_numpy(rng.integers(-2, 3, (n, H * G, D)) * np.float32(scale)).to(DT[dtype])
    q[1] = -q[1].abs() - q[1, :, :1].abs()
    kc[:, 1] = kc[:, 1].abs() + kc[:, 1, :, :1].abs()                # position 1, head 1: no score above 0
    lists = np.tile(np.arange(10, 10 + N, dtype=np.int32), (n, H, 1))
    lists[2, :, 1] = -1
    got, want, mag = _attend(molt_lib, q, kc, vc, [16 * maxb - n], n, lists)
    tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want) + 2.0 ** -12 * mag
    assert np.isfinite(got).all() and (np.abs(got - want) <= tol).all(), np.abs(got - want).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [3, 200])
def test_attention_of_keys_that_score_minus_infinity(molt_lib, dtype, N):
    """Such keys have no weight beside others; a row that sees no others is zeros."""
    rng = np.random.default_rng(7)
    H, G, D, maxb, n = 2, 4, 64, 220, 2
    kc, vc, q = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(DT[dtype])
                 for s in ((maxb, H, 16, D), (maxb, H, D, 16), (n, H * G, D)))
    q[:, :, 5] = q[:, :, 5].abs() + 0.5
    lists = np.tile(np.arange(10, 10 + N, dtype=np.int32), (n, H, 1))
    lists[1, 1, 0] = 4
    kc[10:10 + N, 1, :, 5] = float("-inf")                           # head 1: all but block 4
    kc[10, 0, :, 5], kc[4, 1, :7, 5] = float("-inf"), float("-inf")
    got, _, _ = _attend(molt_lib, q, kc, vc, [16 * maxb - n], n, lists)
    assert (got[0, G:] == 0).all()
    far = kc.clone()
    far[far == float("-inf")] = -(2.0 ** 20)                         # no weight either: scores 2^15 below the others
    far[10:10 + N, 1] = 0                                            # (position 0, head 1 is not compared)
    few = lists.copy()
    few[1, 1, 1:] = -1
    _, want, mag = _attend(molt_lib, q, far, vc, [16 * maxb - n], n, few)
    tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want) + 2.0 ** -12 * mag + 1e-30   # as in test_gpu_blocks.py
    for t, heads in ((0, slice(0, G)), (1, slice(0, G)), (1, slice(G, None))):
        assert (np.abs(got - want)[t, heads] <= tol[t, heads]).all(), (t, heads)


# ---------------------------------------------------------------- refusals

SELECT = dict(n_select=4, n_first=1, n_last=2)


@pytest.mark.parametrize("call,words", [("plan", "too many|too large"), ("read", "head_dim = 96"), ("attend", "head_dim = 96"),
                                        (dict(n_select=2 ** 26 + 1), "n_select = 67108865"),
                                        (dict(n_select=2 ** 31 - 1), "n_select = 2147483647"), (dict(n_first=3), "n_first = 3")])
def test_refused_sizes_make_no_outputs(molt_lib, call, words):
    """Sizes that a call refuses are refused in its own words, before it asks for memory for outputs of such sizes."""
    z = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    bf16, table, ctx, new, have, pool = torch.bfloat16, z(4, 8), z(4), z(4), z(4), molt_lib.block_pool(50)
    q, bounds, odd, ids = z(8, 4, 64, dt=bf16), molt_lib.key_bounds(50, 2, 64), molt_lib.key_bounds(50, 2, 96), z(5)
    q96, kc, vc, lists = z(8, 4, 96, dt=bf16), z(50, 2, 16, 96, dt=bf16), z(50, 2, 96, 16, dt=bf16), z(8, 2, 3)
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    with pytest.raises(molt_lib.MoltError, match=words):
        if call == "plan":
            molt_lib.plan_blocks(table, have, ctx, new, pool, 2 ** 30)
        elif call == "read":
            molt_lib.key_bounds_read(odd, ids)
        elif call == "attend":
            molt_lib.paged_attention_blocks(q96, kc, vc, table, ctx, 1, lists)
        else:
            molt_lib.select_blocks(q, bounds, table, ctx, 1, **{**SELECT, **call})
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before


def _calls_in_full(molt):
    """Every call with arguments that it takes: name -> (function, tensors, numbers, optional tensors), in the order of the
    function's own."""
    z = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    f32 = torch.float32
    kc, vc, rows, q = z(9, 2, 16, 64, dt=f32), z(9, 2, 64, 16, dt=f32), z(6, 2, 64, dt=f32), z(6, 8, 64, dt=f32)
    bounds, table, pool = molt.key_bounds(9, 2, 64), z(2, 4), molt.block_pool(9)
    return {
        "plan": (molt.plan_blocks, dict(block_tables=table, n_blocks=z(2), context_lens=z(2), n_new=z(2), pool=pool), dict(n=3),
                 dict(n_shared=z(2))),
        "write": (molt.kv_write, dict(k=rows, v=rows, k_cache=kc, v_cache=vc, slots=z(6) - 1), {}, {}),
        "update": (molt.key_bounds_update, dict(k_cache=kc, bounds=bounds, block_tables=table, starts=z(2)), dict(n=3),
                   dict(lens=z(2))),
        "read": (molt.key_bounds_read, dict(bounds=bounds, ids=z(5)), {}, {}),
        "select": (molt.select_blocks, dict(q=q, bounds=bounds, block_tables=table, context_lens=z(2)),
                   dict(k=2, n_select=4, n_first=1, n_last=2), dict(lens=z(2), workspace=z(1 << 20))),
        "attend": (molt.paged_attention_blocks, dict(q=q, k_cache=kc, v_cache=vc, block_tables=table, context_lens=z(2),
                                                     blocks=z(6, 2, 3)), dict(k=2), dict(workspace=z(1 << 20))),
    }


@pytest.mark.parametrize("name", ["plan", "write", "update", "read", "select", "attend"])
def test_arguments_of_other_kinds_are_refused_by_name(molt_lib, name):
    """What is no tensor, or no whole number, is a MoltError that names the argument, and so are tensors of other sizes."""
    call, tensors, numbers, optional = _calls_in_full(molt_lib)[name]
    call(**tensors, **numbers, **optional)
    call(**tensors, **numbers)

    def refused(**bad):
        key, value = *bad, *bad.values()
        with pytest.raises(molt_lib.MoltError) as e:
            call(**{**tensors, **numbers, **optional, **bad})
            pytest.fail(f"{key} = {value!r} was taken")
        return str(e.value)

    for key, t in {**tensors, **optional}.items():
        for bad in ([1, 2], 3, "cuda", t.cpu().numpy()) + ((None,) if key in tensors else ()):
            assert key in refused(**{key: bad}), (key, bad)
        assert "must be a GPU tensor" in refused(**{key: t.cpu()})
        assert key in refused(**{key: t[..., None].transpose(0, -1).expand(2, *t.shape[1:], t.shape[0])})
        if key != "workspace":
            for bad in (t.sum(), t[:0].flatten(), t.to(torch.int64), t[None]):
                refused(**{key: bad})
    for key, n in numbers.items():
        for bad in ("3", 1.5, None, [3], torch.tensor(n), -1, 2 ** 31, 10 ** 30):
            assert key in refused(**{key: bad}), (key, bad)


@pytest.mark.parametrize("name", ["plan", "update", "select", "attend"])
def test_whole_numbers_of_other_types(molt_lib, name):
    """numpy's integers are whole numbers, as for the other calls."""
    call, tensors, numbers, _ = _calls_in_full(molt_lib)[name]
    want = call(**{k: t.clone() for k, t in tensors.items()}, **numbers)
    for of in (np.int64, np.int32, np.uint8):
        got = call(**{k: t.clone() for k, t in tensors.items()}, **{k: of(n) for k, n in numbers.items()})
        for a, b in zip(*(x if isinstance(x, tuple) else (x,) for x in (got, want))):
            assert a is b is None or torch.equal(a, b)

"""The 4-bit KV cache in float64: OCP MXFP4 groups of 32 dims (e2m1 elements, e8m0 scale), the paged
record layout of include/molt.h, and the attention over it.

A group with largest magnitude a takes the scale 2^e with a / 2^e in [3.5, 7), e in -125 .. 125; its
elements are the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (with sign), ties to the even code, saturating.
A group with an infinity or NaN has the scale byte 255 and stands for NaN.

Pins: tests/test_oracle_kvq.py.
"""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def encode(x):
    """x [..., D] float64 -> (codes [..., D], scales [..., D / 32]) uint8."""
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], -1, 32)
    a = np.max(np.where(np.isfinite(g), np.abs(g), np.inf), axis=-1)
    e = np.full(a.shape, -125)
    for k in range(-124, 126):                       # the smallest e with a < 7 * 2^e
        e = np.where(a >= 7.0 * 2.0 ** (k - 1), k, e)
    bad = ~np.isfinite(a)
    t = np.where(bad[..., None], 0.0, g) / (2.0 ** e)[..., None]
    gap = np.abs(np.abs(t)[..., None] - GRID)
    best = gap.min(axis=-1, keepdims=True)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])       # even codes first: ties go to them
    code = order[np.argmax(gap[..., order] == best, axis=-1)]
    code = np.where(np.signbit(t), code + 8, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def decode(codes, scales):
    """(codes [..., D], scales [..., D / 32]) -> float64 values [..., D]."""
    c = np.asarray(codes).astype(np.int64)
    v = np.where(c >= 8, -1.0, 1.0) * GRID[c & 7]
    s = np.asarray(scales).astype(np.int64)
    unit = np.where(s == 255, np.nan, 2.0 ** (s - 127.0))
    return (v.reshape(*v.shape[:-1], -1, 32) * unit[..., None]).reshape(v.shape)


def offsets(slot, D, value):
    """Byte offsets in a record: of the code byte of each dim [D], and of each group's scale [D / 32]."""
    d, g = np.arange(D), np.arange(D // 32)
    if value:
        return ((slot // 4) * (D // 8) + d // 8) * 16 + (slot % 4) * 4 + (d % 8) // 2, \
            8 * D + ((slot // 4) * (D // 32) + g) * 4 + slot % 4
    return slot * (D // 2) + d // 2, 8 * D + slot * (D // 32) + g


def write(cache, blk, slot, codes, scales, value):
    """codes [Hkv, D], scales [Hkv, D / 32] into slot `slot` of block blk of cache (uint8, in place)."""
    D = codes.shape[-1]
    at, sc = offsets(slot, D, value)
    cache[blk][:, at[0::2]] = codes[:, 0::2] | (codes[:, 1::2] << 4)
    cache[blk][:, sc] = scales


def read(cache, blk, slot, D, value):
    """Values [Hkv, D] of one slot."""
    at, sc = offsets(slot, D, value)
    byte = cache[blk][:, at]
    return decode(np.where(np.arange(D) % 2 == 1, byte >> 4, byte & 15), cache[blk][:, sc])


def place(table_row, pos, num_blocks):
    """(block, slot) of a position, or None where the table has no such place."""
    if pos < 0 or pos >= 16 * len(table_row):
        return None
    blk = int(table_row[pos // 16])
    return (blk, pos % 16) if 0 <= blk < num_blocks else None


def write_rows(k, v, kc, vc, tables, starts, n, lens=None):
    """Rows k, v [B n, Hkv, D] float64 into the caches, in place."""
    for t in range(len(starts) * n):
        b, j = divmod(t, n)
        at = place(tables[b], int(starts[b]) + j, len(kc))
        if at is None or (lens is not None and j >= lens[b]):
            continue
        write(kc, *at, *encode(k[t]), False)
        write(vc, *at, *encode(v[t]), True)


def read_rows(kc, vc, tables, starts, n, D, lens=None):
    out = [np.zeros((len(starts) * n, kc.shape[1], D)) for _ in range(2)]
    for t in range(len(starts) * n):
        b, j = divmod(t, n)
        at = place(tables[b], int(starts[b]) + j, len(kc))
        if at is None or (lens is not None and j >= lens[b]):
            continue
        out[0][t], out[1][t] = read(kc, *at, D, False), read(vc, *at, D, True)
    return out


def attention(q, kc, vc, tables, ctx, k):
    """q [B (1 + k), Hq, D] float64. Returns (o, a): the outputs, and the sums of w |v| that errors of the
    weights are relative to, both [B (1 + k), Hq, D]. Rows that see no key are zeros."""
    q = np.asarray(q, np.float64)
    T, Hq, D = q.shape
    Hkv = kc.shape[1]
    G = Hq // Hkv
    out, mag = np.zeros_like(q), np.zeros_like(q)
    for b in range(len(ctx)):
        places = [(p, place(tables[b], p, len(kc))) for p in range(max(0, int(ctx[b]) + k + 1))]
        places = [(p, at) for p, at in places if at is not None]
        if not places:
            continue
        pos = np.array([p for p, _ in places])
        K = np.stack([read(kc, *at, D, False) for _, at in places])
        V = np.stack([read(vc, *at, D, True) for _, at in places])
        for j in range(k + 1):
            seen = pos <= int(ctx[b]) + j
            if not seen.any():
                continue
            t = b * (k + 1) + j
            for h in range(Hkv):
                rows = slice(h * G, (h + 1) * G)
                s = q[t, rows] @ K[seen, h].T / np.sqrt(D)
                w = np.exp(s - s.max(axis=-1, keepdims=True))
                w /= w.sum(axis=-1, keepdims=True)
                out[t, rows], mag[t, rows] = w @ V[seen, h], w @ np.abs(V[seen, h])
    return out, mag

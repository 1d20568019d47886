"""Sparse attention over listed blocks of a paged cache, and the cache's upkeep, in float64: block tables that follow
the lengths, rows by slot, bounds of a block's keys, the selection and the attention. Plain loops over sequences."""
import math

import numpy as np

BLOCK = 16
MIN_EXPONENT, NOT_FINITE = -100, 127


# ---------------------------------------------------------------- tables and slots

def plan(tables, n_blocks, ctx, new, pool, n, shared=None):
    """In place on tables [B, max_blocks], n_blocks [B] and pool [2 + cap]; returns (slots [B n], placed [B])."""
    B, max_blocks = tables.shape
    cap = len(pool) - 2
    head, count = int(np.uint32(pool[0]) % cap), min(max(int(pool[1]), 0), cap)
    ring = pool[2:].copy()
    slots, placed = np.full((B, n), -1, np.int32), np.zeros(B, np.int32)
    asked = taken = offered = returned = 0
    for b in range(B):
        c, m, have = int(ctx[b]), int(new[b]), int(n_blocks[b])
        if not 0 <= have <= max_blocks:
            continue
        if m < 0:
            back = tables[b, max(0, int(shared[b])) if shared is not None else 0:have]
            offered += len(back)
            if len(back) and count + offered <= cap:                 # else some id is there twice: dropped
                for i, block in enumerate(back):
                    pool[2 + (head + count + offered - len(back) + i) % cap] = block
                returned = offered
            n_blocks[b] = 0
            continue
        if m > n or c < 0 or c + m > BLOCK * max_blocks:
            continue
        need = max(0, -(-(c + m) // BLOCK) - have) if m else 0
        asked += need
        if need and asked > count:
            continue
        for i in range(need):
            tables[b, have + i] = ring[(head + asked - need + i) % cap]
        if need:
            taken, n_blocks[b] = asked, have + need
        placed[b] = m
        for j in range(m):
            block = int(tables[b, (c + j) // BLOCK])
            if 0 <= block < cap:
                slots[b, j] = block * BLOCK + (c + j) % BLOCK
    pool[0], pool[1] = (head + taken) % cap, count - taken + returned
    return slots.reshape(-1), placed


def write_rows(k, v, k_cache, v_cache, slots):
    """Rows k, v [T, H, D] into k_cache [nb, H, 16, D], v_cache [nb, H, D, 16] at slots [T]."""
    for r, s in enumerate(slots):
        if 0 <= s < BLOCK * len(k_cache):
            k_cache[s // BLOCK, :, s % BLOCK] = k[r]
            v_cache[s // BLOCK, :, :, s % BLOCK] = v[r]


# ---------------------------------------------------------------- bounds and scores

def exponent(a):
    """The smallest integer e >= -100 with a <= 127 * 2^e."""
    e = MIN_EXPONENT
    while a > math.ldexp(127.0, e):
        e += 1
    return e


def bounds_of(keys):
    """(codes of the largest keys, of the smallest, e) of keys [tokens, D]."""
    keys = np.asarray(keys, np.float64)
    D = keys.shape[1]
    if not np.isfinite(keys).all():
        return np.zeros(D, int), np.zeros(D, int), NOT_FINITE
    hi, lo = keys.max(0), keys.min(0)
    e = exponent(max(np.abs(hi).max(), np.abs(lo).max()))
    return np.ceil(np.ldexp(hi, -e)).astype(int), np.floor(np.ldexp(lo, -e)).astype(int), e


def record(keys):
    """The record's bytes."""
    hi, lo, e = bounds_of(keys)
    return np.concatenate([hi, lo, [e], np.zeros(15, int)]).astype(np.int8).view(np.uint8)


def update_bounds(k_cache, bounds, tables, starts, n, lens=None):
    """k_cache holds values; bounds [nb, H, 2 D + 16] uint8, in place."""
    B, max_blocks = tables.shape
    for b in range(B):
        m = n if lens is None else min(max(int(lens[b]), 0), n)
        end = int(starts[b]) + m
        for blk in sorted({p // BLOCK for p in range(int(starts[b]), end)}):
            if not 0 <= blk < max_blocks or not 0 <= tables[b, blk] < len(k_cache):
                continue
            for h in range(k_cache.shape[1]):
                bounds[tables[b, blk], h] = record(k_cache[tables[b, blk], h, :min(BLOCK, end - BLOCK * blk)])


def score(rows, rec):
    """The score of query rows [G, D] for the block of record rec."""
    rec = np.asarray(rec).view(np.int8).astype(int)
    D = (len(rec) - BLOCK) // 2
    hi, lo, e = rec[:D], rec[D:2 * D], int(rec[2 * D])
    if e == NOT_FINITE:
        return math.inf
    best = -math.inf
    for q in np.asarray(rows, np.float64):
        if np.isfinite(q).all():
            f = exponent(np.abs(q).max())
            c = np.rint(np.ldexp(q, -f)).astype(int)
        else:
            f, c = MIN_EXPONENT, np.zeros(D, int)
        best = max(best, math.ldexp(int(np.maximum(c * hi, c * lo).sum()), min(max(e + f, -100), 100)))
    return best


def select(q, bounds, tables, ctx, n, n_select, n_first, n_last, lens=None):
    """q [B n, Hq, D]; returns [B n, H, n_select] int32."""
    B, max_blocks = tables.shape
    H = bounds.shape[1]
    G = q.shape[1] // H
    out = np.full((B * n, H, n_select), -1, np.int32)
    for b in range(B):
        for j in range(n if lens is None else min(max(int(lens[b]), 0), n)):
            seen = min((int(ctx[b]) + j) // BLOCK + 1, max_blocks)
            for h in range(H):
                ranked = []
                for blk in range(max(seen, 0)):
                    block = int(tables[b, blk])
                    if 0 <= block < len(bounds):
                        held = blk < n_first or blk >= seen - n_last
                        s = 0.0 if held else score(q[b * n + j, h * G:(h + 1) * G], bounds[block, h])
                        ranked.append((not held, -s, blk))
                picked = sorted(blk for _, _, blk in sorted(ranked)[:n_select])
                out[b * n + j, h, :len(picked)] = picked
    return out


# ---------------------------------------------------------------- attention

def attend(q, k_cache, v_cache, tables, ctx, n, blocks):
    """q [B n, Hq, D], caches of values, blocks [B n, H, N]; returns (out, sum w |v|) [B n, Hq, D]."""
    T, Hq, D = q.shape
    H, G = blocks.shape[1], Hq // blocks.shape[1]
    max_blocks = tables.shape[1]
    out, mag = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    for t in range(T):
        b, pos = t // n, int(ctx[t // n]) + t % n
        for h in range(H):
            ks, vs = [], []
            for blk in blocks[t, h]:
                if not 0 <= blk < max_blocks or not 0 <= tables[b, blk] < len(k_cache):
                    continue
                m = min(max(pos + 1 - BLOCK * int(blk), 0), BLOCK)
                ks.append(k_cache[tables[b, blk], h, :m])
                vs.append(v_cache[tables[b, blk], h, :, :m].T)
            k, v = (np.concatenate(x) if x else np.zeros((0, D)) for x in (ks, vs))
            if not len(k):
                continue
            s = q[t, h * G:(h + 1) * G] @ k.T / math.sqrt(D)
            w = np.exp(s - s.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            out[t, h * G:(h + 1) * G], mag[t, h * G:(h + 1) * G] = w @ v, w @ np.abs(v)
    return out, mag

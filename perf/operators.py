"""The operators of the 4-bit KV cache: writing rows into it, reading them back, attending over it.

A paged cache whose keys and values are held in MXFP4 (OCP microscaling: 4-bit e2m1 elements, one
power-of-two scale for each group of 32 dims of a token's head vector) takes 17 D / 16 bytes per key
and kv head in place of the 4 D of bf16. The attention over it is bound by those bytes, and so many
more sequences fit one GPU.

For a group x of 32 dims with a = max |x| in (0, inf), the scale is the power of two 2^e with
a / 2^e in [3.5, 7) (e kept within -125 .. 125; stored as the byte e + 127), the element the nearest
of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} to x / 2^e, ties to the even code. A group with an infinity or NaN
gets the scale byte 255 and reads back as NaN.

Cache layout, blocks of 16 tokens with a block table per sequence, uint8 tensors:
  K [num_blocks, Hkv, 17 D / 2]: codes [16 tokens][D / 2] (dim 2i in the low nibble of byte i),
                                 then scales [16 tokens][D / 32]
  V [num_blocks, Hkv, 17 D / 2]: codes [4][D / 8][4 tokens][4] (token 4 a + c, dims 8 i .. 8 i + 7),
                                 then scales [4][D / 32][4 tokens]

Kinds of case:
  attend   paged_attention_kvq: n query positions of each of B sequences behind a cached context
  write    kvq_write of n new positions per sequence, then kvq_read of them: what the cache now holds
  read     kvq_read of n positions of each sequence
  step     kvq_write of the step's new rows, then paged_attention_kvq: one layer's share of a step

Shapes are those of workloads.py (32 query / 4 kv heads x 128, and the tiny f32 decoder's 4 x 64) and
odd ones. Caches hold quantised normal values, keys with uneven channels as after RoPE; physical
blocks are a random permutation, and every block that no sequence owns is filled with 0xFF (NaN).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SPARE = 3                      # blocks of the pool that no sequence owns
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(kind, B, n, Hq, Hkv, D, lo, hi, dtype, name=None, ragged=False, fused=False):
    c = dict(kind=kind, B=B, n=n, Hq=Hq, Hkv=Hkv, D=D, ctx_lo=lo, ctx_hi=hi, dtype=dtype, ragged=ragged,
             fused=fused)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one agent decoding alone without speculation: the smallest call, latency-bound
        _case("attend", 1, 1, 32, 4, 128, 700, 700, "bf16", "attend_one_token"),
        # the tiny f32 decoder's verify step
        _case("attend", 4, 4, 4, 4, 64, 64, 128, "f32", "attend_tiny_f32"),
        # plain decode of a ragged batch, some sequences at their first token
        _case("attend", 64, 1, 32, 4, 128, 0, 8192, "bf16", "attend_decode"),
        # the benchmark's verify step, one layer: 128 sequences at context 8192, 4 drafts
        _case("attend", 128, 5, 32, 4, 128, 8192, 8192, "bf16", "attend_verify"),
        # 8 drafts, many sequences: 72 query rows share each key
        _case("attend", 256, 9, 32, 4, 128, 2048, 2048, "bf16", "attend_many_drafts"),
        # long, variable agent contexts
        _case("attend", 16, 5, 32, 4, 128, 32768, 65536, "bf16", "attend_long"),
        # a tool result appended to cached sessions: a prefill window of odd length (compute-bound)
        _case("attend", 2, 257, 32, 4, 128, 8000, 8200, "bf16", "attend_window"),
        # an odd head layout (7 query heads per kv head, D 64), odd contexts, in a whole step
        _case("step", 33, 3, 14, 2, 64, 1, 5000, "bf16", "step_odd_heads", fused=True),
        # the new rows of the benchmark's verify step, taken from the fused QKV rows
        _case("write", 128, 5, 32, 4, 128, 8192, 8192, "bf16", "write_step", fused=True),
        # first prompts of ragged lengths, f32 rows
        _case("write", 3, 2001, 32, 4, 128, 0, 0, "f32", "write_prompts", ragged=True),
        # a few positions for a consumer of f32 rows
        _case("read", 4, 17, 4, 4, 64, 30, 100, "f32", "read_few"),
        # whole sessions moved to a bf16 consumer
        _case("read", 8, 32768, 32, 4, 128, 0, 0, "bf16", "read_sessions", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "step", "write", "read"])
    Hkv = rng.choice([1, 2, 4, 4, 8])
    G = rng.choice([1, 2, 4, 5, 7, 8, 8, 16])
    D = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind in ("attend", "step"):
        n = rng.choice([1, 1, 2, 4, 5, 5, 9, _log_int(rng, 10, 257)])
        B = _log_int(rng, 1, 256)
        n = max(1, min(n, 60000000 // (B * Hkv * G * D)))
        hi = _log_int(rng, 1, 65536)
        # no more cache or arithmetic than the largest listed cases have
        keys = 4.0e6 * 128 / (Hkv * D)
        flops = 6.0e10 if dtype == "bf16" else 1.5e10
        hi = int(min(hi, keys / B, flops / (4.0 * B * n * Hkv * G * D)))
        lo = rng.choice([hi, hi // 2, 0])
        return _case(kind, B, n, Hkv * G, Hkv, D, lo, hi, dtype, fused=rng.random() < 0.5)
    rows = 250000 * 4 * 128 // (Hkv * D) // (1 if dtype == "bf16" else 2)
    B = _log_int(rng, 1, 128)
    n = min(_log_int(rng, 1, 32768), max(1, rows // B // (8 if kind == "write" else 1)))
    lo = rng.choice([0, 0, rng.randrange(1, 100)])
    return _case(kind, B, n, Hkv * G, Hkv, D, lo, lo + rng.choice([0, rng.randrange(1, 100)]), dtype,
                 ragged=rng.random() < 0.5, fused=kind == "write" and rng.random() < 0.5)


def _contexts(case):
    """Cached tokens of each sequence: evenly spread over the case's range."""
    B, lo, hi = case["B"], case["ctx_lo"], case["ctx_hi"]
    return [lo + (hi - lo) * b // max(1, B - 1) for b in range(B)]


def _lens(case):
    """Rows of each sequence that count (the rest is padding): all, or spread down to one."""
    B, n = case["B"], case["n"]
    return [n - (n - 1) * b // B for b in range(B)] if case["ragged"] else [n] * B


def _pack(x, value):
    """x [blocks, Hkv, 16, D] f32 -> cache records of keys or values (the layout above)."""
    nb, H, _, D = x.shape
    codes, scale = _quantise(x)
    byte = codes[..., 0::2] | (codes[..., 1::2] << 4)          # [nb, H, 16, D / 2]
    if value:
        byte = byte.view(nb, H, 4, 4, D // 8, 4).transpose(3, 4)
        scale = scale.view(nb, H, 4, 4, D // 32).transpose(3, 4)
    return torch.cat([byte.reshape(nb, H, 8 * D), scale.reshape(nb, H, D // 2)], -1)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    B, n, Hq, Hkv, D = (case[k] for k in ("B", "n", "Hq", "Hkv", "D"))
    dt = DTYPES[case["dtype"]]
    order = torch.randperm(B, generator=g, device=dev).tolist()
    ctx = [_contexts(case)[i] for i in order]
    lens = [_lens(case)[i] for i in order]
    owned = [(c + n + 15) // 16 for c in ctx]
    max_blocks = max(owned) + 1
    nb = sum(owned) + SPARE
    perm = torch.randperm(nb, generator=g, device=dev, dtype=torch.int32)
    table = perm[-1:].repeat(B, max_blocks)                    # entries past a row's blocks: a spare block
    at = 0
    for b, c in enumerate(owned):
        table[b, :c] = perm[at:at + c]
        at += c
    st = dict(case=case, table=table, ctx=torch.tensor(ctx, dtype=torch.int32, device=dev), ctx_host=ctx,
              lens_host=lens, lens=torch.tensor(lens, dtype=torch.int32, device=dev) if case["ragged"] else None)
    channel = torch.exp(0.5 * torch.randn(Hkv, 1, D, generator=g, device=dev))
    for name, value in (("kc", False), ("vc", True)):
        cache = torch.empty(nb, Hkv, 17 * D // 2, dtype=torch.uint8, device=dev)
        for i in range(0, nb, 8192):
            x = torch.randn(min(8192, nb - i), Hkv, 16, D, generator=g, device=dev)
            cache[i:i + 8192] = _pack(x if value else x * channel, value)
        cache[perm[at:].long()] = 0xFF
        st[name] = cache
    if case["kind"] in ("attend", "step"):
        st["q"] = torch.randn(B * n, Hq, D, generator=g, device=dev).to(dt)
    if case["kind"] in ("write", "step"):
        rows = torch.randn(B * n, Hq + 2 * Hkv if case["fused"] else 2 * Hkv, D, generator=g, device=dev)
        rows[:, -2 * Hkv:-Hkv] *= channel.view(Hkv, D)
        rows = rows.to(dt)
        st["k"], st["v"] = rows[:, -2 * Hkv:-Hkv], rows[:, -Hkv:]     # views of the projection's rows
        if not case["fused"]:
            st["k"], st["v"] = st["k"].contiguous(), st["v"].contiguous()
    if own and case["kind"] in ("attend", "step"):
        import paper_2607_21653_amd as molt
        size = molt.paged_attention_kvq_workspace_size(B, n - 1, Hq, Hkv, D, max_blocks)
        st["ws"] = torch.empty(size, dtype=torch.uint8, device=dev)
    return st


def run(st):
    case = st["case"]
    kind, n = case["kind"], case["n"]
    if own:
        import paper_2607_21653_amd as molt
        if kind in ("write", "step"):
            molt.kvq_write(st["k"], st["v"], st["kc"], st["vc"], st["table"], st["ctx"], n, lens=st["lens"])
        if kind in ("attend", "step"):
            return molt.paged_attention_kvq(st["q"], st["kc"], st["vc"], st["table"], st["ctx"], n - 1,
                                            workspace=st["ws"])
        return molt.kvq_read(st["kc"], st["vc"], st["table"], st["ctx"], n, lens=st["lens"],
                             dtype=DTYPES[case["dtype"]])
    if kind in ("write", "step"):
        _plain_write(st)
    return _plain_attend(st) if kind in ("attend", "step") else _plain_read(st)


# ---------------------------------------------------------------- plain forms

def _pow2(e):
    """2^e in f32 for integers e in -126 .. 127, from the bits."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """x [..., D] -> codes [..., D] and scale bytes [..., D / 32], both uint8."""
    g = x.float().unflatten(-1, (-1, 32))
    a = g.abs().amax(-1)
    m, e = torch.frexp(a)                                      # a = m 2^e, m in [0.5, 1)
    e = torch.clamp(e - 3 + (m >= 0.875).int(), -125, 125)
    bad = ~torch.isfinite(a)
    r = g * _pow2(-e).unsqueeze(-1)
    r = torch.where(bad.unsqueeze(-1), torch.zeros_like(r), r)
    t = r.abs()
    code = ((t > 0.25).byte() + (t >= 0.75).byte() + (t > 1.25).byte() + (t >= 1.75).byte() + (t > 2.5).byte()
            + (t >= 3.5).byte() + (t > 5.0).byte()) | (torch.signbit(r).byte() << 3)
    scale = torch.where(bad, torch.full_like(e, 255), torch.where(a == 0, torch.full_like(e, 2), e + 127))
    return code.flatten(-2), scale.byte()


def _records(cache, D, value):
    """Views of a cache's codes and scales: [nb, H, 16, ..] of keys, [nb, H, 4, .., 4, ..] of values."""
    codes, scales = cache[..., :8 * D], cache[..., 8 * D:]
    if value:
        return codes.unflatten(-1, (4, D // 8, 4, 4)), scales.unflatten(-1, (4, D // 32, 4))
    return codes.unflatten(-1, (16, D // 2)), scales.unflatten(-1, (16, D // 32))


def _dequantise(codes, scales):
    """codes [..., D / 2] bytes, scales [..., D / 32] -> f32 [..., D]."""
    table = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device)
    v = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).flatten(-2)
    s = _pow2(scales.int().clamp(1, 254) - 127)
    s = torch.where(scales == 255, torch.full_like(s, float("nan")), s)
    return (v.unflatten(-1, (-1, 32)) * s.unsqueeze(-1)).flatten(-2)


def _blocks(cache, ids, D, value):
    """The tokens of the blocks ids, f32 [Hkv, 16 len(ids), D]."""
    codes, scales = _records(cache[ids], D, value)
    if value:
        codes = codes.transpose(3, 4).flatten(4).flatten(2, 3)        # [n, H, 16, D / 2]
        scales = scales.transpose(3, 4).flatten(2, 3)
    x = _dequantise(codes, scales)
    return x.transpose(0, 1).flatten(1, 2)


def _places(st):
    """Block and slot of each of the B n positions, and whether the row counts."""
    case = st["case"]
    B, n = case["B"], case["n"]
    pos = st["ctx"].long()[:, None] + torch.arange(n, device=st["ctx"].device)
    blk = torch.gather(st["table"].long(), 1, pos // 16).flatten()
    j = torch.arange(n, device=pos.device).expand(B, n)
    valid = j < st["lens"][:, None] if st["lens"] is not None else torch.ones_like(j, dtype=torch.bool)
    return blk, (pos % 16).flatten(), valid.flatten()


def _plain_write(st):
    D = st["case"]["D"]
    blk, slot, valid = _places(st)
    T, H = blk.numel(), st["k"].shape[1]
    for x, cache, value in ((st["k"], st["kc"], False), (st["v"], st["vc"], True)):
        codes, scale = _quantise(x)
        byte = codes[..., 0::2] | (codes[..., 1::2] << 4)
        rc, rs = _records(cache, D, value)
        if value:
            byte = byte.view(T, H, D // 8, 4)
            ok = valid.view(T, 1, 1, 1)
            rc[blk, :, slot // 4, :, slot % 4] = torch.where(ok, byte, rc[blk, :, slot // 4, :, slot % 4])
            rs[blk, :, slot // 4, :, slot % 4] = torch.where(ok[..., 0], scale, rs[blk, :, slot // 4, :, slot % 4])
        else:
            ok = valid.view(T, 1, 1)
            rc[blk, :, slot] = torch.where(ok, byte, rc[blk, :, slot])
            rs[blk, :, slot] = torch.where(ok, scale, rs[blk, :, slot])


def _plain_read(st):
    D, dt = st["case"]["D"], DTYPES[st["case"]["dtype"]]
    blk, slot, valid = _places(st)
    out = []
    for cache, value in ((st["kc"], False), (st["vc"], True)):
        rc, rs = _records(cache, D, value)
        if value:
            codes, scales = rc[blk, :, slot // 4, :, slot % 4].flatten(-2), rs[blk, :, slot // 4, :, slot % 4]
        else:
            codes, scales = rc[blk, :, slot], rs[blk, :, slot]
        x = _dequantise(codes, scales)
        out.append(torch.where(valid.view(-1, 1, 1), x, torch.zeros_like(x)).to(dt))
    return tuple(out)


def _plain_attend(st):
    case = st["case"]
    n, Hq, Hkv, D = (case[k] for k in ("n", "Hq", "Hkv", "D"))
    G = Hq // Hkv
    out = torch.empty(case["B"] * n, Hq * D, dtype=st["q"].dtype, device=st["q"].device)
    j = torch.arange(n, device=out.device)
    for b, ctx in enumerate(st["ctx_host"]):
        keys = ctx + n
        ids = st["table"][b, :(keys + 15) // 16].long()
        k = _blocks(st["kc"], ids, D, False)[:, :keys]
        v = _blocks(st["vc"], ids, D, True)[:, :keys]
        q = st["q"][b * n:(b + 1) * n].float().view(n, Hkv, G, D).transpose(0, 1).reshape(Hkv, n * G, D)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(D))
        seen = torch.arange(keys, device=out.device)[None, :] <= (ctx + j)[:, None]        # [n, keys]
        s = s.view(Hkv, n, G, keys).masked_fill(~seen[None, :, None], float("-inf"))
        p = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.matmul(p.view(Hkv, n * G, keys), v) / p.sum(-1).view(Hkv, n * G, 1)
        out[b * n:(b + 1) * n] = o.view(Hkv, n, G, D).transpose(0, 1).reshape(n, Hq * D).to(out.dtype)
    return out


# ---------------------------------------------------------------- the definitions in 64 bits

def _round4(x):
    """x [..., D] f64 -> the values that the format holds: the nearest grid point by distance."""
    g = x.double().unflatten(-1, (-1, 32))
    a = g.abs().amax(-1, keepdim=True)
    power = torch.ceil(torch.log2(a.clamp(2.0 ** -200, 2.0 ** 200) / 7.0)).nan_to_num(0.0).clamp(-125, 125)
    unit = (power.long() + 1023 << 52).view(torch.float64)
    unit = torch.where(a / unit >= 7.0, unit * 2.0, unit).clamp(2.0 ** -125, 2.0 ** 125)
    unit = torch.where((a / unit < 3.5) & (unit > 2.0 ** -125), unit / 2.0, unit)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    t = (g / unit).abs()
    best = torch.zeros_like(t)
    gap = t.clone()
    for i in range(1, 8):
        d = (t - grid[i]).abs()
        take = (d < gap) | ((d == gap) & (i % 2 == 0))
        best, gap = torch.where(take, grid[i], best), torch.where(take, d, gap)
    return torch.where(torch.isfinite(a), torch.copysign(best, g) * unit, torch.full_like(g, float("nan"))).flatten(-2)


def _value(code, scale):
    """e2m1 code and e8m0 byte, from the formats' definitions: (-1)^s 2^(e-1) (1 + m/2), or m/2 at e = 0."""
    c = code.long()
    m, e = (c & 1).double(), ((c >> 1) & 3).double()
    mag = torch.where(e > 0, torch.tensor([0.5, 1.0, 2.0, 4.0], dtype=torch.float64, device=c.device)[e.long()]
                      * (1 + m / 2), m / 2)
    unit = torch.where(scale == 255, float("nan"), (scale.long() + 896 << 52).view(torch.float64))
    return torch.where(c >= 8, -mag, mag) * unit


def _token_values(cache, table, pos, D, value):
    """Values f64 [len(pos), Hkv, D] of positions pos (with the table row of their sequence)."""
    flat = cache.view(cache.shape[0], cache.shape[1], -1)
    blk, t = table[pos // 16].long(), pos % 16
    d = torch.arange(D, device=cache.device)
    if value:
        at = ((t // 4)[:, None] * (D // 8) + d // 8) * 16 + (t % 4)[:, None] * 4 + (d % 8) // 2
        sc = 8 * D + ((t // 4)[:, None] * (D // 32) + d // 32) * 4 + (t % 4)[:, None]
    else:
        at = t[:, None] * (D // 2) + d // 2
        sc = 8 * D + t[:, None] * (D // 32) + d // 32
    h = torch.arange(flat.shape[1], device=cache.device)[None, :, None]
    byte = flat[blk[:, None, None], h, at[:, None]]
    code = torch.where(d % 2 == 1, byte >> 4, byte & 15)
    return _value(code, flat[blk[:, None, None], h, sc[:, None]])


def exact(case, seed):
    st = prepare(case, seed)
    B, n, Hq, Hkv, D = (case[k] for k in ("B", "n", "Hq", "Hkv", "D"))
    dev = st["ctx"].device
    outs = [[], []]
    for b in range(B):
        ctx, ln = st["ctx_host"][b], st["lens_host"][b]
        new = None
        if case["kind"] in ("write", "step"):
            rows = slice(b * n, (b + 1) * n)
            new = [_round4(st["k"][rows]), _round4(st["v"][rows])]
        if case["kind"] in ("write", "read"):
            for i, name in enumerate(("kc", "vc")):
                pos = torch.arange(ctx, ctx + ln, device=dev)
                got = new[i][:ln] if new else _token_values(st[name], st["table"][b], pos, D, i == 1)
                outs[i].append(torch.cat([got, got.new_zeros(n - ln, Hkv, D)]))
            continue
        old = torch.arange(ctx if new else ctx + n, device=dev)
        kv = [_token_values(st[name], st["table"][b], old, D, i == 1) for i, name in enumerate(("kc", "vc"))]
        if new:
            kv = [torch.cat([x, y]) for x, y in zip(kv, new)]
        q = st["q"][b * n:(b + 1) * n].double()
        o = torch.empty(n, Hq, D, dtype=torch.float64, device=dev)
        for h in range(Hq):
            k, v = (x[:, h // (Hq // Hkv)].contiguous() for x in kv)
            s = torch.mm(q[:, h].contiguous(), k.t().contiguous()) / math.sqrt(D)
            hidden = torch.arange(ctx + n, device=dev)[None] > ctx + torch.arange(n, device=dev)[:, None]
            o[:, h] = torch.mm(torch.softmax(s.masked_fill(hidden, float("-inf")), -1), v)
        outs[0].append(o.view(n, Hq * D))
    if case["kind"] in ("write", "read"):
        return torch.cat(outs[0]), torch.cat(outs[1])
    return torch.cat(outs[0])


def work(case):
    """Bytes: the cache's bytes that are needed once, rows in, rows out, tables. Operations: two
    products per key and query row."""
    B, n, Hq, Hkv, D = (case[k] for k in ("B", "n", "Hq", "Hkv", "D"))
    es = 2 if case["dtype"] == "bf16" else 4
    token = Hkv * 17 * D // 16                                 # K and V of one position
    ctx, rows = _contexts(case), sum(_lens(case))
    bytes_ = sum(4 * ((c + n + 15) // 16) + 4 for c in ctx)
    flops = 0
    if case["kind"] in ("write", "step"):
        bytes_ += rows * (2 * Hkv * D * es + token)
    if case["kind"] in ("write", "read"):
        bytes_ += (rows * token if case["kind"] == "read" else 0) + B * n * 2 * Hkv * D * es
    if case["kind"] in ("attend", "step"):
        keys = sum(c if case["kind"] == "step" else c + n for c in ctx)
        bytes_ += keys * token + 2 * B * n * Hq * D * es
        flops += 4 * D * Hq * sum(n * c + n * (n + 1) // 2 for c in ctx)
    if flops == 0:
        flops = 4 * rows * Hkv * D                             # a scaling and a rounding per element
    return {"bytes": bytes_, "flops": flops}

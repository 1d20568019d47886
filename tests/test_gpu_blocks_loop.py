"""The calls of sparse attention together, as a decoding loop makes them: tables that follow the lengths, rows and bounds
of the new positions, lists, attention. Sessions that grow, finish and start again against a plain cache on the host;
lists that hold every block against dense paged attention; other streams; graphs, replayed between the program's own
work, whose workspace they share."""
import numpy as np
import pytest
import torch

from oracle import blocks as ob

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _tol(out, mag, dtype):
    """As in test_gpu_blocks.py: half a step of the output, 2^-12 of sum w |v| for scores, weights and sums."""
    return (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(out) + 2.0 ** -12 * mag + 1e-30


def _i32(a):
    return torch.as_tensor(np.asarray(a, np.int32), device="cuda")


class Loop:
    """A layer's caches and tables on the GPU, and one step over them."""

    def __init__(self, molt, B, n, Hq, Hkv, D, maxb, nb, N, dtype, seed=0):
        self.m, self.n, self.Hkv, self.D, self.N, self.dtype = molt, n, Hkv, D, N, DT[dtype]
        self.rng = np.random.default_rng(seed)
        self.B, self.Hq = B, Hq
        self.kc = torch.full((nb, Hkv, 16, D), float("nan"), dtype=self.dtype, device="cuda")
        self.vc = torch.full((nb, Hkv, D, 16), float("nan"), dtype=self.dtype, device="cuda")
        self.bounds = molt.key_bounds(nb, Hkv, D)
        self.tables, self.n_blocks = torch.full((B, maxb), -1, dtype=torch.int32, device="cuda"), _i32(np.zeros(B))
        self.ctx, self.pool = _i32(np.zeros(B)), molt.block_pool(nb)
        size = max(molt.select_blocks_workspace_size(B, n - 1, Hq, Hkv, D, maxb),
                   molt.paged_attention_blocks_workspace_size(B, n - 1, Hq, Hkv, D, N), 1)
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def rows(self):
        x = self.rng.standard_normal((self.B * self.n, self.Hq + 2 * self.Hkv, self.D)).astype(np.float32)
        return torch.from_numpy(x).to(self.dtype).cuda()

    def step(self, rows, new):
        m, n = self.m, self.n
        q, k, v = (x for x in torch.split(rows, [self.Hq, self.Hkv, self.Hkv], 1))
        slots, placed = m.plan_blocks(self.tables, self.n_blocks, self.ctx, new, self.pool, n)
        m.kv_write(k, v, self.kc, self.vc, slots)
        m.key_bounds_update(self.kc, self.bounds, self.tables, self.ctx, n, lens=placed)
        q = q.contiguous()
        lists = m.select_blocks(q, self.bounds, self.tables, self.ctx, n - 1, self.N, lens=placed, workspace=self.ws)
        out = m.paged_attention_blocks(q, self.kc, self.vc, self.tables, self.ctx, n - 1, lists, workspace=self.ws)
        return out, lists, placed


def _value(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,Hq,Hkv,D,N,maxb,nb", [(1, 1, 8, 1, 128, 4, 12, 12), (5, 4, 14, 2, 64, 5, 20, 5),
                                                    (7, 33, 4, 4, 64, 6, 30, 30)])
def test_sessions(molt_lib, dtype, B, n, Hq, Hkv, D, N, maxb, nb):
    """Against a session's rows on the host: what a step writes, lists and attends to, whatever blocks it got."""
    lo = Loop(molt_lib, B, n, Hq, Hkv, D, maxb, nb, N, dtype)
    keys, values = [[] for _ in range(B)], [[] for _ in range(B)]
    ran_dry = 0
    for step in range(14):
        new = lo.rng.integers(0, n + 1, B)
        new[lo.rng.random(B) < 0.15] = -1
        rows = lo.rows()
        out, lists, placed = lo.step(rows, _i32(new))
        placed, lists, host = placed.cpu().numpy(), lists.cpu().numpy(), _value(rows)
        ran_dry += int(((new > 0) & (placed == 0)).sum())
        for b in range(B):
            if new[b] < 0:
                keys[b], values[b] = [], []
            first = len(keys[b])
            for j in range(placed[b]):
                keys[b].append(host[b * n + j, Hq:Hq + Hkv])
                values[b].append(host[b * n + j, Hq + Hkv:])
            nblk = -(-len(keys[b]) // 16)
            if placed[b] == 0:
                assert (lists[b * n:(b + 1) * n] == -1).all() and (out[b * n:(b + 1) * n] == 0).all()
                continue
            pad = [np.zeros((Hkv, D))] * (16 * nblk - len(keys[b]))
            kc = np.stack(keys[b] + pad).reshape(nblk, 16, Hkv, D).transpose(0, 2, 1, 3)
            vc = np.stack(values[b] + pad).reshape(nblk, 16, Hkv, D).transpose(0, 2, 3, 1)
            table = np.arange(nblk, dtype=np.int32)[None]
            bounds = np.zeros((nblk, Hkv, 2 * D + 16), np.uint8)
            ob.update_bounds(kc, bounds, table, [0], len(keys[b]))
            mine = slice(b * n, b * n + placed[b])
            want = ob.select(host[mine, :Hq], bounds, table, [first], placed[b], N, 1, 2)
            assert np.array_equal(lists[mine], want), (step, b)
            ref, mag = ob.attend(host[mine, :Hq], kc, vc, table, [first], placed[b], want)
            assert (np.abs(_value(out)[mine].reshape(ref.shape) - ref) <= _tol(ref, mag, dtype)).all(), (step, b)
        lo.ctx = _i32([len(k) for k in keys])
    assert ran_dry or n == 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lists_of_every_block_are_dense_attention(molt_lib, dtype):
    lo = Loop(molt_lib, 3, 5, 32, 4, 128, 40, 120, 40, dtype)
    for m in (400, 37, 5):                        # windows, the last one's rows compared
        lo.n = m
        rows = lo.rows()
        out, lists, placed = lo.step(rows, _i32([m, m, m]))
        assert (placed == m).all()
        q = rows[:, :32].contiguous()
        if m == 5:
            dense = molt_lib.paged_attention(q, lo.kc, lo.vc, lo.tables, lo.ctx, m - 1)
            err = (out.double() - dense.double()).abs().max().item()
            assert err <= (2.0 ** -7 if dtype == "bf16" else 2.0 ** -18) * dense.abs().max().item()
        lo.ctx = lo.ctx + m


def test_on_another_stream(molt_lib):
    """Everything on a stream of its own, with new inputs made there; no result waits for the default stream."""
    a = Loop(molt_lib, 4, 5, 16, 2, 128, 80, 400, 8, "bf16", seed=3)
    b = Loop(molt_lib, 4, 5, 16, 2, 128, 80, 400, 8, "bf16", seed=3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for i in range(20):
        rows, new = a.rows(), _i32([5, 3, 5 - i % 6, -1 if i % 5 == 4 else 5])
        got, lists, placed = a.step(rows, new)
        a.ctx = torch.where(new < 0, 0, a.ctx + placed)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again, lists_b, placed_b = b.step(b.rows(), new.clone())
            b.ctx = torch.where(new < 0, 0, b.ctx + placed_b)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, again) and torch.equal(lists, lists_b)


def test_two_loops_at_once(molt_lib):
    """Two streams side by side, each with its own tables, caches and workspace: scores and lists in two launches and lists
    in parts, whose workspaces hold what one launch leaves the next. As one after the other."""
    def run(loops, streams):
        out = [[], []]
        for i in range(12):
            for x, (lo, s) in enumerate(zip(loops, streams)):
                with torch.cuda.stream(s):
                    got, lists, placed = lo.step(lo.rows(), _i32([3, 3]))
                    lo.ctx = lo.ctx + placed
                    out[x] += [got, lists]
        torch.cuda.synchronize()
        return out

    def make():
        loops = [Loop(molt_lib, 2, 3, 16, 2, 128, 600, 1300, 40, "bf16", seed=x) for x in (5, 6)]
        for lo in loops:                                              # 300 blocks of context each, the pool's last ids
            keys = torch.from_numpy(lo.rng.standard_normal((1300, 2, 16, 128)).astype(np.float32)).cuda()
            lo.kc.copy_(keys)
            lo.vc.copy_(keys.flip(0).transpose(2, 3))
            lo.tables[:, :300] = torch.arange(700, 1300, device="cuda").view(2, 300)
            lo.n_blocks.fill_(300)
            lo.ctx.fill_(4790)
            lo.pool[1] = 700
            molt_lib.key_bounds_update(lo.kc, lo.bounds, lo.tables, torch.zeros_like(lo.ctx), 4790)
        assert molt_lib.select_blocks_workspace_size(2, 2, 16, 2, 128, 600) > 0
        assert molt_lib.paged_attention_blocks_workspace_size(2, 2, 16, 2, 128, 40) > 0
        return loops

    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    here = torch.cuda.current_stream()
    want, pair = run(make(), (here, here)), make()
    torch.cuda.synchronize()
    got = run(pair, (one, two))
    assert all(torch.equal(a, b) for x in (0, 1) for a, b in zip(want[x], got[x]))
    assert not torch.equal(want[0][0], want[1][0])


def test_graphs_that_share_a_workspace(molt_lib):
    """Two captured steps (a verify step, and plain decode) on one state and workspace, replayed in turn with the
    program's own work between, against the same steps made eagerly on a second state."""
    kinds = {5: None, 1: None}
    state = Loop(molt_lib, 6, 5, 32, 4, 128, 1300, 3000, 16, "bf16")     # a table of over 1024 blocks: two launches
    eager = Loop(molt_lib, 6, 5, 32, 4, 128, 1300, 3000, 16, "bf16")
    start = [x.clone() for x in (state.tables, state.n_blocks, state.pool, state.kc, state.vc, state.bounds)]
    inputs, new = {n: torch.zeros(6 * n, 40, 128, dtype=torch.bfloat16, device="cuda") for n in kinds}, _i32([0] * 6)
    ctx = state.ctx
    for n in kinds:
        state.n = n
        state.step(inputs[n], new)                # once before the capture
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = state.step(inputs[n], new)
            ctx.copy_(torch.where(new < 0, torch.zeros_like(ctx), ctx + outs[2]))
        kinds[n] = (graph, outs)
    for x, y in zip((state.tables, state.n_blocks, state.pool, state.kc, state.vc, state.bounds), start):
        x.copy_(y)
    ctx.zero_()
    rng = np.random.default_rng(1)
    for i in range(12):
        n = 5 if i % 3 else 1
        rows = torch.from_numpy(rng.standard_normal((6 * n, 40, 128)).astype(np.float32)).bfloat16().cuda()
        count = _i32(np.where(rng.random(6) < 0.15, -1, rng.integers(0, n + 1, 6)))
        inputs[n].copy_(rows)
        new.copy_(count)
        graph, outs = kinds[n]
        graph.replay()
        eager.n = n
        want = eager.step(rows, count)
        eager.ctx = torch.where(count < 0, 0, eager.ctx + want[2])
        torch.cuda.synchronize()
        for x, y in zip(outs, want):
            assert torch.equal(x, y), i
        assert torch.equal(ctx, eager.ctx) and torch.equal(state.tables, eager.tables)
        torch.zeros(1 << 20, device="cuda").sum().item()                 # the program's own work


def test_python_refusals(molt_lib):
    m = molt_lib
    lo = Loop(m, 2, 3, 8, 2, 64, 4, 9, 3, "f32")
    rows = lo.rows()
    q, k, v = rows[:, :8].contiguous(), rows[:, 8:10], rows[:, 10:]
    slots, lists = _i32(np.arange(6)), torch.zeros(6, 2, 3, dtype=torch.int32, device="cuda")
    wide = torch.zeros(2, 8, dtype=torch.int32, device="cuda")[:, ::2]
    bad = [
        lambda: m.plan_blocks(wide, lo.n_blocks, lo.ctx, lo.ctx, lo.pool, 3),
        lambda: m.plan_blocks(lo.tables, lo.n_blocks.long(), lo.ctx, lo.ctx, lo.pool, 3),
        lambda: m.plan_blocks(lo.tables, lo.n_blocks, lo.ctx[:1], lo.ctx, lo.pool, 3),
        lambda: m.plan_blocks(lo.tables, lo.n_blocks, lo.ctx, lo.ctx.cpu(), lo.pool, 3),
        lambda: m.plan_blocks(lo.tables, lo.n_blocks, lo.ctx, lo.ctx, lo.pool[:2], 3),
        lambda: m.plan_blocks(lo.tables, lo.n_blocks, lo.ctx, lo.ctx, lo.pool, 0),
        lambda: m.plan_blocks(lo.tables, lo.n_blocks, lo.ctx, lo.ctx, lo.pool, 3, n_shared=lo.ctx.float()),
        lambda: m.plan_blocks(lo.tables.flatten(), lo.n_blocks, lo.ctx, lo.ctx, lo.pool, 3),
        lambda: m.kv_write(k, v, lo.kc, lo.vc.transpose(2, 3), slots),
        lambda: m.kv_write(k.half(), v, lo.kc, lo.vc, slots),
        lambda: m.kv_write(k[:5], v, lo.kc, lo.vc, slots),
        lambda: m.kv_write(k.flip(1).transpose(1, 2).contiguous().transpose(1, 2), v, lo.kc, lo.vc, slots),
        lambda: m.kv_write(k, v, lo.kc, lo.vc, slots.long()),
        lambda: m.kv_write(k, v, lo.kc.half(), lo.vc.half(), slots),
        lambda: m.kv_write(k, v, lo.kc, lo.vc, slots.cpu()),
        lambda: m.key_bounds_update(lo.kc, lo.bounds[:, :, :-16], lo.tables, lo.ctx, 3),
        lambda: m.key_bounds_update(lo.kc, lo.bounds, lo.tables, lo.ctx, 0),
        lambda: m.key_bounds_update(lo.kc, lo.bounds, lo.tables, lo.ctx, 3, lens=lo.ctx.long()),
        lambda: m.key_bounds_read(lo.bounds, slots.view(2, 3)),
        lambda: m.key_bounds_read(lo.bounds.char(), slots),
        lambda: m.key_bounds_read(lo.bounds, slots[:0]),
        lambda: m.select_blocks(q, lo.bounds, lo.tables, lo.ctx, 2, 0),
        lambda: m.select_blocks(q, lo.bounds, lo.tables, lo.ctx, 2, 2),
        lambda: m.select_blocks(q, lo.bounds, lo.tables, lo.ctx, 1, 3),
        lambda: m.select_blocks(q[:, :7].contiguous(), lo.bounds, lo.tables, lo.ctx, 2, 3),
        lambda: m.select_blocks(rows[:, :8], lo.bounds, lo.tables, lo.ctx, 2, 3),
        lambda: m.select_blocks(q.half(), lo.bounds, lo.tables, lo.ctx, 2, 3),
        lambda: m.select_blocks(q, lo.bounds, lo.tables, lo.ctx, 2, 3, lens=lo.ctx[:1]),
        lambda: m.select_blocks(q, lo.bounds, lo.tables, lo.ctx, 2, 3, workspace=torch.empty(1 << 20, dtype=torch.uint8)),
        lambda: m.paged_attention_blocks(q.bfloat16(), lo.kc, lo.vc, lo.tables, lo.ctx, 2, lists),
        lambda: m.paged_attention_blocks(q, lo.kc, lo.vc, lo.tables, lo.ctx, 2, lists[:5]),
        lambda: m.paged_attention_blocks(q, lo.kc, lo.vc, lo.tables, lo.ctx, 2, lists.long()),
        lambda: m.paged_attention_blocks(q, lo.kc, lo.vc, lo.tables, lo.ctx, 2, lists.flatten()),
        lambda: m.paged_attention_blocks(q, lo.kc, lo.vc[:8], lo.tables, lo.ctx, 2, lists),
        lambda: m.paged_attention_blocks(q, lo.kc, lo.vc, lo.tables, lo.ctx, 2, lists[:, :, :0]),
        lambda: m.paged_attention_blocks(q, lo.kc, lo.vc, lo.tables.cpu(), lo.ctx, 2, lists),
        lambda: m.paged_attention_blocks(q, lo.kc, lo.vc, lo.tables, lo.ctx, 2, lists, workspace=lo.ws[::2]),
    ]
    no = lo.ctx[:0]
    for call in (lambda: m.plan_blocks(lo.tables[:0], no, no, no, lo.pool, 3),
                 lambda: m.key_bounds_update(lo.kc, lo.bounds, lo.tables[:0], no, 3),
                 lambda: m.select_blocks(q[:0], lo.bounds, lo.tables[:0], no, 2, 3),
                 lambda: m.paged_attention_blocks(q[:0], lo.kc, lo.vc, lo.tables[:0], no, 2, lists[:0])):
        with pytest.raises(m.MoltError, match="B = 0"):
            call()
    lo.ws = torch.empty(64, dtype=torch.uint8, device="cuda")
    for i, call in enumerate(bad):
        with pytest.raises(m.MoltError):
            call()
            pytest.fail(f"call {i} was taken")
    torch.cuda.synchronize()

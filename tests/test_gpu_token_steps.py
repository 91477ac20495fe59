"""The token-step operators together, as a serving loop uses them: sequences from the stitch, steps that keep lengths, tables and
slots on the device, against tc_prefill_attn on a second context that appends the same rows; eagerly and replayed from one
captured graph."""
import numpy as np
import pytest
import torch

import step_harness as SH
from paper_2601_08743_amd import workloads as W

pytestmark = pytest.mark.gpu


class Loop:
    """Device state of a batch of sequences, and one step over all layers."""

    def __init__(self, dw, bt, held, n_tokens, n_spare, sink, top, local, theta=1e4):
        from paper_2601_08743_amd import binding as B
        self.dw, self.ctx, self.cfg, self.theta = dw, dw.ctx, dw.cfg, theta
        c, n_seq = dw.cfg, len(held)
        spare = dw.ctx.tc_grow_seqs(np.full((1, n_spare), -1, dtype=np.int32), [16 * n_spare])
        self.owned = [bt, spare]
        self.table = torch.from_numpy(dw.ctx.tc_table_entries(bt)).cuda()
        self.spare = torch.from_numpy(spare[0]).cuda()
        self.seq_len, self.new_len = SH.i32(held), SH.i32(np.zeros(n_seq))
        self.cursor, self.cu, self.status = SH.i32([0]), SH.i32(np.zeros(n_seq + 1)), SH.i32([0, 0])
        self.slot, self.pos, self.seq, self.full = SH.i64(np.zeros(n_tokens)), *(SH.i32(np.zeros(n_tokens)) for _ in range(3))
        dt = torch.bfloat16 if c.dtype == "bf16" else torch.float32
        rows = lambda h: torch.zeros((c.n_layers, n_tokens, h, c.head_dim), dtype=dt, device="cuda")
        self.q, self.k, self.v, self.out, self.qr = rows(c.n_q_heads), rows(c.n_kv_heads), rows(c.n_kv_heads), rows(c.n_q_heads), rows(c.n_q_heads)
        self.shape = (sink, top, local)
        self.lists = SH.i32(np.full((c.n_layers, n_tokens, c.n_kv_heads, sum(self.shape)), -1))
        self.digests = torch.zeros(B.tc_digest_bytes(dw.tc_cfg), dtype=torch.int8, device="cuda")
        self.ws = torch.empty(B.tc_sparse_workspace_bytes(dw.tc_cfg, n_tokens, self.table.shape[1], sum(self.shape)), dtype=torch.uint8, device="cuda")
        self.ctx.tc_digest_blocks(0, c.n_layers, self.table, self.digests)

    def step(self, scale, stream=None):
        c = self.cfg
        self.ctx.tc_step_tables(self.seq_len, self.new_len, self.table, self.spare, self.cursor, self.cursor, self.seq_len, self.cu,
                                self.slot, self.pos, self.seq, self.full, self.status, stream)
        for l in range(c.n_layers):
            self.ctx.tc_rope_append(l, self.q[l], self.k[l], self.v[l], self.pos, self.theta, self.slot, self.qr[l], stream=stream)
        self.ctx.tc_digest_blocks(0, c.n_layers, self.full, self.digests, stream)
        for l in range(c.n_layers):
            self.ctx.tc_select_blocks(l, self.qr[l], self.seq, self.pos, self.table, self.digests, *self.shape, self.lists[l], self.ws, stream)
            self.ctx.tc_block_attn(l, self.qr[l], self.seq, self.pos, self.table, self.lists[l], self.out[l], scale, self.ws, stream)

    def fill(self, seed, new):
        """The step's inputs: new tokens of each request, rows of a projection."""
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        for x in (self.q, self.k, self.v):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda").to(x.dtype))
        self.new_len.copy_(SH.i32(new))


def _setup(cfg, alias, extra):
    import harness as H
    wl = W.make_workload(cfg)
    P = [int(wl.table_len[q].sum()) for q in wl.queries]
    blocks = sum(-(-(p + int(s) + 16) // 16) + 2 for p, s in zip(P, wl.suffix_len)) + extra + 40
    dw = H.DeviceWorkload(wl, seq_blocks=blocks, slot_layout=int(alias))
    max_blocks = max(sum(-(-int(wl.table_len[t]) // 16) for t in q) + -(-int(s) // 16) for q, s in zip(wl.queries, wl.suffix_len)) + 6
    bt, pl = (dw.alias if alias else dw.stitch)(max_blocks)
    for layer in range(cfg.n_layers):           # the prompt's own suffix, as ever
        dw.attn_layer(layer, bt, pl)
    return wl, dw, bt, (np.asarray(pl) + wl.suffix_len).astype(np.int32)


SMALL = {"c2": dict(n_layers=2, n_tables=8, tables_per_query=(2, 5), capacity=8, batch=3, suffix_len=(5, 40)),
         "c1": dict(n_layers=2, n_tables=8, tables_per_query=(1, 3), capacity=8, batch=4, suffix_len=(1, 20))}


def _dense_step(dw, bt, cur, new, loop, scale):
    """The same step through tc_prefill_attn: every query's new rows at once, encoded rows taken from the loop."""
    c, B = dw.cfg, len(cur)
    bt = dw.ctx.tc_grow_seqs(bt, cur + new)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    outs = []
    for l in range(c.n_layers):
        n = int(cu[-1])
        k = torch.empty((n, c.n_kv_heads, c.head_dim), dtype=loop.k.dtype, device="cuda")
        for b in range(B):                      # the encoded keys, read back from the loop's pool
            held, s = int(cur[b]), int(new[b])
            if s:
                row = loop.table[b].cpu().numpy()
                blocks = [int(e) & ((1 << 27) - 1) for e in row[:-(-(held + s) // 16)]]
                kk, _ = loop.ctx.tc_read_seq_kv(l, blocks, held + s, np.uint16 if c.dtype == "bf16" else np.float32)
                kt = torch.from_numpy(kk[held:].copy())
                k[int(cu[b]):int(cu[b + 1])] = (kt.view(torch.bfloat16) if c.dtype == "bf16" else kt).cuda()
        q, v, out = loop.qr[l, :n].contiguous(), loop.v[l, :n].contiguous(), torch.empty_like(loop.qr[l, :n])
        dw.ctx.tc_prefill_attn(l, q, k, v, out, cu, bt, cur, new, scale)
        outs.append(out)
    torch.cuda.synchronize()
    return bt, torch.stack(outs)


@pytest.mark.parametrize("base,alias", [("c2", False), ("c2", True), ("c1", False)])
def test_steps_with_every_block_listed_are_dense_attention(base, alias):
    """Lists long enough for all blocks: a step's rows equal those of tc_prefill_attn on another context that is given the same
    ones, to the rounding of both.  Steps of one token, of several, with waiting requests, across block borders, after
    which the loop's own pool goes on with tc_prefill_attn."""
    cfg = W.scaled(W.CONFIGS[base], **SMALL[base])
    wl, dw, bt, held = _setup(cfg, alias, 60)
    _, ref, rbt, _ = _setup(cfg, alias, 60)
    B, scale = cfg.batch, wl.sm_scale
    n_tokens = 70
    loop = Loop(dw, bt, held, n_tokens, 30, 1, bt.shape[1], 2)
    cur = held.copy()
    rng = np.random.default_rng(1)
    for step in range(6):
        new = np.ones(B, dtype=np.int32) if step % 2 == 0 else rng.integers(0, 23, size=B).astype(np.int32)
        loop.fill(step, new)
        loop.out.fill_(7.0)
        loop.step(scale)
        torch.cuda.synchronize()
        assert loop.status.tolist()[0] == 0
        n = int(new.sum())
        rbt, want = _dense_step(ref, rbt, cur, new, loop, scale)
        got = loop.out[:, :n]
        # both sides round weights and outputs to bf16: 2^-8 each of at most max |v| < 5.6 and of the output; fp32: sums of a few
        # thousand keys, 2e-6 of |v| a side
        tol = 2 * (2.0 ** -8 * (5.6 + float(want.float().abs().max()))) if cfg.dtype == "bf16" else 2 * 2e-6 * 5.6
        assert (got.float() - want.float()).abs().max() <= tol
        assert (loop.out[:, n:] == 7.0).all()
        cur = cur + new
        np.testing.assert_array_equal(loop.seq_len.cpu().numpy(), cur)
    # the loop's own sequences, attended to by the host-planned call
    tab = loop.table.cpu().numpy()
    tab = np.where(tab < 0, -1, tab & ((1 << 27) - 1)).astype(np.int32)
    one = np.ones(B, dtype=np.int32)
    loop.fill(99, one)
    q, k, v = (x[0, :B].contiguous() for x in (loop.q, loop.k, loop.v))
    out_a, out_b = torch.empty_like(q), torch.empty_like(q)
    grown = dw.ctx.tc_grow_seqs(tab, cur + one)
    rgrown = ref.ctx.tc_grow_seqs(rbt, cur + one)
    cu = np.arange(B + 1, dtype=np.int32)
    dw.ctx.tc_prefill_attn(0, q, k, v, out_a, cu, grown, cur, one, scale)
    ref.ctx.tc_prefill_attn(0, q, k, v, out_b, cu, rgrown, cur, one, scale)
    torch.cuda.synchronize()
    assert torch.equal(out_a, out_b)            # the pools hold the same rows
    dw.close()
    ref.close()


@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("shape", [(1, 6, 2), (0, 40, 3)])
def test_one_captured_step_serves_a_growing_batch(alias, shape):
    """A captured step replayed over 40 tokens, with eager work and waits between replays: rows, lists, lengths and pool equal
    those of the same steps made eagerly."""
    cfg = W.scaled(W.CONFIGS["c2"], **SMALL["c2"])
    wl, dw, bt, held = _setup(cfg, alias, 60)
    _, dw2, bt2, held2 = _setup(cfg, alias, 60)
    eager, graphed = Loop(dw, bt, held, 5, 20, *shape), Loop(dw2, bt2, held2, 5, 20, *shape)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):               # a first run with no new tokens: nothing but the kernels' set-up
        graphed.step(wl.sm_scale, side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        graphed.step(wl.sm_scale, torch.cuda.current_stream())
    for step in range(40):
        new = [1, 1, 1] if step % 5 else [2, 0, 3]
        for loop in (eager, graphed):
            loop.fill(1000 + step, new)
        eager.step(wl.sm_scale)
        torch.cuda.synchronize()
        graph.replay()
        if step % 3 == 0:
            torch.randn(1000, device="cuda").sum().item()
        for name in ("seq_len", "cursor", "cu", "slot", "pos", "seq", "full", "status"):
            assert torch.equal(getattr(eager, name), getattr(graphed, name)), (step, name)
        n = sum(new)
        assert torch.equal(eager.lists[:, :n], graphed.lists[:, :n]) and torch.equal(eager.out[:, :n], graphed.out[:, :n]), step
        assert torch.equal(eager.table, graphed.table) and torch.equal(eager.digests, graphed.digests)
    dw.close()
    dw2.close()


def test_a_load_that_evicts_a_table_comes_after_the_steps_that_read_it():
    """Tables read in place by steps on two streams; unpinned, and their slots taken by loads on a third one and a fourth while
    the steps may still run.  The steps' rows are those of undisturbed steps."""
    cfg = W.scaled(W.CONFIGS["c2"], n_layers=2, n_tables=16, tables_per_query=(4, 4), capacity=8, batch=2, suffix_len=(5, 40))
    import harness as H
    wl = W.make_workload(cfg)
    wl.queries[:] = [np.array([0, 1, 2, 3], dtype=np.int32), np.array([4, 5, 6, 7], dtype=np.int32)]
    rows = []
    for disturb in (False, True):
        dw = H.DeviceWorkload(wl, seq_blocks=200, capacity=8, slot_layout=1, load_all=False)
        dw.ctx.tc_pin_tables(list(range(8)))
        dw.ctx.tc_load_async(list(range(8)), 0, cfg.n_layers, None)
        max_blocks = max(sum(-(-int(wl.table_len[t]) // 16) for t in q) for q in wl.queries) + 12
        bt, pl = dw.ctx.tc_stitch_alias(wl.table_ids, wl.cu_tables, wl.suffix_len, max_blocks)
        for layer in range(cfg.n_layers):
            dw.attn_layer(layer, bt, pl)
        held = np.asarray(pl) + wl.suffix_len
        loops = [Loop(dw, bt[i:i + 1], held[i:i + 1], 40, 8, 1, bt.shape[1], 2) for i in range(2)]
        for i, l in enumerate(loops):
            l.fill(i, [40])
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(4)]
        for l, s in zip(loops, streams):
            l.step(wl.sm_scale, s)
        if disturb:
            dw.ctx.tc_unpin_tables(list(range(8)))
            for k, t in enumerate(range(8, 16)):
                dw.ctx.tc_load_async([t], 0, cfg.n_layers, streams[2 + k % 2])
        torch.cuda.synchronize()
        rows.append([l.out.clone() for l in loops])
        dw.close()
    for a, b in zip(*rows):
        assert torch.equal(a, b)


def test_a_first_call_may_be_captured():
    """A program whose first token step is the captured one (in an interpreter of its own: kernels are set up once a process)."""
    import os
    import subprocess
    import sys
    code = """
import sys
sys.path[:0] = [%r, %r]
import numpy as np, torch
import step_harness as SH
pool = SH.Pool(28, 4, 128, "bf16", 200)
pool.fill(1)
table, digests = SH.i32(np.arange(200)[None]), pool.digests()
seq, pos, slot = SH.i32([0] * 3), SH.i32([3000, 3001, 3002]), SH.i64([3000, 3001, 3002])
q, k, v = pool.rows(3, 28, 1), pool.rows(3, 4, 2), pool.rows(3, 4, 3)
lists, ws, out, qr = SH.i32(np.zeros((3, 4, 90))), pool.workspace(3, 200, 90), torch.empty_like(q), torch.empty_like(q)
i = lambda n: SH.i32(np.zeros(n))
tables = (SH.i32([3000]), SH.i32([3]), table, SH.i32([7]), i(1), i(1), i(1), i(2), SH.i64([0] * 3), i(3), i(3), i(3), i(2))
def step():
    s = torch.cuda.current_stream()
    pool.ctx.tc_step_tables(*tables, s)
    pool.ctx.tc_rope_append(0, q, k, v, pos, 1e4, slot, qr, stream=s)
    pool.ctx.tc_digest_blocks(0, 1, table, digests, s)
    pool.ctx.tc_select_blocks(0, qr, seq, pos, table, digests, 1, 80, 9, lists, ws, s)
    pool.ctx.tc_block_attn(0, qr, seq, pos, table, lists, out, 0.1, ws, s)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step()
graph.replay()
torch.cuda.synchronize()
got = out.clone()
out.zero_()
graph.replay()
torch.cuda.synchronize()
assert torch.equal(got, out)
step()
torch.cuda.synchronize()
assert torch.equal(got, out) and torch.isfinite(out).all()
print("captured first: ok")
""" % (os.path.dirname(os.path.dirname(os.path.abspath(__file__))), os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "captured first: ok" in r.stdout, r.stdout + r.stderr


def test_a_step_that_finds_no_spare_blocks_does_nothing():
    cfg = W.scaled(W.CONFIGS["c2"], n_layers=1, n_tables=8, tables_per_query=(2, 3), capacity=8, batch=3, suffix_len=(5, 40))
    wl, dw, bt, held = _setup(cfg, False, 20)
    loop = Loop(dw, bt, held, 60, 2, 1, 4, 1)
    loop.fill(1, [20, 20, 20])
    loop.out.fill_(7.0)
    before, lens, table, digests = dw.pool.clone(), loop.seq_len.clone(), loop.table.clone(), loop.digests.clone()
    loop.step(wl.sm_scale)
    torch.cuda.synchronize()
    assert loop.status.tolist()[0] == -3 and loop.cursor.item() == 0 and loop.cu[-1].item() == 0
    assert torch.equal(before, dw.pool) and torch.equal(lens, loop.seq_len) and torch.equal(table, loop.table)
    assert torch.equal(digests, loop.digests) and (loop.out == 7.0).all() and (loop.lists == -1).all()
    dw.close()


def test_steps_on_two_streams_at_once():
    """Two batches of one context, each with its own state and workspace, on two streams: as one after the other."""
    cfg = W.scaled(W.CONFIGS["c2"], n_layers=1, n_tables=8, tables_per_query=(2, 5), capacity=8, batch=4, suffix_len=(5, 40))
    wl, dw, bt, held = _setup(cfg, False, 60)
    loops = [Loop(dw, bt[:2], held[:2], 4, 8, 1, 6, 2), Loop(dw, bt[2:], held[2:], 4, 8, 1, 6, 2)]
    torch.cuda.synchronize()
    lens = [l.seq_len.clone() for l in loops]
    results = []
    for streams in ([None, None], [torch.cuda.Stream(), torch.cuda.Stream()]):
        for i, l in enumerate(loops):
            l.seq_len.copy_(lens[i])
            l.cursor.zero_()
            l.fill(i, [2, 1])
        torch.cuda.synchronize()
        for _ in range(3):
            for l, s in zip(loops, streams):
                l.step(wl.sm_scale, s)
        torch.cuda.synchronize()
        results.append([l.out[:, :3].clone() for l in loops] + [l.lists[:, :3].clone() for l in loops])
    for a, b in zip(*results):
        assert torch.equal(a, b)
    dw.close()

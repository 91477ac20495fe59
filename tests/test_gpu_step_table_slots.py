"""Token steps over blocks of table slots (block-format slots, device entries that carry the number of unused positions) against the
plain models of oracle/steps.py, fed with the tables as they were registered: digests and lists exactly, attention to its roundings."""
import numpy as np
import pytest
import torch

import step_harness as SH
from oracle import steps as S
from paper_2601_08743_amd import workloads as W
from test_gpu_block_attn_rounding import _tolerance
from test_gpu_token_steps import Loop

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=[(28, 4), (8, 8)])
def batch(request):
    """Two sequences of three and four tables, read in place, with a suffix; and, block by block, the keys and values they are
    made of."""
    import harness as H
    hq, hkv = request.param
    cfg = W.scaled(W.CONFIGS["c2"], n_layers=2, n_q_heads=hq, n_kv_heads=hkv, n_tables=9, table_len=(33, 300), tables_per_query=(3, 4),
                   capacity=9, batch=2, suffix_len=(20, 40))
    wl = W.make_workload(cfg)
    wl.queries[:] = [np.array([5, 0, 7], dtype=np.int32), np.array([2, 8, 1, 5], dtype=np.int32)]
    lens = [int(wl.table_len[t]) for q in wl.queries for t in q]
    assert any(n % 16 for n in lens)
    dw = H.DeviceWorkload(wl, seq_blocks=60, slot_layout=1)
    bt, pl = dw.alias(96)
    suffix = [dw.attn_layer(layer, bt, pl)[1] for layer in range(2)]
    held = (np.asarray(pl) + wl.suffix_len).astype(np.int32)
    f64 = lambda x: W.storage_to_f64(np.ascontiguousarray(x), cfg.dtype)
    parts = []                                  # [layer][sequence] -> list of (K, V) [tokens][Hkv][D], a block each
    for layer in range(2):
        rows = []
        for i, q in enumerate(wl.queries):
            blocks = []
            for t in q:
                k, v = (f64(x[layer]) for x in dw.tables_np[int(t)])
                blocks += [(k[a:a + 16], v[a:a + 16]) for a in range(0, len(k), 16)]
            sl = slice(int(wl.cu_seqlens[i]), int(wl.cu_seqlens[i + 1]))
            k, v = (f64(x[sl]) for x in suffix[layer][1:])
            blocks += [(k[a:a + 16], v[a:a + 16]) for a in range(0, len(k), 16)]
            rows.append(blocks)
        parts.append(rows)
    entries = dw.ctx.tc_table_entries(bt)
    yield dw, bt, entries, held, parts
    dw.close()


def test_entries_carry_the_unused_positions(batch):
    dw, bt, entries, held, parts = batch
    for i, blocks in enumerate(parts[0]):
        n_table = sum(-(-int(dw.wl.table_len[t]) // 16) for t in dw.wl.queries[i])
        for j, (k, _) in enumerate(blocks):
            assert entries[i, j] & ((1 << SH.PAD_SHIFT) - 1) == bt[i, j]
            assert entries[i, j] >> SH.PAD_SHIFT == (16 - len(k) if j < n_table else 0)
            assert (bt[i, j] < dw.first_seq) == (j < n_table)


def _digests(dw, entries):
    B = dw.B
    buf = torch.full((B.tc_digest_bytes(dw.tc_cfg),), 99, dtype=torch.int8, device="cuda")
    dw.ctx.tc_digest_blocks(0, 2, torch.from_numpy(entries).cuda(), buf)
    torch.cuda.synchronize()
    c, n = dw.cfg, dw.tc_cfg.n_pool_blocks
    m = 2 * c.n_kv_heads * n * 2 * c.head_dim
    views = buf[:m].view(2, c.n_kv_heads, n, 2, c.head_dim), buf[m:].view(2, c.n_kv_heads, n)
    return buf, views[0].cpu().numpy(), views[1].cpu().numpy()


def test_digests_of_table_blocks(batch):
    """The zeros in a table's last block are no keys."""
    dw, bt, entries, held, parts = batch
    _, bounds, exps = _digests(dw, entries)
    for layer in range(2):
        for i, blocks in enumerate(parts[layer]):
            for j, (k, _) in enumerate(blocks):
                if j == len(blocks) - 1:
                    continue                    # (partly filled: nobody reads it)
                for h in range(dw.cfg.n_kv_heads):
                    b, e = S.digest(k[:, h])
                    np.testing.assert_array_equal(bounds[layer, h, bt[i, j]], b)
                    assert exps[layer, h, bt[i, j]] == e


@pytest.mark.parametrize("shape", [(1, 5, 2), (0, 9, 1), (2, 0, 3), (0, 96, 1)])
def test_lists_and_attention_over_table_blocks(batch, shape):
    """Tokens in the suffix, at its borders and inside the tables' part; lists whole, and by score.  A token sees the keys up to its own
    position that are in listed blocks: no unused one, and its own."""
    dw, bt, entries, held, parts = batch
    c, layer = dw.cfg, 1
    buf, _, _ = _digests(dw, entries)
    n_pre = [16 * sum(-(-int(dw.wl.table_len[t]) // 16) for t in q) for q in dw.wl.queries]
    at = [(i, p) for i in range(2) for p in (int(held[i]) - 1, n_pre[i], n_pre[i] + 15, n_pre[i] + 16, n_pre[i] - 1, 16 * 7 + 3, 0)]
    seq, pos = [i for i, _ in at], [p for _, p in at]
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q = torch.randn((len(at), c.n_q_heads, c.head_dim), generator=g, device="cuda").to(torch.bfloat16)
    n_list = sum(shape)
    lists, out = SH.i32(np.full((len(at), c.n_kv_heads, n_list), -99)), torch.full_like(q, 7.0)
    ws = torch.empty(dw.B.tc_sparse_workspace_bytes(dw.tc_cfg, len(at), bt.shape[1], n_list), dtype=torch.uint8, device="cuda")
    table, scale = torch.from_numpy(entries).cuda(), 1 / np.sqrt(c.head_dim)
    dw.ctx.tc_select_blocks(layer, q, SH.i32(seq), SH.i32(pos), table, buf, *shape, lists, ws)
    dw.ctx.tc_block_attn(layer, q, SH.i32(seq), SH.i32(pos), table, lists, out, scale, ws)
    torch.cuda.synchronize()
    G = c.n_q_heads // c.n_kv_heads
    q64, got = (x.double().cpu().numpy().reshape(len(at), c.n_kv_heads, G, -1) for x in (q, out))
    for n, (i, p) in enumerate(at):
        blocks = parts[layer][i]
        for h in range(c.n_kv_heads):
            dig = [S.digest(k[:, h]) for k, _ in blocks[:p // 16 + 1]]
            scores = S.scores(q64[n, h], np.stack([b for b, _ in dig]).astype(np.float64), np.array([e for _, e in dig]))
            want = S.block_list(p, scores.__getitem__, *shape)
            np.testing.assert_array_equal(lists[n, h].cpu().numpy(), want)
            seen = [(j, min(len(blocks[j][0]), p - 16 * j + 1)) for j in want if j >= 0]
            keys, vals = (np.concatenate([blocks[j][x][:m, h] for j, m in seen]) for x in (0, 1))
            ref, size_v, size = S.block_attn(q64[n, h], keys, vals, scale)
            assert (np.abs(got[n, h] - ref) <= _tolerance(ref, size_v, size, len(keys))).all(), (n, h)


def test_steps_over_table_blocks_row_by_row(batch):
    """Three steps with every block listed: each token's row against the model over the tables as registered, the prompt's suffix, and
    the keys of the steps themselves as the pool holds them."""
    dw, bt, entries, held, parts = batch
    c, new = dw.cfg, [3, 20]
    loop = Loop(dw, bt, held, 30, 8, 1, bt.shape[1], 2)
    cur = held.copy()
    for step in range(3):
        loop.fill(step, new)
        loop.step(dw.wl.sm_scale)
        torch.cuda.synchronize()
        assert loop.status.tolist()[0] == 0
        tab = loop.table.cpu().numpy()
        n = 0
        for i in range(2):
            n_pre = 16 * sum(-(-int(dw.wl.table_len[t]) // 16) for t in dw.wl.queries[i])
            first, end = n_pre // 16, int(cur[i]) + new[i]
            ids = [int(e) for e in tab[i, first:(end + 15) // 16]]
            for layer in range(2):
                kk, vv = (W.storage_to_f64(x, c.dtype) for x in dw.ctx.tc_read_seq_kv(layer, ids, end - n_pre, np.uint16))
                keys, vals = (np.concatenate([b[x] for b in parts[layer][i][:first]] + [y]) for x, y in ((0, kk), (1, vv)))
                tail = sum(len(b[0]) for b in parts[layer][i][:first])
                qr, out = (x[layer, n:n + new[i]].double().cpu().numpy().reshape(new[i], c.n_kv_heads, -1, c.head_dim) for x in (loop.qr, loop.out))
                for r in range(new[i]):
                    m = tail + int(cur[i]) + r + 1 - n_pre
                    for h in range(c.n_kv_heads):
                        ref, size_v, size = S.block_attn(qr[r, h], keys[:m, h], vals[:m, h], dw.wl.sm_scale)
                        assert (np.abs(out[r, h] - ref) <= _tolerance(ref, size_v, size, m)).all(), (step, i, layer, r, h)
            n += new[i]
        cur = cur + new


@pytest.mark.parametrize("hq,hkv,d,dtype", [(32, 8, 128, "bf16"), (28, 4, 128, "bf16"), (8, 2, 64, "f32")])
def test_one_workspace_against_the_model(hq, hkv, d, dtype):
    """A workspace of a large step for any number of tokens: each against the model, however its lists are shared out."""
    pool = SH.Pool(hq, hkv, d, dtype, 120)
    pool.fill(5)
    rng = np.random.default_rng(1)
    lists = np.stack([np.stack([np.sort(rng.permutation(119)[:100]) for _ in range(hkv)]) for _ in range(12)])
    pos = rng.integers(16 * 119, 16 * 120, size=12)
    table, q = SH.i32(np.arange(120)[None]), pool.rows(12, hq, 3)
    ws = pool.workspace(12, 120, 100)
    k64, v64 = pool.kv64()
    q64 = q.double().cpu().numpy().reshape(12, hkv, -1, d)
    scale = 1 / np.sqrt(d)
    want = [[S.block_attn(q64[n, h], *(x[0, lists[n, h], h].reshape(-1, d) for x in (k64, v64)), scale) for h in range(hkv)] for n in range(12)]
    for n in (12, 7, 4, 2, 1):
        out = torch.full_like(q[:n], 7.0)
        pool.ctx.tc_block_attn(0, q[:n], SH.i32([0] * n), SH.i32(pos[:n]), table, SH.i32(lists[:n]), out, scale, ws)
        torch.cuda.synchronize()
        got = out.double().cpu().numpy().reshape(n, hkv, -1, d)
        for i in range(n):
            for h in range(hkv):
                ref, size_v, size = want[i][h]
                tol = _tolerance(ref, size_v, size, 1600) if dtype == "bf16" else SH.attn_tolerance(ref, size_v, size, False, 1600)
                assert (np.abs(got[i, h] - ref) <= tol).all(), (n, i, h)
    pool.close()

"""Loads into table slots that are still being read: whatever stream a slot's new rows come on, and however the loads are cut, they come
behind the reads of its last occupant."""
import numpy as np
import pytest
import torch

import harness as H
import step_harness as SH
from paper_2601_08743_amd import workloads as W

pytestmark = pytest.mark.gpu


class Busy:
    """Some tens of milliseconds of work for a stream."""

    def __init__(self):
        self.a, self.b = torch.randn((6144, 6144), device="cuda"), torch.empty((6144, 6144), device="cuda")
        torch.mm(self.a, self.a, out=self.b)
        torch.cuda.synchronize()

    def on(self, stream, times=12):
        with torch.cuda.stream(stream):
            for _ in range(times):
                torch.mm(self.a, self.a, out=self.b)


def _resident(n_tables, capacity, blocks):
    cfg = W.scaled(W.CONFIGS["c2"], n_layers=2, n_tables=n_tables, tables_per_query=(2, 2), capacity=capacity, batch=1, suffix_len=(5, 40))
    wl = W.make_workload(cfg)
    wl.queries[:] = [np.array([0, 1], dtype=np.int32)]
    dw = H.DeviceWorkload(wl, seq_blocks=200, capacity=capacity, slot_layout=int(blocks), load_all=False)
    dw.ctx.tc_load_async(list(range(capacity)), 0, cfg.n_layers, None)
    torch.cuda.synchronize()
    return wl, dw


def _step_arrays(dw, wl, bt, pl):
    c, n_list = dw.cfg, bt.shape[1]
    pos = int(pl[0]) - 1
    rng = torch.Generator(device="cuda")
    rng.manual_seed(4)
    q = torch.randn((1, c.n_q_heads, c.head_dim), generator=rng, device="cuda").to(torch.bfloat16)
    return dict(q=q, seq=SH.i32([0]), pos=SH.i32([pos]), table=torch.from_numpy(dw.ctx.tc_table_entries(bt)).cuda(),
                lists=SH.i32(np.tile(np.arange(n_list), (1, c.n_kv_heads, 1))), out=torch.full_like(q, 7.0),
                ws=torch.empty(dw.B.tc_sparse_workspace_bytes(dw.tc_cfg, 1, n_list, n_list), dtype=torch.uint8, device="cuda"))


def _attend(dw, s, stream):
    dw.ctx.tc_block_attn(1, s["q"], s["seq"], s["pos"], s["table"], s["lists"], s["out"], 0.1, s["ws"], stream)


# the second load: of the table whose slot the empty one took (a hit), or of another one, which takes another slot
@pytest.mark.parametrize("second", ["same", "other"])
def test_a_load_of_no_layers_keeps_the_order_behind_steps(second):
    """The slots of two tables that a step reads in place go to others, the first of them by a load of an empty layer range
    on a stream of its own."""
    busy, outs = Busy(), []
    for disturb in (False, True):
        wl, dw = _resident(8, 4, True)
        bt, pl = dw.ctx.tc_stitch_alias(wl.table_ids, wl.cu_tables, wl.suffix_len, 40 + 4 * dw.slot_blocks)
        s = _step_arrays(dw, wl, bt, pl)
        torch.cuda.synchronize()
        reads, empty, copies = (torch.cuda.Stream() for _ in range(3))
        busy.on(reads)
        _attend(dw, s, reads)
        read = torch.cuda.Event()
        read.record(reads)
        if disturb:
            dw.ctx.tc_load_async([4], 0, 0, empty)
            dw.ctx.tc_load_async([4 if second == "same" else 5], 0, wl.cfg.n_layers, copies)
            copies.synchronize()
            assert read.query()                 # (else the rows could have come while the step was reading)
        torch.cuda.synchronize()
        outs.append(s["out"].clone())
        dw.close()
    assert torch.equal(outs[0], outs[1]) and not (outs[0] == 7.0).any()


@pytest.mark.parametrize("second", ["same", "other"])
def test_a_load_of_no_layers_keeps_the_order_behind_dense_attention(second):
    """The same with tc_prefill_attn reading the slots."""
    busy = Busy()
    wl, dw = _resident(8, 4, True)
    bt, pl = dw.ctx.tc_stitch_alias(wl.table_ids, wl.cu_tables, wl.suffix_len, 40 + 4 * dw.slot_blocks)
    q, k, v = (H.to_dev(x, dw.cfg) for x in wl.suffix_qkv(0))
    out, reads, empty, copies = torch.empty_like(q), *(torch.cuda.Stream() for _ in range(3))
    torch.cuda.synchronize()
    busy.on(reads)
    dw.ctx.tc_prefill_attn(0, q, k, v, out, wl.cu_seqlens, bt, pl, wl.suffix_len, wl.sm_scale, reads)
    read = torch.cuda.Event()
    read.record(reads)
    dw.ctx.tc_load_async([4], 1, 1, empty)
    dw.ctx.tc_load_async([4 if second == "same" else 5], 0, wl.cfg.n_layers, copies)
    copies.synchronize()
    assert read.query()
    dw.close()


def test_a_load_of_no_layers_keeps_the_order_behind_a_stitch():
    """Slots of rows: a table takes the slot that a stitch reads in an empty range, and its layers come on another stream."""
    busy = Busy()
    wl, dw = _resident(4, 2, False)
    reads, empty, copies = (torch.cuda.Stream() for _ in range(3))
    busy.on(reads)
    bt, pl = dw.stitch(stream=reads)
    read = torch.cuda.Event()
    read.record(reads)
    dw.ctx.tc_load_async([2], 0, 0, empty)
    dw.ctx.tc_load_async([2], 0, wl.cfg.n_layers, copies)
    copies.synchronize()
    assert read.query()
    torch.cuda.synchronize()
    # the sequence holds the tables that were there
    P = int(pl[0])
    for layer in range(wl.cfg.n_layers):
        got, _ = dw.ctx.tc_read_seq_kv(layer, [int(b) for b in bt[0, :(P + 15) // 16]], P, np.uint16)
        want, _ = H.oracle_sequences(wl, dw.tables_np, layer, 0)
        np.testing.assert_array_equal(got, want)
    dw.close()


def test_layers_of_a_table_on_two_streams_are_all_there_for_a_stitch():
    """A stitch waits for the last load of a table; that of the other layers, on another stream, comes before it."""
    busy = Busy()
    wl, dw = _resident(4, 2, False)
    first, second, third = (torch.cuda.Stream() for _ in range(3))
    wl.queries[:] = [np.array([2, 3], dtype=np.int32)]
    busy.on(first)
    dw.ctx.tc_load_async([2, 3], 0, 1, first)
    dw.ctx.tc_load_async([2, 3], 1, 2, second)
    bt, pl = dw.ctx.tc_stitch_kv([2, 3], [0, 2], wl.suffix_len, 40 + 4 * dw.slot_blocks, third)
    torch.cuda.synchronize()
    P = int(pl[0])
    for layer in range(2):
        got, _ = dw.ctx.tc_read_seq_kv(layer, [int(b) for b in bt[0, :(P + 15) // 16]], P, np.uint16)
        want, _ = H.oracle_sequences(wl, dw.tables_np, layer, 0)
        np.testing.assert_array_equal(got, want)
    dw.close()


def test_steps_on_many_streams_do_not_make_a_load_wait_on_the_host():
    """Steps on the default stream and 32 others, one of them behind long work: the load that takes a slot returns while that runs, and
    its rows come behind all of them."""
    busy = Busy()
    wl, dw = _resident(8, 4, True)
    bt, pl = dw.ctx.tc_stitch_alias(wl.table_ids, wl.cu_tables, wl.suffix_len, 40 + 4 * dw.slot_blocks)
    streams = [torch.cuda.default_stream()] + [torch.cuda.Stream() for _ in range(32)]
    assert len({s.cuda_stream for s in streams}) == 33
    steps = [_step_arrays(dw, wl, bt, pl) for _ in streams]
    _attend(dw, steps[0], streams[0])           # (what a first call sets up)
    torch.cuda.synchronize()
    busy.on(streams[7], 40)
    done = []
    for st, s in zip(streams, steps):
        _attend(dw, s, st)
        done.append(torch.cuda.Event())
        done[-1].record(st)
    dw.ctx.tc_load_async([4], 0, wl.cfg.n_layers, streams[20])
    assert not done[7].query()
    streams[20].synchronize()
    assert all(e.query() for e in done)
    for s in steps[1:]:
        assert torch.equal(s["out"], steps[0]["out"])
    dw.close()

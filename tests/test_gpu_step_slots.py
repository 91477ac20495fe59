"""Steps that take ids of no sequence block: the status says so, and the tokens that fall into them are none - no call makes anything of
their rows."""
import numpy as np
import pytest
import torch

import step_harness as SH
from oracle import steps as S

pytestmark = pytest.mark.gpu
OUT = ("spare_next", "end_len", "cu_new", "slot_map", "token_pos", "token_seq", "full_block", "status")


@pytest.fixture(scope="module")
def pool():
    p = SH.Pool(8, 2, 64, "f32", 400, slot_blocks=3)
    p.fill(3)
    yield p
    p.close()


def _step(pool, held, new, table, spare, used, n_tokens, in_place):
    a = dict(seq_len=SH.i32(held), new_len=SH.i32(new), table=SH.i32(table), spare=SH.i32(spare), used=SH.i32([used]))
    o = dict(spare_next=SH.i32([-77]), end_len=SH.i32(np.full(len(held), -77)), cu_new=SH.i32(np.full(len(held) + 1, -77)),
             slot_map=SH.i64(np.full(n_tokens, -77)), **{k: SH.i32(np.full(n_tokens, -77)) for k in ("token_pos", "token_seq", "full_block")},
             status=SH.i32([-77, -77]))
    if in_place:
        o["end_len"], o["spare_next"] = a["seq_len"], a["used"]
    pool.ctx.tc_step_tables(a["seq_len"], a["new_len"], a["table"], a["spare"], a["used"], *(o[k] for k in OUT))
    torch.cuda.synchronize()
    return o, a["table"]


# one work-group; several that take their inputs' place or not
@pytest.mark.parametrize("n_tokens", [60, 2048, 2049, 20000])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("bad", ["none", "spare_beyond", "spare_of_a_slot", "spare_negative", "spare_not_taken", "partial_missing",
                                 "partial_of_a_slot", "partial_beyond", "partial_of_a_waiting_request"])
def test_status_says_where_tokens_have_no_slot(pool, n_tokens, in_place, bad):
    B = 300 if n_tokens > 2048 else 5
    rng = np.random.default_rng(n_tokens)
    held = rng.integers(0, 60, size=B)
    new = rng.integers(0, min(60, n_tokens // B) + 1, size=B)
    held[3], new[3] = 21, 5                     # goes on in block 1 of its own
    held[4], new[4] = 37, 0                     # waits
    table = np.where(np.arange(10)[None] < (held[:, None] + 15) // 16, rng.integers(3, 400, size=(B, 10)), -1)
    taken = int(((held + new + 15) // 16 - (held + 15) // 16).sum())
    spare, used = rng.integers(3, 400, size=taken + 9), 4
    at = used + taken // 2
    if bad == "spare_beyond":
        spare[at] = 400
    elif bad == "spare_of_a_slot":
        spare[at] = 2
    elif bad == "spare_negative":
        spare[at] = -1
    elif bad == "spare_not_taken":
        spare[[used - 1, used + taken]] = -1
    elif bad == "partial_missing":
        table[3, 1] = -1
    elif bad == "partial_of_a_slot":
        table[3, 1] = 2
    elif bad == "partial_beyond":
        table[3, 1] = 400
    elif bad == "partial_of_a_waiting_request":
        table[4, 2] = -1
    want = S.step_tables(held, new, table, spare, used, n_tokens, pool.first, pool.n)
    got, tab = _step(pool, held, new, table, spare, used, n_tokens, in_place)
    for k in OUT:
        np.testing.assert_array_equal(got[k].cpu().numpy(), np.asarray(want[k]).reshape(got[k].shape), err_msg=k)
    np.testing.assert_array_equal(tab.cpu().numpy(), want["table"])
    assert want["status"][0] == int(bad not in ("none", "spare_not_taken", "partial_of_a_waiting_request"))
    slots, total = np.asarray(want["slot_map"]), int(new.sum())
    assert ((slots[:total] < 0).any()) == bool(want["status"][0]) and (np.asarray(want["token_seq"])[slots < 0] == -1).all()


def test_rows_without_a_slot_are_passed_over_by_every_call(pool):
    """A request whose new block is none, beside one that is whole: its rows of q_out, lists and outputs stay, the other's are as in
    a step of its own."""
    held, new, n = [16, 20], [3, 2], 6
    o, table = _step(pool, held, new, np.array([[5, -1, -1], [7, 9, -1]]), np.array([400, 30]), 0, n, False)
    assert o["status"].tolist() == [1, 1] and o["slot_map"][:3].tolist() == [-1] * 3 and o["cu_new"].tolist() == [0, 3, 5]
    q, k, v = pool.rows(n, 8, 1), pool.rows(n, 2, 2), pool.rows(n, 2, 3)
    qr, out = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    lists, ws = SH.i32(np.full((n, 2, 3), -99)), pool.workspace(n, 3, 3)
    digests = pool.digests()
    pool.ctx.tc_rope_append(0, q, k, v, o["token_pos"], 1e4, o["slot_map"], qr)
    pool.ctx.tc_digest_blocks(0, 1, table, digests)
    pool.ctx.tc_select_blocks(0, qr, o["token_seq"], o["token_pos"], table, digests, 1, 1, 1, lists, ws)
    pool.ctx.tc_block_attn(0, qr, o["token_seq"], o["token_pos"], table, lists, out, 0.1, ws)
    torch.cuda.synchronize()
    rest = [0, 1, 2, 5]
    assert (qr[rest] == 7.0).all() and (out[rest] == 7.0).all() and (lists[rest] == -99).all()
    assert (lists[3:5] == SH.i32([0, 1, -1])).all()
    k64, v64 = pool.kv64()
    q64 = qr.double().cpu().numpy()
    for i, p in ((3, 20), (4, 21)):
        for h in range(2):
            keys, vals = (np.concatenate([x[0, 4, h], x[0, 6, h, :p - 15]]) for x in (k64, v64))
            ref, size_v, size = S.block_attn(q64[i, 4 * h:4 * h + 4], keys, vals, 0.1)
            got = out[i, 4 * h:4 * h + 4].double().cpu().numpy()
            assert (np.abs(got - ref) <= SH.attn_tolerance(ref, size_v, size, False, len(keys))).all()

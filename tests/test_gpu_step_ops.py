"""Block tables from lengths, encoded append and digests (tc_step_tables, tc_rope_append, tc_digest_blocks) against the plain
models of oracle/steps.py.  Integers exactly; encoded rows to the rounding of one result and the arithmetic before it."""
import numpy as np
import pytest
import torch

import step_harness as SH
from oracle import steps as S

pytestmark = pytest.mark.gpu
OUT = ("spare_next", "end_len", "cu_new", "slot_map", "token_pos", "token_seq", "full_block", "status")


# ------------------------------------------------------------------------------------------------ tables

def _step(pool, seq_len, new_len, table, spare, used, n_tokens, in_place=False):
    """The call's arrays as numpy, outputs poisoned before it."""
    B = len(seq_len)
    a = dict(seq_len=SH.i32(seq_len), new_len=SH.i32(new_len), table=SH.i32(table), spare=SH.i32(spare),
             spare_used=SH.i32([used]))
    o = dict(spare_next=SH.i32([-77]), end_len=SH.i32(np.full(B, -77)), cu_new=SH.i32(np.full(B + 1, -77)),
             slot_map=SH.i64(np.full(n_tokens, -77)), **{k: SH.i32(np.full(n_tokens, -77)) for k in ("token_pos", "token_seq", "full_block")},
             status=SH.i32([-77, -77]))
    if in_place:
        o["end_len"], o["spare_next"] = a["seq_len"], a["spare_used"]
    pool.ctx.tc_step_tables(a["seq_len"], a["new_len"], a["table"], a["spare"], a["spare_used"], *(o[k] for k in OUT))
    torch.cuda.synchronize()
    return dict({k: o[k].cpu().numpy() for k in OUT}, table=a["table"].cpu().numpy())


def _check_step(pool, seq_len, new_len, max_blocks, spare, used, n_tokens, in_place=False, table=None):
    rng = np.random.default_rng(len(seq_len) * 131 + n_tokens)
    if table is None:
        table = np.full((len(seq_len), max_blocks), -1)
        for b, l in enumerate(seq_len):
            have = min(max_blocks, max(0, (int(l) + 15) // 16))
            table[b, :have] = rng.integers(pool.first, pool.n, size=have)
    want = S.step_tables(seq_len, new_len, table, spare, used, n_tokens, pool.first, pool.n)
    got = _step(pool, seq_len, new_len, table, spare, used, n_tokens, in_place)
    for k in OUT + ("table",):
        np.testing.assert_array_equal(got[k], np.asarray(want[k]).reshape(got[k].shape), err_msg=k)
    return got


@pytest.fixture(scope="module")
def small_pool():
    p = SH.Pool(8, 2, 64, "f32", 400, slot_blocks=3)
    yield p
    p.close()


@pytest.mark.parametrize("seq_len,new_len,n_tokens", [
    ([0], [1], 1), ([15], [1], 1), ([16], [1], 4), ([31], [2], 2), ([0], [0], 0), ([5], [0], 3), ([], [], 0), ([], [], 5),
    ([0, 0, 0], [0, 7, 0], 7), ([3, 16, 0, 47, 48], [1, 1, 33, 1, 1], 37), ([100, 0, 20], [0, 160, 12], 180),
    ([7] * 70, [1] * 70, 77)])
@pytest.mark.parametrize("in_place", [False, True])
def test_tables_of_small_steps(small_pool, seq_len, new_len, n_tokens, in_place):
    spare = np.random.default_rng(3).permutation(np.arange(3, 400))[:40]
    got = _check_step(small_pool, seq_len, new_len, 20, spare, 2, n_tokens, in_place)
    assert got["status"][0] == 0


@pytest.mark.parametrize("B,n_tokens,most", [(256, 1024, 4), (257, 1024, 4), (300, 8192, 50), (300, 8193, 50), (1500, 9000, 9),
                                             (8192, 8192, 1), (3, 30000, 9000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_tables_of_large_steps(small_pool, B, n_tokens, most, in_place):
    """One work-group and many, requests in several rounds, every third request waiting."""
    rng = np.random.default_rng(B + n_tokens)
    new = np.where(np.arange(B) % 3 == 1, 0, rng.integers(0, most + 1, size=B))
    assert new.sum() <= n_tokens
    held = rng.integers(0, 700, size=B)
    spare = rng.integers(3, 400, size=int((most // 16 + 1) * B + 5))
    got = _check_step(small_pool, held, new, (700 + most) // 16 + 2, spare, 4, n_tokens, in_place)
    assert got["status"][0] == 0


@pytest.mark.parametrize("n_tokens", [64, 9000])
@pytest.mark.parametrize("seq_len,new_len,used,spare,code", [
    ([10, 20], [10, 30], 0, 2, -3),            # three blocks wanted, two there
    ([10, 20], [10, 30], 3, 5, -3),            # .. two left
    ([10, -1], [1, 1], 0, 9, -1), ([10, 3], [1, -1], 0, 9, -1),
    ([10, 300], [1, 21], 0, 99, -1),           # ends at 321 > 320
    ([10, 300], [1, 20], 0, 99, 0),
    ([0, 0], [9000, 9000], 0, 99, -1), ([0, 2147483647], [1, 2147483647], 0, 9, -1),
    ([1, 1], [1, 1], -1, 9, -1), ([1, 1], [1, 1], 10, 9, -1), ([1, 1], [1, 1], 9, 9, 0)])
def test_steps_that_cannot_be_made_change_nothing(small_pool, seq_len, new_len, used, spare, code, n_tokens):
    for in_place in (False, True):
        got = _check_step(small_pool, seq_len, new_len, 20, np.arange(3, 3 + spare), used, n_tokens, in_place)
        assert got["status"][0] == code


def test_entries_that_are_no_blocks_give_no_slots(small_pool):
    """Spare ids beyond the pool or of a table slot, a missing entry under the partial last block, unused-position counts."""
    table = np.array([[5, -1, -1, -1], [7, -1, -1, -1], [9 | (3 << 27), 11, -1, -1]])
    got = _check_step(small_pool, [16, 20, 17], [33, 2, 1], 4, np.array([2, 400, 8, -5]), 0, 40, table=table)
    assert (got["slot_map"][:32] == -1).all() and got["table"][0].tolist() == [5, -1, -1, 8]


# ------------------------------------------------------------------------------------------------ encode and append

def _append_case(hq, hkv, d, dtype, slots, pos, sections, theta, fused, in_place=False, slot_blocks=0, n_blocks=12, layers=2, layer=1):
    pool = SH.Pool(hq, hkv, d, dtype, n_blocks, layers, slot_blocks)
    n = len(slots)
    if fused:
        rows = pool.rows(n, hq + 2 * hkv + 1, 5)
        q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:hq + 2 * hkv]
    else:
        q, k, v = pool.rows(n, hq, 5), pool.rows(n, hkv, 6), pool.rows(n, hkv, 7)
    q64, k64, v64 = (x.double().cpu().numpy() for x in (q, k, v))
    before = pool.raw.clone()
    q_out = q if in_place else torch.full((n, hq, d), float("nan"), dtype=pool.dt, device="cuda")
    pool.ctx.tc_rope_append(layer, q, k, v, SH.i32(pos), theta, SH.i64(slots), q_out, sections)
    torch.cuda.synchronize()

    pos2 = np.asarray(pos).reshape(-1, n)
    sec = [d // 2] if sections is None else sections
    want_q, want_k = S.rotate(q64, pos2, sec, theta), S.rotate(k64, pos2, sec, theta)

    def close(got, want, x):
        half = d // 2
        rad = np.sqrt(x[..., :half] ** 2 + x[..., half:] ** 2)
        # one rounding of the result, and fp32 sine, cosine, products and sum: 2e-6 of the pair's radius (test_gpu_reencode)
        tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want) + 2e-6 * np.concatenate([rad, rad], -1) + 1e-30
        assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) - tol).max())

    kk, vv = pool.kv64()
    live = [i for i, s in enumerate(slots) if s >= 0 and slot_blocks <= s // 16 < n_blocks]
    touched = np.zeros(kk.shape[1] * 16, dtype=bool)
    q_got = q_out.double().cpu().numpy()
    for i in range(n):
        if i not in live:
            if in_place:
                np.testing.assert_array_equal(q_got[i], q64[i])
            else:
                assert np.isnan(q_got[i]).all()
    close(q_got[live], want_q[live], q64[live])
    for i in live:
        b, t = slots[i] // 16 - slot_blocks, slots[i] % 16
        close(kk[layer, b, :, t][None], want_k[i][None], k64[i][None])
        np.testing.assert_array_equal(vv[layer, b, :, t], v64[i])
        touched[b * 16 + t] = True
    for i in live:                              # blocks begun here: zeros behind what was written
        b, t = slots[i] // 16 - slot_blocks, slots[i] % 16
        if t == 0:
            run = 1
            while run < 16 and i + run < n and slots[i + run] == slots[i] + run:
                run += 1
            assert (kk[layer, b, :, run:] == 0).all() and (vv[layer, b, :, run:] == 0).all()
            touched[b * 16:b * 16 + 16] = True
    # everything else as it was
    clean = pool.raw.clone()
    pool.raw.copy_(before)
    k0, v0 = pool.kv()
    kn, vn = k0.clone(), v0.clone()
    pool.raw.copy_(clean)
    k1, v1 = pool.kv()
    rest = torch.from_numpy(~touched).cuda().view(-1, 16)
    for was, now in ((kn, k1), (vn, v1)):
        same = (was.nan_to_num(7.5) == now.nan_to_num(7.5)).all(-1).all(2)                    # [layers][blocks][16]
        same[layer] |= ~rest
        assert same.all()
    pool.close()


SHAPES = [(8, 2, 64, "f32"), (8, 2, 128, "f32"), (28, 4, 128, "bf16"), (5, 1, 128, "bf16"), (3, 3, 128, "bf16")]


@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_append_one_token(hq, hkv, d, dtype):
    _append_case(hq, hkv, d, dtype, [35], [4711], None, 1e6, False)
    _append_case(hq, hkv, d, dtype, [48], [0], None, 1e4, False, in_place=True)


@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
@pytest.mark.parametrize("axes", [1, 3])
@pytest.mark.parametrize("fused", [False, True])
def test_append_ragged_runs(hq, hkv, d, dtype, axes, fused):
    """Runs that begin inside a block, fill it, go on in another one, one token of a block, padded rows, slots of no sequence block."""
    slots = list(range(16 * 5 + 9, 16 * 6)) + list(range(16 * 3, 16 * 4)) + list(range(16 * 9, 16 * 9 + 5)) + [-1, 16 * 2 + 7, -1] + \
        [16 * 12, 5, 16 * 400 + 3, -(1 << 40), 1 << 40] + [16 * 11 + 15, 16 * 10] + [-1]
    rng = np.random.default_rng(8)
    pos = rng.integers(0, 1 << 17, size=(axes, len(slots)))
    sections = None if axes == 1 else ([16, 24, 24] if d == 128 else [8, 12, 12])
    _append_case(hq, hkv, d, dtype, slots, pos[0] if axes == 1 else pos, sections, 1e6, fused, slot_blocks=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_far_and_negative_positions_and_empty_sections(dtype):
    pos = np.array([[0, 1, 1 << 27, -5, 99999], [3, 1 << 27, 7, 8, -9], [1, 2, 3, 4, 5], [6, 1 << 27, 0, 9, 4]])
    _append_case(4, 2, 128, dtype, [3, 17, 16 * 4, 16 * 4 + 1, 16 * 7 + 15], pos, [0, 33, 0, 31], 1e4, False)


def test_append_many_tokens():
    """Long suffixes of three sequences, blocks in mixed order: every token in its slot."""
    rng = np.random.default_rng(17)
    blocks = rng.permutation(90)
    slots = [int(blocks[p // 16]) * 16 + p % 16 for p in range(5, 700)]
    slots += [int(blocks[44 + p // 16]) * 16 + p % 16 for p in range(16, 500)]
    slots += [int(blocks[76 + p // 16]) * 16 + p % 16 for p in range(0, 33)]
    _append_case(8, 2, 128, "bf16", slots, rng.integers(0, 30000, size=len(slots)), None, 1e6, True, n_blocks=90, layers=1, layer=0)
    _append_case(8, 2, 64, "f32", slots, rng.integers(0, 30000, size=len(slots)), None, 1e6, True, n_blocks=90, layers=1, layer=0)


# ------------------------------------------------------------------------------------------------ digests

@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_digests_are_the_definition(hq, hkv, d, dtype):
    pool = SH.Pool(hq, hkv, d, dtype, 40, layers=3, slot_blocks=2)
    pool.fill(3)
    k, v = (x.clone() for x in pool.kv())
    k[:, 4] = 0
    k[:, 5] *= 1e-39 if dtype == "f32" else 1e-38                  # subnormal keys
    k[:, 6] *= 1e37
    k[:, 7, :, 3, 5] = float("inf")
    k[:, 8, :, 15, 0] = float("nan")
    k[:, 9, 0, 0, 1] = -float("inf")
    k[:, 10] = 127.0 * 2.0 ** -3                                   # the exponent's edge, and the next number above it
    k[:, 11] = 127.5 if dtype == "f32" else 127.5
    k[:, 12] = -128.0
    k[:, 13, :, 9:] = float("nan")                                 # unused positions of a table block
    k[:, 14] = -k[:, 14].abs()                                     # one sign only
    pool.put(k, v)
    ids = np.arange(2, 40)
    entries = ids.copy()
    entries[13] |= 7 << SH.PAD_SHIFT
    entries[20] |= 15 << SH.PAD_SHIFT
    listed = np.concatenate([entries[:37], [-1, entries[5], 40, 1, 0, (1 << 27) - 1]])        # block 39 is not listed
    buf = pool.digests()
    pool.ctx.tc_digest_blocks(1, 3, SH.i32(listed).view(-1, 1), buf)
    torch.cuda.synchronize()
    bounds, exps = (x.cpu().numpy() for x in pool.digest_views(buf))
    k64, _ = pool.kv64()
    assert (bounds[0] == 99).all() and (exps[0] == 99).all()       # layer 0 not asked for
    assert (bounds[:, :, [0, 1, 39]] == 99).all() and (exps[:, :, [0, 1, 39]] == 99).all()
    for layer in (1, 2):
        for i, entry in enumerate(entries[:37]):
            n = 16 - (int(entry) >> SH.PAD_SHIFT)
            for h in range(hkv):
                b, e = S.digest(k64[layer, i, h, :n])
                np.testing.assert_array_equal(bounds[layer, h, ids[i]], b, err_msg="layer %d block %d" % (layer, ids[i]))
                assert exps[layer, h, ids[i]] == e
    pool.close()


def test_digests_of_a_table_that_is_mostly_empty():
    """More rows than one launch takes, nearly all of them -1."""
    pool = SH.Pool(8, 8, 128, "bf16", 6)
    pool.fill(3)
    n = (1 << 23) + 20
    entries = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    for at, block in ((0, 4), ((1 << 23) - 2, 0), ((1 << 23) + 1, 5), (n - 1, 2)):
        entries[at] = block
    buf = pool.digests()
    pool.ctx.tc_digest_blocks(0, 1, entries, buf)
    whole = pool.digests()
    pool.ctx.tc_digest_blocks(0, 1, SH.i32([0, 2, 4, 5]), whole)
    torch.cuda.synchronize()
    assert torch.equal(buf, whole)
    pool.close()


# ------------------------------------------------------------------------------------------------ refusals

def test_refusals(small_pool):
    from paper_2601_08743_amd import binding as B
    p, c = small_pool, small_pool.ctx
    one, i8 = SH.i32([1]), torch.zeros(B.tc_digest_bytes(p.cfg), dtype=torch.int8, device="cuda")
    q, kv, slot = p.rows(1, 8, 1), p.rows(1, 2, 2), SH.i64([16 * 5])

    def refused(f, code=B.TC_ERR_INVALID):
        with pytest.raises(B.TcError) as e:
            f()
        assert e.value.code == code, e.value

    def append(layer=0, q=q, k=kv, v=kv, pos=one, theta=1e4, slot=slot, out=q, sections=None):
        c.tc_rope_append(layer, q, k, v, pos, theta, slot, out, sections)

    append()
    refused(lambda: append(layer=1))
    refused(lambda: append(layer=-1))
    for theta in (1.0, 0.5, float("inf"), float("nan")):
        refused(lambda: append(theta=theta))
    refused(lambda: append(sections=[31]))
    refused(lambda: append(sections=[16, 16]))                                      # one axis of positions
    refused(lambda: append(pos=SH.i32([[1], [1]])))                                 # two axes, no sections
    refused(lambda: append(pos=SH.i32([[1], [1]]), sections=[40, -8]))
    refused(lambda: append(pos=SH.i32([[1]] * 5), sections=[8, 8, 8, 4, 4]))
    refused(lambda: append(q=q.bfloat16()))
    refused(lambda: append(k=p.rows(1, 3, 2)))
    refused(lambda: append(slot=SH.i32([80])))
    refused(lambda: append(pos=SH.i32([1, 2])))
    refused(lambda: append(pos=one.cpu()))
    wide = torch.zeros((2, 2, 66), device="cuda")
    two = dict(q=p.rows(2, 8, 1), pos=SH.i32([1, 2]), slot=SH.i64([80, 81]), out=p.rows(2, 8, 1))
    refused(lambda: append(k=wide[..., :64], v=p.rows(2, 2, 1), **two))             # heads apart
    refused(lambda: append(k=torch.zeros((1, 2, 64), device="cuda").expand(2, 2, 64), v=p.rows(2, 2, 1), **two))
    off = torch.zeros(2 * 131, device="cuda").as_strided((2, 2, 64), (131, 64, 1))  # rows not at 16 bytes
    refused(lambda: append(k=off, v=p.rows(2, 2, 1), **two))

    refused(lambda: c.tc_digest_blocks(0, 2, one, i8))
    refused(lambda: c.tc_digest_blocks(1, 0, one, i8))
    refused(lambda: c.tc_digest_blocks(0, 1, one, i8[:-1]))
    refused(lambda: c.tc_digest_blocks(0, 1, one.long(), i8))
    c.tc_digest_blocks(0, 1, SH.i32([]), i8)
    c.tc_digest_blocks(0, 0, one, i8)

    def tables(seq=one, table=SH.i32([[5, -1]]), n=1, **kw):
        a = dict(spare=one, spare_used=SH.i32([0]), spare_next=SH.i32([0]), end_len=SH.i32([0]), cu_new=SH.i32([0, 0]), slot_map=SH.i64([0] * n),
                 token_pos=SH.i32([0] * n), token_seq=SH.i32([0] * n), full_block=SH.i32([0] * n), status=SH.i32([0, 0]))
        a.update(kw)
        c.tc_step_tables(seq, one, table, *a.values())

    tables()
    refused(lambda: tables(cu_new=SH.i32([0])))
    refused(lambda: tables(status=SH.i32([0])))
    refused(lambda: tables(token_pos=SH.i64([0])))
    refused(lambda: tables(seq=SH.i32([1, 2])))
    refused(lambda: tables(full_block=SH.i32([0, 0])))
    many = 8193
    refused(lambda: c.tc_step_tables(SH.i32([1] * many), SH.i32([1] * many), SH.i32([[5]] * many), one, SH.i32([0]), SH.i32([0]),
                                     SH.i32([0] * many), SH.i32([0] * (many + 1)), SH.i64([0]), SH.i32([0]), SH.i32([0]), SH.i32([0]), SH.i32([0, 0])))
    torch.cuda.synchronize()


def test_table_entries(small_pool):
    c = small_pool.ctx
    got = c.tc_table_entries(np.array([[3, 399, -1], [-1, 7, 3]]))
    np.testing.assert_array_equal(got, [[3, 399, -1], [-1, 7, 3]])
    from paper_2601_08743_amd import binding as B
    for bad in (400, 2, 0):
        with pytest.raises(B.TcError) as e:
            c.tc_table_entries(np.array([5, bad]))
        assert e.value.code == B.TC_ERR_INVALID


def test_encoded_queries_do_not_overwrite_rows_still_to_be_read(small_pool):
    from paper_2601_08743_amd import binding as B
    p = small_pool
    wide = p.rows(2, 12, 1)                                                         # queries and keys of one projection
    q, kv, out = wide[:, :8], wide[:, 8:10], wide.view(-1)[:2 * 8 * 64].view(2, 8, 64)
    before, slot = wide.clone(), SH.i64([16 * p.first, 16 * p.first + 1])
    with pytest.raises(B.TcError) as e:
        p.ctx.tc_rope_append(0, q, kv, kv, SH.i32([1, 2]), 1e4, slot, out)
    assert e.value.code == B.TC_ERR_INVALID
    torch.cuda.synchronize()
    assert torch.equal(wide, before)
    p.ctx.tc_rope_append(0, q[:1], kv[:1], kv[:1], SH.i32([1]), 1e4, slot[:1], out[:1])        # one row is read before it is written


def test_tensors_of_another_device_are_refused(small_pool):
    """As seen from a context of device 7: none of this machine's tensors are its own."""
    from paper_2601_08743_amd import _py_step, binding as B
    c, one = small_pool.ctx, SH.i32([1])
    other = c._step[:6] + (7,)
    assert c._step[6] == torch.cuda.current_device()
    with pytest.raises(B.TcError, match="entries.* on device 7, got Int . 1 . on device 0"):
        _py_step.digest_blocks(0, other, 0, 1, one, small_pool.digests(), None)
    q, kv = small_pool.rows(1, 8, 1), small_pool.rows(1, 2, 2)
    with pytest.raises(B.TcError, match="q: .* on device 7"):
        _py_step.rope_append(0, other, 0, q, kv, kv, one, None, 0, 1e4, SH.i64([80]), q, None)
    with pytest.raises(B.TcError, match="on device 7"):
        _py_step.block_attn(0, other, 0, q, one, one, SH.i32([[1]]), SH.i32([[[0], [0]]]), q, 0.1, torch.zeros(16, dtype=torch.uint8, device="cuda"), None)

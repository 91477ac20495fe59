"""Block lists by the integer score and attention over listed blocks (tc_select_blocks, tc_block_attn) against the plain
models of oracle/steps.py: lists exactly, attention to the rounding that step_harness.attn_tolerance counts."""
import math

import numpy as np
import pytest
import torch

import step_harness as SH
from oracle import steps as S

pytestmark = pytest.mark.gpu


def _table(pool, lens, max_blocks, seed):
    rng = np.random.default_rng(seed)
    ids = rng.permutation(np.arange(pool.first, pool.n))
    table = np.full((len(lens), max_blocks), -1)
    at = 0
    for b, l in enumerate(lens):
        have = (l + 15) // 16
        table[b, :have] = ids[at:at + have]
        at += have
    assert at <= len(ids)
    return table


def _lists(pool, q, seq, pos, table, digests, sink, top, local, layer=0, workspace=None):
    n = len(seq)
    lists = SH.i32(np.full((n, pool.hkv, sink + top + local), -99))
    ws = pool.workspace(n, table.shape[1], sink + top + local) if workspace is None else workspace
    pool.ctx.tc_select_blocks(layer, q, SH.i32(seq), SH.i32(pos), SH.i32(table), digests, sink, top, local, lists, ws)
    torch.cuda.synchronize()
    return lists.cpu().numpy()


def _want_lists(pool, q, seq, pos, table, digests, sink, top, local, layer=0):
    bounds, exps = (x.cpu().numpy().astype(np.int64) for x in pool.digest_views(digests))
    q64 = q.double().cpu().numpy().reshape(len(seq), pool.hkv, -1, pool.d)
    out = np.full((len(seq), pool.hkv, sink + top + local), -99)
    for i, (b, p) in enumerate(zip(seq, pos)):
        if not (0 <= b < len(table) and 0 <= p < 16 * table.shape[1]):
            continue
        for h in range(pool.hkv):
            e = table[b].astype(np.int64)
            bid = e & ((1 << 27) - 1)
            ok = (e >= 0) & (bid >= pool.first) & (bid < pool.n)
            row = np.full(len(e), -np.inf, dtype=np.float32)
            some = np.unique(bid[ok])
            if len(some):
                at = S.scores(q64[i, h], bounds[layer, h, some].astype(np.float64), exps[layer, h, some])
                row[ok] = at[np.searchsorted(some, bid[ok])]
            score = row.__getitem__
            out[i, h] = S.block_list(p, score, sink, top, local)
    return out


def _digested(pool, table, layer=0):
    buf = pool.digests()
    pool.ctx.tc_digest_blocks(layer, layer + 1, SH.i32(table), buf)
    return buf


SHAPES = [(8, 2, 64, "f32"), (8, 2, 128, "f32"), (28, 4, 128, "bf16"), (6, 6, 128, "bf16"), (20, 1, 128, "bf16"), (17, 1, 64, "f32")]


@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
@pytest.mark.parametrize("sink,top,local", [(1, 5, 2), (0, 1, 1), (2, 0, 3), (0, 400, 1), (40, 3, 1)])
def test_lists(hq, hkv, d, dtype, sink, top, local):
    """Positions in the first block, at block borders, where the window just holds everything, and long ones; a padded row and rows
    that name no request or position."""
    lens = [1, 16, 17, 160, 700, 3000]
    pool = SH.Pool(hq, hkv, d, dtype, 260, slot_blocks=1)
    pool.fill(11)
    table = _table(pool, lens, 190, 4)
    digests = _digested(pool, table)
    seq = [0, 1, 2, 3, 3, 4, 5, 5, -1, 6, 4, 4]
    pos = [0, 15, 16, 159, 96, 690, 2999, 1503, 5, 3, -1, 190 * 16]
    q = pool.rows(len(seq), hq, 21)
    got = _lists(pool, q, seq, pos, table, digests, sink, top, local)
    np.testing.assert_array_equal(got, _want_lists(pool, q, seq, pos, table, digests, sink, top, local))
    assert (got[8:] == -99).all()
    pool.close()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_lists_with_ties_and_values_that_are_not_finite(dtype, d):
    """The same block many times over (every score tied), blocks with an infinity or a NaN, queries that are not finite or
    zero, entries that name no block."""
    pool = SH.Pool(8, 2, d, dtype, 30)
    pool.fill(2)
    k, v = (x.clone() for x in pool.kv())
    k[:, 6, 0, 3, 3] = float("nan")
    k[:, 7, 1, 0, 0] = float("inf")
    k[:, 8] = 0
    pool.put(k, v)
    table = np.full((5, 130), -1)
    table[0] = 3
    table[1] = np.resize([3, 4, 5], 130)
    table[2] = np.resize(np.arange(30), 130)
    table[3] = np.resize([9, -1, 30, 10, 1 << 26, 11, -1], 130)
    table[4] = 8
    digests = _digested(pool, np.arange(30))
    seq = [0, 1, 2, 3, 4] * 3
    pos = [2000] * 5 + [2079] * 5 + [700] * 5
    q = pool.rows(len(seq), 8, 5)
    q[5, 0, 1] = float("nan")                   # one head of a group
    q[6, :4] = float("inf")                     # all heads of one
    q[7] = float("nan")
    q[8] = 0
    q[9] = 0
    for sink, top, local in ((1, 20, 3), (0, 64, 1), (0, 127, 1)):
        got = _lists(pool, q, seq, pos, table, digests, sink, top, local)
        np.testing.assert_array_equal(got, _want_lists(pool, q, seq, pos, table, digests, sink, top, local))
    pool.close()


def test_lists_of_values_of_all_sizes():
    """Scores that overflow, that vanish, and that lie a step apart."""
    pool = SH.Pool(4, 1, 64, "f32", 60)
    pool.fill(2)
    k, v = (x.clone() for x in pool.kv())
    k *= (10.0 ** torch.linspace(-38, 37, 60, device="cuda")).view(1, -1, 1, 1, 1)
    pool.put(k, v)
    table = np.random.default_rng(1).permutation(60)[None]
    digests = _digested(pool, table)
    q = pool.rows(6, 4, 3) * torch.tensor([1e-38, 1e-20, 1.0, 1e18, 1e38, 1e-44], device="cuda").view(6, 1, 1)
    seq, pos = [0] * 6, [959] * 6
    for top in (1, 7, 31, 58):
        got = _lists(pool, q, seq, pos, table, digests, 0, top, 1)
        np.testing.assert_array_equal(got, _want_lists(pool, q, seq, pos, table, digests, 0, top, 1))
    pool.close()


@pytest.mark.parametrize("max_blocks", [16384, 16385, 40000])
def test_lists_of_very_long_sequences(max_blocks):
    """Candidates beyond what the selection keeps in LDS; few different blocks, so ties by the hundred."""
    pool = SH.Pool(4, 1, 128, "bf16", 700)
    pool.fill(9)
    table = np.random.default_rng(max_blocks).integers(0, 700, size=(2, max_blocks))
    digests = _digested(pool, np.arange(700))
    seq, pos = [0, 1, 1], [16 * max_blocks - 1, 16 * max_blocks - 1, 16 * 4000]
    q = pool.rows(3, 4, 3)
    for top in (100, 3001):
        got = _lists(pool, q, seq, pos, table, digests, 2, top, 2)
        np.testing.assert_array_equal(got, _want_lists(pool, q, seq, pos, table, digests, 2, top, 2))
    pool.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(28, 4, 128, "bf16"), (8, 8, 128, "bf16"), (32, 2, 128, "bf16"), (20, 1, 128, "bf16"),
                                            (10, 2, 64, "f32"), (8, 2, 128, "f32")])
def test_lists_of_suffixes(hq, hkv, d, dtype):
    """Many tokens of a few requests: those of one request share the digests that are read, and groups of them hold tokens of two
    or three requests, of requests whose candidates are all listed, padded rows in between and at the end."""
    lens = [300, 40, 2100, 2500, 17]
    pool = SH.Pool(hq, hkv, d, dtype, 330, slot_blocks=1)
    pool.fill(13)
    table = _table(pool, lens, 160, 4)
    table[3, 7] = -1
    table[2, 9] = pool.n
    digests = _digested(pool, table)
    seq, pos = [], []
    for b, n_new in ((0, 3), (1, 5), (2, 250), (3, 150), (0, 70), (4, 2), (2, 130)):
        seq += [b] * n_new
        pos += list(range(lens[b] - min(n_new, lens[b]), lens[b])) + [lens[b] - 1] * max(0, n_new - lens[b])
    for i in (9, 100, 101, 300):
        seq[i] = -1
    seq += [-1] * 5
    pos += [0] * 5
    q = pool.rows(len(seq), hq, 3)
    q[20, :, 3] = float("nan")
    got = _lists(pool, q, seq, pos, table, digests, 1, 13, 2)
    np.testing.assert_array_equal(got, _want_lists(pool, q, seq, pos, table, digests, 1, 13, 2))
    # in rounds of few tokens
    small = torch.full((hkv * 160 * 4 * 77,), 0x22, dtype=torch.uint8, device="cuda")
    np.testing.assert_array_equal(got, _lists(pool, q, seq, pos, table, digests, 1, 13, 2, workspace=small))
    pool.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(7, 1, 128, "bf16"), (34, 1, 128, "bf16"), (20, 1, 64, "f32"), (4, 2, 128, "f32")])
@pytest.mark.parametrize("max_blocks", [1536, 1537, 2048, 2049, 2700])
def test_lists_over_tables_of_some_thousand_blocks(hq, hkv, d, dtype, max_blocks):
    """One token of each request, tables around the length from which scores and list are launches of their own."""
    pool = SH.Pool(hq, hkv, d, dtype, 500)
    pool.fill(8)
    table = np.random.default_rng(max_blocks).integers(0, 500, size=(3, max_blocks))
    table[1, 5:60:7] = -1
    digests = _digested(pool, np.arange(500))
    pos = [16 * max_blocks - 1, 16 * max_blocks - 9, 16 * 520]
    q = pool.rows(3, hq, 3)
    for sink, top, local in ((0, 600, 1), (3, 31, 5)):
        got = _lists(pool, q, [0, 1, 2], pos, table, digests, sink, top, local)
        np.testing.assert_array_equal(got, _want_lists(pool, q, [0, 1, 2], pos, table, digests, sink, top, local))
    pool.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, "bf16"), (40, 2, 128, "bf16"), (34, 2, 64, "f32")])
@pytest.mark.parametrize("max_blocks", [900, 1900])
def test_lists_of_queries_that_are_not_finite(hq, hkv, d, dtype, max_blocks):
    """One head, the first or the last ones of a group, or all of it, for one launch and for two."""
    pool = SH.Pool(hq, hkv, d, dtype, 60)
    pool.fill(8)
    table = np.random.default_rng(max_blocks).integers(0, 60, size=(6, max_blocks))
    digests = _digested(pool, np.arange(60))
    G = hq // hkv
    q = pool.rows(6, hq, 3)
    q[0, :, 5] = float("nan")
    q[1, 0, 0] = float("inf")
    q[2, G:, 7] = float("-inf")
    q[3, :G - 1, 1] = float("nan")
    q[4, 1:G, 1] = float("nan")
    seq, pos = list(range(6)), [16 * max_blocks - 1] * 6
    for sink, top, local in ((1, 30, 2), (0, 300, 1)):
        got = _lists(pool, q, seq, pos, table, digests, sink, top, local)
        np.testing.assert_array_equal(got, _want_lists(pool, q, seq, pos, table, digests, sink, top, local))
    pool.close()


@pytest.mark.parametrize("max_blocks", [257, 1024, 1025])
def test_lists_of_many_tokens_over_long_tables(max_blocks):
    """More than a thousand lists, from every number of candidates; few different blocks, so scores are tied."""
    pool = SH.Pool(8, 8, 128, "bf16", 90)
    pool.fill(6)
    table = np.random.default_rng(max_blocks).integers(0, 90, size=(2, max_blocks))
    table[1, 3:50:9] = -1
    digests = _digested(pool, np.arange(90))
    seq = [0] * 70 + [1] * 71
    pos = [int(x) for x in np.linspace(0, 16 * max_blocks - 1, 70)] + [int(x) for x in np.linspace(16 * 7, 16 * max_blocks - 1, 71)]
    q = pool.rows(len(seq), 8, 3)
    for sink, top, local in ((0, 1, 1), (2, 100, 3)):
        got = _lists(pool, q, seq, pos, table, digests, sink, top, local)
        np.testing.assert_array_equal(got, _want_lists(pool, q, seq, pos, table, digests, sink, top, local))
    pool.close()


def test_lists_do_not_depend_on_the_workspace():
    pool = SH.Pool(8, 2, 128, "bf16", 120)
    pool.fill(1)
    table = _table(pool, [900, 1000], 70, 3)
    digests = _digested(pool, table)
    seq, pos = [0, 1] * 150, [890, 999] * 150
    q = pool.rows(300, 8, 2)
    whole = _lists(pool, q, seq, pos, table, digests, 1, 9, 2)
    for tokens in (1, 5):
        ws = torch.full((2 * 70 * 4 * tokens + 3,), 0x11, dtype=torch.uint8, device="cuda")
        np.testing.assert_array_equal(whole, _lists(pool, q, seq, pos, table, digests, 1, 9, 2, workspace=ws))
    np.testing.assert_array_equal(whole, _want_lists(pool, q, seq, pos, table, digests, 1, 9, 2))
    pool.close()


# ------------------------------------------------------------------------------------------------ attention

def _attend(pool, q, seq, pos, table, lists, scale=None, layer=0):
    n, n_list = len(seq), lists.shape[2]
    out = torch.full((n, pool.hq, pool.d), 7.0, dtype=pool.dt, device="cuda")
    pool.ctx.tc_block_attn(layer, q, SH.i32(seq), SH.i32(pos), SH.i32(table), SH.i32(lists), out,
                           1 / math.sqrt(pool.d) if scale is None else scale, pool.workspace(n, table.shape[1], n_list))
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


def _check_attn(pool, q, seq, pos, table, lists, scale=None, layer=0):
    got = _attend(pool, q, seq, pos, table, lists, scale, layer)
    scale = 1 / math.sqrt(pool.d) if scale is None else scale
    k64, v64 = pool.kv64()
    q64 = q.double().cpu().numpy().reshape(len(seq), pool.hkv, -1, pool.d)
    worst = 0.0
    for i, (b, p) in enumerate(zip(seq, pos)):
        if not (0 <= b < len(table) and 0 <= p < 16 * table.shape[1]):
            assert (got[i] == 7.0).all()
            continue
        for h in range(pool.hkv):
            keys, vals = [], []
            for j in lists[i, h]:
                if not 0 <= j <= p // 16:
                    continue
                e = int(table[b, j])
                bid = e & ((1 << 27) - 1)
                if e < 0 or not pool.first <= bid < pool.n:
                    continue
                m = min(16 - (e >> SH.PAD_SHIFT), p - 16 * j + 1)
                keys.append(k64[layer, bid - pool.first, h, :m])
                vals.append(v64[layer, bid - pool.first, h, :m])
            keys = np.concatenate(keys) if keys else np.zeros((0, pool.d))
            vals = np.concatenate(vals) if vals else np.zeros((0, pool.d))
            ref, size_v, size = S.block_attn(q64[i, h], keys, vals, scale)
            tol = SH.attn_tolerance(ref, size_v, size, pool.bf16, len(keys))
            G = pool.hq // pool.hkv
            diff = np.abs(got[i, h * G:(h + 1) * G] - ref)
            assert (diff <= tol).all(), (i, h, float((diff - tol).max()), float(diff.max()))
            worst = max(worst, float((diff / tol).max()))
    return worst


ATTN_SHAPES = SHAPES + [(40, 8, 128, "bf16"), (32, 1, 128, "bf16"), (33, 1, 128, "bf16"), (9, 1, 128, "f32")]


@pytest.mark.parametrize("hq,hkv,d,dtype", ATTN_SHAPES)
@pytest.mark.parametrize("n_list", [1, 2, 7, 8, 9, 64, 131])
def test_attention_over_lists(hq, hkv, d, dtype, n_list):
    """Lists with blocks in any order, twice, missing, behind the token and beyond the table; positions at every kind of
    border; what a token does not see is NaN."""
    lens = [1, 16, 17, 160, 1000]
    pool = SH.Pool(hq, hkv, d, dtype, 100, layers=2, slot_blocks=1)
    pool.fill(31)
    table = _table(pool, lens, 70, 4)
    table[4, 5] = -1
    table[4, 6] = pool.n
    table[4, 7] = 0
    table[3, 4] |= 5 << SH.PAD_SHIFT
    seq = [0, 1, 2, 3, 3, 4, 4, -1, 5, 4]
    pos = [0, 15, 16, 159, 97, 999, 500, 3, 3, 70 * 16]
    k, v = (x.clone() for x in pool.kv())
    for b, l in enumerate(lens):                # behind the sequence's end, and the unused tail of a table block
        if l % 16:
            k[:, int(table[b, l // 16]) - 1, :, l % 16:] = float("nan")
            v[:, int(table[b, l // 16]) - 1, :, l % 16:] = float("nan")
    tail = (int(table[3, 4]) & ((1 << 27) - 1)) - 1
    v[:, tail, :, 11:] = float("inf")
    k[:, tail, :, 11:] = -3e38
    pool.put(k, v)
    rng = np.random.default_rng(n_list)
    lists = rng.integers(-2, 66, size=(len(seq), hkv, n_list))
    lists[4, :, 0] = 6                          # the token's own block, in part
    lists[:3, :, 0] = [[0], [0], [1]]
    lists[5, 0] = -1                            # nothing at all
    lists[0, 0, -1] = 0x7fffffff
    worst = _check_attn(pool, pool.rows(len(seq), hq, 3), seq, pos, table, lists, layer=1)
    print("worst error / tolerance %.3f" % worst)
    pool.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(28, 4, 128, "bf16"), (8, 2, 64, "f32"), (8, 2, 128, "f32")])
@pytest.mark.parametrize("n_tokens", [1, 3, 150])
def test_attention_in_one_range_and_many(hq, hkv, d, dtype, n_tokens):
    """A long list shared by many work-groups, and many tokens with a work-group each."""
    pool = SH.Pool(hq, hkv, d, dtype, 300)
    pool.fill(5)
    table = _table(pool, [300 * 16 - 3], 300, 4)
    rng = np.random.default_rng(n_tokens)
    pos = np.sort(rng.integers(2000, 300 * 16 - 3, size=n_tokens))
    lists = np.stack([np.stack([np.sort(rng.permutation(p // 16 + 1)[:100]) for _ in range(hkv)]) for p in pos])
    if n_tokens > 3:
        lists = lists[:, :, :40]
    _check_attn(pool, pool.rows(n_tokens, hq, 3), [0] * n_tokens, pos, table, lists)
    pool.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(32, 8, 128, "bf16"), (28, 4, 128, "bf16"), (8, 2, 64, "f32")])
def test_one_workspace_for_any_number_of_tokens(hq, hkv, d, dtype):
    """A workspace sized for the largest step serves smaller ones, whose lists are shared out further; its bytes behind what was
    asked for stay as they were."""
    pool = SH.Pool(hq, hkv, d, dtype, 300)
    pool.fill(5)
    table, rng = SH.i32(np.arange(300)[None]), np.random.default_rng(1)
    need = pool.B.tc_sparse_workspace_bytes(pool.cfg, 40, 300, 200)
    ws = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    lists = SH.i32(rng.integers(0, 280, size=(40, hkv, 200)))
    q = pool.rows(40, hq, 3)
    whole = None
    for n in (40, 31, 16, 9, 8, 5, 4, 3, 2, 1):
        out = torch.empty_like(q[:n])
        pool.ctx.tc_block_attn(0, q[:n], SH.i32([0] * n), SH.i32([4790] * n), table, lists[:n], out, 0.1, ws[:need])
        torch.cuda.synchronize()
        whole = out.float() if whole is None else whole
        # (another number of ranges: other roundings, each of 2^-8 of |v| < 5.6, or in fp32 of sums of 3200 keys)
        assert (out.float() - whole[:n]).abs().max() <= (2 * 2.0 ** -8 * 5.6 if dtype == "bf16" else 2 * 3200 * 2.0 ** -24 * 5.6)
    assert (ws[need:] == 0x5A).all()
    pool.close()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 128), ("f32", 64)])
def test_attention_with_extreme_values(dtype, d):
    """Scores far apart (one weight takes all), large ones that are equal, a key of minus infinity, a score of plus infinity, keys and
    values that are NaN: as the formula has it, row by row."""
    pool = SH.Pool(4, 1, d, dtype, 40)
    pool.fill(5)
    k, v = (x.clone() for x in pool.kv())
    k[:, 3, :, 2] = 300.0
    k[:, 5] = k[:, 5, :, :1]                    # sixteen equal keys
    pool.put(k, v)
    table = np.arange(40)[None]
    q = pool.rows(4, 4, 8)
    q[1] *= 40
    q[2] = 50.0
    lists = np.stack([np.arange(30)[None]] * 4)
    _check_attn(pool, q, [0] * 4, [479] * 4, table, lists)
    _check_attn(pool, q * 0, [0] * 4, [479, 3, 16, 17], table, lists)
    # a score of minus infinity has no weight; all of them give zeros; plus infinity and NaN reach every output of the row
    k, v = (x.clone() for x in pool.kv())
    q = torch.ones_like(q)
    k[:, 7] = -float("inf")
    k[:, 8, :, 4] = float("inf")
    k[:, 9, :, 4, 1] = float("nan")
    v[:, 10, :, 4, 5] = float("nan")
    k[:, 10] = 1.0
    pool.put(k, v)
    one = lambda *blocks: np.array([[list(blocks) + [-1] * (3 - len(blocks))]])
    out = _attend(pool, q[:1], [0], [639], table, one(7))
    assert (out == 0).all()
    a, b = _attend(pool, q[:1], [0], [639], table, one(7, 2)), _attend(pool, q[:1], [0], [639], table, one(2))
    np.testing.assert_array_equal(a, b)
    assert np.isnan(_attend(pool, q[:1], [0], [639], table, one(2, 8))).all()
    assert np.isnan(_attend(pool, q[:1], [0], [639], table, one(2, 9))).all()
    bad = _attend(pool, q[:1], [0], [639], table, one(2, 10))
    assert np.isnan(bad[..., 5]).all() and np.isfinite(np.delete(bad, 5, axis=-1)).all()
    pool.close()


def test_the_largest_number_of_tokens():
    """2^20 tokens of 17 KV heads are more work-groups than one launch takes; all but some at both ends are padded rows, which
    stay as they are."""
    pool = SH.Pool(17, 17, 64, "f32", 12)
    pool.fill(5)
    n, few = 1 << 20, [0, 1, (1 << 24) // 17 - 1, (1 << 24) // 17, (1 << 24) // 17 + 1, (1 << 20) - 2, (1 << 20) - 1]
    at = torch.tensor(few, device="cuda")
    table = SH.i32(np.arange(12)[None])
    digests = _digested(pool, np.arange(12))
    seq, pos = SH.i32(np.full(n, -1)), SH.i32(np.full(n, 190))
    seq[at] = 0
    q = torch.zeros((n, 17, 64), device="cuda")
    q[at] = pool.rows(len(few), 17, 3)
    lists, out = torch.full((n, 17, 3), -99, dtype=torch.int32, device="cuda"), torch.full((n, 17, 64), 7.0, device="cuda")
    ws = pool.workspace(n, 12, 3)
    pool.ctx.tc_select_blocks(0, q, seq, pos, table, digests, 1, 1, 1, lists, ws)
    pool.ctx.tc_block_attn(0, q, seq, pos, table, lists, out, 0.1, ws)
    few_lists = torch.full((len(few), 17, 3), -99, dtype=torch.int32, device="cuda")
    few_out = torch.full((len(few), 17, 64), 7.0, device="cuda")
    pool.ctx.tc_select_blocks(0, q[at], seq[at], pos[at], table, digests, 1, 1, 1, few_lists, ws)
    pool.ctx.tc_block_attn(0, q[at], seq[at], pos[at], table, few_lists, few_out, 0.1, ws)
    torch.cuda.synchronize()
    want = _want_lists(pool, q[at], [0] * len(few), [190] * len(few), np.arange(12)[None], digests, 1, 1, 1)
    np.testing.assert_array_equal(few_lists.cpu().numpy(), want)
    assert torch.equal(lists[at], few_lists) and torch.equal(out[at], few_out)      # (lists of one range in both)
    lists[at], out[at] = -99, 7.0
    assert bool((lists == -99).all()) and bool((out == 7.0).all())
    pool.close()


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB in its last layer: the last blocks are read, digested and scored where they are."""
    pool = SH.Pool(8, 8, 128, "bf16", 72000)
    assert pool.raw.numel() * 4 > 2 ** 32
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    pool.raw.zero_()
    pool.seq[0, -40:] = torch.randn((40, 2, 8 * 16 * 128), generator=g, device="cuda").to(torch.bfloat16)
    pool.seq[0, :40] = torch.randn((40, 2, 8 * 16 * 128), generator=g, device="cuda").to(torch.bfloat16)
    table = np.arange(72000 - 1, 72000 - 41, -1)[None]
    digests = _digested(pool, table)
    q = pool.rows(2, 8, 2)
    lists = _lists(pool, q, [0, 0], [639, 600], table, digests, 1, 9, 2)
    np.testing.assert_array_equal(lists, _want_lists(pool, q, [0, 0], [639, 600], table, digests, 1, 9, 2))
    out = _attend(pool, q, [0, 0], [639, 600], table, lists)
    last = SH.Pool(8, 8, 128, "bf16", 40)
    last.seq[0] = pool.seq[0, -40:]
    np.testing.assert_array_equal(out, _attend(last, q, [0, 0], [639, 600], table - (72000 - 40), lists))
    # the append as well
    k, v = pool.rows(1, 8, 6), pool.rows(1, 8, 7)
    pool.ctx.tc_rope_append(0, q[:1].clone(), k, v, SH.i32([0]), 1e4, SH.i64([72000 * 16 - 1]), torch.empty_like(q[:1]))
    torch.cuda.synchronize()
    assert torch.equal(pool.seq[0, -1, 0].view(8, 16, 128)[:, 15], k[0])
    last.close()
    pool.close()


def test_refusals():
    from paper_2601_08743_amd import binding as B
    pool = SH.Pool(8, 2, 64, "f32", 20)
    pool.fill(1)
    table, digests, ws = SH.i32(np.arange(20)[None]), pool.digests(), pool.workspace(1, 20, 100)
    q, seq, pos = pool.rows(1, 8, 1), SH.i32([0]), SH.i32([300])

    def refused(f, code=B.TC_ERR_INVALID):
        with pytest.raises(B.TcError) as e:
            f()
        assert e.value.code == code, e.value

    def select(layer=0, q=q, seq=seq, pos=pos, table=table, digests=digests, sink=1, top=3, local=1, n_list=5, ws=ws):
        pool.ctx.tc_select_blocks(layer, q, seq, pos, table, digests, sink, top, local, SH.i32(np.zeros((1, 2, n_list))), ws)

    def attend(layer=0, q=q, seq=seq, pos=pos, table=table, n_list=5, out=None, scale=0.1, ws=ws):
        pool.ctx.tc_block_attn(layer, q, seq, pos, table, SH.i32(np.zeros((1, 2, n_list))), torch.empty_like(q) if out is None else out, scale, ws)

    pool.ctx.tc_digest_blocks(0, 1, table, digests)
    select()
    attend()
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    for f in (select, attend):
        refused(lambda: f(layer=1))
        refused(lambda: f(layer=-1))
        refused(lambda: f(q=q.bfloat16()))
        refused(lambda: f(q=pool.rows(2, 8, 1)))
        refused(lambda: f(seq=SH.i64([0])))
        refused(lambda: f(pos=SH.i32([0, 1])))
        refused(lambda: f(table=table.cpu()))
        refused(lambda: f(n_list=0))
    refused(lambda: select(n_list=4))
    refused(lambda: select(local=0, n_list=4))
    refused(lambda: select(sink=-1, n_list=3))
    refused(lambda: select(top=-1, n_list=1))
    refused(lambda: select(digests=digests[1:]))
    refused(lambda: select(ws=none), B.TC_ERR_CAPACITY)
    refused(lambda: select(ws=ws[:159]), B.TC_ERR_CAPACITY)
    select(ws=ws[:160])
    select(top=20, n_list=22, ws=none)          # no score is needed
    select(top=0, n_list=2, ws=none)
    refused(lambda: attend(n_list=100, ws=none), B.TC_ERR_CAPACITY)
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        refused(lambda: attend(scale=scale))
    refused(lambda: attend(out=pool.rows(1, 7, 1)))
    torch.cuda.synchronize()
    pool.close()

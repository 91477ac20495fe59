"""The plain models of the token-step operators (oracle/steps.py) against hand-worked cases and brute force, and what of the
entry points can be asked without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from oracle import steps as S


def test_step_tables_by_hand():
    table = np.array([[9, -1, -1], [4, 6, -1], [-1, -1, -1]])
    r = S.step_tables([15, 20, 0], [2, 0, 17], table, [30, 31, 32, 33], 1, 21, 3, 40)
    assert r["table"].tolist() == [[9, 31, -1], [4, 6, -1], [32, 33, -1]]
    assert r["cu_new"].tolist() == [0, 2, 2, 19] and r["end_len"].tolist() == [17, 20, 17] and r["spare_next"] == 4
    assert r["slot_map"].tolist() == [9 * 16 + 15, 31 * 16] + list(range(32 * 16, 33 * 16)) + [33 * 16, -1, -1]
    assert r["full_block"].tolist() == [9, -1] + [-1] * 15 + [32, -1, -1, -1]
    assert r["token_pos"].tolist() == [15, 16] + list(range(17)) + [-1, -1] and r["status"].tolist() == [0, 3]
    short = S.step_tables([15, 20, 0], [2, 0, 17], table, [30, 31, 32], 1, 21, 3, 40)
    assert short["status"].tolist() == [-3, 3] and short["table"].tolist() == table.tolist() and short["cu_new"].tolist() == [0] * 4


def test_rotate_is_the_reencoding_of_the_stitch():
    """With one axis the model is the oracle's re-encoding; with several, each section is that of its own axis alone."""
    rng = np.random.default_rng(2)
    x, pos = rng.standard_normal((6, 2, 64)), rng.integers(0, 90000, size=(3, 6))
    np.testing.assert_allclose(S.rotate(x, pos[:1], [32], 1e4), oracle.reencode_keys(x, pos[0], 1e4), atol=1e-9)
    mixed = S.rotate(x, pos, [5, 0, 27], 1e4)
    for axis, cols in ((0, np.r_[0:5, 32:37]), (2, np.r_[5:32, 37:64])):
        np.testing.assert_allclose(mixed[..., cols], S.rotate(x, pos[axis:axis + 1], [32], 1e4)[..., cols], atol=1e-12)


def test_digest_bounds_hold_and_are_tight():
    rng = np.random.default_rng(3)
    for scale in (1e-38, 1e-3, 1.0, 3e5, 1e37):
        k = rng.standard_normal((16, 64)) * scale
        b, e = S.digest(k)
        step = 2.0 ** e
        assert (b[0] * step >= k.max(0)).all() and (b[1] * step <= k.min(0)).all() and np.abs(b).max() <= 127
        assert (b[0] * step - k.max(0) < step).all() and (e == -126 or np.abs(k).max() > 127 * 2.0 ** (e - 1))
    assert S.exponent(127.0) == 0 and S.exponent(127.00001) == 1 and S.exponent(0.0) == -126


def test_score_bounds_every_key():
    """No key of the block scores higher, up to the rounding of q: half a step of 2^f in each channel."""
    rng = np.random.default_rng(4)
    for _ in range(20):
        k, q = rng.standard_normal((16, 64)) * np.exp(rng.standard_normal(64)), rng.standard_normal((3, 64))
        b, e = S.digest(k)
        slack = max(0.5 * 2.0 ** S.exponent(np.abs(row).max()) for row in q) * np.abs(k).sum(1).max()
        assert S.score(q, b, e) >= (q @ k.T).max() - slack
    assert S.score(q, b, 127) == np.inf and S.score(np.full((1, 64), np.nan), b, e) == -np.inf


def test_scores_of_many_blocks_are_the_scores():
    rng = np.random.default_rng(6)
    q = rng.standard_normal((5, 32)) * 3
    q[2, 4] = np.inf
    dig = [S.digest(rng.standard_normal((16, 32)) * 10.0 ** x) for x in np.linspace(-30, 30, 9)] + [(np.zeros((2, 32), np.int64), 127)]
    many = S.scores(q, np.stack([b for b, _ in dig]).astype(np.float64), np.array([e for _, e in dig]))
    assert many.tolist() == [S.score(q, b, e) for b, e in dig]
    assert (S.scores(q * np.nan, np.stack([b for b, _ in dig]).astype(np.float64), np.array([0] * 10)) == -np.inf).all()


def test_block_list_by_hand():
    score = lambda j: {1: 5.0, 2: 7.0, 3: 7.0, 4: 1.0, 5: 7.0}[j]
    assert S.block_list(7 * 16 + 3, score, 1, 2, 2).tolist() == [0, 2, 3, 6, 7]
    assert S.block_list(7 * 16, score, 1, 4, 2).tolist() == [0, 1, 2, 3, 5, 6, 7]
    assert S.block_list(3 * 16, score, 1, 2, 2).tolist() == [0, 1, 2, 3, -1]
    assert S.block_list(0, score, 3, 2, 2).tolist() == [0] + [-1] * 6


def test_block_attn_is_softmax_attention():
    rng = np.random.default_rng(5)
    q, k, v = (torch.from_numpy(rng.standard_normal((n, 32))) for n in (4, 37, 37))
    want = torch.nn.functional.scaled_dot_product_attention(q[None], k[None], v[None], scale=0.3)[0]
    got, _, _ = S.block_attn(q.numpy(), k.numpy(), v.numpy(), 0.3)
    np.testing.assert_allclose(got, want.numpy(), atol=1e-12)
    assert (S.block_attn(q.numpy(), k.numpy()[:0], v.numpy()[:0], 0.3)[0] == 0).all()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(28, 4, 128, 1), (8, 2, 64, 0), (40, 8, 128, 1), (33, 1, 128, 0)])
def test_a_workspace_does_for_fewer_tokens_and_shorter_lists(hq, hkv, d, dtype):
    from paper_2601_08743_amd import binding as B
    cfg = B.make_config(1, hq, hkv, d, dtype, 4000, 0, 16)
    size = lambda n, nl: B.tc_sparse_workspace_bytes(cfg, n, 1, nl)
    for nl in (1, 5, 60, 100, 129, 500, 4000):
        sizes = [size(n, nl) for n in list(range(1, 140)) + [256, 257, 600, 5000]]
        assert sizes == sorted(sizes)
    for n in (1, 3, 17, 200):
        sizes = [size(n, nl) for nl in range(1, 700, 13)]
        assert sizes == sorted(sizes)


def test_sizes_and_null_contexts_need_no_gpu():
    from paper_2601_08743_amd import binding as B
    cfg = B.make_config(28, 28, 4, 128, B.TC_BF16, 4000, 40, 600)
    assert B.tc_digest_bytes(cfg) == 28 * 4 * 4000 * 257
    assert B.tc_digest_bytes(B.make_config(28, 28, 5, 128, B.TC_BF16, 4000, 40, 600)) == 0
    one = B.tc_sparse_workspace_bytes(cfg, 1, 100, 1)
    assert one >= 4 * 100 * 4 and one % 256 == 0
    assert B.tc_sparse_workspace_bytes(cfg, 4096, 1 << 20, 64) >= 4 * (1 << 20) * 4         # a round of at least one token
    for bad in ((-1, 1, 1), (1 << 21, 1, 1), (1, -1, 1), (1, 1 << 27, 1), (1, 1, 0)):
        assert B.tc_sparse_workspace_bytes(cfg, *bad) == 0
    lib = B._lib
    for name in ("tc_table_entries", "tc_step_tables", "tc_rope_append", "tc_digest_blocks", "tc_select_blocks", "tc_block_attn"):
        f = getattr(lib, name)
        assert f(*[None if t is ctypes.c_void_p else 0 for t in f.argtypes]) == B.TC_ERR_INVALID, name

"""Lists by either kernel for scores, on both sides of the rule that chooses it (csrc/score_route.h): padded batches of one token each over
long tables, suffixes of few and of many tokens, whole and in rounds."""
import numpy as np
import pytest
import torch

import step_harness as SH
from test_gpu_block_sparse import _digested, _lists, _want_lists

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d,dtype", [(32, 8, 128, "bf16"), (28, 4, 128, "bf16"), (2, 2, 64, "f32")])
@pytest.mark.parametrize("requests,tokens,pad", [(20, 1, 3), (9, 2, 0), (9, 3, 1), (2, 30, 2)])
def test_lists_on_both_sides_of_the_rule(hq, hkv, d, dtype, requests, tokens, pad):
    pool = SH.Pool(hq, hkv, d, dtype, 150)
    pool.fill(4)
    max_blocks = 1600
    rng = np.random.default_rng(requests)
    table = rng.integers(0, 150, size=(requests, max_blocks))
    table[0, 20:400:17] = -1
    digests = _digested(pool, np.arange(150))
    seq, pos = np.repeat(np.arange(requests), tokens), []
    for b in range(requests):
        end = int(rng.integers(16 * 300, 16 * max_blocks))
        pos += list(range(end - tokens, end))
    seq, pos = list(seq) + [-1] * pad, pos + [-1] * pad
    q = pool.rows(len(seq), hq, 3)
    got = _lists(pool, q, seq, pos, table, digests, 1, 50, 2)
    np.testing.assert_array_equal(got, _want_lists(pool, q, seq, pos, table, digests, 1, 50, 2))
    assert (got[len(seq) - pad:] == -99).all()
    pool.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(32, 8, 128, "bf16"), (16, 1, 128, "bf16"), (10, 2, 64, "f32")])
def test_groups_in_rounds(hq, hkv, d, dtype):
    """A workspace for some of the tokens: groups that end with a round, and begin the next one inside a request."""
    pool = SH.Pool(hq, hkv, d, dtype, 200)
    pool.fill(9)
    max_blocks = 1200
    table = np.random.default_rng(2).integers(0, 200, size=(3, max_blocks))
    digests = _digested(pool, np.arange(200))
    seq = [0] * 300 + [1] * 210 + [2] * 250
    pos = list(range(16 * 1100, 16 * 1100 + 300)) + list(range(16 * 700, 16 * 700 + 210)) + list(range(250))
    for i in (3, 299, 300, 301, 555):
        seq[i] = -1
    q = pool.rows(len(seq), hq, 3)
    want = _want_lists(pool, q, seq, pos, table, digests, 1, 13, 2)
    np.testing.assert_array_equal(_lists(pool, q, seq, pos, table, digests, 1, 13, 2), want)
    ws = torch.full((hkv * max_blocks * 4 * 293,), 0x22, dtype=torch.uint8, device="cuda")
    np.testing.assert_array_equal(_lists(pool, q, seq, pos, table, digests, 1, 13, 2, workspace=ws), want)
    pool.close()

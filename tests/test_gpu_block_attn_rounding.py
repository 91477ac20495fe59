"""What the attention over listed blocks rounds in bf16: the output, once.  Few keys and values of both signs, so that the output is
small against the weights times the values, and a weight kept in 8 bits shows."""
import math

import numpy as np
import pytest
import torch

import step_harness as SH
from oracle import steps as S

pytestmark = pytest.mark.gpu


def _tolerance(ref, p_abs_v, size, n_keys):
    """One rounding of the output (half a step of bf16, 2^-8 of it).  Weights as step_harness.attn_tolerance has them for fp32 - scores
    of 128 products, the exponential, a quotient of two sums over n keys - and kept as a sum of two bf16 numbers, which
    leaves 2^-8 of 2^-8 of a weight."""
    delta = 130 * 2.0 ** -24 * size[..., None] + 2.0 ** -21
    rel = 2 * delta + 2 * (n_keys + 8) * 2.0 ** -24
    return 2.0 ** -8 * np.abs(ref) + (rel + 2.0 ** -16) * p_abs_v * (1 + 2.0 ** -8) + 1e-30


def _run(pool, q, pos, lists, scale):
    n = q.shape[0]
    out = torch.full_like(q, 7.0)
    table = SH.i32(np.arange(pool.n)[None])
    pool.ctx.tc_block_attn(0, q, SH.i32([0] * n), SH.i32(pos), table, SH.i32(lists), out, scale,
                           pool.workspace(n, pool.n, lists.shape[2]))
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


@pytest.mark.parametrize("hq,hkv", [(28, 4), (8, 8), (20, 1)])
@pytest.mark.parametrize("n_list", [1, 3, 8, 131])
def test_only_the_output_is_rounded_to_bf16(hq, hkv, n_list):
    """Lists of one to three blocks; of 131 places, where they are shared out over work-groups, three are filled."""
    pool = SH.Pool(hq, hkv, 128, "bf16", 40)
    pool.fill(7)
    k, v = (x.clone() for x in pool.kv())
    pool.put(k, torch.where(v > 0, 1.0, -1.0) * (1 + 0.25 * v.abs()))
    q = (0.3 * pool.rows(6, hq, 3).float()).to(pool.dt)
    pos = [639, 500, 47, 40, 300, 21]
    rng = np.random.default_rng(n_list)
    lists = np.full((6, hkv, n_list), -1)
    for i, p in enumerate(pos):
        for h in range(hkv):
            at = rng.permutation(n_list)[:3]
            lists[i, h, at] = rng.permutation(p // 16 + 1)[:len(at)] if p // 16 + 1 >= len(at) else rng.integers(0, p // 16 + 1, size=len(at))
    scale = 1 / math.sqrt(128)
    got = _run(pool, q, pos, lists, scale)
    k64, v64 = pool.kv64()
    q64, G = q.double().cpu().numpy().reshape(6, hkv, -1, 128), hq // hkv
    for i, p in enumerate(pos):
        for h in range(hkv):
            m = [(int(j), min(16, p - 16 * int(j) + 1)) for j in lists[i, h] if j >= 0]
            keys, vals = (np.concatenate([x[0, j, h, :n] for j, n in m]) for x in (k64, v64))
            ref, size_v, size = S.block_attn(q64[i, h], keys, vals, scale)
            diff = np.abs(got[i, h * G:(h + 1) * G] - ref)
            tol = _tolerance(ref, size_v, size, len(keys))
            assert (diff <= tol).all(), (i, h, float((diff / tol).max()))
    pool.close()


def test_infinite_values_reach_the_output_as_they_are():
    """A value of plus or minus infinity under a weight that is not zero, whether or not that weight is a bf16 number."""
    pool = SH.Pool(4, 1, 128, "bf16", 6)
    pool.fill(5)
    k, v = (x.clone() for x in pool.kv())
    k[:, 2] = k[:, 2, :, :1]                    # sixteen equal keys: weights of 1 / 16 where the block is alone
    v[:, 2, :, 3, 10] = float("inf")
    v[:, 2, :, 9, 20] = -float("inf")
    v[:, 2, :, 9, 30], v[:, 2, :, 11, 30] = float("inf"), -float("inf")
    pool.put(k, v)
    q = pool.rows(1, 4, 8)
    for blocks in ([2, -1, -1], [1, 2, 3]):
        out = _run(pool, q, [95], np.array([[blocks]]), 0.1)
        assert (out[..., 10] == np.inf).all() and (out[..., 20] == -np.inf).all() and np.isnan(out[..., 30]).all()
        assert np.isfinite(np.delete(out, [10, 20, 30], axis=-1)).all()
    pool.close()

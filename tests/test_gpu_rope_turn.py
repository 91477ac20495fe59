"""The turn of the encoded append in fp32: sine and cosine to a few units of their own last place, at any fraction of a revolution."""
import numpy as np
import pytest
import torch

import step_harness as SH

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("theta", [1e4, 1e6])
def test_small_sines_and_cosines_keep_their_bits(d, theta):
    """Queries (1, 0) in every pair become (cos, sin).  Sine and cosine of the fp32 library are off by 4 units of the last place at
    most, 2^-21; products by 1 and 0 and sums with 0 are exact; the turn in fp64, pos * theta^(-2j/D) revolutions as a product
    of three rounded numbers, is off by 4 * 2^-53 of itself.  What is left to the fraction of a revolution in fp32 is 2^-22 of
    the result."""
    pool = SH.Pool(2, 1, d, "f32", 4)
    n, half = 20000, d // 2
    q = torch.zeros((n, 2, d), device="cuda")
    q[..., :half] = 1
    kv = torch.zeros((n, 1, d), device="cuda")
    slots = np.full(n, -1)
    pos = np.concatenate([np.arange(n // 2), np.random.default_rng(d).integers(0, 1 << 22, size=n - n // 2)])
    # (a row needs a slot to be encoded: 63 of them at a time, without the block's first position)
    out = torch.full_like(q, float("nan"))
    for a in range(0, n, 60):
        m = min(60, n - a)
        slot = [16 * (i // 15) + 1 + i % 15 for i in range(m)]
        pool.ctx.tc_rope_append(0, q[a:a + m], kv[a:a + m], kv[a:a + m], SH.i32(pos[a:a + m]), theta, SH.i64(slot), out[a:a + m])
    torch.cuda.synchronize()
    turn = pos[:, None].astype(np.longdouble) * np.longdouble(theta) ** (-np.arange(half, dtype=np.longdouble) / half)
    slack = (turn * (4 * 2.0 ** -53 + 2.0 ** -60)).astype(np.float64)[:, None]
    got = out.double().cpu().numpy()
    for have, want in ((got[..., :half], np.cos(turn)), (got[..., half:], np.sin(turn))):
        want = want.astype(np.float64)[:, None]
        diff, tol = np.abs(have - want), (2.0 ** -21 + 2.0 ** -22) * np.abs(want) + slack + 1e-30
        assert (diff <= tol).all(), (int((diff > tol).sum()), float((diff - tol).max()))
    pool.close()

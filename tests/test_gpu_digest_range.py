"""Digests of blocks whose channels are far apart in size: a bound that is not zero stays one, however small it is against the block's
largest key."""
import numpy as np
import pytest
import torch

import step_harness as SH
from oracle import steps as S

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("f32", 128)])
def test_bounds_of_channels_far_below_the_largest(dtype, d):
    """Channels from 1e38 down to the smallest subnormal numbers, of one sign, of the other, of both and zero: a quotient by the block's
    power of two that no fp32 number can hold still rounds up to 1, or down to -1."""
    pool = SH.Pool(2, 1, d, dtype, 12)
    pool.fill(3)
    k, v = (x.clone() for x in pool.kv())
    size = 10.0 ** torch.linspace(38, -44, d, dtype=torch.float64, device="cuda").roll(7)
    for b in range(11):
        x = k[0, b].double() * size * 10.0 ** (-6.0 * b)
        sign = torch.arange(d, device="cuda") % 4
        x = torch.where(sign == 0, x.abs(), torch.where(sign == 1, -x.abs(), x)).clamp(-3e38, 3e38)
        x[..., 5] = 0
        k[0, b] = x.to(pool.dt)
    pool.put(k, v)
    buf = pool.digests()
    pool.ctx.tc_digest_blocks(0, 1, SH.i32(np.arange(12)), buf)
    torch.cuda.synchronize()
    bounds, exps = (x.cpu().numpy() for x in pool.digest_views(buf))
    k64, _ = pool.kv64()
    for b in range(12):
        want, e = S.digest(k64[0, b, 0])
        assert exps[0, 0, b] == e
        np.testing.assert_array_equal(bounds[0, 0, b], want, err_msg="block %d" % b)
    pool.close()

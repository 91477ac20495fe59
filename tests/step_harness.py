"""Set-up shared by the tests of the token-step operators: a pool of sequence blocks that the test fills itself, and the same
keys and values as fp64 arrays."""
from __future__ import annotations

import numpy as np
import torch

VPOS = np.array([(t & 3) | ((t & 4) << 1) | ((t & 8) >> 1) for t in range(16)])
PAD_SHIFT = 27


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def i64(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int64)).cuda()


class Pool:
    """A context whose pool holds `n_blocks` blocks in each of `layers` layers, `first` of them (a table slot) before the first
    sequence block.  Every byte starts as a NaN of either type."""

    def __init__(self, hq, hkv, d, dtype, n_blocks, layers=1, slot_blocks=0):
        from paper_2601_08743_amd import binding as B
        self.B, self.hq, self.hkv, self.d, self.layers, self.n = B, hq, hkv, d, layers, n_blocks
        self.bf16 = dtype == "bf16"
        self.dt = torch.bfloat16 if self.bf16 else torch.float32
        self.first = slot_blocks
        self.cfg = B.make_config(layers, hq, hkv, d, B.TC_BF16 if self.bf16 else B.TC_F32, n_blocks, 1 if slot_blocks else 0,
                                 16 * max(1, slot_blocks))
        self.raw = torch.full((B.tc_pool_bytes(self.cfg) // 4,), 0x7FC07FC0, dtype=torch.int32, device="cuda")
        self.ctx = B.Context(self.cfg, self.raw, self.raw.numel() * 4)
        elems = self.raw.view(self.dt)
        per = 2 * hkv * 16 * d
        self.seq = elems[layers * slot_blocks * per:].view(layers, n_blocks - slot_blocks, 2, hkv * 16 * d)

    def kv(self):
        """(K, V) of every sequence block as the kernels left them, torch [layers][blocks][Hkv][16][D]."""
        k = self.seq[:, :, 0].reshape(self.layers, -1, self.hkv, 16, self.d)
        if not self.bf16:
            return k, self.seq[:, :, 1].reshape(self.layers, -1, self.hkv, 16, self.d)
        v = self.seq[:, :, 1].reshape(self.layers, -1, self.hkv, self.d, 16)
        return k, v[..., torch.from_numpy(VPOS).cuda()].transpose(-1, -2)

    def kv64(self):
        return tuple(x.double().cpu().numpy() for x in self.kv())

    def put(self, k, v):
        """K, V as torch [layers][blocks][Hkv][16][D] into the sequence blocks."""
        n = self.seq.shape[1]
        self.seq[:, :, 0] = k.to(self.dt).reshape(self.layers, n, -1)
        if self.bf16:
            t = torch.empty((self.layers, n, self.hkv, self.d, 16), dtype=self.dt, device="cuda")
            t[..., torch.from_numpy(VPOS).cuda()] = v.to(self.dt).transpose(-1, -2)
            self.seq[:, :, 1] = t.reshape(self.layers, n, -1)
        else:
            self.seq[:, :, 1] = v.reshape(self.layers, n, -1)

    def fill(self, seed, spread=1.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        shape = (self.layers, self.seq.shape[1], self.hkv, 16, self.d)
        centre = torch.randn(shape[:3] + (1, self.d), generator=g, device="cuda")
        k = centre * spread + 0.5 * torch.randn(shape, generator=g, device="cuda")
        self.put(k, torch.randn(shape, generator=g, device="cuda"))

    def rows(self, n, heads, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        return torch.randn((n, heads, self.d), generator=g, device="cuda").to(self.dt)

    def digests(self):
        return torch.full((self.B.tc_digest_bytes(self.cfg),), 99, dtype=torch.int8, device="cuda")

    def digest_views(self, buf):
        m = self.layers * self.hkv * self.n * 2 * self.d
        return buf[:m].view(self.layers, self.hkv, self.n, 2, self.d), buf[m:].view(self.layers, self.hkv, self.n)

    def workspace(self, n_tokens, max_blocks, n_list):
        need = self.B.tc_sparse_workspace_bytes(self.cfg, n_tokens, max_blocks, n_list)
        assert need > 0
        return torch.full((need,), 0xAB, dtype=torch.uint8, device="cuda")

    def close(self):
        torch.cuda.synchronize()
        self.ctx.tc_destroy()


def attn_tolerance(ref, p_abs_v, size, bf16, n_keys):
    """What rounding may leave between the kernels' output and the fp64 one, from the number of roundings.

    A score is a sum of D products taken in fp32: off by at most (D + 2) 2^-24 of sum |q_d k_d| scale (`size`), here with
    D <= 128; the weight that follows is off by that and by the exponential's 2^-21, relatively: delta.  The quotient of two sums
    of such weights over n keys adds 2 n 2^-24 and doubles delta.  In bf16 each weight is also rounded for the product with
    the values, by 2^-8 of it at most, and the output by 2^-8 of itself; in fp32 the output's rounding is 2^-24."""
    delta = 130 * 2.0 ** -24 * size[..., None] + 2.0 ** -21
    rel = 2 * delta + 2 * (n_keys + 8) * 2.0 ** -24
    if bf16:
        return 2.0 ** -8 * np.abs(ref) + (rel + 2.0 ** -8 * (1 + rel)) * p_abs_v * (1 + 2.0 ** -8) + 1e-30
    return 2.0 ** -24 * np.abs(ref) + rel * p_abs_v + 1e-30

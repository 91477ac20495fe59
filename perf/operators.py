"""Operators of a token step that stays on the GPU, as cases that can be timed: each is one pass through one operator.

``tables``   block tables and slot maps of a step from the requests' lengths
``append``   queries and keys encoded by position (one axis, or time / height / width), keys and values put into the pool
``digest``   bounds of the keys of pool blocks, in 8 bits
``sparse``   lists of blocks chosen by those bounds, and attention over the listed blocks

With ``own`` false a pass computes the operator with elementary torch operations, with ``own`` true through
``paper_2601_08743_amd.binding``.  Both work on the same buffers: a pool of sequence blocks in one layer,
``[n_blocks][2][Hkv * 16 * D]`` - K as ``[Hkv][16][D]``, V likewise in fp32 and as ``[Hkv][D][16]`` in bf16, where token t
of a block stands at position ``_VPOS[t]`` - and digests, int8 ``[Hkv][n_blocks][2][D]`` (upper, lower bounds) followed by
an exponent each, ``[Hkv][n_blocks]``.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

ROPE_THETA = 1.0e6
_VPOS = [(t & 3) | ((t & 4) << 1) | ((t & 8) >> 1) for t in range(16)]
_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# attention heads and element type of the configurations the framework is built for
_SHAPES = {"small": dict(q_heads=8, kv_heads=2, head_dim=64, dtype="f32"),
           "wide32": dict(q_heads=8, kv_heads=2, head_dim=128, dtype="f32"),
           "7b": dict(q_heads=28, kv_heads=4, head_dim=128, dtype="bf16"),
           "8b": dict(q_heads=32, kv_heads=8, head_dim=128, dtype="bf16"),
           "14b": dict(q_heads=40, kv_heads=8, head_dim=128, dtype="bf16")}


def _tables(requests, held, new, layout):
    return dict(op="tables", requests=requests, held_min=held[0], held_max=held[1], new_min=new[0], new_max=new[1], layout=layout)


def _append(shape, requests, held, new, layout, axes=1, fused=False):
    return dict(op="append", **_SHAPES[shape], requests=requests, held_min=held[0], held_max=held[1], new_min=new[0],
                new_max=new[1], layout=layout, axes=axes, fused=fused)


def _digest(shape, blocks, layers, layout):
    return dict(op="digest", **_SHAPES[shape], blocks=blocks, layers=layers, layout=layout)


def _sparse(shape, requests, held, new, layout, sink, top, local, padded=0):
    return dict(op="sparse", **_SHAPES[shape], requests=requests, held_min=held[0], held_max=held[1], new_min=new[0],
                new_max=new[1], layout=layout, sink=sink, top=top, local=local, padded=padded)


def listed():
    return [
        # the next token of four sequences: the smallest call, launches and latency
        dict(_tables(4, (700, 5000), (1, 1), 11), name="tables_token"),
        # a service's whole round: 300 requests, some at their first chunk of prompt, some waiting (no new token), most decoding
        dict(_tables(300, (0, 20000), (0, 120), 12), name="tables_round"),
        # the next token of a batch of 32, a layer
        dict(_append("7b", 32, (700, 5000), (1, 1), 21), name="append_token"),
        # suffixes of four long-schema queries with positions in time, height and width, rows of one fused projection
        dict(_append("8b", 4, (20000, 24600), (512, 512), 22, axes=3, fused=True), name="append_suffix"),
        # an fp32 reference run: ragged suffixes
        dict(_append("wide32", 7, (0, 900), (1, 90), 23), name="append_f32"),
        # the long-schema batch after its stitch: 6168 blocks in two layers
        dict(_digest("8b", 6168, 2, 31), name="digest_long"),
        # one small sequence in fp32
        dict(_digest("small", 47, 1, 32), name="digest_f32"),
        # a token of one sequence over twelve tables
        dict(_sparse("7b", 1, (4600, 4600), (1, 1), 41, 1, 48, 4), name="sparse_one"),
        # a token of 32 sequences, a batch padded to 34 rows
        dict(_sparse("7b", 32, (700, 5000), (1, 1), 42, 1, 40, 8, padded=2), name="sparse_batch"),
        # a token of four sequences over long schemas
        dict(_sparse("8b", 4, (22000, 27000), (1, 1), 43, 2, 118, 8), name="sparse_long"),
        # questions of some tokens against long schemas
        dict(_sparse("8b", 8, (6000, 14000), (33, 128), 44, 1, 60, 3), name="sparse_suffix"),
        # the same step in fp32
        dict(_sparse("small", 5, (100, 3000), (1, 3), 45, 1, 21, 2), name="sparse_f32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of the same ranges: 1..300 requests that hold 0..27000 tokens, 0..512 new ones each, 1..8 KV heads with
    1..8 query heads, lists of 2..160 blocks."""
    while True:
        c = dict(op=rng.choice(["tables", "append", "digest", "sparse", "sparse"]), layout=rng.randrange(1 << 30))
        if rng.random() < 0.4:
            c.update(_SHAPES[rng.choice(sorted(_SHAPES))])
        else:
            f32 = rng.random() < 0.3
            kv = rng.choice([1, 2, 3, 4, 8])
            c.update(q_heads=kv * rng.randint(1, 8), kv_heads=kv, head_dim=rng.choice([64, 128]) if f32 else 128,
                     dtype="f32" if f32 else "bf16")
        held = _log_int(rng, 1, 27000)
        c.update(held_min=held // 3 if rng.random() < 0.7 else 0, held_max=held)
        if c["op"] == "tables":
            for k in ("q_heads", "kv_heads", "head_dim", "dtype"):
                del c[k]
            new = _log_int(rng, 1, 512)
            c.update(requests=_log_int(rng, 1, 300), new_min=rng.choice([0, 1, new]), new_max=new)
        elif c["op"] == "append":
            new = _log_int(rng, 1, 512)
            c.update(requests=_log_int(rng, 1, 32), new_min=rng.choice([0, 1, new]), new_max=new, axes=rng.choice([1, 1, 2, 3]),
                     fused=rng.random() < 0.5)
        elif c["op"] == "digest":
            del c["held_min"], c["held_max"]
            c.update(blocks=_log_int(rng, 1, 6000), layers=rng.randint(1, 3))
        else:
            new = _log_int(rng, 1, 64) if rng.random() < 0.4 else 1
            c.update(requests=_log_int(rng, 1, 48), new_min=rng.choice([1, new]), new_max=new, sink=rng.randint(0, 2),
                     top=_log_int(rng, 1, 150), local=rng.randint(1, 8), padded=rng.choice([0, 0, 3]))
        if c["op"] == "tables" and c["requests"] * c["new_max"] > 40000:
            continue
        w = work(c)
        limit = {"tables": 1e6, "append": 4.5e7, "digest": 4.2e8, "sparse": 2.5e8}[c["op"]]
        if w["bytes"] <= limit and w["flops"] <= 8e9 and _pool_bytes(c) <= 1.2e9:
            return c


# ------------------------------------------------------------------------------------------------ structure

def _lengths(c):
    """How many tokens each request holds, and how many new ones it brings."""
    rng = np.random.default_rng([c["layout"], 1])
    n = c["requests"]
    held = rng.integers(c["held_min"], c["held_max"] + 1, size=n)
    new = rng.integers(c["new_min"], c["new_max"] + 1, size=n)
    if c["op"] == "tables" and c["new_min"] == 0 and n >= 8:        # most requests of a service's round decode
        new = np.where(rng.random(n) < 0.75, np.minimum(new, 1), new)
    return held.astype(np.int64), new.astype(np.int64)


def _n_blocks(tokens):
    return (tokens + 15) // 16


def _esize(c):
    return 4 if c["dtype"] == "f32" else 2


def _block_elems(c):
    return 2 * c["kv_heads"] * 16 * c["head_dim"]


def _pool_blocks(c):
    if c["op"] == "digest":
        return c["blocks"] + 3
    held, new = _lengths(c)
    return int(_n_blocks(held + new).sum()) + 3


def _pool_bytes(c):
    return 0 if c["op"] == "tables" else _pool_blocks(c) * _block_elems(c) * _esize(c) * c.get("layers", 1)


def work(c):
    """Bytes: lengths, positions and lists once, the rows of q, k, v once in and once out; digests of the candidates and the
    listed blocks once for each request and KV head (a request's tokens choose much the same blocks).  Operations: the
    products of the score (counted as those of q with both bounds) and of the attention."""
    if c["op"] == "digest":
        n = c["blocks"] * c["kv_heads"] * c["layers"]
        return {"bytes": n * (16 * c["head_dim"] * _esize(c) + 2 * c["head_dim"] + 1) + 4 * c["blocks"],
                "flops": 2.0 * n * 16 * c["head_dim"]}
    held, new = _lengths(c)
    n_tok = int(new.sum())
    if c["op"] == "tables":
        taken = int((_n_blocks(held + new) - _n_blocks(held)).sum())
        return {"bytes": 16 * c["requests"] + 20 * n_tok + 8 * taken, "flops": float(4 * n_tok)}
    hq, hkv, d, e = c["q_heads"], c["kv_heads"], c["head_dim"], _esize(c)
    if c["op"] == "append":
        return {"bytes": 2 * n_tok * (hq + 2 * hkv) * d * e + n_tok * (8 + 4 * c["axes"]), "flops": 3.0 * n_tok * (hq + hkv) * d}
    n_bytes, n_flops = 0.0, 0.0
    for h, s in zip(held, new):
        if not s:
            continue
        cand = max(0, (int(h) + int(s)) // 16 - c["sink"] - c["local"])
        blocks = min(_n_blocks(int(h) + int(s)), c["sink"] + c["top"] + c["local"] + (int(s) + 15) // 16)
        n_bytes += hkv * (cand * (2 * d + 1) + blocks * 32 * d * e) + 2.0 * s * hq * d * e
        n_flops += float(s) * hq * d * (4.0 * cand + 64.0 * blocks)
    return {"bytes": n_bytes + 4.0 * n_tok * hkv * (c["sink"] + c["top"] + c["local"]), "flops": n_flops}


# ------------------------------------------------------------------------------------------------ inputs

def _gpu_rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _block_table(c, held, new, rng, spread):
    """Tables over a pool whose free blocks have been mixed by earlier sequences; entries of the step's new blocks are
    filled where `spread`, and listed as spare otherwise."""
    have, want = _n_blocks(held), _n_blocks(held + new)
    n = _pool_blocks(c)
    ids = rng.permutation(n).astype(np.int32)
    table = np.full((len(held), int(want.max()) + 2), -1, dtype=np.int32)
    at = 0
    for i in range(len(held)):
        k = int(want[i] if spread else have[i])
        table[i, :k] = ids[at:at + k]
        at += k
    return table, ids[at:]


def _tokens(held, new, table):
    """Request, position and slot of each new token."""
    seq = np.repeat(np.arange(len(held)), new)
    first = np.concatenate([[0], np.cumsum(new)])[:-1]
    pos = held[seq] + np.arange(len(seq)) - first[seq]
    slot = table[seq, pos // 16].astype(np.int64) * 16 + pos % 16
    return seq, pos, slot


def _normal(g, shape, dtype, scale=None):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if scale is not None:
        x *= scale
    return x.to(dtype)


def _keys_like(c, g, layers, n):
    """A pool: keys with channels of unequal size that are alike within a block (a table's rows), values N(0, 1)."""
    hkv, d, dt = c["kv_heads"], c["head_dim"], _DTYPES[c["dtype"]]
    channel = torch.exp(0.5 * torch.randn((hkv, 1, d), generator=g, device="cuda"))
    pool = torch.empty((layers, n, 2, hkv * 16 * d), dtype=dt, device="cuda")
    for layer in range(layers):
        for a in range(0, n, 2048):
            m = min(2048, n - a)
            centre = torch.randn((m, hkv, 1, d), generator=g, device="cuda")
            k = (0.8 * centre + 0.6 * torch.randn((m, hkv, 16, d), generator=g, device="cuda")) * channel
            pool[layer, a:a + m, 0] = k.reshape(m, -1).to(dt)
            pool[layer, a:a + m, 1] = _normal(g, (m, hkv * 16 * d), dt)
    return pool


def _inputs(c, seed):
    rng, g = np.random.default_rng([c["layout"], 2, seed]), _gpu_rng(seed * 1000003 + 17)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    s = {}
    if c["op"] == "digest":
        s["pool"] = _keys_like(c, g, c["layers"], c["blocks"] + 3)
        s["entries"] = i32(rng.permutation(c["blocks"] + 3)[:c["blocks"]])
        return s
    held, new = _lengths(c)
    if c["op"] == "tables":
        table, spare = _block_table(c, held, new, rng, False)
        s.update(seq_len=i32(held), new_len=i32(new), table=i32(table), spare=i32(spare), spare_used=i32([0]))
        s["n_tokens"] = int(new.sum()) + 5                           # rows a program keeps for a fuller round
        return s
    hq, hkv, d, dt = c["q_heads"], c["kv_heads"], c["head_dim"], _DTYPES[c["dtype"]]
    table, _ = _block_table(c, held, new, rng, True)
    seq, pos, slot = _tokens(held, new, table)
    n = len(seq)
    s["pool"] = _keys_like(c, g, 1, _pool_blocks(c))
    if c["op"] == "append":
        if c["fused"]:
            rows = _normal(g, (n, hq + 2 * hkv, d), dt)
            s["q"], s["k"], s["v"] = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
        else:
            s["q"], s["k"], s["v"] = (_normal(g, (n, h, d), dt) for h in (hq, hkv, hkv))
        axes = np.stack([pos] + [pos // 2 + rng.integers(0, 60, size=n) for _ in range(c["axes"] - 1)])
        s["pos"] = i32(axes)
        cut = np.linspace(0, d // 2, c["axes"] + 1).round().astype(int)
        s["sections"] = [int(b - a) for a, b in zip(cut[:-1], cut[1:])]
        s["slot_map"] = torch.from_numpy(slot).cuda()
        return s
    s["q"] = _normal(g, (n + c["padded"], hq, d), dt)
    pad = -np.ones(c["padded"], dtype=np.int64)
    s["token_seq"], s["token_pos"] = i32(np.concatenate([seq, pad])), i32(np.concatenate([pos, pad]))
    s["table"] = i32(table)
    s["digests"] = torch.zeros(hkv * _pool_blocks(c) * (2 * d + 1), dtype=torch.int8, device="cuda")
    bounds, exps = _digest_views(c, s["digests"], 1, _pool_blocks(c))
    b, e = _plain_digest(s["pool"][0, :, 0].reshape(-1, hkv, 16, d))
    bounds[0], exps[0] = b.transpose(0, 1), e.transpose(0, 1)
    return s


def _digest_views(c, buf, layers, n):
    hkv, d = c["kv_heads"], c["head_dim"]
    m = layers * hkv * n * 2 * d
    return buf[:m].view(layers, hkv, n, 2, d), buf[m:m + layers * hkv * n].view(layers, hkv, n)


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s["case"] = c
    dev = "cuda"
    if c["op"] == "tables":
        n, b = s["n_tokens"], c["requests"]
        s["out"] = dict(spare_next=torch.zeros(1, dtype=torch.int32, device=dev), end_len=torch.zeros(b, dtype=torch.int32, device=dev),
                        cu_new=torch.zeros(b + 1, dtype=torch.int32, device=dev), slot_map=torch.zeros(n, dtype=torch.int64, device=dev),
                        token_pos=torch.zeros(n, dtype=torch.int32, device=dev), token_seq=torch.zeros(n, dtype=torch.int32, device=dev),
                        full_block=torch.zeros(n, dtype=torch.int32, device=dev), status=torch.zeros(2, dtype=torch.int32, device=dev))
    elif c["op"] == "append":
        s["q_out"] = torch.zeros(s["q"].shape, dtype=s["q"].dtype, device=dev)
    elif c["op"] == "digest":
        s["digests"] = torch.zeros(c["layers"] * c["kv_heads"] * (c["blocks"] + 3) * (2 * c["head_dim"] + 1), dtype=torch.int8, device=dev)
    else:
        n_list = c["sink"] + c["top"] + c["local"]
        s["lists"] = torch.full((s["q"].shape[0], c["kv_heads"], n_list), -1, dtype=torch.int32, device=dev)
        s["attn_out"] = torch.zeros_like(s["q"])
    if own:
        from paper_2601_08743_amd import binding as B
        shape = dict(_SHAPES["7b"], **{k: c[k] for k in ("q_heads", "kv_heads", "head_dim", "dtype") if k in c})
        pool = s.get("pool")
        if pool is None:                                             # the tables' blocks live in some pool
            pool = torch.empty((1, _pool_blocks(c), _block_elems(shape)), dtype=_DTYPES[shape["dtype"]], device=dev)
        cfg = B.make_config(c.get("layers", 1), shape["q_heads"], shape["kv_heads"], shape["head_dim"],
                            B.TC_F32 if shape["dtype"] == "f32" else B.TC_BF16, _pool_blocks(c), 0, 16)
        s["ctx"] = B.Context(cfg, pool)
        if c["op"] == "sparse":
            need = B.tc_sparse_workspace_bytes(cfg, s["q"].shape[0], s["table"].shape[1], s["lists"].shape[2])
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device=dev)
    return s


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    s, c = state, state["case"]
    st = torch.cuda.current_stream()
    if c["op"] == "tables":
        o = s["out"]
        if own:
            s["ctx"].tc_step_tables(s["seq_len"], s["new_len"], s["table"], s["spare"], s["spare_used"], o["spare_next"], o["end_len"],
                                    o["cu_new"], o["slot_map"], o["token_pos"], o["token_seq"], o["full_block"], o["status"], st)
            return dict(o, table=s["table"])
        return _plain_tables(s)
    if c["op"] == "append":
        if own:
            s["ctx"].tc_rope_append(0, s["q"], s["k"], s["v"], s["pos"], ROPE_THETA, s["slot_map"], s["q_out"], s["sections"], st)
            return s["q_out"], s["pool"]
        return _plain_append(s)
    if c["op"] == "digest":
        n = c["blocks"] + 3
        if own:
            s["ctx"].tc_digest_blocks(0, c["layers"], s["entries"], s["digests"], st)
        else:
            bounds, exps = _digest_views(c, s["digests"], c["layers"], n)
            ids = s["entries"].long()
            for layer in range(c["layers"]):
                for part in ids.split(1024):
                    b, e = _plain_digest(s["pool"][layer, part, 0].view(-1, c["kv_heads"], 16, c["head_dim"]))
                    bounds[layer, :, part] = b.transpose(0, 1)
                    exps[layer, :, part] = e.transpose(0, 1)
        return s["digests"]
    scale = 1.0 / math.sqrt(c["head_dim"])
    if own:
        s["ctx"].tc_select_blocks(0, s["q"], s["token_seq"], s["token_pos"], s["table"], s["digests"], c["sink"], c["top"], c["local"],
                                  s["lists"], s["workspace"], st)
        s["ctx"].tc_block_attn(0, s["q"], s["token_seq"], s["token_pos"], s["table"], s["lists"], s["attn_out"], scale, s["workspace"], st)
        return s["lists"], s["attn_out"]
    return _plain_sparse(s, scale)


def _plain_tables(s):
    held, new, table = s["seq_len"].long(), s["new_len"].long(), s["table"]
    have, want = (held + 15) // 16, (held + new + 15) // 16
    need = want - have
    before = torch.cumsum(need, 0) - need
    used = s["spare_used"].long()
    j = torch.arange(table.shape[1], device="cuda")
    fresh = (j >= have[:, None]) & (j < want[:, None])
    at = torch.where(fresh, used + before[:, None] + j - have[:, None], 0)
    table = torch.where(fresh, s["spare"][at], table)
    end = torch.cumsum(new, 0)
    cu = torch.cat([torch.zeros_like(end[:1]), end])
    n = torch.arange(s["n_tokens"], device="cuda")
    live = n < end[-1]
    seq = torch.clamp(torch.searchsorted(end, n, right=True), max=len(held) - 1)
    pos = torch.where(live, held[seq] + n - cu[seq], 0)
    block = table[seq, pos // 16]
    none = torch.full_like(n, -1)
    taken = need.sum().reshape(1)
    return dict(spare_next=(used + taken).int(), end_len=(held + new).int(), cu_new=cu.int(),
                slot_map=torch.where(live, block.long() * 16 + pos % 16, none), token_pos=torch.where(live, pos, none).int(),
                token_seq=torch.where(live, seq, none).int(), full_block=torch.where(live & (pos % 16 == 15), block.long(), none).int(),
                status=torch.cat([torch.zeros_like(taken), taken]).int(), table=table)


def _rotate(x, turn):
    """Pairs (j, j + D/2) of every head turned; `turn` in radians, [n][1][D/2]."""
    half = x.shape[-1] // 2
    a, b = x[..., :half], x[..., half:]
    cos, sin = torch.cos(turn).to(x.dtype), torch.sin(turn).to(x.dtype)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _turns(pos, sections, d):
    """Angles in 64 bits: the axis of a pair is that of the section it falls into."""
    axis = torch.repeat_interleave(torch.arange(len(sections), device="cuda"), torch.tensor(sections, device="cuda"))
    freq = ROPE_THETA ** (-2.0 * torch.arange(d // 2, device="cuda", dtype=torch.float64) / d)
    return (pos[axis].T.double() * freq)[:, None, :]


def _put(pool, c, slot, k, v):
    """Rows to their slots of one layer's pool; a block that gets its first token is zero behind the step's last one."""
    hkv, d = c["kv_heads"], c["head_dim"]
    blk, t = slot // 16, slot % 16
    kp = pool[:, 0].view(-1, hkv, 16, d)
    vp = pool[:, 1].view(-1, hkv, d, 16) if c["dtype"] == "bf16" else pool[:, 1].view(-1, hkv, 16, d)
    begun = blk[t == 0]
    kp[begun] = 0
    vp[begun] = 0
    kp[blk, :, t] = k
    if c["dtype"] == "bf16":
        vp[blk, :, :, torch.tensor(_VPOS, device="cuda")[t]] = v
    else:
        vp[blk, :, t] = v


def _plain_append(s):
    c, dt = s["case"], s["q"].dtype
    turn = _turns(s["pos"], s["sections"], c["head_dim"])
    s["q_out"].copy_(_rotate(s["q"].float(), turn).to(dt))
    _put(s["pool"][0], c, s["slot_map"], _rotate(s["k"].float(), turn).to(dt), s["v"])
    return s["q_out"], s["pool"]


def _pow2(e):
    """2^e in fp32, -126 <= e <= 127."""
    return ((e + 127).int() << 23).view(torch.float32)


def _exponent(size):
    """The smallest e >= -126 with size <= 127 * 2^e (size finite, fp32)."""
    e = torch.clamp((size.view(torch.int32) >> 23) - 127 - 6, min=-126)
    return e + (size * _pow2(-e) > 127).int()


def _plain_digest(k):
    """Keys [..][16][D] -> bounds int8 [..][2][D] and exponents int8 [..] (127: a key that is not finite)."""
    k = k.float()
    hi, lo = k.amax(-2), k.amin(-2)
    size = torch.maximum(hi.abs(), lo.abs()).amax(-1)
    ok = torch.isfinite(size)
    e = _exponent(torch.where(ok, size, torch.zeros_like(size)))
    up = _pow2(-e)[..., None]
    bounds = torch.stack([torch.ceil(hi * up), torch.floor(lo * up)], dim=-2)
    bounds = torch.where(ok[..., None, None], bounds, torch.zeros_like(bounds))
    return bounds.to(torch.int8), torch.where(ok, e, torch.full_like(e, 127)).to(torch.int8)


def _plain_scores(c, q, ids, bounds, exps):
    """Scores [n][Hkv][blocks] of the blocks `ids` [n][blocks] for queries [n][Hq][D]."""
    hkv, d = c["kv_heads"], c["head_dim"]
    q = q.float().view(q.shape[0], hkv, -1, d)
    size = q.abs().amax(-1)
    ok = torch.isfinite(size)
    f = _exponent(torch.where(ok, size, torch.zeros_like(size)))
    qi = torch.where(ok[..., None], torch.round(q * _pow2(-f)[..., None]), torch.zeros_like(q))
    both = torch.cat([torch.clamp(qi, min=0), torch.clamp(qi, max=0)], dim=-1)               # [n][Hkv][G][2D]
    dig = bounds[:, ids].transpose(0, 1).reshape(q.shape[0], hkv, ids.shape[1], 2 * d).float()
    dot = both @ dig.transpose(-1, -2)                                                        # integers below 2^24
    e = exps[:, ids].transpose(0, 1).int()[:, :, None]                                        # [n][Hkv][1][blocks]
    score = dot * _pow2(f)[..., None] * _pow2(torch.clamp(e, max=126))
    score = torch.where(ok[..., None], score, torch.full_like(score, -math.inf))
    return torch.where(e[:, :, 0] == 127, torch.full_like(score[:, :, 0], math.inf), score.amax(2))


def _plain_lists(c, score, pos):
    """The first `sink` blocks, the `top` best of those between, the last `local`, in ascending order, then -1."""
    n, hkv, m = score.shape
    j = torch.arange(m, device="cuda")
    own_block = (pos // 16)[:, None]
    w0 = torch.clamp(own_block - (c["local"] - 1), min=0)
    first = torch.clamp(w0, max=c["sink"])
    cand = ((j >= first) & (j < w0))[:, None].expand(n, hkv, m)
    order = torch.sort(torch.where(cand, score, torch.full_like(score, -math.inf)), dim=-1, descending=True, stable=True).indices
    # a candidate that scores -infinity still goes before what is no candidate
    order = torch.gather(order, -1, torch.sort((~torch.gather(cand, -1, order)).int(), dim=-1, stable=True).indices)
    taken = torch.zeros((n, hkv, m), dtype=torch.bool, device="cuda")
    taken.scatter_(-1, order[..., :c["top"]], True)
    taken = (taken & cand) | ((j < first) | ((j >= w0) & (j <= own_block)))[:, None]
    n_list = c["sink"] + c["top"] + c["local"]
    key = torch.sort(torch.where(taken, j, m), dim=-1).values[..., :n_list]
    key = torch.where(key < m, key, -1)
    if key.shape[-1] < n_list:
        key = torch.nn.functional.pad(key, (0, n_list - key.shape[-1]), value=-1)
    return key


def _plain_attend(c, q, lists, table_rows, pos, pool, scale, dtype):
    """Attention of queries [n][Hq][D] over the listed blocks, in `dtype`."""
    hkv, d, n = c["kv_heads"], c["head_dim"], q.shape[0]
    phys = torch.gather(table_rows, 1, torch.clamp(lists, min=0).reshape(n, -1)).view(lists.shape).long()
    phys = torch.clamp(phys, min=0)
    head = torch.arange(hkv, device="cuda")[None, :, None]
    k = pool[:, 0].view(-1, hkv, 16, d)[phys, head].to(dtype)                                 # [n][Hkv][L][16][D]
    if c["dtype"] == "bf16":
        v = pool[:, 1].view(-1, hkv, d, 16)[phys, head][..., _VPOS].transpose(-1, -2).to(dtype)
    else:
        v = pool[:, 1].view(-1, hkv, 16, d)[phys, head].to(dtype)
    k, v = k.reshape(n, hkv, -1, d), v.reshape(n, hkv, -1, d)
    at = (lists[..., None] * 16 + torch.arange(16, device="cuda")).reshape(n, hkv, 1, -1)
    seen = (lists[..., None].expand(*lists.shape, 16).reshape(n, hkv, 1, -1) >= 0) & (at <= pos[:, None, None, None])
    s = (q.to(dtype).view(n, hkv, -1, d) @ k.transpose(-1, -2)) * scale
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    v = torch.where(seen.transpose(-1, -2), v, torch.zeros_like(v))
    return (p @ v).reshape(n, -1, d)


def _plain_sparse(s, scale):
    c, m = s["case"], s["table"].shape[1]
    n_blocks = s["pool"].shape[1]
    bounds, exps = _digest_views(c, s["digests"], 1, n_blocks)
    live = s["q"].shape[0] - c["padded"]                             # (padded rows stay as they were)
    lists = s["lists"]
    at_once = max(1, int(1.5e8 / (c["kv_heads"] * max(m * 2 * c["head_dim"], lists.shape[2] * 32 * c["head_dim"]))))
    for a in range(0, live, at_once):
        part = slice(a, min(live, a + at_once))
        rows = s["table"][s["token_seq"][part].long()].long()
        pos = s["token_pos"][part].long()
        score = _plain_scores(c, s["q"][part], torch.clamp(rows, min=0), bounds[0], exps[0])
        key = _plain_lists(c, score, pos)
        lists[part] = key.int()
        s["attn_out"][part] = _plain_attend(c, s["q"][part], key, rows, pos, s["pool"][0], scale, torch.float32).to(s["q"].dtype)
    return lists, s["attn_out"]


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    """Whole numbers have no other value in 64 bits and are not repeated here, but for the digests, whose bounds come from
    the definition; the attention takes the blocks that the integer score selects, computed token by token."""
    c = case
    if c["op"] == "tables":
        return None
    s = _inputs(c, seed)
    if c["op"] == "append":
        return _exact_append(c, s)
    if c["op"] == "digest":
        return _exact_digest(c, s)
    return _exact_sparse(c, s)


def _two_to(e):
    """2^e for whole e, in 64 bits (a power computed by exp and log is a rounding off, and ties would break)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_append(c, s):
    hq, hkv, d, n = c["q_heads"], c["kv_heads"], c["head_dim"], s["q"].shape[0]
    axis = [a for a, width in enumerate(s["sections"]) for _ in range(width)]
    pos = s["pos"].cpu().numpy()[axis].T.astype(np.float64)                                   # [n][D/2]
    z = np.exp(1j * pos * np.power(ROPE_THETA, -np.arange(0, d, 2) / d))[:, None, :]

    def turned(x):
        x = x.double().cpu().numpy()
        y = (x[..., :d // 2] + 1j * x[..., d // 2:]) * z
        return np.concatenate([y.real, y.imag], axis=-1)

    q, k, v = turned(s["q"]), turned(s["k"]), s["v"].double().cpu().numpy()
    pool = s["pool"].double().cpu().numpy()
    slots = s["slot_map"].cpu().numpy()
    transposed = c["dtype"] == "bf16"
    for i in range(n):
        b, t = divmod(int(slots[i]), 16)
        if t == 0:
            pool[0, b] = 0.0
        pool[0, b, 0].reshape(hkv, 16, d)[:, t] = k[i]
        if transposed:
            pool[0, b, 1].reshape(hkv, d, 16)[:, :, _VPOS[t]] = v[i]
        else:
            pool[0, b, 1].reshape(hkv, 16, d)[:, t] = v[i]
    return torch.from_numpy(q), torch.from_numpy(pool)


def _exact_digest(c, s):
    layers, hkv, d, n = c["layers"], c["kv_heads"], c["head_dim"], c["blocks"] + 3
    bounds = torch.zeros((layers, hkv, n, 2, d), dtype=torch.float64)
    exps = torch.zeros((layers, hkv, n), dtype=torch.float64)
    ids = s["entries"].long()
    for layer in range(layers):
        k = s["pool"][layer, ids, 0].view(-1, hkv, 16, d).double()
        hi, lo = k.max(2).values, k.min(2).values
        size = torch.maximum(hi, -lo).max(-1).values.clamp(min=1e-300)
        e = torch.ceil(torch.log2(size / 127.0))                    # then put right where the logarithm was rounded
        e = torch.where(size > 127.0 * _two_to(e), e + 1, e)
        e = torch.where(size <= 127.0 * _two_to(e - 1), e - 1, e).clamp(min=-126.0)
        step = _two_to(e)[..., None]
        both = torch.stack([torch.ceil(hi / step), torch.floor(lo / step)], dim=2).transpose(0, 1).cpu()
        bounds[layer][:, ids.cpu()] = both
        exps[layer][:, ids.cpu()] = e.transpose(0, 1).cpu()
    return torch.cat([bounds.flatten(), exps.flatten()])


def _exact_sparse(c, s):
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    n = s["q"].shape[0] - c["padded"]
    if n > 1200:
        return None
    bounds, exps = _digest_views(c, s["digests"], 1, s["pool"].shape[1])
    seqs, poss, rows = s["token_seq"].tolist(), s["token_pos"].tolist(), s["table"].long()
    kp = s["pool"][0, :, 0].view(-1, hkv, 16, d)
    vp = s["pool"][0, :, 1].view(-1, hkv, d, 16) if c["dtype"] == "bf16" else s["pool"][0, :, 1].view(-1, hkv, 16, d)
    order = torch.tensor(_VPOS, device="cuda")
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    heads = torch.arange(hkv, device="cuda")[:, None]
    for i in range(n):
        p, last = poss[i], poss[i] // 16
        ids = rows[seqs[i], :last + 1]
        w0 = max(0, last - c["local"] + 1)
        first = min(c["sink"], w0)
        q = s["q"][i].double().view(hkv, -1, d)
        keep = [list(range(first)) + list(range(w0, last + 1)) for _ in range(hkv)]
        if first < w0:
            size = q.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -126)
            f = torch.ceil(torch.log2(size / 127.0))
            f = torch.where(size > 127.0 * _two_to(f), f + 1, f)
            f = torch.where(size <= 127.0 * _two_to(f - 1), f - 1, f).clamp(min=-126.0)
            qi = torch.round(q / _two_to(f))
            dig = bounds[0][:, ids[first:w0]].double()                                        # [Hkv][cand][2][D]
            dot = qi.clamp(min=0) @ dig[:, :, 0].transpose(1, 2) + qi.clamp(max=0) @ dig[:, :, 1].transpose(1, 2)
            score = (dot * _two_to(f) * _two_to(exps[0][:, ids[first:w0]])[:, None]).amax(1)
            ranked = torch.sort(score, dim=-1, descending=True, stable=True).indices[:, :c["top"]]
            keep = [sorted(a + [first + x for x in r]) for a, r in zip(keep, ranked.tolist())]
        at = torch.tensor(keep, device="cuda")                                                # [Hkv][blocks]
        k = kp[ids[at], heads].double().reshape(hkv, -1, d)
        v = vp[ids[at], heads].double()
        v = (v[..., order].transpose(-1, -2) if c["dtype"] == "bf16" else v).reshape(hkv, -1, d)
        seen = ((at[..., None] * 16 + torch.arange(16, device="cuda")) <= p).reshape(hkv, 1, -1)
        x = (q @ k.transpose(1, 2)) / math.sqrt(d)
        w = torch.softmax(torch.where(seen, x, torch.full_like(x, -math.inf)), dim=-1)
        out[i] = (w @ v).reshape(hq, d)
    return None, out

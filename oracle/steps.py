"""fp64 / integer models of the token-step operators (test infrastructure only): block tables and slot maps from lengths,
multi-axis rotary encoding, digests of blocks' keys, block lists by the integer score, attention over listed blocks.
Plain loops over requests, tokens and heads, from the definitions in include/tablecache.h."""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np


def step_tables(seq_len, new_len, table, spare, used: int, n_tokens: int, first_seq: int, n_blocks: int) -> dict:
    """What tc_step_tables leaves in its arrays; `table` is copied."""
    table = np.array(table, dtype=np.int64)
    B, max_blocks = table.shape
    seq_len, new_len = [int(x) for x in seq_len], [int(x) for x in new_len]
    rows = dict(slot_map=np.full(n_tokens, -1, np.int64), token_pos=np.full(n_tokens, -1, np.int64),
                token_seq=np.full(n_tokens, -1, np.int64), full_block=np.full(n_tokens, -1, np.int64))

    def refused(code, blocks):
        return dict(rows, table=table, spare_next=used, end_len=np.array(seq_len, dtype=np.int64),
                    cu_new=np.zeros(B + 1, np.int64), status=np.array([code, blocks]))

    if used < 0 or used > len(spare) or any(l < 0 or s < 0 or l + s > 16 * max_blocks for l, s in zip(seq_len, new_len)) or \
            sum(new_len) > n_tokens:
        return refused(-1, 0)
    need = [(l + s + 15) // 16 - (l + 15) // 16 for l, s in zip(seq_len, new_len)]
    if sum(need) > len(spare) - used:
        return refused(-3, sum(need))
    at, n, whole = used, 0, True
    for b in range(B):
        have = (seq_len[b] + 15) // 16
        for j in range(have, have + need[b]):
            table[b, j] = spare[at] if first_seq <= spare[at] < n_blocks else -1
            at += 1
        for p in range(seq_len[b], seq_len[b] + new_len[b]):
            block = int(table[b, p // 16])
            block = block & ((1 << 27) - 1) if block >= 0 else -1
            if first_seq <= block < n_blocks:
                rows["token_seq"][n], rows["token_pos"][n] = b, p
                rows["slot_map"][n] = 16 * block + p % 16
                if p % 16 == 15:
                    rows["full_block"][n] = block
            else:
                whole = False
            n += 1
    return dict(rows, table=table, spare_next=at, end_len=np.array(seq_len) + np.array(new_len),
                cu_new=np.concatenate([[0], np.cumsum(new_len)]), status=np.array([0 if whole else 1, sum(need)]))


def rotate(x: np.ndarray, pos: np.ndarray, sections: Sequence[int], theta: float) -> np.ndarray:
    """x [n][heads][D] in fp64 turned by pos [axes][n]; pair (j, j + D/2) belongs to the section that j falls into."""
    half = x.shape[-1] // 2
    axis = np.repeat(np.arange(len(sections)), sections)
    turn = np.asarray(pos, dtype=np.float64)[axis].T * theta ** (-np.arange(half) / half)
    c, s = np.cos(turn)[:, None], np.sin(turn)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


def exponent(size: float) -> int:
    """The smallest e >= -126 with size <= 127 * 2^e."""
    e = -126
    while size > 127.0 * 2.0 ** e:
        e += 1
    return e


def digest(keys: np.ndarray):
    """keys [tokens][D] (fp64, the block's own tokens) -> (bounds int [2][D], exponent)."""
    if not np.isfinite(keys).all():
        return np.zeros((2, keys.shape[1]), np.int64), 127
    hi, lo = keys.max(axis=0), keys.min(axis=0)
    e = exponent(max(np.abs(hi).max(), np.abs(lo).max()))
    return np.stack([np.ceil(hi / 2.0 ** e), np.floor(lo / 2.0 ** e)]).astype(np.int64), e


def score(q: np.ndarray, bounds: np.ndarray, e: int) -> float:
    """q [G][D] fp64 of one KV head's query heads; a block's digest -> its score (fp32 arithmetic on exact integers)."""
    best = -np.inf
    if e == 127:
        return np.inf
    for row in q:
        if not np.isfinite(row).all():
            continue
        f = exponent(np.abs(row).max())
        i = np.rint(row / 2.0 ** f).astype(np.int64)
        dot = int((np.maximum(i, 0) * bounds[0] + np.minimum(i, 0) * bounds[1]).sum())
        with np.errstate(over="ignore", under="ignore"):
            best = max(best, np.float32(np.float32(dot) * np.float32(2.0) ** np.float32(f)) * np.float32(2.0) ** np.float32(e))
    return float(best)


def scores(q: np.ndarray, bounds: np.ndarray, exps: np.ndarray) -> np.ndarray:
    """``score`` of many blocks at once: bounds [n][2][D], exps [n] (products of whole numbers, exact in fp64)."""
    ok = np.isfinite(q).all(axis=1)
    best = np.full(len(bounds), -np.inf, dtype=np.float32)
    for row in q[ok]:
        f = exponent(np.abs(row).max())
        i = np.rint(row / 2.0 ** f)
        dot = (bounds[:, 0] @ np.maximum(i, 0) + bounds[:, 1] @ np.minimum(i, 0)).astype(np.float32)
        with np.errstate(over="ignore", under="ignore", invalid="ignore"):
            best = np.maximum(best, dot * np.float32(2.0) ** np.float32(f) * np.float32(2.0) ** exps.astype(np.float32))
    return np.where(exps == 127, np.float32(np.inf), best)


def block_list(pos: int, scores, n_sink: int, n_top: int, n_local: int) -> np.ndarray:
    """The list of a token at `pos`; scores(j) for a candidate block j."""
    own = pos // 16
    w0 = max(0, own - n_local + 1)
    first = min(n_sink, w0)
    ranked = sorted(range(first, w0), key=lambda j: (-scores(j), j))[:n_top] if w0 - first > n_top else range(first, w0)
    chosen = list(range(first)) + sorted(ranked) + list(range(w0, own + 1))
    out = np.full(n_sink + n_top + n_local, -1, np.int64)
    out[:len(chosen)] = chosen
    return out


def block_attn(q: np.ndarray, keys: np.ndarray, values: np.ndarray, scale: float):
    """q [G][D], keys / values [n][D] of the keys that are seen -> (output [G][D], sum p |v| [G][D], largest sum |q_d k_d| scale
    of a row [G]): the latter two size the error that rounding may leave."""
    if len(keys) == 0:
        z = np.zeros_like(q)
        return z, z, np.zeros(len(q))
    s = (q @ keys.T) * scale
    p = np.exp(s - s.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    return p @ values, p @ np.abs(values), (np.abs(q) @ np.abs(keys).T).max(axis=1) * scale

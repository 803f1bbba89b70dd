"""Plain definitions of the serving step over the 4-bit key-value cache, in 64 bits on the CPU.

The formats and the rules are those of include/lt_indexer.h ("A serving step over a key-value cache held in 4 bits"); nothing here
shares code with the kernels.
"""
from __future__ import annotations

import numpy as np

PAGE = 64
GROUP = 32


def bf16_round(x):
    """float64/float32 -> nearest bf16 value (ties to even), as float64.  x must be representable in float32."""
    bits = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    bits = (bits + 0x7FFF + ((bits >> 16) & 1)) >> 16 << 16
    return bits.astype(np.uint32).view(np.float32).astype(np.float64)


def quantise(x):
    """x float32 [..., D] -> (codes uint8 [..., D] 1..15, scales float16 [..., D / 32])."""
    x = np.asarray(x, np.float32)
    groups = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    clean = np.where(np.isnan(groups), np.float32(0), groups)
    amax = np.abs(clean).max(-1)
    scale = np.minimum(bf16_round((amax / np.float32(7)).astype(np.float32)), 2048.0).astype(np.float16)
    s = scale.astype(np.float64)[..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        n = np.where(s > 0, np.rint(clean.astype(np.float64) / s), 0.0)
    return (np.clip(np.nan_to_num(n), -7, 7) + 8).astype(np.uint8).reshape(x.shape), scale


def values(codes, scales):
    """What the codes stand for, float64 [..., D]."""
    return (codes.astype(np.float64) - 8) * np.repeat(scales.astype(np.float64), GROUP, axis=-1)


def pack_rows(k, v):
    """Rows uint8 [..., D + D / 8] of keys and values float32 [..., D]."""
    halves, scales = [], []
    for x in (k, v):
        c, s = quantise(x)
        halves.append(c[..., 0::2] | (c[..., 1::2] << 4))
        scales.append(np.ascontiguousarray(s).view(np.uint8))
    return np.concatenate(halves + scales, -1)


def unpack_rows(rows):
    """(keys, values) float64 [..., D] of rows uint8 [..., D + D / 8]."""
    D = rows.shape[-1] // 9 * 8
    out = []
    for j in range(2):
        b = rows[..., j * D // 2:(j + 1) * D // 2]
        c = np.stack([b & 15, b >> 4], -1).reshape(*rows.shape[:-1], D)
        s = np.ascontiguousarray(rows[..., D + j * D // 16:D + (j + 1) * D // 16]).view(np.float16)
        out.append(values(c, s))
    return out


def page_tables(context_len, new_len, free_pages, page_table, T):
    """One request after the other, one token after the other.  Returns (page_table, total_len, query_start, slot_map, position,
    status)."""
    table = np.array(page_table, np.int32)
    B, max_pages = table.shape
    free = list(np.asarray(free_pages, np.int64))
    total_len = np.zeros(B, np.int32)
    start = np.zeros(B + 1, np.int32)
    slots, position = np.full(T, -1, np.int32), np.full(T, -1, np.int32)
    tokens = asked = 0
    short = False
    for b in range(B):
        ctx, new = int(context_len[b]), int(new_len[b])
        short |= ctx < 0 or new < 0
        ctx, new = max(ctx, 0), max(new, 0)
        start[b] = min(tokens, T)
        total_len[b] = min(ctx + new, 2**31 - 1)
        old, need = -(-ctx // PAGE), -(-(ctx + new) // PAGE)
        short |= need > max_pages
        for p in range(min(old, max_pages), min(need, max_pages)):
            table[b, p] = free[asked] if asked < len(free) else -1
            asked += 1
        for j in range(min(new, max(T - tokens, 0))):
            pos = ctx + j
            page = int(table[b, pos // PAGE]) if pos // PAGE < max_pages else -1
            slots[tokens + j] = page * PAGE + pos % PAGE if page >= 0 else -1
            position[tokens + j] = pos
        tokens += new
    start[B] = min(tokens, T)
    missing = max(asked - len(free), 0)
    short |= missing > 0 or tokens > T
    status = np.array([8 if short else 0, tokens, asked - missing, missing, 0, 0, 0, 0], np.int32)
    return table, total_len, start, slots, position, status


def attend(q, k, v, scale):
    """One query q [D] over k, v [n, D] (float64): (out [D], lse, sum_s p_s |v_s| [D])."""
    D = q.shape[0]
    if k.shape[0] == 0:
        return np.zeros(D), -np.inf, np.zeros(D)
    s = scale * (k @ q)
    m = s.max()
    e = np.exp(s - m)
    p = e / e.sum()
    return p @ v, m + np.log(e.sum()), p @ np.abs(v)


def attention(q, pool, page_table, query_start, context_len, scale, idx=None):
    """q float64 [T, Hq, D] over the pool uint8 [pages, Hkv, 64, row].  Returns (out, lse, spread, weight, mass), all float64:
    spread [T, Hq, D] = sum_s p_s |v_s|, weight [T, Hq] = the largest scale * sum_d |q_d k_d| of any position seen, and mass
    [T, Hq, D] = sum_s |v_s| bound what a rounding can do.  Rows that are nobody's are NaN."""
    T, Hq, D = q.shape
    pages, Hkv = pool.shape[:2]
    group = Hq // Hkv
    out, lse = np.full((T, Hq, D), np.nan), np.full((T, Hq), np.nan)
    spread, weight, mass = np.full((T, Hq, D), np.nan), np.zeros((T, Hq)), np.zeros((T, Hq, D))
    for b in range(len(context_len)):
        ctx, t0, t1 = int(context_len[b]), int(query_start[b]), int(query_start[b + 1])
        if t1 <= t0:
            continue
        at = np.arange(min(ctx + t1 - t0, page_table.shape[1] * PAGE))
        page = page_table[b][at // PAGE]
        ok = (page >= 0) & (page < pages)
        for h in range(Hkv):
            k, v = unpack_rows(pool[np.where(ok, page, 0), h, at % PAGE])
            for t in range(t0, t1):
                last = min(ctx + t - t0, at.size - 1)
                if idx is None:
                    see = np.flatnonzero(ok[:last + 1])
                else:
                    see = np.array([i for i in idx[t] if 0 <= i <= last and ok[i]], np.int64)
                for j in range(h * group, (h + 1) * group):
                    out[t, j], lse[t, j], spread[t, j] = attend(q[t, j], k[see], v[see], scale)
                    mass[t, j] = np.abs(v[see]).sum(0)
                    if see.size:
                        weight[t, j] = abs(scale) * (np.abs(k[see]) @ np.abs(q[t, j])).max()
    return out, lse, spread, weight, mass

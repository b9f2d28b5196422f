"""Plain fp64 forms of the operators that serve a receiver from pages -- TEST INFRASTRUCTURE ONLY.

numpy only, loops over requests and tokens, written from the definitions; values of 16- and 8-bit arrays come in as the
float64 numbers they stand for.
"""
from __future__ import annotations

import math

import numpy as np


def page_tables(ctx_lens, q_lens, free_pages, page_size, block_table, max_tokens):
    """One request after the other, one token after the other.  Returns a dict of int32 arrays."""
    table = np.array(block_table, dtype=np.int32)
    width = table.shape[1]
    q_starts, kv_lens, info = [0], [], []
    slots = np.full(max_tokens, -1, np.int32)
    positions = np.full(max_tokens, -1, np.int32)
    used, dry, rows = 0, False, 0
    for r, (ctx, q) in enumerate(zip(map(int, ctx_lens), map(int, q_lens))):
        if ctx < 0 or q < 0:
            why, q_eff = 3, 0
        else:
            have, total = -(-ctx // page_size), -(-(ctx + q) // page_size)
            why, q_eff = 0, q
            if total > width:
                why = 2
            elif rows + q > max_tokens:
                why = 4
            elif total > have and (dry or used + total - have > len(free_pages)):
                why, dry = 1, True
        if why == 0:
            for j in range(have, total):
                table[r, j] = free_pages[used]
                used += 1
            for i in range(q):
                pos = ctx + i
                page = int(table[r, pos // page_size])
                positions[rows + i] = pos
                slots[rows + i] = page * page_size + pos % page_size if page >= 0 else -1
        rows += q_eff
        q_starts.append(min(rows, max_tokens))
        kv_lens.append(ctx + q if why == 0 else 0)
        info.append(why)
    i32 = lambda x: np.asarray(x, dtype=np.int32)
    return dict(block_table=table, q_starts=i32(q_starts), kv_lens=i32(kv_lens), slots=slots, positions=positions,
                info=i32(info), n_used=i32([used]))


def turn(x, table, positions, axis, style, inverse=False):
    """x [token][...][d] float64 turned pair by pair; table [n_pos][d/2][2], positions [axes][token].  Also the sum of
    the absolute values of the two products behind every element."""
    n, d = x.shape[0], x.shape[-1]
    y, mag = np.empty_like(x), np.empty_like(x)
    for i in range(d // 2):
        a, b = (i, i + d // 2) if style == 0 else (2 * i, 2 * i + 1)
        pos = np.asarray(positions)[axis[i]][:n]
        ok = (pos >= 0) & (pos < table.shape[0])
        cs = np.where(ok[:, None], table[np.clip(pos, 0, table.shape[0] - 1), i].astype(np.float64), np.nan)
        shape = (n,) + (1,) * (x.ndim - 2)
        c, s = cs[:, 0].reshape(shape), cs[:, 1].reshape(shape) * (-1 if inverse else 1)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        mag[..., a], mag[..., b] = abs(x[..., a] * c) + abs(x[..., b] * s), abs(x[..., b] * c) + abs(x[..., a] * s)
    return y, mag


def attention(q, K, V, kv_len, scale, window=0, sinks=0, hidden=()):
    """One request and KV head.  q [new token][G][d], K and V [>= kv_len][d] float64; keys in ``hidden`` are on no page.
    Returns out, lse, sum_j w_j |v_j| (w normalised) and the largest sum_i |scale q_i k_i| over the visible keys."""
    n, G, d = q.shape
    out, lse = np.zeros((n, G, d)), np.full((n, G), -math.inf)
    mag, smag = np.zeros((n, G, d)), np.zeros((n, G))
    hidden = set(hidden)
    for i in range(n):
        p = kv_len - n + i
        keys = [j for j in range(min(p + 1, kv_len)) if (not window or j > p - window or j < sinks) and j not in hidden]
        if not keys:
            continue
        k, v = K[keys], V[keys]
        for g in range(G):
            s = scale * (k @ q[i, g])
            m = s.max()
            e = np.exp(s - m)
            w = e / e.sum()
            out[i, g], lse[i, g] = w @ v, m + math.log(e.sum())
            mag[i, g] = w @ np.abs(v)
            smag[i, g] = (abs(scale) * (np.abs(k) @ np.abs(q[i, g]))).max()
    return out, lse, mag, smag

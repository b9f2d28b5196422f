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


# ------------------------------------------------------------------ pages whose scales belong to a page

E_MIN, E_MAX = -64, 119              # exponents of the smallest and largest scale


def e4m3(x):
    """x rounded to the nearest e4m3 number (ties to even); beyond the largest, and infinities: NaN."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.where(x != 0, np.floor(np.log2(np.abs(np.where(x != 0, x, 1.0)))), -6)
    step = 2.0 ** (np.clip(np.nan_to_num(e, nan=0.0, posinf=0.0), -6, 8) - 3)
    y = np.round(x / step) * step
    return np.where(np.abs(y) <= 448, y, np.nan)


def block_exponent(rows, turned):
    """The exponent of a block's scale from its rows (any shape)."""
    a = np.abs(rows[np.isfinite(rows)])
    m = float(a.max()) if a.size else 0.0
    e = E_MIN
    while e < E_MAX and m > (316.0 if turned else 448.0) * 2.0 ** e:
        e += 1
    return e


def page_spans(row_starts, q_lens, kv_lens, page_size, n_rows, width):
    """(request, entry, first place, tokens, first row) of every page that a request's last q tokens lie in."""
    out = []
    for r, (b, q, kv) in enumerate(zip(map(int, row_starts), map(int, q_lens), map(int, kv_lens))):
        if q <= 0 or kv < q or kv > width * page_size or b < 0 or b + q > n_rows:
            continue
        pos = kv - q
        while pos < kv:
            n = min(kv - pos, page_size - pos % page_size)
            out.append((r, pos // page_size, pos % page_size, n, b + pos - (kv - q)))
            pos += n
    return out


def page_quantize(rows, turned, codes, exps, spans, block_table):
    """rows, turned [row][layer][2][head][d] as they come and turned (K) float64; codes [layer][2][page][head][place][d]
    and exps [layer][page][head][2] are updated, the new rows' codes before they are rounded.  turned None: nothing is
    turned."""
    y = rows if turned is None else turned
    _, L, _, H, _ = rows.shape
    for r, entry, at, n, t in spans:
        page = int(block_table[r][entry])
        if not 0 <= page < codes.shape[2]:
            continue
        for l in range(L):
            for z in range(2):
                for h in range(H):
                    e = block_exponent(rows[t:t + n, l, z, h], turned is not None and z == 0)
                    was = int(exps[l, page, h, z])
                    if at > 0 and was >= e:
                        e = was
                    elif at > 0:
                        codes[l, z, page, h, :at] = e4m3(codes[l, z, page, h, :at] * 2.0 ** (was - e))
                    codes[l, z, page, h, at:at + n] = y[t:t + n, l, z, h] * 2.0 ** -e
                    exps[l, page, h, z] = e


# ------------------------------------------------------------------ selected pages

def page_bounds(keys):
    """Least and greatest of every channel of keys [token][d]; a NaN is both."""
    return np.stack([keys.min(0), keys.max(0)])


def page_scores(q, bounds):
    """q [head of the group][d], bounds [page][2][d] float64: the pages' scores, rounded to 32 bits once."""
    with np.errstate(invalid="ignore", over="ignore"):
        out = np.zeros(len(bounds))
        for u in q:
            out = out + (np.maximum(u, 0) * bounds[:, 1] + np.minimum(u, 0) * bounds[:, 0]).sum(-1)
        return out.astype(np.float32)


def page_select(scores, there, n_first, n_last, k):
    """scores of the pages 0 .. own (the last), there: which of them are in the pool.  The chosen ones, ascending."""
    own = len(scores) - 1
    always = [i for i in range(own + 1) if there[i] and (i < n_first or i > own - n_last)]
    s = np.where(np.isnan(scores), np.inf, scores)
    rest = sorted((i for i in range(own + 1) if there[i] and i not in set(always)), key=lambda i: (-s[i], i))
    return sorted(always + rest[:k - len(always)])

"""GPU tests of serving a receiver from pages: tables, rotary positions with several axes, page writes and attention
against the plain fp64 forms of ``oracle.serve``.

Tolerances are the operators' own roundings, counted element by element:
  a rounding to bf16 is off by at most 2^-8 of the value, to e4m3 by 2^-4 of it (2^-10 below 2^-6), fp32 by 2^-24;
  a turned pair a c - b s takes three fp32 roundings of terms no larger than |a c| + |b s|;
  an attention row: every weight is rounded to bf16 for its product with V (2^-8 of sum_j w_j |v_j|) and is off by its
  score's error (d fp32 sums of products of at most S = max_j sum_i |scale q_i k_i|: (d + 4) 2^-23 S, counted for the
  weight and for their sum), the sums over n keys take n 2^-24, exp2 and log2 a few ulps; the output rounds once more.
"""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F32 = 2.0 ** -8, 2.0 ** -24
THETA = 1e4


@pytest.fixture(scope="module")
def cb():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    import paper_2609_00891_amd as mod
    return mod


@pytest.fixture(scope="module")
def serve():
    from oracle import serve as mod
    return mod


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def f64(t):
    return t.float().double().cpu().numpy()


def gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(shape, generator=g).to(torch.bfloat16)


# ------------------------------------------------------------------ tables

def run_tables(cb, ctx, q, free, ps, table, tokens):
    bt = i32(table)
    n = len(ctx)
    r = dict(block_table=bt, q_starts=i32([-7] * (n + 1)), kv_lens=i32([-7] * n), slots=i32([-7] * tokens),
             positions=i32([-7] * tokens), info=i32([-7] * n), n_used=i32([-7]))
    cb.cb_page_tables(i32(ctx), i32(q), i32(free), ps, bt, r["q_starts"], r["kv_lens"], r["slots"], r["positions"],
                      r["info"], r["n_used"])
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in r.items()}


@pytest.mark.parametrize("n,ps,ctx_max,q_max,free,tokens,width", [
    (1, 16, 0, 1, 4, 1, 2), (3, 1, 5, 3, 40, 20, 12), (7, 16, 100, 1, 30, 7, 9), (5, 24, 0, 300, 200, 2000, 20),
    (64, 16, 900, 1, 200, 72, 60), (300, 8, 50, 40, 5000, 20000, 16), (300, 8, 50, 40, 500, 20000, 16),
    (300, 8, 50, 40, 0, 4000, 11), (257, 7, 3, 2, 600, 300, 2), (2000, 16, 64, 5, 9000, 12000, 6), (4096, 3, 9, 4, 20000, 20000, 6)])
def test_tables(cb, serve, n, ps, ctx_max, q_max, free, tokens, width):
    rng = np.random.default_rng(n + ps)
    ctx, q = rng.integers(0, ctx_max + 1, n), rng.integers(0, q_max + 1, n)
    if n > 4:
        ctx[2], q[3] = -1, -5
    pool = rng.permutation(free + n * width)
    table = np.full((n, width), -1)
    for r in range(n):
        have = min(width, -(-max(int(ctx[r]), 0) // ps))
        table[r, :have] = pool[free + r * width:free + r * width + have]
    want = serve.page_tables(ctx, q, pool[:free], ps, table, tokens)
    got = run_tables(cb, ctx, q, pool[:free], ps, table, tokens)
    for k in want:
        assert np.array_equal(got[k], want[k]), k


def test_tables_without_requests_or_tokens(cb):
    e = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    starts, used, slots, pos = i32([9]), i32([9]), i32([9, 9]), i32([9, 9])
    cb.cb_page_tables(e(0), e(0), e(0), 16, e(0, 4), starts, e(0), slots, pos, e(0), used)
    assert starts.tolist() == [0] and used.tolist() == [0] and slots.tolist() == [-1, -1] and pos.tolist() == [-1, -1]
    starts, kv, info, used = i32([9, 9]), i32([9]), i32([9]), i32([9])
    cb.cb_page_tables(i32([5]), i32([0]), e(0), 16, i32([[3, -1]]), starts, kv, e(0), e(0), info, used)
    assert starts.tolist() == [0, 0] and kv.tolist() == [5] and info.tolist() == [0] and used.tolist() == [0]


# ------------------------------------------------------------------ rows

def axis_of(d, axes):
    return [(i * 7 // 3) % axes for i in range(d // 2)]


def make_rope(cb, d, axes, n, seed, n_pos=64, bad=()):
    """A table and positions (on the device and as numbers); ``bad`` tokens stand outside the table."""
    rng = np.random.default_rng(seed)
    pos = rng.integers(0, n_pos, (axes, n)).astype(np.int32)
    for t in bad:
        pos[0, t] = n_pos if t % 2 else -1
    table = torch.empty((n_pos, d // 2, 2), dtype=torch.float32, device="cuda")
    cb.cb_rope_table(THETA, d, n_pos, table)
    return table, pos, axis_of(d, axes)


def check_turned(got, want, mag, what):
    tol = BF * np.abs(want) + 4 * F32 * mag
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    ok = ~np.isnan(want)
    assert (np.abs(got - want)[ok] <= tol[ok]).all(), what


@pytest.mark.parametrize("d,axes,style,L,H,B,T,token_major", [
    (128, 3, 0, 2, 2, 2, 33, False), (128, 3, 1, 1, 3, 1, 1, True), (64, 1, 0, 3, 1, 2, 17, True), (96, 2, 1, 1, 2, 3, 50, False),
    (16, 4, 0, 2, 2, 1, 40, False), (256, 3, 1, 1, 1, 1, 9, True), (80, 3, 0, 1, 5, 1, 7, False), (128, 3, 0, 12, 8, 1, 300, False)])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_axes(cb, serve, d, axes, style, L, H, B, T, token_major, inverse):
    g = gen(d + T)
    x = randn(g, L, 2, B, T, H, d) if token_major else randn(g, L, 2, B, H, T, d)
    x = x.cuda()
    x = x.permute(0, 1, 2, 4, 3, 5) if token_major else x
    n = B * T
    bad = [n // 2] if n > 8 else []
    table, pos, axis = make_rope(cb, d, axes, n, T, bad=bad)
    rope = cb.rope_axes_spec(table, i32(pos), axis, style)
    out = torch.full((L, 2, B, H, T, d), 7.0, dtype=torch.bfloat16, device="cuda")
    cb.cb_rope_axes(x, out, rope, inverse=inverse)
    xk = f64(x[:, 0]).transpose(1, 3, 0, 2, 4).reshape(n, L, H, d)
    y, mag = serve.turn(xk, table.cpu().numpy(), pos, axis, style, inverse)
    got = f64(out[:, 0]).transpose(1, 3, 0, 2, 4).reshape(n, L, H, d)
    check_turned(got, y, mag, "keys")
    assert torch.equal(out[:, 1], x[:, 1].contiguous())
    inplace = x.clone(memory_format=torch.preserve_format)
    cb.cb_rope_axes(inplace, inplace, rope, inverse=inverse)
    assert torch.equal(inplace[:, 0].nan_to_num(3.0), out[:, 0].nan_to_num(3.0)) and torch.equal(inplace[:, 1], x[:, 1])


@pytest.mark.parametrize("d", [16, 48, 64, 80, 96, 112, 176, 240])
def test_long_calls_of_narrow_rows(cb, serve, d):
    """Rows whose halves are no whole lines, in calls of many (layer, head) rows: an odd number of tokens, some of them
    without a slot, some positions outside the table; in place, out of place and into pages are the same."""
    L, H, B, T = 10, 8, 3, 401
    g, n = gen(d), 3 * 401
    x = randn(g, L, 2, B, H, T, d).cuda()
    table, pos, axis = make_rope(cb, d, 2, n, seed=d, bad=(7, n - 1))
    rope = cb.rope_axes_spec(table, i32(pos), axis)

    def same(u, v):
        return torch.equal(u.isnan(), v.isnan()) and torch.equal(u.nan_to_num(1.0), v.nan_to_num(1.0))

    out = torch.full_like(x, 3.0)
    cb.cb_rope_axes(x, out, rope)
    y = x.clone()
    cb.cb_rope_axes(y, y, rope)
    assert same(y, out) and torch.equal(out[:, 1], x[:, 1])
    rows = f64(x).transpose(2, 4, 0, 1, 3, 5).reshape(n, L, 2, H, d)
    want, mag = serve.turn(rows[:, :2, 0], table.cpu().numpy(), pos, axis, 0)
    got = f64(out).transpose(2, 4, 0, 1, 3, 5).reshape(n, L, 2, H, d)[:, :2, 0]
    check_turned(got, want, mag, "keys")
    pool = torch.full((L, 2, n, H, 1, d), 5.0, dtype=torch.bfloat16, device="cuda")
    slots = torch.randperm(n, generator=g).int()
    slots[[0, 5, 6, 7, 400, n - 2]] = -1
    q = randn(g, n, 5, d).cuda()
    q_out, q_ref = torch.full_like(q, 7.0), torch.empty((1, 2, 1, 5, n, d), dtype=torch.bfloat16, device="cuda")
    cb.cb_page_write(x, cb.page_pool(pool), slots.cuda(), rope=rope, q=q, q_out=q_out)
    cb.cb_rope_axes(q.transpose(0, 1)[None, None, None].expand(1, 2, 1, 5, n, d), q_ref, rope)
    keep = slots >= 0
    flat = out.permute(2, 4, 0, 1, 3, 5).reshape(n, L, 2, H, d).cpu()
    moved = pool.permute(2, 4, 0, 1, 3, 5).reshape(n, L, 2, H, d).cpu()
    assert same(moved[slots[keep].long()], flat[keep])
    left = torch.ones(n, dtype=torch.bool)
    left[slots[keep].long()] = False
    assert (moved[left] == 5.0).all()
    assert same(q_out.cpu()[keep], q_ref[0, 0, 0].transpose(0, 1).cpu()[keep])
    assert (q_out.cpu()[~keep] == 7.0).all()
    z = torch.full_like(pool, 5.0)                              # without a turn: the rows themselves
    cb.cb_page_write(x, cb.page_pool(z), slots.cuda())
    plain = x.permute(2, 4, 0, 1, 3, 5).reshape(n, L, 2, H, d).cpu()
    assert torch.equal(z.permute(2, 4, 0, 1, 3, 5).reshape(n, L, 2, H, d).cpu()[slots[keep].long()], plain[keep])


def test_rope_axes_with_one_axis_is_rope(cb):
    """Positions 3 .. 3 + T - 1 in one axis: the transform that cb_rope makes from an offset, bit for bit."""
    x = randn(gen(1), 2, 2, 1, 3, 40, 128).cuda()
    table = torch.empty((64, 64, 2), dtype=torch.float32, device="cuda")
    cb.cb_rope_table(THETA, 128, 64, table)
    for style in (0, 1):
        a, b = torch.empty_like(x), torch.empty_like(x)
        cb.cb_rope(x, a, table, style, pos_offset=3)
        cb.cb_rope_axes(x, b, cb.rope_axes_spec(table, torch.arange(3, 43, dtype=torch.int32, device="cuda"), None, style))
        assert torch.equal(a, b)


def make_pool(L, H, P, ps, d, token_major, f8, seed=0):
    """A pool full of a recognisable value, stored by head or by token inside a page, and its scales."""
    shape = (L, 2, P, ps, H, d) if token_major else (L, 2, P, H, ps, d)
    pool = torch.full(shape, 0.375, dtype=torch.bfloat16, device="cuda")
    scales = None
    if f8:
        pool = pool.to(torch.float8_e4m3fn)
        scales = (0.01 + 0.03 * torch.rand((L, 2, H), generator=gen(seed))).cuda()
    return (pool.permute(0, 1, 2, 4, 3, 5) if token_major else pool), scales


@pytest.mark.parametrize("d,axes,style,L,H,G,B,T,ps,token_major,f8", [
    (128, 1, 0, 1, 2, 4, 1, 9, 16, True, False), (128, 3, 0, 2, 2, 0, 2, 37, 16, False, True), (64, 0, 0, 2, 3, 0, 1, 50, 7, False, False),
    (96, 2, 1, 1, 2, 5, 1, 33, 32, True, True), (64, 3, 1, 1, 1, 1, 3, 5, 1, False, True), (128, 0, 0, 1, 4, 0, 2, 64, 64, True, True),
    (256, 1, 0, 1, 1, 2, 1, 3, 4, False, False), (80, 3, 0, 2, 2, 1, 1, 11, 8, True, False), (128, 3, 0, 8, 8, 0, 2, 300, 100, False, False)])
def test_page_write(cb, serve, d, axes, style, L, H, G, B, T, ps, token_major, f8):
    g, n = gen(d + T), B * T
    x = randn(g, L, 2, B, H, T, d)
    x[0, 0, 0, 0, 0, 3], x[0, 1, 0, 0, 0, 5] = 3e4, -3e4                  # beyond e4m3's range at these scales
    x = x.cuda()
    P = n // ps + 3
    pool, scales = make_pool(L + 1, H, P, ps, d, token_major, f8)
    if f8 and token_major and (H * d) % 16:
        pytest.skip("rows not 16-byte aligned")
    rng = np.random.default_rng(n)
    slots = rng.permutation(P * ps)[:n].astype(np.int32)
    skip = [1] if n > 3 else []
    for t in skip:
        slots[t] = -1
    if n > 8:
        slots[7] = P * ps                                                   # outside the pool
        skip.append(7)
    keep = np.array([t for t in range(n) if t not in skip])
    before = pool.clone(memory_format=torch.preserve_format)
    rope = q = q_out = None
    if axes:
        table, pos, axis = make_rope(cb, d, axes, n, T, bad=[2] if n > 30 else [])
        rope = cb.rope_axes_spec(table, i32(pos), axis, style)
    if G:
        q = randn(g, n, H * G, d).cuda()
        q_out = torch.full_like(q, 5.0)
    cb.cb_page_write(x, cb.page_pool(pool, scales), i32(slots), layer=1, rope=rope, q=q, q_out=q_out)
    torch.cuda.synchronize()
    rows = f64(x).transpose(2, 4, 0, 1, 3, 5).reshape(n, L, 2, H, d)[keep]
    want, mag = rows.copy(), np.zeros_like(rows)
    if axes:
        pk = pos[:, keep]
        want[:, :, 0], mag[:, :, 0] = serve.turn(rows[:, :, 0], table.cpu().numpy(), pk, axis, style)
    page, off = slots[keep] // ps, slots[keep] % ps
    got = np.stack([f64(pool[1:, :, int(p), :, int(o)]) for p, o in zip(page, off)])
    if f8:
        inv = (1.0 / scales[1:].cpu()).double().numpy()[None, :, :, :, None]
        want, mag = np.clip(want * inv, -448, 448), mag * inv
        tol = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) + 5 * F32 * (mag + np.abs(want))
    else:
        tol = BF * np.abs(want) + 4 * F32 * mag if axes else 0 * want
        if axes:
            tol[:, :, 1] = 0
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    assert (np.abs(got - want)[fine] <= tol[fine]).all()
    # nothing else was written
    mask = torch.ones_like(pool, dtype=torch.bool)
    for p, o in zip(page, off):
        mask[1:, :, int(p), :, int(o)] = False
    assert torch.equal(pool.view(torch.uint8 if f8 else torch.int16)[mask], before.view(torch.uint8 if f8 else torch.int16)[mask])
    if G:
        y, m2 = serve.turn(f64(q)[keep], table.cpu().numpy(), pk, axis, style)
        check_turned(f64(q_out)[keep], y, m2, "queries")
        assert (q_out[torch.tensor(skip)] == 5.0).all() if skip else True
        q2 = q.clone()
        cb.cb_page_write(x, cb.page_pool(pool, scales), i32(slots), layer=1, rope=rope, q=q2, q_out=q2)
        assert torch.equal(q2[keep].nan_to_num(1.0), q_out[keep].nan_to_num(1.0)) and torch.equal(q2[skip], q[skip])


# ------------------------------------------------------------------ attention

class Step:
    """Requests of (new tokens, keys) in a shuffled pool whose unused places hold NaN (e4m3: its NaN)."""

    def __init__(self, cb, lens, H, G, d, ps, f8=False, token_major=False, pad=0, seed=0, layers=2, layer=1, spread=1.0):
        g, rng = gen(seed), np.random.default_rng(seed)
        self.cb, self.lens, self.H, self.G, self.d, self.ps, self.f8, self.layer = cb, lens, H, G, d, ps, f8, layer
        used = [-(-kv // ps) for _, kv in lens]
        self.width = max(1, max(used) + 1)
        P = sum(used) + 2
        order = rng.permutation(P)
        self.table = np.full((len(lens), self.width), -1, np.int32)
        at = 0
        for r, u in enumerate(used):
            self.table[r, :u] = order[at:at + u]
            at += u
        shape = (layers, 2, P, ps, H, d) if token_major else (layers, 2, P, H, ps, d)
        self.scales = None
        host = torch.full(shape, float("nan"), dtype=torch.bfloat16)
        host = host.permute(0, 1, 2, 4, 3, 5) if token_major else host
        if f8:
            self.scales = (0.01 + 0.02 * torch.rand((layers, 2, H), generator=g)).cuda()
        self.K, self.V = [], []                                            # [request][head][key][d] as numbers
        for r, (_, kv) in enumerate(lens):
            k, v = randn(g, H, kv, d) * spread, randn(g, H, kv, d)
            if f8:
                k, v = (40 * k).clamp(-448, 448).to(torch.float8_e4m3fn), (40 * v).clamp(-448, 448).to(torch.float8_e4m3fn)
            for z, x in enumerate((k, v)):
                xb = x.to(torch.bfloat16)                                  # e4m3 values are exact in bf16
                for j in range(0, kv, ps):
                    m = min(ps, kv - j)
                    host[layer, z, self.table[r, j // ps], :, :m] = xb[:, j:j + m]
            sc = np.ones((2, H, 1, 1)) if not f8 else self.scales[layer].double().cpu().numpy()[:, :, None, None]
            self.K.append(f64(k) * sc[0])
            self.V.append(f64(v) * sc[1])
        dev = host.to(torch.float8_e4m3fn) if f8 else host
        self.pool = dev.cuda() if not token_major else dev.permute(0, 1, 2, 4, 3, 5).contiguous().cuda().permute(0, 1, 2, 4, 3, 5)
        self.n = sum(q for q, _ in lens) + pad
        self.q = randn(g, self.n, H * G, d).cuda()
        self.starts = np.concatenate([[0], np.cumsum([q for q, _ in lens])])
        self.max_q = max([q for q, _ in lens] + [1])

    def run(self, window=0, sinks=0, ws=True, scale=None, table=None, max_q=None, lse=True, stream=None, q=None, kv=None):
        cb = self.cb
        self.out = torch.full((self.n, self.H * self.G, self.d), 9.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((self.n, self.H * self.G), 9.0, dtype=torch.float32, device="cuda") if lse else None
        need = cb.cb_attn_paged_workspace_bytes(self.n, len(self.lens), self.H * self.G, self.H, self.d, self.max_q)
        w = torch.empty((need if ws is True else int(ws),), dtype=torch.uint8, device="cuda") if ws else None
        cb.cb_attn_paged(self.q if q is None else q, cb.page_pool(self.pool, self.scales), self.layer, i32(self.starts),
                         i32([k for _, k in self.lens] if kv is None else kv), i32(self.table if table is None else table),
                         self.out, self.max_q if max_q is None else max_q, scale=scale, window=window, sinks=sinks,
                         lse=self.lse, workspace=w, stream=stream)
        torch.cuda.synchronize()
        return self.out, self.lse

    def check(self, serve, window=0, sinks=0, scale=None, hidden=None, rows=None):
        """Every row (or the requests ``rows``) against the plain form; rows of no request are left as they were."""
        sc = self.d ** -0.5 if scale is None else scale
        got, gl, qd = f64(self.out), f64(self.lse), f64(self.q)
        H, G, d = self.H, self.G, self.d
        for r, (nq, kv) in enumerate(self.lens):
            if rows is not None and r not in rows:
                continue
            s = slice(self.starts[r], self.starts[r + 1])
            for h in range(H):
                hs = slice(h * G, (h + 1) * G)
                o, l, mag, smag = serve.attention(qd[s, hs], self.K[r][h], self.V[r][h], kv, sc, window, sinks,
                                                  () if hidden is None else hidden[r])
                es = (d + 8) * 2 * F32 * smag
                few = (kv + 64) * 2 * F32
                tol = BF * np.abs(o) * 1.01 + mag * (BF * 1.01 + (2 * es + few)[..., None])
                assert (np.abs(got[s, hs] - o) <= tol).all(), (r, h, np.max(np.abs(got[s, hs] - o) / np.maximum(tol, 1e-30)))
                seen = np.isfinite(l)
                assert np.array_equal(np.isneginf(gl[s, hs]), ~seen), (r, h)
                lt = (es + few)[seen] + 8 * F32 * (np.abs(l[seen]) + 1)
                assert (np.abs(gl[s, hs][seen] - l[seen]) <= lt).all(), (r, h)
        assert (got[self.starts[-1]:] == 9.0).all() and (gl[self.starts[-1]:] == 9.0).all()


CASES = [
    # lens, H, G, d, page, e4m3, token major
    ([(1, 1)], 1, 1, 64, 16, False, False),
    ([(1, 5), (1, 64), (1, 33)], 2, 4, 128, 16, False, False),
    ([(1, 700), (1, 31), (1, 32), (1, 1)], 2, 8, 128, 16, False, True),
    ([(1, 300), (1, 257)], 2, 5, 96, 24, False, False),
    ([(1, 300), (1, 257)], 1, 16, 96, 32, True, True),
    ([(1, 300), (1, 257)], 2, 3, 64, 7, True, False),
    ([(1, 1500)], 1, 8, 128, 64, True, False),
    ([(3, 3), (0, 40), (5, 90), (1, 17)], 2, 2, 64, 16, False, True),
    ([(7, 260), (4, 4)], 1, 7, 128, 1, False, False),
    ([(40, 100), (1, 200), (33, 33)], 1, 4, 128, 16, False, False),
    ([(130, 300)], 1, 1, 96, 100, False, False),
    ([(65, 129), (2, 600)], 1, 2, 64, 16, True, False),
    ([(20, 85)], 1, 33, 128, 128, True, True),
    ([(1, 90), (2, 40)], 1, 40, 64, 16, False, False),
    ([(150, 150)], 2, 2, 128, 32, True, False),
]


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(cb, serve, case, ws):
    lens, H, G, d, ps, f8, tm = CASES[case]
    s = Step(cb, lens, H, G, d, ps, f8, tm, pad=case % 3, seed=case)
    s.run(ws=ws)
    s.check(serve)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (33, 4), (64, 70), (100, 1), (2 ** 31 - 1, 0), (50, 2 ** 31 - 1)])
@pytest.mark.parametrize("case", [2, 5, 7, 9, 10, 11])
def test_attention_window(cb, serve, case, window, sinks):
    lens, H, G, d, ps, f8, tm = CASES[case]
    s = Step(cb, lens, H, G, d, ps, f8, tm, pad=1, seed=case)
    s.run(window, sinks)
    s.check(serve, window, sinks)


@pytest.mark.parametrize("f8", [False, True])
def test_attention_long_rows_in_parts(cb, serve, f8):
    """Long rows beside short ones: divided among workgroups as the workspace allows, the same within rounding, and the
    same bits from call to call."""
    s = Step(cb, [(1, 9000), (1, 40), (2, 3001), (1, 1)], 1, 4, 128, 16, f8, pad=2, seed=3)
    s.run()
    s.check(serve)
    a, al = s.out.clone(), s.lse.clone()
    s.run()
    assert torch.equal(a, s.out) and torch.equal(al, s.lse)
    for ws in (70000, 300000, 16):
        s.run(ws=ws)
        s.check(serve, rows=[0, 2, 3])
    for hint in (0, 2, 1000):
        s.run(max_q=hint)
        s.check(serve, rows=[0, 1, 2])


@pytest.mark.parametrize("d,f8", [(64, False), (96, False), (128, False), (64, True), (96, True), (128, True)])
def test_attention_rows_in_many_parts(cb, serve, d, f8):
    """Rows in dozens of parts, of single tokens and of chunks, joined by a workgroup each; the same bits every time."""
    s = Step(cb, [(1, 20000), (40, 12000), (3, 5000), (2, 300)], 2, 2, d, 16, f8, pad=1, seed=80)
    s.run()
    s.check(serve)
    a, al = s.out.clone(), s.lse.clone()
    s.run()
    assert torch.equal(a, s.out) and torch.equal(al, s.lse)
    s.run(max_q=1)
    s.check(serve)


def test_attention_chunk_in_parts(cb, serve):
    s = Step(cb, [(70, 2100), (1, 50)], 1, 2, 64, 16, seed=4)
    s.run()
    s.check(serve)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("lens,G", [([(1, 100), (1, 70)], 4), ([(70, 200)], 2)])
def test_attention_hidden_pages(cb, serve, lens, G, f8):
    """Entries outside the pool (-1, its size, a large number) hide their keys; all of them: zeros and -inf."""
    s = Step(cb, lens, 1, G, 128, 16, f8, seed=6)
    P = s.pool.shape[2]
    table = s.table.copy()
    table[0, 0], table[0, 3] = -1, P
    hidden = [set(range(16)) | set(range(48, 64))] + [set()] * (len(lens) - 1)
    s.run(table=table)
    s.check(serve, hidden=hidden)
    table[0, :] = 2 ** 31 - 1
    s.run(table=table)
    s.check(serve, hidden=[set(range(lens[0][1]))] + [set()] * (len(lens) - 1))
    # behind a window the pages may be given back
    table = s.table.copy()
    first = lens[0][1] - lens[0][0] - 20 + 1
    table[0, 1:first // 16] = -1
    s.run(20, 5, table=table)
    s.check(serve, 20, 5)


@pytest.mark.parametrize("G,q,kv", [(2, 3, 60), (4, 40, 90), (1, 130, 130)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_attention_bad_values_stay_with_their_rows(cb, serve, G, q, kv, bad):
    """A NaN or infinity in a key or value that later rows see does not reach the rows before it."""
    for what in ("k", "v"):
        s = Step(cb, [(q, kv)], 1, G, 64, 16, seed=8)
        j = kv - q + q // 2                                                 # seen by the new tokens q // 2 ... only
        at = (s.layer, 0 if what == "k" else 1, int(s.table[0, j // 16]), 0, j % 16, 3)
        s.pool[at] = bad
        s.run()
        got = f64(s.out)
        early, late = got[:q // 2], got[q // 2:]
        o, _, mag, smag = serve.attention(f64(s.q), s.K[0][0], s.V[0][0], kv, 64 ** -0.5)
        tol = BF * 1.01 * np.abs(o) + mag * (BF * 1.01 + (2 * 72 * 2 * F32 * smag + (kv + 64) * 2 * F32)[..., None])
        assert (np.abs(early - o[:q // 2]) <= tol[:q // 2]).all(), what
        if what == "v":
            assert not np.isfinite(late[..., 3]).any()
            keep = [c for c in range(64) if c != 3]
            assert (np.abs(late - o[q // 2:]) <= tol[q // 2:])[..., keep].all()
        elif math.isnan(bad):
            assert np.isnan(late).all()


def test_attention_more_new_tokens_than_keys(cb, serve):
    """Rows before position 0 and requests with kv_lens 0 see nothing: zeros and -inf."""
    s = Step(cb, [(5, 5), (3, 40)], 2, 2, 64, 16, seed=9)
    s.run(kv=[2, 0])
    got, l = f64(s.out), f64(s.lse)
    assert (got[:3] == 0).all() and np.isneginf(l[:3]).all()
    assert (got[5:] == 0).all() and np.isneginf(l[5:]).all()
    o, _, mag, _ = serve.attention(f64(s.q)[3:5, :2], s.K[0][0], s.V[0][0], 2, 64 ** -0.5)
    assert (np.abs(got[3:5, :2] - o) <= 2 * BF * 1.02 * (mag + np.abs(o))).all()


@pytest.mark.parametrize("G,q", [(2, 5), (4, 70)])
def test_attention_largest_window_with_more_new_tokens_than_keys(cb, serve, G, q):
    s = Step(cb, [(q, q), (3, 40)], 2, G, 64, 16, seed=9)
    whole = s.run(kv=[q - 3, 40])
    wide = s.run(kv=[q - 3, 40], window=2 ** 31 - 1)
    assert torch.equal(wide[0], whole[0]) and torch.equal(wide[1], whole[1])
    got = f64(s.out)
    assert (got[:3] == 0).all()
    for h in range(2):
        hs = slice(h * G, (h + 1) * G)
        o, _, mag, _ = serve.attention(f64(s.q)[3:q, hs], s.K[0][h], s.V[0][h], q - 3, 64 ** -0.5)
        assert (np.abs(got[3:q, hs] - o) <= 2 * BF * 1.02 * (mag + np.abs(o))).all()


def test_attention_lengths_out_of_range_stay_in_bounds(cb, serve):
    """Lengths beyond the table and starts beyond the rows are cut to them; negative ones are none."""
    s = Step(cb, [(1, 60), (1, 30)], 1, 2, 64, 16, seed=10)
    s.run(kv=[2 ** 31 - 1, -5])
    # request 0 counts as 80 keys, the table's five entries: keys 60 .. 63, the NaN behind its last page's rows, are
    # among those that it sees, and the fifth entry (-1) hides the rest
    assert torch.isnan(s.out[0]).all()
    assert (f64(s.out)[1] == 0).all()
    s.starts = np.array([0, 1, 2 ** 31 - 1])
    s.run()
    s.starts = np.array([-3, 1, 2])
    s.run()
    s.check(serve, rows=[1])


def test_attention_scores_of_large_size_and_no_scale(cb, serve):
    s = Step(cb, [(1, 200), (9, 77)], 1, 4, 128, 16, seed=11, spread=30.0)
    s.run()
    s.check(serve)
    s.run(scale=0.0)
    s.check(serve, scale=0.0)
    s.run(scale=-0.2)
    s.check(serve, scale=-0.2)


def test_attention_over_a_contiguous_cache(cb, serve):
    """A mapped cache [layer][kv][seq][head][tok][dim] is a pool whose pages are its sequences: no copy."""
    g = gen(12)
    x = randn(g, 2, 2, 3, 2, 70, 128).cuda()
    q = randn(g, 3, 4, 128).cuda()
    out, lse = torch.empty_like(q), torch.empty((3, 4), dtype=torch.float32, device="cuda")
    cb.cb_attn_paged(q, cb.page_pool(x), 1, i32([0, 1, 2, 3]), i32([70, 13, 1]), i32([[0], [1], [2]]), out, 1, lse=lse)
    for r, kv in enumerate((70, 13, 1)):
        for h in range(2):
            o, l, mag, _ = serve.attention(f64(q[r:r + 1, 2 * h:2 * h + 2]), f64(x[1, 0, r, h]), f64(x[1, 1, r, h]), kv, 128 ** -0.5)
            assert (np.abs(f64(out[r:r + 1, 2 * h:2 * h + 2]) - o) <= 1.1 * BF * (np.abs(o) + mag)).all()


def test_attention_strided_queries(cb, serve):
    """Queries inside a fused projection [token][q heads + k heads + v heads], outputs inside a wider buffer."""
    s = Step(cb, [(2, 40), (1, 90)], 2, 2, 64, 16, seed=13)
    wide = torch.zeros((s.n, 8, 64), dtype=torch.bfloat16, device="cuda")
    wide[:, :4] = s.q
    s.run()
    a = s.out.clone()
    s.run(q=wide[:, :4])
    assert torch.equal(a, s.out)


def test_attention_pool_beyond_32_bits(cb, serve):
    """Rows more than 2^32 bytes apart: the last page of a pool of over 4 GiB per layer."""
    ps, H, d = 64, 8, 128
    P = (5 << 30) // (ps * H * d * 2)
    pool = torch.empty((1, 2, P, H, ps, d), dtype=torch.bfloat16, device="cuda")
    g = gen(14)
    ids = [P - 1, 3, P - 2]
    kv = 150
    K, V = randn(g, H, kv, d), randn(g, H, kv, d)
    for j, p in enumerate(ids):
        m = min(ps, kv - 64 * j)
        pool[0, 0, p, :, :m] = K[:, 64 * j:64 * j + m].cuda()
        pool[0, 1, p, :, :m] = V[:, 64 * j:64 * j + m].cuda()
        pool[0, :, p, :, m:] = float("nan")
    q = randn(g, 1, H, d).cuda()
    out = torch.empty_like(q)
    cb.cb_attn_paged(q, cb.page_pool(pool), 0, i32([0, 1]), i32([kv]), i32([ids]), out, 1)
    for h in range(H):
        o, _, mag, _ = serve.attention(f64(q[:, h:h + 1]), f64(K[h]), f64(V[h]), kv, d ** -0.5)
        assert (np.abs(f64(out[:, h:h + 1]) - o) <= 1.1 * BF * (np.abs(o) + mag)).all()
    del pool
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ together

def test_a_step_after_a_handoff(cb, serve):
    """cb_apply's mapped cache into pages, then two steps of new tokens: tables, write with queries, attention."""
    L, H, G, d, ps, B, T = 2, 2, 4, 64, 16, 3, 40
    g = gen(20)
    src = randn(g, L, 2, B, H, T, d).cuda()
    hm = {k: np.array(v, np.int32) for k, v in dict(
        tgt_layer=[l for l in range(L) for z in range(2) for h in range(H)], tgt_head=[h for l in range(L) for z in range(2) for h in range(H)],
        kv=[z for l in range(L) for z in range(2) for h in range(H)], src_layer=[l for l in range(L) for z in range(2) for h in range(H)],
        src_head=[h for l in range(L) for z in range(2) for h in range(H)], weight_row=[0] * (2 * L * H)).items()}
    plan = cb.cb_plan_create(hm, src, src, B * T)
    maps = (torch.randn((2 * L * H, d + 1, d), generator=g) * d ** -0.5).cuda()
    mapped = torch.empty_like(src)
    cb.cb_apply(plan, maps, src, mapped)
    lens = [40, 17, 33]
    P = 16
    pool = torch.full((L, 2, P, H, ps, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    pages = cb.page_pool(pool)
    free = i32(np.random.default_rng(0).permutation(P))
    table = i32(np.full((B, 6), -1))
    ctx = i32([0] * B)
    q_starts, kv, info, used = i32([0] * (B + 1)), i32([0] * B), i32([0] * B), i32([0])
    slots, pos = i32([0] * (B * T)), i32([0] * (B * T))
    # the handoff: sequence b's token t is row q_starts[b] + t of the step; the padded batch takes its slots from there
    cb.cb_page_tables(ctx, i32(lens), free, ps, table, q_starts, kv, slots, pos, info, used)
    assert info.tolist() == [0, 0, 0] and kv.tolist() == lens
    padded = torch.full((B, T), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(lens):
        padded[b, :n] = slots[int(q_starts[b]):int(q_starts[b]) + n]
    n_pos = 64
    rt = torch.empty((n_pos, d // 2, 2), dtype=torch.float32, device="cuda")
    cb.cb_rope_table(THETA, d, n_pos, rt)
    in_seq = torch.arange(T, dtype=torch.int32, device="cuda").repeat(B)
    cb.cb_page_write(mapped, pages, padded.reshape(-1), rope=cb.rope_axes_spec(rt, in_seq))
    # host copy of what every request holds, as numbers, in every layer
    hold = [[[serve.turn(f64(mapped[l, 0, b]).transpose(1, 0, 2)[:n], rt.cpu().numpy(), np.arange(n)[None], [0] * (d // 2), 0)[0],
              f64(mapped[l, 1, b]).transpose(1, 0, 2)[:n]] for l in range(L)] for b, n in enumerate(lens)]
    ws = torch.empty((cb.cb_attn_paged_workspace_bytes(8, B, H * G, H, d, 3),), dtype=torch.uint8, device="cuda")
    have = list(lens)
    for new in ([1, 0, 3], [2, 1, 1]):
        free = free[int(used):].contiguous()
        n = 8                                                                # rows of a padded step
        slots, pos = i32([0] * n), i32([0] * n)
        cb.cb_page_tables(i32(have), i32(new), free, ps, table, q_starts, kv, slots, pos, info, used)
        for l in range(L):
            kvq = randn(g, n, 2 * H + H * G, d).cuda()                       # a fused projection of the new tokens
            rows = kvq[:, :2 * H].view(n, 2, H, d).permute(1, 2, 0, 3)[None, :, None]
            q = kvq[:, 2 * H:]
            qr = torch.full((n, H * G, d), 3.0, dtype=torch.bfloat16, device="cuda")
            out = torch.full((n, H * G, d), 9.0, dtype=torch.bfloat16, device="cuda")
            cb.cb_page_write(rows, pages, slots, layer=l, rope=cb.rope_axes_spec(rt, pos), q=q, q_out=qr)
            cb.cb_attn_paged(qr, pages, l, q_starts, kv, table, out, max(new), workspace=ws)
            torch.cuda.synchronize()
            at = 0
            for b, m in enumerate(new):
                tok = slice(at, at + m)
                p = np.arange(have[b], have[b] + m)[None]
                for z, x in enumerate((rows[0, 0, 0], rows[0, 1, 0])):
                    y = f64(x).transpose(1, 0, 2)[tok]
                    y = serve.turn(y, rt.cpu().numpy(), p, [0] * (d // 2), 0)[0] if z == 0 else y
                    hold[b][l][z] = np.concatenate([hold[b][l][z], y])
                qt = serve.turn(f64(q)[tok], rt.cpu().numpy(), p, [0] * (d // 2), 0)[0]
                for h in range(H):
                    o, _, mag, smag = serve.attention(qt[:, h * G:(h + 1) * G], hold[b][l][0][:, h], hold[b][l][1][:, h],
                                                      have[b] + m, d ** -0.5)
                    # keys and queries were rounded to bf16 after their turn: scores off by 2 * 2^-8 of smag
                    tol = 1.05 * BF * (np.abs(o) + mag) + 2 * mag * (2.02 * BF * smag)[..., None]
                    assert (np.abs(f64(out[tok, h * G:(h + 1) * G]) - o) <= tol).all(), (b, l, h)
                at += m
            assert (out[at:] == 9.0).all() and (qr[at:] == 3.0).all()
        have = [a + b for a, b in zip(have, new)]
    plan.close()


def test_a_step_in_a_graph_with_other_lengths(cb, serve):
    """A captured step replayed as its lengths grow, eager work in between, on a stream of its own; two graphs with a
    workspace each.  Every replay equals the eager call on the same lengths."""
    H, G, d, ps, B = 2, 2, 64, 16, 3
    g = gen(21)
    P, n = 120, 8
    pool = randn(g, 1, 2, P, H, ps, d).cuda()
    pages = cb.page_pool(pool)
    base = i32(np.arange(P))
    rt = torch.empty((2048, d // 2, 2), dtype=torch.float32, device="cuda")
    cb.cb_rope_table(THETA, d, 2048, rt)

    def state():
        s = dict(ctx=i32([0] * B), q=i32([0] * B), free=base.clone(), table=i32(np.full((B, 40), -1)), q_starts=i32([0] * (B + 1)),
                 kv=i32([0] * B), slots=i32([0] * n), pos=i32([0] * n), info=i32([0] * B), used=i32([0]),
                 x=torch.zeros((1, 2, 1, H, n, d), dtype=torch.bfloat16, device="cuda"),
                 qin=torch.zeros((n, H * G, d), dtype=torch.bfloat16, device="cuda"),
                 qr=torch.zeros((n, H * G, d), dtype=torch.bfloat16, device="cuda"),
                 out=torch.zeros((n, H * G, d), dtype=torch.bfloat16, device="cuda"),
                 ws=torch.empty((cb.cb_attn_paged_workspace_bytes(n, B, H * G, H, d, 4),), dtype=torch.uint8, device="cuda"))
        s["rope"] = cb.rope_axes_spec(rt, s["pos"])
        return s

    def step(s, pg):
        cb.cb_page_tables(s["ctx"], s["q"], s["free"], ps, s["table"], s["q_starts"], s["kv"], s["slots"], s["pos"], s["info"], s["used"])
        cb.cb_page_write(s["x"], pg, s["slots"], rope=s["rope"], q=s["qin"], q_out=s["qr"])
        cb.cb_attn_paged(s["qr"], pg, 0, s["q_starts"], s["kv"], s["table"], s["out"], 4, window=700, sinks=2, workspace=s["ws"])

    graphs = []
    for _ in range(2):
        s = state()
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            step(s, pages)
        torch.cuda.current_stream().wait_stream(st)
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step(s, pages)
        graphs.append((gr, s))
    e = state()
    rng = np.random.default_rng(3)
    for it in range(6):
        gr, s = graphs[it % 2]
        ctx, q = rng.integers(0, 600, B), rng.integers(0, 3, B)
        x, qin = randn(g, 1, 2, 1, H, n, d).cuda(), randn(g, n, H * G, d).cuda()
        table = np.full((B, 40), -1)
        perm = rng.permutation(P)
        for b in range(B):
            table[b, :-(-int(ctx[b]) // ps)] = perm[40 * b:40 * b + -(-int(ctx[b]) // ps)]
        left = np.array([p for p in range(P) if p not in set(table.ravel().tolist())])
        left = np.concatenate([left, np.full(P - len(left), left[0])])
        for t in (s, e):
            t["ctx"].copy_(i32(ctx)); t["q"].copy_(i32(q)); t["free"].copy_(i32(left)); t["table"].copy_(i32(table))
            t["x"].copy_(x); t["qin"].copy_(qin); t["out"].fill_(4.0); t["qr"].fill_(4.0)
        gr.replay()
        torch.cuda.synchronize()
        step(e, pages)
        torch.cuda.synchronize()
        for k in ("q_starts", "kv", "slots", "pos", "info", "used", "table", "out", "qr"):
            assert torch.equal(s[k], e[k]), (it, k)
        assert torch.isfinite(s["out"]).all()


def test_calls_on_two_streams_with_a_workspace_each(cb, serve):
    a, b = (Step(cb, [(1, 4000), (2, 900)], 1, 4, 128, 16, f8, seed=30 + f8) for f8 in (False, True))
    st = [torch.cuda.Stream(), torch.cuda.Stream()]
    want = []
    for s in (a, b):
        s.run()
        want.append(s.out.clone())
    outs = []
    wss = [torch.empty((cb.cb_attn_paged_workspace_bytes(s.n, 2, 4, 1, 128, 2),), dtype=torch.uint8, device="cuda") for s in (a, b)]
    args = [(s.q, cb.page_pool(s.pool, s.scales), 1, i32(s.starts), i32([k for _, k in s.lens]), i32(s.table)) for s in (a, b)]
    torch.cuda.synchronize()
    for rep in range(5):
        for i in range(2):
            o = torch.empty_like(want[i])
            torch.cuda.synchronize()
            cb.cb_attn_paged(*args[i], o, 2, workspace=wss[i], stream=st[i])
            outs.append((i, o))
    torch.cuda.synchronize()
    for i, o in outs:
        assert torch.equal(o, want[i])


# ------------------------------------------------------------------ many requests, parts, e4m3's NaN

@pytest.mark.parametrize("d,G,f8,hint", [(64, 3, False, None), (128, 2, True, None), (96, 5, False, None), (64, 1, True, 1)])
def test_attention_many_requests(cb, serve, d, G, f8, hint):
    """More requests than a workgroup has threads: idle ones, single tokens, chunks, long rows in parts among them."""
    rng = np.random.default_rng(G)
    lens = []
    for r in range(600):
        q = int(rng.choice([0, 1, 1, 1, 2, 9]))
        lens.append((q, int(rng.integers(q, 40))))
    lens[3], lens[255], lens[256], lens[300], lens[599] = (1, 5000), (60, 300), (1, 2500), (200, 700), (3, 4100)
    s = Step(cb, lens, 1, G, d, 16, f8, pad=4, seed=40 + G, layers=1, layer=0)
    s.run(max_q=hint)
    s.check(serve, rows=[0, 1, 2, 3, 4, 100, 254, 255, 256, 257, 300, 511, 512, 513, 598, 599])
    # the others at least as numbers: nothing is left out
    named = s.starts[-1]
    assert torch.isfinite(s.out[:named]).all() and not (s.lse[:named] == 9.0).any()


@pytest.mark.parametrize("d,G,f8", [(128, 4, True), (96, 4, False)])
def test_attention_window_in_parts(cb, serve, d, G, f8):
    """Windows of several thousand keys, divided, with sinks far in front of them."""
    s = Step(cb, [(1, 9000), (2, 7000), (40, 9000)], 1, G, d, 24, f8, pad=1, seed=50)
    for ws in (True, False):
        s.run(5000, 40, ws=ws)
        s.check(serve, 5000, 40)


@pytest.mark.parametrize("G,q,kv", [(2, 3, 60), (4, 40, 90), (1, 130, 130)])
def test_attention_e4m3_nan_stays_with_its_rows(cb, serve, G, q, kv):
    for z in (0, 1):
        s = Step(cb, [(q, kv)], 1, G, 128, 16, True, seed=8)
        s.run()
        clean = f64(s.out)
        j = kv - q + q // 2
        raw = s.pool.view(torch.uint8)
        raw[s.layer, z, int(s.table[0, j // 16]), 0, j % 16, 77] = 0x7f
        s.run()
        got = f64(s.out)
        # without a NaN in sight the tiles go another way than with one, but with the same sums
        assert np.array_equal(got[:q // 2], clean[:q // 2])
        if z == 1:
            assert np.isnan(got[q // 2:, :, 77]).all()
            keep = [c for c in range(128) if c != 77]
            assert np.array_equal(got[q // 2:, :, keep], clean[q // 2:, :, keep])
        else:
            assert np.isnan(got[q // 2:]).all()


def test_attention_many_heads_few_workgroups(cb, serve):
    """More KV heads than workgroups that rows are divided into, head groups beyond a row tile."""
    s = Step(cb, [(1, 3000), (2, 60)], 40, 2, 64, 16, seed=60)
    s.run(ws=40000)
    s.check(serve, rows=[1])
    s.run()
    s.check(serve)
    s = Step(cb, [(1, 2000), (3, 2100)], 1, 150, 64, 64, seed=61)
    s.run()
    s.check(serve)


def test_calls_on_a_stream_object_and_a_handle(cb, serve):
    s = Step(cb, [(1, 500), (33, 120)], 1, 2, 64, 16, seed=62)
    s.run()
    want = s.out.clone()
    st = torch.cuda.Stream()
    s.run(stream=st)
    assert torch.equal(s.out, want)
    s.run(stream=st.cuda_stream)
    assert torch.equal(s.out, want)
    with torch.cuda.stream(st):
        s.run()
    assert torch.equal(s.out, want)


def check_tokens(serve, s, tokens, heads, window=0, sinks=0):
    """Some tokens (request, new token) and KV heads of a large step against the plain form, each as its request's last."""
    got, gl, qd, G, d = f64(s.out), f64(s.lse), f64(s.q), s.G, s.d
    for r, i in tokens:
        nq, kv = s.lens[r]
        t, p = s.starts[r] + i, kv - nq + i
        for h in heads:
            hs = slice(h * G, (h + 1) * G)
            o, l, mag, smag = serve.attention(qd[t:t + 1, hs], s.K[r][h], s.V[r][h], p + 1, d ** -0.5, window, sinks)
            es, few = (d + 8) * 2 * F32 * smag, (kv + 64) * 2 * F32
            tol = BF * np.abs(o) * 1.01 + mag * (BF * 1.01 + (2 * es + few)[..., None])
            assert (np.abs(got[t:t + 1, hs] - o) <= tol).all(), (r, i, h)
            assert (np.abs(gl[t:t + 1, hs] - l) <= es + few + 8 * F32 * (np.abs(l) + 1)).all(), (r, i, h)


@pytest.mark.parametrize("d,f8", [(128, False), (128, True), (64, False), (64, True), (96, False)])
def test_attention_large_alike_chunks(cb, serve, d, f8):
    """Chunks that fill the chip with 256 rows a workgroup (heads of 96: 128), a single token among them, with and
    without a window, a value of V that only the later rows see, and rows in parts."""
    s = Step(cb, [(512, 600), (512, 1500), (1, 700), (512, 512), (513, 513)], 8, 8, d, 16, f8, pad=2, seed=70, layers=1, layer=0)
    some = [(0, 0), (0, 511), (1, 100), (1, 255), (1, 256), (2, 0), (3, 0), (3, 31), (3, 32), (3, 300), (4, 1), (4, 512)]
    s.run()
    check_tokens(serve, s, some, [0, 5])
    assert (s.out[-2:] == 9.0).all()
    clean = f64(s.out)
    s.run(300, 4)
    check_tokens(serve, s, some, [2, 7], 300, 4)
    s.run(max_q=100)                                            # the same with 128 rows a workgroup
    check_tokens(serve, s, some, [0, 5])
    j = 200                                                     # of request 3: its rows from 200 on see it
    at = (0, 1, int(s.table[3, j // 16]), 5, j % 16, 9)
    if f8:
        s.pool.view(torch.uint8)[at] = 0x7f
    else:
        s.pool[at] = float("inf")
    s.run()
    got = f64(s.out)
    t0, hs = s.starts[3], slice(40, 48)
    assert not np.isfinite(got[t0 + 200:t0 + 512, hs, 9]).any()
    got[t0 + 200:t0 + 512, hs, 9] = clean[t0 + 200:t0 + 512, hs, 9]
    assert np.array_equal(got, clean)


def test_attention_large_chunk_in_parts(cb, serve):
    """One chunk of 256-row tiles over a long context in few heads: its keys in parts."""
    s = Step(cb, [(2050, 9000)], 1, 64, 64, 64, seed=71, layers=1, layer=0)
    s.run()
    check_tokens(serve, s, [(0, 0), (0, 3), (0, 4), (0, 1025), (0, 2049)], [0])
    s.run(ws=False)
    check_tokens(serve, s, [(0, 0), (0, 2049)], [0])


def one_hot(cb, lens, G, d, f8, exponent, sign=1.0, scale=None):
    """A step whose scores are exact and so far apart that a row's largest visible one takes all the weight: key j is
    c_j in every channel, c_j whole numbers that fit both types, queries 2^exponent in every channel."""
    s = Step(cb, lens, 1, G, d, 16, f8, seed=90)
    c = [np.random.default_rng(r).permutation(kv) % 13 * 16 + 16.0 for r, (_, kv) in enumerate(lens)]
    for r, (nq, kv) in enumerate(lens):
        for j in range(kv):
            s.pool[s.layer, 0, int(s.table[r, j // 16]), :, j % 16] = torch.full((1, d), c[r][j]).to(s.pool.dtype).cuda()
    s.q = torch.full_like(s.q, sign * 2.0 ** exponent)
    s.run(scale=scale)
    sc = d ** -0.5 if scale is None else scale
    kscale = 1.0 if not f8 else float(s.scales[s.layer, 0, 0])
    for r, (nq, kv) in enumerate(lens):
        for i in range(nq):
            t, p = s.starts[r] + i, kv - nq + i
            score = sc * kscale * d * sign * 2.0 ** exponent * c[r][:p + 1]
            best = np.flatnonzero(score == score.max())
            v = s.V[r][0][best]                                             # equal scores share the weight
            got, l = f64(s.out)[t], f64(s.lse)[t]
            tol = BF * 1.01 * np.abs(v.mean(0)) + (BF + (kv + 64) * 2 * F32) * np.abs(v).mean(0)
            assert (np.abs(got - v.mean(0)) <= tol).all(), (r, i)
            want = score.max() + math.log(len(best))
            assert (np.abs(l - want) <= 8 * F32 * (np.abs(want) + 1)).all(), (r, i)


@pytest.mark.parametrize("sign,scale", [(1.0, None), (-1.0, None), (1.0, -0.3)])
@pytest.mark.parametrize("exponent", [12, 17, 20, 24, 27, 28, 40, 90])
@pytest.mark.parametrize("f8", [False, True])
def test_attention_scores_beyond_the_places_of_fp32(cb, f8, exponent, sign, scale):
    """Scores of 2^20 .. 2^100: fp32 has no fractions there, but the differences are whole scores and the largest one's
    weight is 1 in every kernel."""
    for lens, G in (([(1, 70), (3, 40)], 4), ([(70, 200), (40, 40)], 2), ([(300, 300)], 1)):
        one_hot(cb, lens, G, 128, f8, exponent, sign, scale)
    one_hot(cb, [(40, 100), (1, 60)], 4, 96, f8, exponent, sign, scale)


def test_attention_scores_beyond_the_places_of_fp32_in_large_chunks(cb):
    for exponent in (20, 28):
        s = Step(cb, [(520, 520)], 8, 64, 64, 16, seed=91, layers=1, layer=0)
        c = torch.arange(520) % 251 + 1
        pool = s.pool
        for j in range(520):
            pool[0, 0, int(s.table[0, j // 16]), :, j % 16] = float(c[j])
        s.q = torch.full_like(s.q, 2.0 ** exponent)
        s.run()
        best = [int(max(range(i + 1), key=lambda j: (int(c[j]), j))) for i in range(520)]
        got = f64(s.out)
        for i in (0, 1, 63, 64, 200, 250, 251, 519):
            rows = [j for j in range(i + 1) if c[j] == c[best[i]]]
            for h in (0, 7):
                v = s.V[0][h][rows]
                tol = BF * 1.01 * np.abs(v.mean(0)) + (BF + 584 * 2 * F32) * np.abs(v).mean(0)
                assert (np.abs(got[i, 64 * h:64 * h + 64] - v.mean(0)) <= tol).all(), (exponent, i, h)


@pytest.mark.parametrize("d,f8", [(64, False), (96, True), (128, False), (128, True)])
@pytest.mark.parametrize("nq,kv", [(1, 300), (2, 700), (4, 2600)])
def test_attention_of_a_request_beside_others(cb, serve, d, f8, nq, kv):
    """A request alone, beside a chunk (which picks the other kernel for it) and beside rows long enough to be divided:
    other orders of sums and other bf16 weights, each within its roundings, the same bits for the same call.  Two results
    differ by the two outputs' roundings and, for weights w whose bf16 numbers differ by up to 2^-8 w on either side, by
    twice the weights' share."""
    H, G = 2, 8
    beside = ([], [(90, 400)], [(1, 30000)], [(300, 2000), (1, 9000), (2, 40)])
    results, first = [], None
    for others in beside:
        s = Step(cb, [(nq, kv)] + others, H, G, d, 16, f8, seed=95, layers=1, layer=0)
        if first is None:
            first = s
        else:                                                   # the request's own keys, values and queries are the first step's
            s.K[0], s.V[0] = first.K[0], first.V[0]
            s.scales = first.scales
            s.q[:nq] = first.q[:nq]
            for j in range(-(-kv // 16)):
                s.pool[0, :, int(s.table[0, j])] = first.pool[0, :, int(first.table[0, j])]
        s.run()
        s.check(serve, rows=[0])
        a, l = s.out[:nq].clone(), s.lse[:nq].clone()
        s.run()
        assert torch.equal(a, s.out[:nq]) and torch.equal(l, s.lse[:nq])
        results.append((f64(a), f64(l)))
    for h in range(H):
        hs = slice(h * G, (h + 1) * G)
        o, l, mag, smag = serve.attention(f64(first.q)[:nq, hs], first.K[0][h], first.V[0][h], kv, d ** -0.5)
        es, few = (d + 8) * 2 * F32 * smag, (kv + 64) * 2 * F32
        tol = 2 * (BF * 1.01 * np.abs(o) + mag * (BF * 1.01 + (2 * es + few)[..., None]))
        for a, al in results[1:]:
            assert (np.abs(a[:, hs] - results[0][0][:, hs]) <= tol).all()
            assert (np.abs(al[:, hs] - results[0][1][:, hs]) <= 2 * (es + few + 8 * F32 * (np.abs(l) + 1))).all()


# ------------------------------------------------------------------ rows whose halves two tokens' lanes exchange

@pytest.fixture(scope="module")
def rows_cut(tmp_path_factory):
    """The launch of a call on rows, from the library's own rule: (group, whether pairs of tokens exchange halves)."""
    d = tmp_path_factory.mktemp("rows_cut")
    (d / "cut.cpp").write_text('#include "cb_paged_rules.h"\nextern "C" int cut(int64_t n, int rows, int d, int f8) {\n'
                               '    cb::RowsCut c = cb::rows_cut(n, rows, d, f8); return 2 * c.group + c.pairs; }\n')
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_00891_amd", "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", csrc, str(d / "cut.cpp"), "-o", str(d / "cut.so")],
                   check=True)
    lib = ctypes.CDLL(str(d / "cut.so"))
    lib.cut.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int]
    return lambda n, rows, d, f8=False: divmod(lib.cut(n, rows, d, int(f8)), 2)


@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("d,L,H,B,T,token_major", [
    (64, 54, 8, 3, 401, False), (96, 54, 8, 3, 401, True), (16, 103, 16, 3, 401, False), (112, 40, 8, 1, 801, False),
    (240, 30, 8, 3, 401, True), (64, 80, 128, 1, 1, False), (96, 200, 8, 2, 150, False)])
def test_rows_that_exchange_halves(cb, serve, rows_cut, d, L, H, B, T, token_major, style):
    """Every form of the exchange, in calls that the rule gives to it: out of place and in place, forward and back, into
    pages with tokens without a slot (of pairs one, the other or both) and query rows, turned or not.  The same bits as
    layer by layer, calls that the rule gives to the other form, and the plain form in some layers."""
    n, QH = B * T, 5
    for rows in (L * H, 2 * L * H, 2 * L * H + QH):
        group, pairs = rows_cut(n, rows, d)
        assert pairs and group >= 4
    assert not rows_cut(n, 2 * H, d)[1]
    g = gen(d + T)
    shape = (L, 2, B, T, H, d) if token_major else (L, 2, B, H, T, d)
    x = torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(d + T), device="cuda").to(torch.bfloat16)
    x = x.permute(0, 1, 2, 4, 3, 5) if token_major else x
    table, pos, axis = make_rope(cb, d, 3, n, seed=d, bad=(n - 1, 7) if n > 8 else ())
    rope = cb.rope_axes_spec(table, i32(pos), axis, style)

    def same(u, v):
        return torch.equal(u.isnan(), v.isnan()) and torch.equal(u.nan_to_num(1.0), v.nan_to_num(1.0))

    for inverse in (False, True):
        out = torch.full((L, 2, B, H, T, d), 3.0, dtype=torch.bfloat16, device="cuda")
        cb.cb_rope_axes(x, out, rope, inverse=inverse)
        one = torch.full_like(out, 3.0)
        for l in range(L):
            cb.cb_rope_axes(x[l:l + 1], one[l:l + 1], rope, inverse=inverse)
        assert same(out, one)
        y = x.clone(memory_format=torch.preserve_format)
        cb.cb_rope_axes(y, y, rope, inverse=inverse)
        assert same(y, one)
        for l in (0, L - 1):
            want, mag = serve.turn(f64(x[l, 0, :, :2]).transpose(0, 2, 1, 3).reshape(n, -1, d), table.cpu().numpy(), pos, axis,
                                   style, inverse)
            check_turned(f64(out[l, 0, :, :2]).transpose(0, 2, 1, 3).reshape(n, -1, d), want, mag, "keys")
    slots = torch.randperm(n + 3, generator=g)[:n].int()
    if n > 8:
        slots[[0, 5, 6, 7, 10, 11, n // 2, n - 2]] = -1
        slots[3] = n + 3
    keep = ((slots >= 0) & (slots < n + 3)).cuda()
    at = slots.cuda()[keep].long()
    left = torch.ones(n + 3, dtype=torch.bool, device="cuda")
    left[at] = False
    q = randn(g, n, QH, d).cuda()
    q_ref = torch.empty((1, 2, 1, QH, n, d), dtype=torch.bfloat16, device="cuda")
    cb.cb_rope_axes(q.transpose(0, 1)[None, None, None].expand(1, 2, 1, QH, n, d), q_ref, rope)
    for turned in (True, False):
        ref = x
        if turned:
            ref = torch.full((L, 2, B, H, T, d), 3.0, dtype=torch.bfloat16, device="cuda")
            cb.cb_rope_axes(x, ref, rope)
        pool = torch.full((L, 2, n + 3, H, 1, d), 5.0, dtype=torch.bfloat16, device="cuda")
        q_out = torch.full_like(q, 7.0)
        kw = dict(rope=rope, q=q, q_out=q_out) if turned else {}
        cb.cb_page_write(x, cb.page_pool(pool), slots.cuda(), **kw)
        moved = pool.squeeze(4)                                 # [layer][kv][slot][head][d]
        flat = ref.permute(0, 1, 2, 4, 3, 5).reshape(L, 2, n, H, d)
        assert same(moved[:, :, at], flat[:, :, keep])
        assert (moved[:, :, left] == 5.0).all()
        if turned:
            assert same(q_out[keep], q_ref[0, 0, 0].transpose(0, 1)[keep]) and (q_out[~keep] == 7.0).all()
            cb.cb_page_write(x, cb.page_pool(pool), slots.cuda(), rope=rope, q=q_out, q_out=q_out)   # in place: once more
            twice = torch.empty_like(q_ref)
            cb.cb_rope_axes(q_ref, twice, rope)
            assert same(q_out[keep], twice[0, 0, 0].transpose(0, 1)[keep]) and (q_out[~keep] == 7.0).all()


# ------------------------------------------------------------------ calls at once, captured steps

def test_calls_on_two_streams_at_once(cb, serve):
    """Divided rows and chunks on two streams, a workspace each, enqueued in turn without a wait between them: what one
    leaves in a buffer the other could read, it would read here."""
    steps = [Step(cb, [(1, 40000), (200, 6000), (1, 20000), (3, 50)], 2, 4, 128, 64, f8, seed=100 + f8, layers=1, layer=0)
             for f8 in (False, True)]
    st = [torch.cuda.Stream(), torch.cuda.Stream()]
    want, args, ws, outs = [], [], [], []
    for s in steps:
        s.run()
        check_tokens(serve, s, [(0, 0), (1, 0), (1, 199), (3, 2)], [1])
        want.append((s.out.clone(), s.lse.clone()))
        args.append((s.q, cb.page_pool(s.pool, s.scales), 0, i32(s.starts), i32([k for _, k in s.lens]), i32(s.table)))
        need = cb.cb_attn_paged_workspace_bytes(s.n, len(s.lens), 8, 2, 128, s.max_q)
        ws.append(torch.empty((need,), dtype=torch.uint8, device="cuda"))
        outs.append([(torch.full_like(s.out, 5.0), torch.full_like(s.lse, 5.0)) for _ in range(20)])
    first, last = ([torch.cuda.Event(enable_timing=True) for _ in st] for _ in range(2))
    torch.cuda.synchronize()
    for i in range(2):
        first[i].record(st[i])
    for rep in range(20):
        for i in range(2):
            o, l = outs[i][rep]
            cb.cb_attn_paged(*args[i], o, steps[i].max_q, lse=l, workspace=ws[i], stream=st[i])
    for i in range(2):
        last[i].record(st[i])
    torch.cuda.synchronize()
    assert first[0].elapsed_time(last[1]) > 0 and first[1].elapsed_time(last[0]) > 0    # both were under way together
    for i in range(2):
        for o, l in outs[i]:
            assert torch.equal(o, want[i][0]) and torch.equal(l, want[i][1])


@pytest.mark.parametrize("max_q,G,window,sinks", [(3, 2, 0, 0), (40, 4, 0, 0), (40, 4, 3000, 40), (3, 2, 3000, 40), (40, 4, 700, 2)])
def test_a_captured_step_of_long_requests(cb, serve, max_q, G, window, sinks):
    """A step captured with a table of 12,000 keys and replayed with lengths that move requests between one part, several
    and as many as a workgroup joins, between the kernels of short rows and of chunks, and out of the step.  Two graphs
    with a workspace each take turns; every replay equals the eager call on its lengths and, in some tokens, the plain
    form."""
    H, d, ps, B, width, n = 2, 64, 16, 3, 750, 90
    g = gen(110 + max_q)
    P = B * width + 4
    pool = torch.randn((1, 2, P, H, ps, d), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").to(torch.bfloat16)
    pages = cb.page_pool(pool)
    rt = torch.empty((width * ps, d // 2, 2), dtype=torch.float32, device="cuda")
    cb.cb_rope_table(THETA, d, width * ps, rt)
    need = cb.cb_attn_paged_workspace_bytes(n, B, H * G, H, d, max_q)

    def state():
        z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
        s = dict(ctx=i32([0] * B), q=i32([0] * B), free=i32([0] * 8), table=i32(np.full((B, width), -1)), q_starts=i32([0] * (B + 1)),
                 kv=i32([0] * B), slots=i32([0] * n), pos=i32([0] * n), info=i32([0] * B), used=i32([0]), x=z(1, 2, 1, H, n, d),
                 qin=z(n, H * G, d), qr=z(n, H * G, d), out=z(n, H * G, d),
                 lse=torch.zeros((n, H * G), dtype=torch.float32, device="cuda"),
                 ws=torch.empty((need,), dtype=torch.uint8, device="cuda"))
        s["rope"] = cb.rope_axes_spec(rt, s["pos"])
        return s

    def step(s):
        cb.cb_page_tables(s["ctx"], s["q"], s["free"], ps, s["table"], s["q_starts"], s["kv"], s["slots"], s["pos"], s["info"], s["used"])
        cb.cb_page_write(s["x"], pages, s["slots"], rope=s["rope"], q=s["qin"], q_out=s["qr"])
        cb.cb_attn_paged(s["qr"], pages, 0, s["q_starts"], s["kv"], s["table"], s["out"], max_q, window=window, sinks=sinks,
                         lse=s["lse"], workspace=s["ws"])

    graphs = []
    for _ in range(2):
        s = state()
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            step(s)
        torch.cuda.current_stream().wait_stream(st)
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step(s)
        graphs.append((gr, s))
    e = state()
    # contexts and new tokens: short rows, one part, two, dozens (joined by a workgroup), a chunk of either, none
    lengths = [([40, 300, 700], [1, 1, 1]), ([11900, 20, 0], [1, 2, 3]), ([1500, 11000, 9000], [3, 1, 2]),
               ([9000, 30, 11500], [max_q, 1, 0]), ([100, 10000, 2000], [1, max_q, max_q]), ([0, 0, 0], [0, 0, 0]),
               ([5000, 5000, 5000], [2, 1, 2]), ([11990, 3, 600], [1, max_q, 1])]
    rng = np.random.default_rng(7)
    for it, (ctx, q) in enumerate(lengths):
        gr, s = graphs[it % 2]
        x, qin = randn(g, 1, 2, 1, H, n, d).cuda(), randn(g, n, H * G, d).cuda()
        perm = rng.permutation(P)
        table, at = np.full((B, width), -1), 0
        for b in range(B):
            m = -(-ctx[b] // ps)
            table[b, :m] = perm[at:at + m]
            at += m
        free = perm[at:at + 8]
        assert len(free) == 8
        for t in (s, e):
            for k, v in (("ctx", ctx), ("q", q), ("free", free), ("table", table)):
                t[k].copy_(i32(v))
            t["x"].copy_(x); t["qin"].copy_(qin); t["out"].fill_(4.0); t["qr"].fill_(4.0); t["lse"].fill_(4.0)
        torch.cuda.synchronize()
        gr.replay()
        torch.cuda.synchronize()
        step(e)
        torch.cuda.synchronize()
        for k in ("q_starts", "kv", "slots", "pos", "info", "used", "table", "out", "qr", "lse"):
            assert torch.equal(s[k], e[k]), (it, k)
        total = sum(q)
        assert s["info"].tolist() == [0] * B and (s["out"][total:] == 4.0).all() and (s["lse"][total:] == 4.0).all()
        final, out, lse, qr = s["table"].cpu().numpy(), f64(s["out"]), f64(s["lse"]), f64(s["qr"])
        start = 0
        for b in range(B):
            kv = ctx[b] + q[b]
            ids = torch.tensor(final[b, :-(-kv // ps)].astype(np.int64), device="cuda")
            for i in sorted({0, q[b] // 2, q[b] - 1} if q[b] else ()):
                t, p, h = start + i, ctx[b] + i, (it + b) % H
                rows = [f64(pool[0, z, ids, h].reshape(-1, d)[:p + 1]) for z in range(2)]
                hs = slice(h * G, (h + 1) * G)
                o, l, mag, smag = serve.attention(qr[t:t + 1, hs], *rows, p + 1, d ** -0.5, window, sinks)
                es, few = (d + 8) * 2 * F32 * smag, (kv + 64) * 2 * F32
                tol = BF * np.abs(o) * 1.01 + mag * (BF * 1.01 + (2 * es + few)[..., None])
                assert (np.abs(out[t:t + 1, hs] - o) <= tol).all(), (it, b, i)
                assert (np.abs(lse[t:t + 1, hs] - l) <= es + few + 8 * F32 * (np.abs(l) + 1)).all(), (it, b, i)
            start += q[b]


def test_more_workspace_than_the_call_asks_for_changes_nothing(cb, serve):
    """One chunk, and heads with more queries than a short row tile: the bits of a workspace of twice the size."""
    for lens, H, G, d in (([(70, 9000)], 2, 2, 64), ([(1, 9000), (3, 5000)], 1, 40, 64), ([(1, 20000)], 1, 4, 96)):
        s = Step(cb, lens, H, G, d, 16, seed=120, layers=1, layer=0)
        need = cb.cb_attn_paged_workspace_bytes(s.n, len(lens), H * G, H, d, s.max_q)
        s.run(ws=need)
        a, l = s.out.clone(), s.lse.clone()
        check_tokens(serve, s, [(0, 0)], [H - 1])
        s.run(ws=2 * need)
        assert torch.equal(a, s.out) and torch.equal(l, s.lse)

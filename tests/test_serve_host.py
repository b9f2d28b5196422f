"""Host checks (no GPU) of serving from pages: how attention is cut into workgroups, and what the calls refuse."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_00891_amd", "csrc")
SOURCE = """
#include "cb_paged_rules.h"
extern "C" {
void tiles(int p_lo, int p_hi, int window, int sinks, int KT, int *out) {
    cb::KeyTiles k = cb::key_tiles(p_lo, p_hi, window, sinks, KT);
    out[0] = k.n; out[1] = k.sink; out[2] = k.first;
}
int tile_at(int n, int sink, int first, int v) { cb::KeyTiles k = {n, sink, first}; return k.tile(v); }
int64_t bound(int kv, int tokens, int window, int sinks, int KT) { return cb::key_tiles_bound(kv, tokens, window, sinks, KT); }
int64_t part_tiles(int64_t W, int H, int target, int c_min) { return cb::part_tiles(W, H, target, c_min); }
int parts_of(int64_t b, int64_t c) { return cb::parts_of(b, c); }
int parts_least(int64_t b, int64_t c, int least) { return cb::parts_of(b, c, least); }
int part_begin(int n, int s, int parts) { return cb::part_begin(n, s, parts); }
void work(int q, int kv, int G, int M, int KT, int64_t lo, int64_t hi, int window, int sinks, int64_t *out) {
    cb::RequestWork w = cb::request_work(q, kv, G, M, KT, lo, hi, window, sinks);
    out[0] = w.tiles; out[1] = w.tokens; out[2] = w.bound;
}
int64_t row_tiles_bound(int64_t t, int64_t n, int64_t G, int64_t M, int64_t hi) { return cb::row_tiles_bound(t, n, G, M, hi); }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged_rules")
    (d / "rules.cpp").write_text(SOURCE)
    so = str(d / "librules.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(d / "rules.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    i32, i64 = ctypes.c_int, ctypes.c_int64
    for name, res, args in (("tiles", None, [i32] * 5 + [ctypes.c_void_p]), ("tile_at", i32, [i32] * 4),
                            ("bound", i64, [i32] * 5), ("part_tiles", i64, [i64, i32, i32, i32]),
                            ("parts_of", i32, [i64, i64]), ("part_begin", i32, [i32] * 3),
                            ("work", None, [i32] * 5 + [i64, i64, i32, i32, ctypes.c_void_p]),
                            ("row_tiles_bound", i64, [i64] * 5)):
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    return lib


def _key_tiles(rules, *args):
    out = (ctypes.c_int * 3)()
    rules.tiles(*args, ctypes.addressof(out))
    n, sink, first = out
    return [rules.tile_at(n, sink, first, v) for v in range(n)]


@pytest.mark.parametrize("KT", [32, 64])
def test_key_tiles_are_those_with_a_visible_key(rules, KT):
    rng = np.random.default_rng(KT)
    for _ in range(400):
        p_lo = int(rng.integers(-40, 900))
        p_hi = p_lo + int(rng.integers(0, 40))
        window = int(rng.choice([0, 1, 2, 31, 32, 33, 100, 500, 2 ** 31 - 1]))
        sinks = int(rng.choice([0, 1, 4, 32, 33, 70, 2 ** 31 - 1]))
        got = _key_tiles(rules, p_lo, p_hi, window, sinks, KT)
        want = {j // KT for p in range(max(p_lo, 0), p_hi + 1) for j in range(p + 1)
                if not window or j > p - window or j < sinks}
        assert len(set(got)) == len(got) and set(got) >= want, (p_lo, p_hi, window, sinks)
        # no tile without a visible key (windows that both rows' ranges share leave none between)
        assert set(got) - want <= {t for t in range(max(p_lo, 0) // KT + 1)} if p_lo < 0 else set(got) == want


def test_key_tiles_with_the_largest_window_and_rows_before_the_first_key(tmp_path):
    """Sums that wrap, as a compiler may form them, must not turn the largest window into a small one."""
    (tmp_path / "rules.cpp").write_text(SOURCE)
    so = str(tmp_path / "librules.so")
    subprocess.run(["g++", "-O2", "-fwrapv", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(tmp_path / "rules.cpp"), "-o", so],
                   check=True)
    lib = ctypes.CDLL(so)
    for window in (2 ** 31 - 1, 2 ** 31 - 40):
        for p_lo, p_hi in ((-100, 70), (-41, 0), (-40, 200), (-2, 1), (0, 33), (2 ** 31 - 70, 2 ** 31 - 60)):
            out = (ctypes.c_int * 3)()
            lib.tiles(p_lo, p_hi, window, 0, 32, out)
            hidden = max(0, p_lo - window + 1)                  # keys before this one are seen by no row
            assert tuple(out) == (p_hi // 32 + 1 - hidden // 32, 0, hidden // 32), (window, p_lo, p_hi, tuple(out))


def test_every_key_tile_of_every_row_tile_has_one_part(rules):
    """The workgroups' division, evaluated as they do: every (request, row tile, key tile) once, partial results and
    workgroups within what the host provides."""
    rng = np.random.default_rng(5)
    out = (ctypes.c_int64 * 3)()
    for trial in range(300):
        M, KT = [(16, 32), (32, 32), (128, 64), (256, 64)][trial % 4]
        H, G = int(rng.choice([1, 2, 4, 8, 40])), int(rng.choice([1, 2, 5, 8, 16, 33]))
        n = int(rng.choice([1, 2, 7, 60, 300]))
        q = rng.integers(0, 1 + int(rng.choice([1, 9, 200])), n)
        kv = (np.exp(rng.uniform(0, np.log(1 + int(rng.choice([40, 3000, 100000]))), n))).astype(int)
        window, sinks = int(rng.choice([0, 0, 50, 4000])), int(rng.choice([0, 4, 70]))
        target, c_min = int(rng.choice([0, 1, 7, 512, 2048])), int(rng.choice([1, 8]))
        lo, hi = [(0, 2 ** 62), (16, 2 ** 62), (0, 16)][int(rng.integers(3))]
        per = []
        for a, b in zip(q, kv):
            rules.work(int(a), int(b), G, M, KT, lo, hi, window, sinks, ctypes.addressof(out))
            per.append(tuple(out))
        W = sum(t * b for t, _, b in per)
        c = rules.part_tiles(W, H, target, c_min)
        items = slots = joined = 0
        for (tiles, tokens, bound), a, b in zip(per, map(int, q), map(int, kv)):
            rows = a * G
            assert tiles == (-(-rows // M) if lo < rows <= hi else 0)
            parts = rules.parts_of(bound, c)
            assert parts >= 1
            items += tiles * parts
            slots += tiles * parts if parts > 1 else 0
            joined += tiles if parts > 1 else 0
            for t in range(min(tiles, 3)):
                t0, t1 = t * M // G, (min(rows, (t + 1) * M) - 1) // G
                assert t1 - t0 + 1 <= tokens
                n_keys = len(_key_tiles(rules, b - a + t0, b - a + t1, window, sinks, KT))
                assert n_keys <= max(bound, 0)
                cuts = [rules.part_begin(n_keys, s, parts) for s in range(parts + 1)]
                assert cuts[0] == 0 and cuts[-1] == n_keys and cuts == sorted(cuts)
        tiles_bound = rules.row_tiles_bound(int(q.sum()), n, G, M, hi)
        assert items <= tiles_bound + target // H
        assert 3 * slots * H <= 4 * target
        assert joined <= min(tiles_bound, target // H)
        assert slots < 1 << 24


def test_short_rows_have_one_part(rules):
    rules.parts_least.restype, rules.parts_least.argtypes = ctypes.c_int, [ctypes.c_int64, ctypes.c_int64, ctypes.c_int]
    for b in range(0, 200):
        for c in (8, 16, 50, 2 ** 63 - 1):
            assert rules.parts_least(b, c, 36) == (1 if b < 36 else rules.parts_of(b, c))


# ------------------------------------------------------------------ refusals (nothing is enqueued: no GPU needed)

OK, ARG, SHAPE, ALIGN, UNSUP = 0, 1, 2, 3, 6
P = 1 << 20                                     # an aligned address that is never read


@pytest.fixture(scope="module")
def cb():
    import paper_2609_00891_amd as mod
    return mod


def cache(cb, **kw):
    c = cb.CbCache()
    d = dict(data=P, n_layers=1, n_heads=2, head_dim=64, n_seqs=4, seq_len=16, s_layer=8192, s_kv=4096, s_seq=2048,
             s_head=1024, s_tok=64)
    d.update(kw)
    for k, v in d.items():
        setattr(c, k, v)
    return c


def pages(cb, dtype=0, scales=None, **kw):
    p = cb.CbPages()
    p.cache, p.dtype, p.scales = cache(cb, **kw), dtype, scales
    return p


def rows(cb, **kw):
    r = cb.CbRows()
    d = dict(data=2 * P, n_tokens=3, n_heads=4, head_dim=64, s_tok=256, s_head=64)
    d.update(kw)
    for k, v in d.items():
        setattr(r, k, v)
    return r


def rope(cb, **kw):
    r = cb.CbRopeAxesSpec()
    d = dict(table=P, head_dim=64, n_pos=100, style=0, n_axes=1, positions=P, axis_stride=1 << 20)
    d.update(kw)
    axis = d.pop("axis", None)
    for k, v in d.items():
        setattr(r, k, v)
    for i, a in enumerate(axis or []):
        r.axis[i] = a
    return r


ATTN = dict(q={}, out=dict(data=3 * P), pages={}, layer=0, n_reqs=2, qs=P, kv=P, bt=P, stride=8, width=8, max_q=1, scale=0.1,
            window=0, sinks=0, lse=None, ws=None, ws_bytes=0)


def attn(cb, **kw):
    a = dict(ATTN)
    a.update(kw)
    ref = lambda f, x: None if x is None else ctypes.byref(f(cb, **x))
    return cb.library().cb_attn_paged(ref(rows, a["q"]), ref(pages, a["pages"]), a["layer"], a["n_reqs"], a["qs"], a["kv"],
                                      a["bt"], a["stride"], a["width"], ref(rows, a["out"]), a["max_q"], a["scale"],
                                      a["window"], a["sinks"], a["lse"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), ARG), (dict(out=None), ARG), (dict(pages=None), ARG),
    (dict(pages=dict(dtype=2)), ARG), (dict(pages=dict(dtype=1)), ARG), (dict(pages=dict(n_seqs=0)), SHAPE),
    (dict(pages=dict(seq_len=0)), SHAPE), (dict(pages=dict(head_dim=80)), UNSUP), (dict(pages=dict(s_tok=68)), ALIGN),
    (dict(pages=dict(data=P + 8)), ALIGN), (dict(pages=dict(dtype=1, scales=P, s_tok=72)), ALIGN),
    (dict(pages=dict(dtype=1, scales=P + 2)), ALIGN), (dict(pages=dict(s_seq=1 << 36)), UNSUP),
    (dict(pages=dict(n_seqs=1 << 20, seq_len=1 << 20)), UNSUP), (dict(pages=dict(s_head=-64)), SHAPE),
    (dict(layer=1), ARG), (dict(layer=-1), ARG), (dict(q=dict(head_dim=128)), SHAPE), (dict(q=dict(n_heads=5)), SHAPE),
    (dict(q=dict(n_heads=3), out=dict(data=3 * P, n_heads=3)), SHAPE), (dict(q=dict(s_head=36)), ALIGN),
    (dict(q=dict(data=P + 4)), ALIGN), (dict(q=dict(s_tok=-256)), SHAPE), (dict(out=dict(data=3 * P, n_tokens=2)), SHAPE),
    (dict(out=dict(data=None)), ARG), (dict(out=dict(data=2 * P)), ARG), (dict(n_reqs=-1), ARG), (dict(qs=None), ARG),
    (dict(kv=None), ARG), (dict(bt=None), ARG), (dict(qs=P + 2), ALIGN), (dict(stride=7), SHAPE), (dict(width=-1), ARG),
    (dict(width=1 << 28, stride=1 << 28), UNSUP), (dict(max_q=-1), ARG), (dict(scale=float("nan")), ARG),
    (dict(scale=float("inf")), ARG), (dict(window=-1), ARG), (dict(sinks=-1), ARG), (dict(ws=P + 4, ws_bytes=64), ALIGN),
    (dict(ws_bytes=-1), ARG), (dict(lse=P + 1), ALIGN),
    (dict(q=dict(n_tokens=0), out=dict(n_tokens=0)), OK), (dict(n_reqs=0), OK),
    (dict(out=dict(data=3 * P, s_tok=0)), SHAPE), (dict(out=dict(data=3 * P, s_head=32)), SHAPE), (dict(scale=3e38), ARG),
    (dict(q=dict(s_tok=0, s_head=0), n_reqs=0), OK),
    (dict(q=dict(n_tokens=1, n_heads=2), out=dict(data=3 * P, n_tokens=1, n_heads=2, s_tok=0), n_reqs=0), OK),
])
def test_attention_refuses(cb, kw, status):
    assert attn(cb, **kw) == status, cb.cb_last_error()
    assert (cb.cb_last_error() != "") == (status != OK)


WRITE = dict(rows=dict(n_seqs=1, seq_len=5, data=4 * P), pages={}, layer=0, slots=P, rope=None, q=None, qo=None)


def write(cb, **kw):
    a = dict(WRITE)
    a.update(kw)
    ref = lambda f, x: None if x is None else ctypes.byref(f(cb, **x))
    return cb.library().cb_page_write(ref(cache, a["rows"]), ref(pages, a["pages"]), a["layer"], a["slots"],
                                      ref(rope, a["rope"]), ref(rows, a["q"]), ref(rows, a["qo"]), None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=None), ARG), (dict(pages=None), ARG), (dict(slots=None), ARG), (dict(slots=P + 1), ALIGN),
    (dict(layer=1), ARG), (dict(layer=-1), ARG), (dict(pages=dict(n_heads=3)), SHAPE), (dict(pages=dict(head_dim=128)), SHAPE),
    (dict(rows=dict(head_dim=72, s_tok=72)), UNSUP), (dict(rows=dict(n_heads=0)), SHAPE), (dict(q={}), ARG),
    (dict(qo={}), ARG), (dict(q={}, qo={}), ARG), (dict(rope=dict(table=None)), ARG), (dict(rope=dict(positions=None)), ARG),
    (dict(rope=dict(style=2)), ARG), (dict(rope=dict(head_dim=128)), SHAPE), (dict(rope=dict(n_axes=0)), ARG),
    (dict(rope=dict(n_axes=5)), ARG), (dict(rope=dict(axis=[1])), ARG), (dict(rope=dict(n_axes=2, axis_stride=4)), SHAPE),
    (dict(rope=dict(table=P + 8)), ALIGN), (dict(rope=dict(n_pos=-1)), ARG),
    (dict(rope={}, q=dict(n_tokens=4), qo=dict(n_tokens=4)), SHAPE),
    (dict(rope={}, q=dict(n_tokens=5), qo=dict(n_tokens=5, n_heads=2)), SHAPE),
    (dict(rope={}, q=dict(n_tokens=5), qo=dict(n_tokens=5, s_tok=512)), ARG),
    (dict(rows=dict(n_seqs=1, seq_len=0)), OK),
    (dict(rope={}, q=dict(n_tokens=5), qo=dict(n_tokens=5, data=3 * P, s_tok=0)), SHAPE),
    (dict(rope={}, q=dict(n_tokens=5), qo=dict(n_tokens=5, data=3 * P, s_head=0)), SHAPE),
])
def test_page_write_refuses(cb, kw, status):
    assert write(cb, **kw) == status, cb.cb_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(inn=None), ARG), (dict(out=None), ARG), (dict(rope=None), ARG), (dict(out=dict(seq_len=4)), SHAPE),
    (dict(out=dict(s_tok=128)), ARG), (dict(out=dict(head_dim=96)), SHAPE), (dict(inn=dict(head_dim=24, s_tok=24)), UNSUP),
    (dict(rope=dict(axis=[3])), ARG), (dict(inn=dict(seq_len=0), out=dict(seq_len=0)), OK),
])
def test_rope_axes_refuses(cb, kw, status):
    a = dict(inn={}, out={}, rope={})
    a.update(kw)
    ref = lambda f, x: None if x is None else ctypes.byref(f(cb, **x))
    assert cb.library().cb_rope_axes(ref(cache, a["inn"]), ref(cache, a["out"]), ref(rope, a["rope"]), 0, None) == status


TABLES = dict(n=2, ctx=P, q=P, free=P, n_free=3, ps=16, bt=P, stride=4, width=4, tokens=8, qs=P, kv=P, slots=P, pos=P, info=P,
              used=P)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), ARG), (dict(n=4097), UNSUP), (dict(ctx=None), ARG), (dict(q=None), ARG), (dict(free=None), ARG),
    (dict(n_free=-1), ARG), (dict(ps=0), ARG), (dict(bt=None), ARG), (dict(stride=3), SHAPE), (dict(width=-1), ARG),
    (dict(ps=1 << 30), UNSUP), (dict(tokens=-1), ARG), (dict(qs=None), ARG), (dict(kv=None), ARG), (dict(slots=None), ARG),
    (dict(pos=None), ARG), (dict(info=None), ARG), (dict(used=None), ARG), (dict(used=P + 2), ALIGN),
])
def test_page_tables_refuse(cb, kw, status):
    a = dict(TABLES)
    a.update(kw)
    assert cb.library().cb_page_tables(a["n"], a["ctx"], a["q"], a["free"], a["n_free"], a["ps"], a["bt"], a["stride"],
                                       a["width"], a["tokens"], a["qs"], a["kv"], a["slots"], a["pos"], a["info"], a["used"],
                                       None) == status


def test_binding_refuses_wrong_tensors(cb):
    z = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t)
    i = lambda *s: z(*s, t=torch.int32)
    pool = z(1, 2, 3, 2, 16, 64)
    with pytest.raises(ValueError, match="scales"):
        cb.page_pool(pool, scales=z(1, 2, 2, t=torch.float32))
    with pytest.raises(ValueError, match="scales"):
        cb.page_pool(pool.to(torch.float8_e4m3fn))
    with pytest.raises(ValueError, match="bfloat16 or float8"):
        cb.page_pool(pool.half())
    pg = cb.page_pool(pool)
    assert pg.cache.n_seqs == 3 and pg.cache.seq_len == 16 and pg.cache.s_tok == 64
    q, out = z(2, 4, 64), z(2, 4, 64)
    good = dict(q=q, pages=pg, layer=0, q_starts=i(3), kv_lens=i(2), block_table=i(2, 3), out=out, max_q_len=1)
    for bad, match in ((dict(q=q.float()), "q is"), (dict(q_starts=i(2)), "q_starts"), (dict(kv_lens=i(2).long()), "kv_lens"),
                       (dict(block_table=i(3, 3)), "block_table"), (dict(lse=z(2, 4)), "lse"), (dict(), "current CUDA device")):
        with pytest.raises(ValueError, match=match):
            cb.cb_attn_paged(**dict(good, **bad))
    for name in ("layer", "max_q_len", "window", "sinks"):
        with pytest.raises(ValueError, match="32-bit"):
            cb.cb_attn_paged(**dict(good, **{name: 2 ** 32 + 1}))
    with pytest.raises(ValueError, match="32-bit"):
        cb.cb_page_write(z(1, 2, 1, 2, 9, 64), pg, i(9), layer=2 ** 32)
    with pytest.raises(ValueError, match="32-bit"):
        cb.cb_page_tables(i(2), i(2), i(4), 2 ** 32 + 16, i(2, 3), i(3), i(2), i(8), i(8), i(2), i(1))
    table = z(10, 32, 2, t=torch.float32)
    with pytest.raises(ValueError, match="axis"):
        cb.rope_axes_spec(table, i(3, 8), axis=[0] * 31)
    sp = cb.rope_axes_spec(table, i(3, 8), axis=[0, 1, 2, 0] * 8)
    assert sp.head_dim == 64 and sp.n_axes == 3 and sp.axis_stride == 8 and list(sp.axis[:4]) == [0, 1, 2, 0]
    rows_ = z(1, 2, 1, 2, 9, 64)
    with pytest.raises(ValueError, match="positions hold 8"):
        cb.cb_page_write(rows_, pg, i(9), rope=sp)
    with pytest.raises(ValueError, match="slots"):
        cb.cb_page_write(rows_, pg, i(8))
    with pytest.raises(ValueError, match="slots|positions"):
        cb.cb_page_tables(i(2), i(2), i(4), 16, i(2, 3), i(3), i(2), i(8), i(7), i(2), i(1))


def test_plain_tables_by_hand():
    """The plain form that the kernel is held against, on an example worked out by hand: page size 4."""
    from oracle import serve
    table = np.array([[7, -1, -1], [-1, -1, -1], [9, 8, -1], [-1, -1, -1]])
    r = serve.page_tables([3, 0, 8, 0], [2, 1, 5, 4], [20, 21, 22, 23], 4, table, 9)
    assert r["info"].tolist() == [0, 0, 2, 4]                   # 13 tokens need 4 entries; rows 8 + 4 > 9
    assert r["n_used"].tolist() == [2] and r["q_starts"].tolist() == [0, 2, 3, 8, 9]
    assert r["kv_lens"].tolist() == [5, 1, 0, 0]
    assert r["block_table"].tolist() == [[7, 20, -1], [21, -1, -1], [9, 8, -1], [-1, -1, -1]]
    assert r["positions"].tolist() == [3, 4, 0] + [-1] * 6
    assert r["slots"].tolist() == [7 * 4 + 3, 80, 84] + [-1] * 6


# ------------------------------------------------------------------ rows that are written

@pytest.mark.parametrize("s_tok,s_head,ok", [
    (64, 64, False), (64, 128, False), (128, 64, False), (192, 64, False), (256, 64, True), (264, 64, True), (64, 192, True),
    (64, 184, False), (64, 0, False), (0, 64, False), (56, 256, False)])
def test_rows_that_meet_are_refused_where_they_are_written(cb, s_tok, s_head, ok):
    """Three tokens of four heads of 64: two (token, head) rows may not share an element in an output."""
    at = sorted((t * s_tok + h * s_head) for t in range(3) for h in range(4))
    assert ok == all(b - a >= 64 for a, b in zip(at, at[1:]))
    r = dict(n_tokens=3, n_heads=4, s_tok=s_tok, s_head=s_head)
    assert attn(cb, out=dict(r, data=3 * P), n_reqs=0) == (OK if ok else SHAPE)
    # (rows without tokens: with good strides the call ends at the next check, that of the token counts)
    q = dict(n_tokens=3, n_heads=4)
    assert write(cb, rope={}, q=q, qo=dict(r, data=3 * P)) == SHAPE
    assert ("must not overlap" in cb.cb_last_error()) == (not ok)
    assert attn(cb, q=dict(r, data=3 * P), n_reqs=0) == OK                  # what is only read may meet


def test_rows_that_interleave_without_nesting_are_refused(cb):
    """Apart, but neither dimension's stride spans the other: refused as the header says."""
    assert attn(cb, out=dict(data=3 * P, n_tokens=3, n_heads=4, s_tok=320, s_head=128), n_reqs=0) == SHAPE


def test_rows_far_apart_do_not_wrap(cb):
    for s_tok, s_head, ok in ((1 << 62, 1 << 61, False), (1 << 62, 1 << 60, True), (64, 1 << 62, True)):
        out = dict(data=3 * P, n_tokens=3, n_heads=4, s_tok=s_tok, s_head=s_head)
        assert attn(cb, out=out, n_reqs=0) == (OK if ok else SHAPE)


# a cache of three layers, four sequences or pages, two heads, 16 tokens of 64 channels, every dimension beside the others
NESTED = dict(n_layers=3, n_seqs=4, n_heads=2, seq_len=16, head_dim=64, s_layer=16384, s_kv=8192, s_seq=2048, s_head=1024,
              s_tok=64)
MEET = [dict(s_tok=0), dict(s_head=0), dict(s_seq=0), dict(s_kv=0), dict(s_layer=0), dict(s_tok=48), dict(s_head=64),
        dict(s_seq=1024), dict(s_kv=2048), dict(s_layer=8192), dict(s_kv=8176), dict(s_layer=4096, s_kv=16384)]


def refused_as_written(cb, status, name):
    return status == SHAPE and f"{name} is written" in cb.cb_last_error()


@pytest.mark.parametrize("kw", MEET)
@pytest.mark.parametrize("dtype,scales", [(0, None), (1, P)])
def test_a_pool_whose_rows_meet_is_refused_where_it_is_written(cb, kw, dtype, scales):
    bad = {**NESTED, "dtype": dtype, "scales": scales, **kw}
    r = dict(data=4 * P, n_layers=2, n_seqs=1, seq_len=5)
    assert refused_as_written(cb, write(cb, rows=r, pages=bad), "pages"), cb.cb_last_error()
    # without tokens nothing is written; what attention reads may meet (a broadcast pool)
    assert write(cb, rows=dict(r, seq_len=0), pages=bad) == OK
    assert attn(cb, pages=bad, n_reqs=0) == OK


@pytest.mark.parametrize("kw", MEET)
def test_a_turned_cache_whose_rows_meet_is_refused(cb, kw):
    def turn(inn, out):
        return cb.library().cb_rope_axes(ctypes.byref(cache(cb, **inn)), ctypes.byref(cache(cb, **out)),
                                         ctypes.byref(rope(cb)), 0, None)
    bad = {**NESTED, **kw}
    assert refused_as_written(cb, turn(NESTED, dict(bad, data=8 * P)), "out"), cb.cb_last_error()
    if "s_kv" not in kw and kw != dict(s_layer=8192):           # in place only keys are written, and those are apart
        assert refused_as_written(cb, turn(bad, bad), "out"), cb.cb_last_error()
    assert turn(dict(bad, n_seqs=0), dict(bad, n_seqs=0, data=8 * P)) == OK


def test_the_launch_of_rows_covers_every_token_and_row(tmp_path):
    """The rule that cuts a call on rows: every token in a wave, every row in a group, whole pairs of tokens, and the
    exchange of halves only for long calls on 16-bit rows whose half is no whole number of lines."""
    (tmp_path / "cut.cpp").write_text(
        '#include "cb_paged_rules.h"\nextern "C" void cut(int64_t n, int rows, int d, int f8, int64_t *o) {\n'
        '    cb::RowsCut c = cb::rows_cut(n, rows, d, f8);\n'
        '    o[0] = c.tok_per_wave; o[1] = c.group; o[2] = c.blocks; o[3] = c.groups; o[4] = c.pairs; }\n')
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(tmp_path / "cut.cpp"), "-o",
                    str(tmp_path / "cut.so")], check=True)
    lib = ctypes.CDLL(str(tmp_path / "cut.so"))
    lib.cut.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p]
    rng, out, seen = np.random.default_rng(2), (ctypes.c_int64 * 5)(), set()
    for _ in range(3000):
        d, f8 = 16 * int(rng.integers(1, 17)), int(rng.integers(2))
        n, rows = int(np.exp(rng.uniform(0, 17))), int(np.exp(rng.uniform(0, 16)))
        lib.cut(n, rows, d, f8, ctypes.addressof(out))
        per_wave, group, blocks, groups, pairs = out
        lanes = d // 16
        assert per_wave % 2 == 0 and 2 <= per_wave and per_wave * lanes <= 64
        assert (blocks - 1) * 4 * per_wave < n <= blocks * 4 * per_wave
        assert (groups - 1) * group < rows <= groups * group and groups <= 65535
        assert group <= 16 or groups * 2 > 65535
        assert group == 1 or blocks * -(-rows // group) >= 2048 or -(-rows * 2 // group) > 65535
        assert pairs == (not f8 and d % 128 != 0 and group >= 4)
        seen.add((pairs, d))
    assert {(1, 16 * k) for k in range(1, 17) if k % 8} <= seen


def test_workspace_holds_what_the_call_can_use(cb):
    """Partial results of 16 rows (short rows: 4,096 slots) and of 128 (chunks: 1,024), both only in calls that can have
    both: chunks in one request, or heads with more queries than a short row tile, have no short rows beside them."""
    for d in (64, 96, 128):
        short, chunk = 4096 * 16 * (d + 2) * 4, 1024 * 128 * (d + 2) * 4
        for n_reqs, qheads, heads, max_q, want in ((5, 16, 2, 1, short), (1, 16, 2, 4, short), (1, 64, 2, 1, short),
                                                   (5, 16, 2, 5, short + chunk), (1, 16, 2, 5, chunk), (1, 16, 1, 3, chunk),
                                                   (9, 16, 1, 3, short + chunk), (9, 34, 2, 2, chunk), (9, 40, 1, 1, chunk)):
            got = cb.cb_attn_paged_workspace_bytes(100, n_reqs, qheads, heads, d, max_q)
            assert got == want, (n_reqs, qheads, heads, max_q)
    for bad in ((0, 1, 8, 8, 64, 1), (1, 0, 8, 8, 64, 1), (1, 1, 8, 3, 64, 1), (1, 1, 8, 8, 64, 0)):
        assert cb.cb_attn_paged_workspace_bytes(*bad) == 0


def test_workspace_sizes_do_not_wrap(cb):
    good = [100, 5, 16, 2, 64, 40]
    assert cb.cb_attn_paged_workspace_bytes(*good) > 0
    for i in range(6):
        with pytest.raises(ValueError, match="32-bit"):
            cb.cb_attn_paged_workspace_bytes(*(v + (2 ** 32 if i == j else 0) for j, v in enumerate(good)))

"""Host checks (no GPU) of pages whose scales belong to a page and head: the plain forms by hand, and what the calls
refuse (nothing is enqueued)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from test_serve_host import ALIGN, ARG, OK, P, SHAPE, UNSUP, cache, cb, pages, rope, rows  # noqa: F401


def blocks(cb, **kw):
    return pages(cb, **{**dict(dtype=2, scales=P), **kw})


SPANS = dict(n_reqs=2, starts=P, q=P, kv=P, bt=P, stride=8, width=8)
QUANT = dict(rows=dict(n_seqs=1, seq_len=5, data=4 * P), pages={}, layer=0, rope=None, qr=None, qo=None, **SPANS)


def ref(f, cb, x):
    return None if x is None else ctypes.byref(f(cb, **x))


def quantize(cb, **kw):
    a = {**QUANT, **kw}
    return cb.library().cb_page_quantize(ref(cache, cb, a["rows"]), ref(blocks, cb, a["pages"]), a["layer"], a["n_reqs"],
                                         a["starts"], a["q"], a["kv"], a["bt"], a["stride"], a["width"],
                                         ref(rope, cb, a["rope"]), ref(rows, cb, a["qr"]), ref(rows, cb, a["qo"]), None)


def read(cb, **kw):
    a = {**QUANT, **kw}
    return cb.library().cb_page_read(ref(blocks, cb, a["pages"]), a["layer"], ref(cache, cb, a["rows"]), a["n_reqs"],
                                     a["starts"], a["q"], a["kv"], a["bt"], a["stride"], a["width"],
                                     ref(rope, cb, a["rope"]), 1, None)


SPAN_REFUSALS = [
    (dict(n_reqs=-1), ARG), (dict(width=-1), ARG), (dict(stride=7), SHAPE), (dict(width=1 << 28, stride=1 << 28), UNSUP),
    (dict(starts=None), ARG), (dict(q=None), ARG), (dict(kv=None), ARG), (dict(bt=None), ARG), (dict(starts=P + 1), ALIGN),
    (dict(q=P + 2), ALIGN), (dict(kv=P + 2), ALIGN), (dict(bt=P + 2), ALIGN), (dict(n_reqs=0, starts=None, q=None), OK),
    (dict(rows=dict(n_seqs=1, seq_len=0)), OK), (dict(rows=None), ARG), (dict(pages=None), ARG),
    (dict(pages=dict(seq_len=1 << 25, n_seqs=1), width=1), UNSUP), (dict(layer=1), ARG), (dict(layer=-1), ARG),
    (dict(pages=dict(n_heads=3)), SHAPE), (dict(pages=dict(head_dim=128)), SHAPE), (dict(pages=dict(scales=None)), ARG),
    (dict(pages=dict(scales=P + 2)), ALIGN), (dict(pages=dict(s_tok=72)), ALIGN), (dict(pages=dict(dtype=3)), ARG),
    (dict(rows=dict(head_dim=72, s_tok=72)), UNSUP), (dict(rope=dict(style=2)), ARG), (dict(rope=dict(head_dim=128)), SHAPE),
    (dict(rope=dict(table=None)), ARG), (dict(rope=dict(n_axes=2, axis_stride=4)), SHAPE),
]


@pytest.mark.parametrize("kw,status", SPAN_REFUSALS + [
    (dict(pages=dict(dtype=1)), ARG), (dict(pages=dict(dtype=0, scales=None)), ARG), (dict(qr={}), ARG), (dict(qo={}), ARG),
    (dict(qr={}, qo={}), ARG), (dict(rope={}, qr=dict(n_tokens=4), qo=dict(n_tokens=4)), SHAPE),
    (dict(rope={}, qr=dict(n_tokens=5), qo=dict(n_tokens=5, n_heads=2)), SHAPE),
    (dict(rope={}, qr=dict(n_tokens=5), qo=dict(n_tokens=5, s_tok=512)), ARG),
    (dict(rope={}, qr=dict(n_tokens=5), qo=dict(n_tokens=5, data=3 * P, s_tok=0)), SHAPE),
    (dict(pages=dict(s_seq=0)), SHAPE), (dict(pages=dict(s_kv=0)), SHAPE),
])
def test_quantize_refuses(cb, kw, status):
    assert quantize(cb, **kw) == status, cb.cb_last_error()
    assert (cb.cb_last_error() != "") == (status != OK)


@pytest.mark.parametrize("kw,status", SPAN_REFUSALS + [
    (dict(rows=dict(n_seqs=2, seq_len=5, s_seq=0)), SHAPE), (dict(rows=dict(n_seqs=1, seq_len=5, s_kv=0)), SHAPE),
    (dict(pages=dict(s_seq=0), n_reqs=0), OK), (dict(pages=dict(dtype=0, scales=None), n_reqs=0), OK),
    (dict(pages=dict(dtype=1), n_reqs=0), OK),
])
def test_read_refuses(cb, kw, status):
    assert read(cb, **kw) == status, cb.cb_last_error()


def test_write_refuses_pages_with_scales_of_their_own(cb):
    c, p = cache(cb, n_seqs=1, seq_len=5, data=4 * P), blocks(cb)
    assert cb.library().cb_page_write(ctypes.byref(c), ctypes.byref(p), 0, P, None, None, None, None) == ARG
    assert "cb_page_quantize" in cb.cb_last_error()


def test_binding_refuses_wrong_tensors(cb):
    z = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t)  # noqa: E731
    i = lambda *s: z(*s, t=torch.int32)  # noqa: E731
    pool = z(2, 2, 3, 2, 16, 64).to(torch.float8_e4m3fn)
    for shape in ((2, 3, 2), (2, 3, 2, 1), (2, 2, 3, 2), (2, 2, 2, 2)):
        with pytest.raises(ValueError, match="scales"):
            cb.page_pool(pool, z(*shape, t=torch.float32))
    pg = cb.page_pool(pool, z(2, 3, 2, 2, t=torch.float32))
    assert pg.dtype == cb.CB_PAGES_E4M3_BLOCKS and cb.page_pool(pool, z(2, 2, 2, t=torch.float32)).dtype == cb.CB_PAGES_E4M3
    x = z(1, 2, 1, 2, 9, 64)
    good = dict(rows=x, pages=pg, row_starts=i(2), q_lens=i(2), kv_lens=i(2), block_table=i(2, 3))
    for f in (cb.cb_page_quantize, cb.cb_page_read):
        for bad, match in ((dict(rows=x.float()), "cache tensors"), (dict(row_starts=i(3)), "row_starts"),
                           (dict(q_lens=i(2).long()), "q_lens"), (dict(block_table=i(3, 3)), "block_table"),
                           (dict(layer=2 ** 32), "32-bit"), (dict(), "current CUDA device")):
            with pytest.raises(ValueError, match=match):
                f(**{**good, **bad})
        sp = cb.rope_axes_spec(z(10, 32, 2, t=torch.float32), i(3, 8), axis=[0, 1, 2, 0] * 8)
        with pytest.raises(ValueError, match="positions hold 8"):
            f(**good, rope=sp)


def test_plain_e4m3_by_hand():
    from oracle import serve
    x = [0.0, 1.0, 1.06, 1.0625, 1.1875, 17.0, 447.0, 448.0, 463.0, 465.0, 500.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9,
         -2.0 ** -11, 0.015]
    want = [0.0, 1.0, 1.0, 1.0, 1.25, 16.0, 448.0, 448.0, 448.0, np.nan, np.nan, 2.0 ** -9, 0.0, 2.0 ** -8, -0.0, 2.0 ** -6]
    assert np.array_equal(serve.e4m3(np.array(x)), np.array(want), equal_nan=True)
    assert np.isnan(serve.e4m3(np.array([np.inf, -np.inf, np.nan]))).all()
    ours = serve.e4m3(np.linspace(-447, 447, 9999))
    theirs = torch.linspace(-447, 447, 9999, dtype=torch.float64).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ours, theirs)


def test_plain_quantize_by_hand():
    """Page of two places: a first token of size 448, then one of 900, whose scale 4 the first goes over to."""
    from oracle import serve
    rows = np.zeros((2, 1, 2, 1, 2))
    rows[0, 0, :, 0] = [448.0, -3.0]
    rows[1, 0, :, 0] = [900.0, 1.0]
    codes, exps, table = np.full((1, 2, 2, 1, 2, 2), 5.0), np.full((1, 2, 1, 2), 3), np.array([[1]])
    assert serve.page_spans([0, 1], [1, 9], [1, 9], 2, 2, 1) == [(0, 0, 0, 1, 0)]
    serve.page_quantize(rows, None, codes, exps, serve.page_spans([0], [1], [1], 2, 2, 1), table)
    assert exps[0, :, 0].tolist() == [[3, 3], [0, 0]] and codes[0, 0, 1, 0].tolist() == [[448, -3], [5, 5]]
    serve.page_quantize(rows, None, codes, exps, serve.page_spans([1], [1], [2], 2, 2, 1), table)
    assert exps[0, 1, 0].tolist() == [2, 2] and codes[0, 1, 1, 0].tolist() == [[112, -0.75], [225, 0.25]]
    assert serve.block_exponent(np.array([0.0]), False) == serve.E_MIN
    assert [serve.block_exponent(np.array([v, np.inf, np.nan]), t) for v, t in ((448.0, 0), (449.0, 0), (316.0, 1), (317.0, 1))] == [0, 1, 0, 1]


# ------------------------------------------------------------------ selected pages

STEP = dict(q={}, pages={}, layer=0, n_reqs=2, qs=P, kv=P, bt=P, stride=8, width=8)
SELECT = dict(STEP, bounds=P, first=1, last=1, k=4, sel=P, ws=P, ws_bytes=1 << 20)
ATTEND = dict(STEP, sel=P, k=4, out=dict(data=3 * P), scale=0.1, lse=None, ws=None, ws_bytes=0)


def select(cb, **kw):
    a = {**SELECT, **kw}
    return cb.library().cb_page_select(ref(rows, cb, a["q"]), ref(blocks, cb, a["pages"]), a["layer"], a["bounds"], a["n_reqs"],
                                       a["qs"], a["kv"], a["bt"], a["stride"], a["width"], a["first"], a["last"], a["k"], a["sel"],
                                       a["ws"], a["ws_bytes"], None)


def attend(cb, **kw):
    a = {**ATTEND, **kw}
    return cb.library().cb_attn_selected(ref(rows, cb, a["q"]), ref(blocks, cb, a["pages"]), a["layer"], a["n_reqs"], a["qs"],
                                         a["kv"], a["bt"], a["stride"], a["width"], a["sel"], a["k"], ref(rows, cb, a["out"]),
                                         a["scale"], a["lse"], a["ws"], a["ws_bytes"], None)


STEP_REFUSALS = [
    (dict(q=None), ARG), (dict(pages=None), ARG), (dict(pages=dict(head_dim=80)), UNSUP), (dict(layer=1), ARG), (dict(layer=-1), ARG),
    (dict(pages=dict(scales=None)), ARG), (dict(pages=dict(scales=P + 4)), ALIGN), (dict(q=dict(s_tok=-256)), SHAPE),
    (dict(n_reqs=-1), ARG), (dict(qs=None), ARG), (dict(kv=None), ARG), (dict(bt=None), ARG), (dict(qs=P + 2), ALIGN),
    (dict(stride=7), SHAPE), (dict(width=-1), ARG), (dict(width=1 << 28, stride=1 << 28), UNSUP), (dict(sel=None), ARG),
    (dict(sel=P + 2), ALIGN), (dict(ws_bytes=-1), ARG), (dict(n_reqs=0, qs=None, kv=None, bt=None, sel=None), OK),
]


@pytest.mark.parametrize("kw,status", STEP_REFUSALS + [
    (dict(q=dict(head_dim=128)), SHAPE), (dict(q=dict(n_heads=5)), SHAPE), (dict(first=-1), ARG), (dict(last=0), ARG),
    (dict(first=4), ARG), (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), ARG), (dict(k=1), ARG), (dict(bounds=None), ARG),
    (dict(bounds=P + 8), ALIGN), (dict(ws=P + 2), ALIGN), (dict(ws_bytes=(8 + 4) * 2 * 4 - 1), SHAPE), (dict(ws=None), SHAPE),
    (dict(q=dict(n_tokens=0)), OK), (dict(width=1 << 25, stride=1 << 25, pages=dict(seq_len=1)), UNSUP),
    (dict(k=(1 << 30) + 1), UNSUP), (dict(q=dict(n_tokens=1 << 27)), UNSUP), (dict(q=dict(n_tokens=1 << 23), n_reqs=1 << 23), UNSUP),
])
def test_select_refuses(cb, kw, status):
    assert select(cb, **kw) == status, cb.cb_last_error()
    assert (cb.cb_last_error() != "") == (status != OK)


@pytest.mark.parametrize("kw,status", STEP_REFUSALS + [
    (dict(out=None), ARG), (dict(out=dict(data=3 * P, n_tokens=2)), SHAPE), (dict(out=dict(data=3 * P, s_tok=0)), SHAPE),
    (dict(out=dict(data=2 * P)), ARG), (dict(k=0), ARG), (dict(k=1 << 27), UNSUP), (dict(scale=float("nan")), ARG),
    (dict(scale=3e38), ARG), (dict(lse=P + 1), ALIGN), (dict(ws=P + 4), ALIGN),
    (dict(q=dict(n_tokens=0), out=dict(data=3 * P, n_tokens=0)), OK),
    (dict(q=dict(n_tokens=1 << 23), out=dict(data=3 * P, n_tokens=1 << 23)), UNSUP),
])
def test_selected_attention_refuses(cb, kw, status):
    assert attend(cb, **kw) == status, cb.cb_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(pages=None), ARG), (dict(layer=1), ARG), (dict(layers=0), ARG), (dict(layers=2), ARG), (dict(bounds=None), ARG),
    (dict(bounds=P + 8), ALIGN), (dict(n_reqs=-1), ARG), (dict(q=None), ARG), (dict(kv=None), ARG), (dict(bt=None), ARG),
    (dict(kv=P + 1), ALIGN), (dict(stride=7), SHAPE), (dict(width=1 << 28, stride=1 << 28), UNSUP), (dict(max_q=-1), ARG),
    (dict(pages=dict(seq_len=1 << 25, n_seqs=1), width=1), UNSUP), (dict(n_reqs=0, bounds=None), OK),
])
def test_bounds_refuses(cb, kw, status):
    a = {**dict(SPANS, pages={}, layer=0, layers=1, bounds=P, max_q=1), **kw}
    assert cb.library().cb_page_bounds(ref(blocks, cb, a["pages"]), a["layer"], a["layers"], a["bounds"], a["n_reqs"], a["q"],
                                       a["kv"], a["bt"], a["stride"], a["width"], a["max_q"], None) == status, cb.cb_last_error()


def test_binding_refuses_wrong_tensors_of_a_selection(cb):
    z = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t)  # noqa: E731
    i = lambda *s: z(*s, t=torch.int32)  # noqa: E731
    pg = cb.page_pool(z(1, 2, 3, 2, 16, 64))
    good = dict(q=z(2, 4, 64), pages=pg, layer=0, q_starts=i(3), kv_lens=i(2), block_table=i(2, 3), selected=i(2, 2, 4))
    sel = dict(good, bounds=z(1, 3, 2, 2, 64))
    att = dict(good, out=z(2, 4, 64))
    common = [(dict(q=z(2, 4, 64).float()), "q is"), (dict(q_starts=i(2)), "q_starts"), (dict(kv_lens=i(2).long()), "kv_lens"),
              (dict(block_table=i(3, 3)), "block_table"), (dict(selected=i(2, 4)), "selected"), (dict(selected=i(2, 1, 4)), "selected"),
              (dict(selected=i(2, 2, 4).long()), "selected"), (dict(layer=2 ** 32), "32-bit"),
              (dict(workspace=z(8, 8).T), "workspace"), (dict(), "current CUDA device")]
    for f, a, more in ((cb.cb_page_select, sel, [(dict(bounds=z(1, 3, 2, 2, 64).float()), "bounds"), (dict(bounds=z(1, 2, 2, 2, 64)), "bounds"),
                                                 (dict(first=2 ** 32 + 1), "32-bit")]),
                       (cb.cb_attn_selected, att, [(dict(lse=z(2, 4)), "lse"), (dict(out=z(2, 4, 64).float()), "out is")])):
        for bad, match in common + more:
            with pytest.raises(ValueError, match=match):
                f(**{**a, **bad})
    with pytest.raises(ValueError, match="bounds"):
        cb.cb_page_bounds(pg, z(1, 3, 2, 1, 64), i(2), i(2), i(2, 3), 1)
    with pytest.raises(ValueError, match="32-bit"):
        cb.cb_page_bounds(pg, z(1, 3, 2, 2, 64), i(2), i(2), i(2, 3), 2 ** 32)
    with pytest.raises(ValueError, match="32-bit"):
        cb.cb_page_select_workspace_bytes(2 ** 32 + 1, 1, 1)
    with pytest.raises(ValueError, match="32-bit"):
        cb.cb_attn_selected_workspace_bytes(1, 8, 8, 64, 2 ** 32 + 16, 4)


def test_workspaces(cb):
    """Scores of every token, head and entry, and four numbers for 256 entries; partial results of row tiles that are
    divided, none for others."""
    assert cb.cb_page_select_workspace_bytes(7, 2, 100) == 7 * 2 * (100 + 4) * 4
    assert cb.cb_page_select_workspace_bytes(7, 2, 257) == 7 * 2 * (257 + 8) * 4
    assert cb.cb_page_select_workspace_bytes(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1) == 2 ** 63 - 1
    assert cb.cb_page_select_workspace_bytes(0, 2, 100) == 0
    # 1 token, 8 heads, 128 tiles of 32 keys: parts of 16 tiles
    assert cb.cb_attn_selected_workspace_bytes(1, 64, 8, 128, 64, 64) == 8 * 8 * 16 * 130 * 4
    assert cb.cb_attn_selected_workspace_bytes(1, 8 * 33, 8, 128, 64, 64) == 3 * 8 * 8 * 16 * 130 * 4
    assert cb.cb_attn_selected_workspace_bytes(512, 64, 8, 128, 64, 64) == 0             # enough row tiles undivided
    assert cb.cb_attn_selected_workspace_bytes(1, 64, 8, 128, 16, 64) == 0               # 32 tiles: short
    for bad in ((0, 8, 8, 64, 16, 4), (1, 8, 3, 64, 16, 4), (1, 8, 8, 64, 16, 0), (1, 8, 8, 64, 1 << 20, 1 << 20)):
        assert cb.cb_attn_selected_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("n,qh,h,ps,k", [
    (1, 2 ** 31 - 1, 1, 1 << 20, 1 << 10), (2 ** 31 - 1, 2 ** 31 - 1, 1, 1, 1 << 30), (2 ** 31 - 1, 64, 8, 64, 64),
    (1 << 24, 16, 1, 1, 1 << 30), (1, 1 << 24, 1 << 24, 1, 1 << 30), (1 << 20, 16 * 17, 1, 64, 64), (2, 1 << 27, 1, 32, 1 << 25)])
def test_no_workspace_for_selected_attention_that_is_refused(cb, n, qh, h, ps, k):
    """2^24 rows of up to 16 query heads and more: the call refuses them, and their sizes would leave 64 bits."""
    assert n * -(-qh // h // 16) * h >= 1 << 24
    assert cb.cb_attn_selected_workspace_bytes(n, qh, h, 64, ps, k) == 0


@pytest.mark.parametrize("d", [64, 2 ** 31 - 1])
def test_workspace_of_the_largest_selected_attention(cb, d):
    """One row tile below the limit, and the longest lists: whole numbers that 64 bits hold, by parts as the rule counts
    them."""
    for n, qh, h in (((1 << 24) - 1, 1, 1), (1, 16 * ((1 << 24) - 1), 1), (1, (1 << 24) - 1, (1 << 24) - 1), (1, 1, 1), (64, 64, 8)):
        tiles, keys = -(-qh // h // 16), 1 << 25
        c = max(16, -(-n * tiles * keys * h // 2048))
        parts = 1 if keys <= c else keys // c + (keys % c >= c - c // 2)
        want = n * tiles * parts * h * 16 * (d + 2) * 4 if parts > 1 else 0
        assert cb.cb_attn_selected_workspace_bytes(n, qh, h, d, 1 << 20, 1 << 10) == want and 0 <= want < 2 ** 63


RULES = """
#include "cb_paged_rules.h"
extern "C" {
void selected(int64_t n, int32_t H, int32_t G, int32_t ps, int32_t k, int32_t *out) {
    const cb::SelectedCut c = cb::selected_cut(n, H, G, ps, k);
    out[0] = c.tiles;
    out[1] = c.parts;
}
int32_t shared(int64_t n, int64_t reqs, int64_t H, int32_t G, int32_t k, int32_t entries) {
    return cb::shared_tokens(n, reqs, H, G, k, entries);
}
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.cpp").write_text(RULES)
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_00891_amd", "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", csrc, str(d / "rules.cpp"), "-o", str(d / "r.so")], check=True)
    lib = ctypes.CDLL(str(d / "r.so"))
    i32, i64 = ctypes.c_int32, ctypes.c_int64
    lib.selected.argtypes, lib.selected.restype = [i64, i32, i32, i32, i32, ctypes.POINTER(i32)], None
    lib.shared.argtypes, lib.shared.restype = [i64, i64, i64, i32, i32, i32], i32
    return lib


@pytest.mark.parametrize("H", [1, 2, 8, 40])
@pytest.mark.parametrize("G", [1, 3, 8, 9, 33])
def test_selected_rows_are_cut_into_parts(rules, H, G):
    """A row tile has each of its query heads once; parts have at least 12 key tiles (nearest number to parts of 16 and
    more), there are none of short lists, and about 2,048 workgroups at most where rows are divided."""
    out = (ctypes.c_int32 * 2)()
    for n in (1, 7, 64, 500, 5000):
        for ps, k in ((1, 1), (16, 64), (16, 80), (64, 17), (64, 64), (1000, 5), (128, 4000), (1 << 20, 1 << 10)):
            rules.selected(n, H, G, ps, k, out)
            tiles, parts = out
            keys = -(-ps * k // 32)
            assert (tiles - 1) * 16 < G <= tiles * 16 and parts >= 1
            assert parts == 1 or (keys >= 36 and keys >= 12 * parts and n * tiles * H * parts <= 4 / 3 * 2048), (n, ps, k, parts)
            assert parts > 1 or keys < 36 or n * tiles * H > 2048 / 1.5 or keys <= 24, (n, ps, k)


def test_tokens_that_share_a_row_tile(rules):
    """Their heads fit 16 rows, their lists the entries, and 1,024 workgroups are left; requests of few tokens share none."""
    assert [rules.shared(4096, 1, 8, g, 64, 1024) for g in (1, 2, 3, 5, 8, 9, 16, 17)] == [16, 8, 5, 3, 2, 1, 1, 1]
    assert [rules.shared(4096, 1, 8, 1, k, 1024) for k in (1, 64, 65, 512, 513, 5000)] == [16, 16, 15, 2, 1, 1]
    assert [rules.shared(n, 1, 8, 2, 4, 1024) for n in (1, 128, 255, 256, 511, 1023, 1024, 9999)] == [1, 1, 1, 2, 3, 7, 8, 8]
    assert [rules.shared(600, r, 8, 4, 4, 1024) for r in (1, 200, 201, 600)] == [4, 4, 1, 1]
    assert rules.shared(2 ** 31 - 1, 1, 2 ** 16, 1, 1, 1024) == 16


def test_plain_selection_by_hand():
    from oracle import serve
    b = serve.page_bounds(np.array([[1.0, -2.0], [3.0, 0.5]]))
    assert b.tolist() == [[1.0, -2.0], [3.0, 0.5]]
    # q = (2, -1): 2 * 3 + -1 * -2 = 8; q = (-1, 0): -1 * 1 = -1
    assert serve.page_scores(np.array([[2.0, -1.0], [-1.0, 0.0]]), b[None]).tolist() == [7.0]
    s = np.array([5, 1, 9, 9, np.nan, -3, 0], np.float32)
    assert serve.page_select(s, [True] * 7, 1, 1, 4) == [0, 2, 4, 6]
    assert serve.page_select(s, [True] * 7, 0, 2, 4) == [2, 4, 5, 6]
    assert serve.page_select(s, [False, True, True, False, False, True, False], 1, 1, 2) == [1, 2]
    assert serve.page_select(s[:2], [True] * 2, 1, 1, 4) == [0, 1]


SPAN_RULES = """
#include "cb_paged_rules.h"
extern "C" void spans(int64_t n, int64_t reqs, int32_t ps, int32_t d, int32_t rows, int64_t *out) {
    const cb::SpanCut c = cb::span_cut(n, reqs, ps, d, rows);
    out[0] = c.lgc;
    out[1] = c.wide;
    out[2] = c.pairs;
    out[3] = c.group;
    out[4] = c.blocks;
    out[5] = c.groups;
}
"""


def build_span_cut(d):
    """span_cut(tokens, requests, page size, head_dim, rows) as a function that returns its numbers."""
    (d / "spans.cpp").write_text(SPAN_RULES)
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_00891_amd", "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", csrc, str(d / "spans.cpp"), "-o", str(d / "s.so")], check=True)
    lib = ctypes.CDLL(str(d / "s.so"))
    i32, i64 = ctypes.c_int32, ctypes.c_int64
    lib.spans.argtypes, lib.spans.restype = [i64, i64, i32, i32, i32, ctypes.POINTER(i64)], None

    def cut(*args):
        out = (i64 * 6)()
        lib.spans(*args, out)
        return dict(zip(("lgc", "wide", "pairs", "group", "blocks", "groups"), out))
    return cut


@pytest.fixture(scope="module")
def span_cut(tmp_path_factory):
    return build_span_cut(tmp_path_factory.mktemp("spans"))


@pytest.mark.parametrize("d", [16, 48, 64, 96, 128, 256])
def test_spans_are_cut_into_workgroups(span_cut, d):
    """Every row of every page has a workgroup, within a launch's limits; a page that a team takes in one turn has a place
    for each of its units (256 threads of the team, `pairs` each)."""
    for ps in (1, 7, 16, 64, 100, 1024, 1 << 24):
        for n, reqs in ((1, 1), (63, 64), (263, 64), (1811, 3), (5, 9), (1 << 24, 1), (2 ** 31 - 1, 1)):
            for rows in (2, 10, 80, 5120, 3 << 24):
                c = span_cut(n, reqs, ps, d, rows)
                assert 1 << c["lgc"] >= d // 16 > 1 << c["lgc"] >> 1
                assert (c["groups"] - 1) * c["group"] < rows <= c["groups"] * c["group"] and c["groups"] <= 65535
                assert 1 <= c["blocks"] <= min(max(n, 1), 1 << 22)
                units = ps << c["lgc"]
                assert units <= 256 * c["pairs"] if c["pairs"] else units > 1024


def test_a_call_of_single_tokens_and_a_chunk_has_narrow_teams(span_cut):
    """The rule goes by the call's tokens for each request: chunks' whole pages come to teams that were made for single
    tokens, larger than a wave and, where the page has more than 256 units, in turns."""
    assert [span_cut(n, 64, 64, 128, 12)["wide"] for n in (64, 263, 512, 513)] == [0, 0, 1, 1]
    assert not span_cut(63 + 200, 64, 16, 128, 12)["wide"] and not span_cut(30 + 150, 31, 64, 64, 12)["wide"]

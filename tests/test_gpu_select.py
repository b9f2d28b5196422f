"""GPU tests of attention over selected pages: bounds of pages, the choice of pages, attention over them, against the
plain fp64 forms of ``oracle.serve``.  Bounds and choices are exact; tolerances of attention as in ``test_gpu_serve``."""
import numpy as np
import pytest
import torch

from test_gpu_serve import BF, F32, THETA, Step, cb, f64, gen, i32, randn, serve  # noqa: F401
from test_gpu_serve_blocks import BlockStep

pytestmark = pytest.mark.gpu


def make_step(cb, kind, lens, H, G, d, ps, **kw):
    return BlockStep(cb, lens, H, G, d, ps, **kw) if kind == "blocks" else Step(cb, lens, H, G, d, ps, kind == "e4m3", **kw)


def stored_keys(s, r):
    """Request r's keys [head][key][d] in units of their scale, as bounds count them."""
    _, kv = s.lens[r]
    k = s.pool[s.layer, 0].float().double().cpu().numpy()
    return np.stack([np.concatenate([k[int(s.table[r, j // s.ps]), h, :min(s.ps, kv - j)] for j in range(0, kv, s.ps)])
                     for h in range(s.H)])


def empty_bounds(s, value=3.0):
    L, _, P, H, _, d = s.pool.shape
    return torch.full((L, P, H, 2, d), value, device="cuda").to(s.pool.dtype)


def all_bounds(cb, s):
    b = empty_bounds(s)
    kv = i32([k for _, k in s.lens])
    cb.cb_page_bounds(cb.page_pool(s.pool, s.scales), b, kv, kv, i32(s.table), max(k for _, k in s.lens), layer=s.layer)
    return b


# ------------------------------------------------------------------ bounds

@pytest.mark.parametrize("kind,d,ps,tm", [("bf16", 64, 16, False), ("bf16", 128, 7, True), ("bf16", 96, 64, False),
                                          ("e4m3", 64, 24, True), ("blocks", 128, 16, False), ("blocks", 96, 100, True)])
def test_bounds(cb, serve, kind, d, ps, tm):
    """The pages of the new tokens in one layer of three, the others' bounds left as they were."""
    lens = [(1, 1), (1, ps), (3, 2 * ps + 1), (2 * ps, 3 * ps), (0, 9), (5, 40)]
    s = make_step(cb, kind, lens, 3, 1, d, ps, token_major=tm, layers=3, layer=1, seed=d + ps)
    b = empty_bounds(s)
    before = f64(b)
    for hint in (1, 0, 500):
        cb.cb_page_bounds(cb.page_pool(s.pool, s.scales), b, i32([q for q, _ in lens]), i32([k for _, k in lens]), i32(s.table),
                          hint, layer=1)
    want = before.copy()
    for r, (q, kv) in enumerate(lens):
        x = stored_keys(s, r)
        for i in range((kv - q) // ps, (kv - 1) // ps + 1) if q else ():
            for h in range(3):
                want[1, int(s.table[r, i]), h] = serve.page_bounds(x[h, i * ps:min(kv, (i + 1) * ps)])
    assert np.array_equal(f64(b), want)


@pytest.mark.parametrize("d", [16, 48, 80, 256])
def test_bounds_of_other_widths_in_several_layers(cb, serve, d):
    g = gen(d)
    pool = randn(g, 3, 2, 5, 2, 8, d).cuda()
    b = torch.zeros((3, 5, 2, 2, d), dtype=torch.bfloat16, device="cuda")
    cb.cb_page_bounds(cb.page_pool(pool), b, i32([20]), i32([20]), i32([[4, 0, 2]]), 20, layer=1, layers=2)
    for l in (1, 2):
        for i, p in enumerate((4, 0, 2)):
            for h in range(2):
                assert np.array_equal(f64(b[l, p, h]), serve.page_bounds(f64(pool[l, 0, p, h, :min(8, 20 - 8 * i)])))
    assert (b[0] == 0).all() and (b[:, [1, 3]] == 0).all()


def test_bounds_of_nan_and_infinity(cb):
    pool = randn(gen(1), 1, 2, 2, 1, 4, 64).cuda()
    pool[0, 0, 0, 0, 2, 5], pool[0, 0, 0, 0, 1, 7], pool[0, 0, 0, 0, 3, 8] = float("nan"), float("inf"), -float("inf")
    b = torch.zeros((1, 2, 1, 2, 64), dtype=torch.bfloat16, device="cuda")
    cb.cb_page_bounds(cb.page_pool(pool), b, i32([4]), i32([4]), i32([[0]]), 4)
    assert b[0, 0, 0, :, 5].isnan().all() and b[0, 0, 0, 1, 7] == float("inf") and b[0, 0, 0, 0, 8] == -float("inf")
    assert b[0, 0, 0].isnan().sum() == 2


def test_bounds_of_requests_that_take_no_part(cb):
    pool = randn(gen(2), 1, 2, 3, 1, 4, 64).cuda()
    b = torch.full((1, 3, 1, 2, 64), 2.0, dtype=torch.bfloat16, device="cuda")
    cb.cb_page_bounds(cb.page_pool(pool), b, i32([0, -1, 3, 4, 1]), i32([3, 3, 2, 9, 4]), i32([[0, 1], [0, 1], [1, 0], [1, 2], [3, 0]]), 4)
    assert (b == 2.0).all()


# ------------------------------------------------------------------ selection

def choose(cb, s, b, k, first, last, q=None, table=None, kv=None, rows=None):
    n = s.n if q is None else q.shape[0]
    sel = torch.full((n, s.H, k), -7, dtype=torch.int32, device="cuda")
    width = s.table.shape[1]
    need = cb.cb_page_select_workspace_bytes(n if rows is None else rows, s.H, width)
    ws = torch.empty((need,), dtype=torch.uint8, device="cuda")
    cb.cb_page_select(s.q if q is None else q, cb.page_pool(s.pool, s.scales), s.layer, b, i32(s.starts),
                      i32([c for _, c in s.lens] if kv is None else kv), i32(s.table if table is None else table), sel,
                      first=first, last=last, workspace=ws)
    torch.cuda.synchronize()
    return sel.cpu().numpy()


def expected(serve, s, b, k, first, last, table=None):
    """As the definition says, token by token."""
    table = s.table if table is None else table
    P, ps, G = s.pool.shape[2], s.ps, s.G
    bn, qd = f64(b)[s.layer], f64(s.q)
    out = np.full((s.n, s.H, k), -7)
    for r, (nq, kv) in enumerate(s.lens):
        there = (table[r] >= 0) & (table[r] < P)
        pages = np.where(there, table[r], 0)
        for h in range(s.H):
            f = np.ones(len(pages))
            if s.scales is not None and s.scales.dim() == 4:
                f = s.scales[s.layer, :, h, 0].double().cpu().numpy()[pages]
            for t in range(nq):
                p = kv - nq + t
                row = out[s.starts[r] + t, h]
                row[:] = -1
                if p < 0:
                    continue
                m = p // ps + 1
                scores = serve.page_scores(qd[s.starts[r] + t, h * G:(h + 1) * G], bn[pages[:m], h] * f[:m, None, None])
                got = serve.page_select(scores, there[:m], first, last, k)
                row[:len(got)] = got
    return out


SELECT = [
    # kind, lens, H, G, d, page, k, first, last
    ("bf16", [(1, 1)], 1, 1, 64, 16, 3, 1, 1),
    ("bf16", [(1, 300), (1, 77), (1, 16), (1, 17)], 2, 4, 128, 16, 5, 1, 2),
    ("bf16", [(3, 200), (0, 40), (5, 5), (1, 700)], 1, 2, 96, 7, 9, 0, 1),
    ("e4m3", [(1, 900), (1, 33)], 2, 8, 64, 16, 16, 2, 2),
    ("blocks", [(1, 1000), (2, 500)], 2, 5, 128, 16, 12, 1, 2),
    ("blocks", [(40, 800), (17, 17)], 1, 3, 96, 24, 6, 0, 1),
    ("bf16", [(35, 600)], 2, 1, 64, 1, 40, 1, 3),
    ("blocks", [(1, 9000), (1, 3)], 1, 16, 64, 8, 64, 1, 1),
    ("bf16", [(16, 1200), (16, 300)], 1, 40, 128, 64, 8, 1, 1),
    ("e4m3", [(2, 20000)], 1, 2, 128, 16, 1000, 4, 30),
]


@pytest.mark.parametrize("case", range(len(SELECT)))
def test_select(cb, serve, case):
    kind, lens, H, G, d, ps, k, first, last = SELECT[case]
    s = make_step(cb, kind, lens, H, G, d, ps, pad=case % 3, seed=case)
    b = all_bounds(cb, s)
    got = choose(cb, s, b, k, first, last)
    assert np.array_equal(got, expected(serve, s, b, k, first, last))
    for rows in (1, 3):                                         # the tokens take turns
        assert np.array_equal(choose(cb, s, b, k, first, last, rows=rows), got)


def test_select_equal_scores_go_to_the_lower_page(cb, serve):
    """Pages with the same bounds, and queries of zero, whose scores are all zeros, of both signs."""
    s = make_step(cb, "bf16", [(1, 640), (3, 320)], 2, 2, 64, 16, seed=3)
    b = all_bounds(cb, s)
    for r in range(2):
        rows = torch.tensor(s.table[r][s.table[r] >= 0], device="cuda").long()
        b[s.layer, rows] = b[s.layer, rows[torch.arange(len(rows), device="cuda") % 5]]
    s.q[1] = 0
    s.q[2] = -0.0
    for k, first, last in ((7, 1, 2), (2, 0, 1), (30, 3, 1)):
        got = choose(cb, s, b, k, first, last)
        assert np.array_equal(got, expected(serve, s, b, k, first, last))


def test_select_scores_in_the_last_places(cb, serve):
    """Scores that 32-bit sums would confuse: large terms that cancel beside the small ones that decide."""
    s = make_step(cb, "bf16", [(2, 512)], 1, 4, 128, 16, seed=4)
    b = all_bounds(cb, s)
    s.q[:, :, 0], s.q[:, :, 1] = 2.0 ** 12, 2.0 ** 12
    b[s.layer, :, :, :, 0], b[s.layer, :, :, :, 1] = 2.0 ** 11, -2.0 ** 11
    got = choose(cb, s, b, 6, 1, 1)
    assert np.array_equal(got, expected(serve, s, b, 6, 1, 1))


@pytest.mark.parametrize("kind", ["bf16", "blocks"])
def test_select_among_many_nearly_alike_pages(cb, serve, kind):
    """Hundreds of pages whose scores differ in their last places or not at all: more than are looked at in one go."""
    s = make_step(cb, kind, [(2, 5000), (1, 400)], 2, 3, 64, 16, seed=40)
    b = all_bounds(cb, s)
    g = gen(41)
    one = randn(g, 2, 1, 64).abs()
    one[0] = -one[0]
    alike = (one[:, 0] * 8).to(b.dtype)                            # [least and greatest][channel]
    raw = b.view(torch.uint8 if kind == "blocks" else torch.int16)
    for r in range(2):
        rows = torch.tensor(s.table[r][s.table[r] >= 0]).long()
        for i, p in enumerate(rows.tolist()):
            if i % 5:
                x = alike.clone().view(raw.dtype)
                x[i % 2, (7 * i) % 64] += i % 3                  # a channel one or two steps away
                raw[s.layer, p] = x.cuda()
    if kind == "blocks":
        s.scales[s.layer, :, :, 0] = 0.5
    for k, first, last in ((40, 1, 2), (150, 0, 1), (299, 2, 2)):
        got = choose(cb, s, b, k, first, last)
        assert np.array_equal(got, expected(serve, s, b, k, first, last))


def test_select_in_large_tables(cb, serve):
    """More entries than a wave keeps, with tokens that have few and many candidates."""
    s = make_step(cb, "bf16", [(3, 9000), (1, 40)], 1, 2, 64, 1, seed=42)
    b = all_bounds(cb, s)
    assert s.table.shape[1] > 8192
    for k, first, last in ((20, 1, 2), (700, 0, 5)):
        got = choose(cb, s, b, k, first, last)
        assert np.array_equal(got, expected(serve, s, b, k, first, last))


def large_table(cb, kind, d, seed):
    """Requests whose rows of the table have more entries than a wave keeps: pages of one key."""
    s = make_step(cb, kind, [(3, 9000), (1, 40), (2, 8300)], 2 if d == 96 else 1, 3, d, 1, seed=seed)
    assert s.table.shape[1] > 8192
    return s, all_bounds(cb, s)


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "blocks"])
def test_select_in_large_tables_of_every_kind(cb, serve, kind, d):
    """All tokens at once and in turns; equal scores, pages that are hidden, and NaN among bounds and queries."""
    s, b = large_table(cb, kind, d, seed=d)
    for k, first, last in ((33, 1, 2), (1500, 0, 1)):
        got = choose(cb, s, b, k, first, last)
        assert np.array_equal(got, expected(serve, s, b, k, first, last))
        for rows in (1, 4):
            assert np.array_equal(choose(cb, s, b, k, first, last, rows=rows), got)
    # a seventh of the pages differ, in bounds and scales
    for r in range(3):
        rows = torch.tensor(s.table[r][s.table[r] >= 0], device="cuda").long()
        alike = rows[torch.arange(len(rows), device="cuda") % -(-len(rows) // 7)]
        raw = b.view(torch.int16 if kind == "bf16" else torch.uint8)
        raw[s.layer, rows] = raw[s.layer, alike]
        if kind == "blocks":
            s.scales[s.layer, rows] = s.scales[s.layer, alike]
    s.q[1], s.q[4] = 0, -0.0
    table = s.table.copy()
    table[0, [0, 5, 4000, 8999]] = -1, s.pool.shape[2], 2 ** 31 - 1, -7
    table[2, 100:8290] = -1
    got = choose(cb, s, b, 40, 2, 3, table=table)
    assert np.array_equal(got, expected(serve, s, b, 40, 2, 3, table=table))
    raw = b.view(torch.uint8)
    nan = [0xc0, 0x7f] if kind == "bf16" else [0x7f]
    for i in (7, 3000, 8700):
        page, c = int(s.table[0, i]), 9 * len(nan)
        raw[s.layer, page, 0, 1, c:c + len(nan)] = torch.tensor(nan, dtype=torch.uint8, device="cuda")
    s.q[5, 0, 3] = float("nan")                                  # every page of request 2
    got = choose(cb, s, b, 40, 0, 1)
    assert np.array_equal(got, expected(serve, s, b, 40, 0, 1))
    assert {7, 3000, 8700} <= set(got[0, 0]) and got[5, 0].tolist() == list(range(39)) + [8299]


@pytest.mark.parametrize("kind,large", [("blocks", False), ("bf16", False), ("e4m3", True)])
def test_strided_queries_and_tables(cb, serve, kind, large):
    """Queries head by head in memory and among others, a table that is part of a wider one, another stream: the same
    bounds, choices and answers."""
    lens = [(3, 9000), (1, 40)] if large else [(3, 900), (17, 400), (1, 33)]
    s = make_step(cb, kind, lens, 2, 3, 64, 1 if large else 16, pad=2, seed=44)
    b = all_bounds(cb, s)
    want = choose(cb, s, b, 9, 1, 2)
    attend(cb, s, want)
    table = torch.full((len(lens), s.table.shape[1] + 5), 2 ** 30, dtype=torch.int32, device="cuda")
    table[:, 2:-3] = i32(s.table)
    table = table[:, 2:-3]
    starts, kv = i32(s.starts), i32([k for _, k in s.lens])
    pages, side = cb.page_pool(s.pool, s.scales), torch.cuda.Stream()
    by_head = s.q.transpose(0, 1).contiguous().transpose(0, 1)
    among = torch.full((s.n, 10, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    among[:, 3:9] = s.q
    torch.cuda.synchronize()
    for q in (by_head, among[:, 3:9]):
        with torch.cuda.stream(side):
            bounds = empty_bounds(s)
            cb.cb_page_bounds(pages, bounds, kv, kv, table, max(k for _, k in lens), layer=s.layer)
            sel = torch.full((s.n, 2, 9), -7, dtype=torch.int32, device="cuda")
            ws = torch.empty(cb.cb_page_select_workspace_bytes(s.n, 2, table.shape[1]), dtype=torch.uint8, device="cuda")
            cb.cb_page_select(q, pages, s.layer, bounds, starts, kv, table, sel, first=1, last=2, workspace=ws)
            out = torch.full((6, s.n, 64), 9.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
            lse = torch.full((s.n, 6), 9.0, dtype=torch.float32, device="cuda")
            cb.cb_attn_selected(q, pages, s.layer, starts, kv, table, sel, out, lse=lse)
        side.synchronize()
        raw = torch.int16 if kind == "bf16" else torch.uint8
        assert torch.equal(bounds.view(raw), b.view(raw))
        assert np.array_equal(sel.cpu().numpy(), want) and torch.equal(out, s.out) and torch.equal(lse, s.lse)


@pytest.mark.parametrize("large", [False, True])
def test_select_pages_with_infinities(cb, serve, large):
    """A page whose bounds hold an infinity or a NaN counts as +infinity, whatever the queries' signs."""
    if large:
        s, b = large_table(cb, "bf16", 64, seed=6)
    else:
        s = make_step(cb, "bf16", [(3, 900), (1, 40), (2, 830)], 1, 3, 64, 8, seed=6)
        b = all_bounds(cb, s)
    own = (s.lens[0][1] - 1) // s.ps                             # of token 2; behind the others of its request where pages are small
    for i, z, v in ((11, 0, -float("inf")), (12, 1, float("inf")), (own, 1, float("inf")), (40, 0, float("nan"))):
        b[s.layer, int(s.table[0, i]), 0, z, 9] = v
    for sign in (1.0, -1.0):
        s.q.copy_(s.q.abs() * sign)
        got = choose(cb, s, b, 20, 0, 1)
        assert np.array_equal(got, expected(serve, s, b, 20, 0, 1))
        assert all({11, 12, 40} <= set(got[t, 0]) for t in range(3))


def test_select_scores_of_extreme_size(cb, serve):
    """Queries and bounds near the ends of bf16's range: estimates that leave fp32's say nothing, and the scores decide."""
    for qs, bs in ((2.0 ** 60, 2.0 ** 60), (2.0 ** 100, 2.0 ** 20), (2.0 ** -70, 2.0 ** -50), (2.0 ** -120, 2.0 ** 100), (2.0 ** 126, 1.0)):
        s = make_step(cb, "bf16", [(1, 600), (2, 300)], 1, 2, 64, 16, seed=43)
        s.q *= qs
        b = all_bounds(cb, s)
        b *= bs
        got = choose(cb, s, b, 6, 1, 1)
        assert np.array_equal(got, expected(serve, s, b, 6, 1, 1)), (qs, bs)


@pytest.mark.parametrize("small", ["bounds", "queries", "both parts"])
def test_select_by_denormal_numbers(cb, serve, small):
    """Channels whose bounds, or queries, are denormal bf16 numbers decide, beside larger ones of ordinary channels that do
    not; queries whose lower part, behind the first bf16 number of their sum, is denormal."""
    s = make_step(cb, "bf16", [(2, 1500), (1, 700)], 1, 2, 64, 16, seed=45)
    b = all_bounds(cb, s)
    g = gen(46)
    if small == "both parts":
        s.q *= 2.0 ** -122                                        # sums of two heads have more bits than one number
        b *= 2.0 ** 60
    else:
        s.q *= 2.0 ** -35
        b *= 2.0 ** -60                                           # terms of about 2^-95
        k = torch.randint(1, 128, (*b.shape[:3], 1), generator=g).cuda().float()
        if small == "bounds":                                      # k 2^-133 by 2^40
            s.q[..., 0] = 2.0 ** 40
            b[..., 0] = (k * 2.0 ** -133).to(torch.bfloat16)
        else:                                                      # 3 2^-132 by k 2^39
            s.q[..., 0] = 3 * 2.0 ** -132
            b[..., 0] = (k * 2.0 ** 39).to(torch.bfloat16)
        assert (s.q[..., 0] > 0).all() and (b[..., 0] > 0).all() and b.isfinite().all()
    for n, first, last in ((5, 1, 1), (20, 0, 2)):
        got = choose(cb, s, b, n, first, last)
        assert np.array_equal(got, expected(serve, s, b, n, first, last))


def test_select_nan_and_infinity_come_first(cb, serve):
    s = make_step(cb, "bf16", [(1, 400), (1, 350)], 1, 2, 64, 16, seed=5)
    b = all_bounds(cb, s)
    for i, v in ((7, float("nan")), (3, float("inf")), (11, -float("inf"))):
        b[s.layer, int(s.table[0, i]), 0, 1, 9] = v
    s.q[1, 0, 3] = float("nan")                                  # every page of request 1
    got = choose(cb, s, b, 5, 0, 1)
    assert np.array_equal(got, expected(serve, s, b, 5, 0, 1))
    assert {3, 7} <= set(got[0, 0]) and got[1, 0].tolist() == [0, 1, 2, 3, 21]


def test_select_hidden_pages(cb, serve):
    """Pages outside the pool are no candidates, nor among the first and last; the others take their places."""
    s = make_step(cb, "blocks", [(1, 300), (9, 200), (1, 50)], 2, 3, 64, 16, seed=6)
    b = all_bounds(cb, s)
    table = s.table.copy()
    table[0, [0, 4, 17, 18]] = -1, s.pool.shape[2], 2 ** 31 - 1, -5
    table[1, :11] = -1
    table[2, :] = -1
    got = choose(cb, s, b, 4, 2, 2, table=table)
    assert np.array_equal(got, expected(serve, s, b, 4, 2, 2, table=table))
    assert (got[10] == -1).all()


def test_select_more_new_tokens_than_keys(cb, serve):
    s = make_step(cb, "bf16", [(5, 5), (3, 40)], 1, 2, 64, 16, seed=7)
    b = all_bounds(cb, s)
    got = choose(cb, s, b, 3, 1, 1, kv=[2, 0])
    assert (got[:3] == -1).all() and got[3:5].tolist() == [[[0, -1, -1]]] * 2 and (got[5:] == -1).all()


def test_select_many_requests(cb, serve):
    rng = np.random.default_rng(3)
    lens = [(int(q), int(q + k)) for q, k in zip(rng.choice([0, 1, 1, 2, 20], 300), rng.integers(0, 200, 300))]
    lens = [(q, max(1, k)) for q, k in lens]
    s = make_step(cb, "bf16", lens, 1, 1, 64, 16, pad=4, seed=8)
    b = all_bounds(cb, s)
    got = choose(cb, s, b, 4, 1, 1)
    assert np.array_equal(got, expected(serve, s, b, 4, 1, 1))


# ------------------------------------------------------------------ attention over the selected pages

def attend(cb, s, sel, ws=True, table=None, scale=None, lse=True, q=None):
    s.out = torch.full((s.n, s.H * s.G, s.d), 9.0, dtype=torch.bfloat16, device="cuda")
    s.lse = torch.full((s.n, s.H * s.G), 9.0, dtype=torch.float32, device="cuda") if lse else None
    need = cb.cb_attn_selected_workspace_bytes(s.n, s.H * s.G, s.H, s.d, s.ps, sel.shape[2])
    w = torch.empty((need if ws is True else int(ws),), dtype=torch.uint8, device="cuda") if ws else None
    cb.cb_attn_selected(s.q if q is None else q, cb.page_pool(s.pool, s.scales), s.layer, i32(s.starts),
                        i32([k for _, k in s.lens]), i32(s.table if table is None else table), i32(sel), s.out, scale=scale,
                        lse=s.lse, workspace=w)
    torch.cuda.synchronize()
    return s.out, s.lse


def check_attend(serve, s, sel, table=None, scale=None, rows=None):
    sc = s.d ** -0.5 if scale is None else scale
    table = s.table if table is None else table
    got, gl, qd = f64(s.out), f64(s.lse), f64(s.q)
    H, G, d, ps, P = s.H, s.G, s.d, s.ps, s.pool.shape[2]
    for r, (nq, kv) in enumerate(s.lens):
        there = (table[r] >= 0) & (table[r] < P)
        for t in range(nq) if rows is None else [t for t in range(nq) if s.starts[r] + t in rows]:
            p = kv - nq + t
            for h in range(H):
                pages = {int(i) for i in sel[s.starts[r] + t, h] if 0 <= i < len(there) and there[i]}
                at, hs = s.starts[r] + t, slice(h * G, (h + 1) * G)
                keys = np.array([j for j in range(max(p, -1) + 1) if j // ps in pages], dtype=int)
                n = len(keys)
                o, l, mag, smag = serve.attention(qd[at:at + 1, hs], s.K[r][h][keys], s.V[r][h][keys], n, sc)
                es, few = (d + 8) * 2 * F32 * smag, (n + 64) * 2 * F32
                tol = BF * np.abs(o) * 1.01 + mag * (BF * 1.01 + (2 * es + few)[..., None])
                assert (np.abs(got[at:at + 1, hs] - o) <= tol).all(), (r, t, h)
                assert np.array_equal(np.isneginf(gl[at:at + 1, hs]), np.isneginf(l)), (r, t, h)
                if n:
                    assert (np.abs(gl[at:at + 1, hs] - l) <= es + few + 8 * F32 * (np.abs(l) + 1)).all(), (r, t, h)
    if rows is None:
        assert (got[s.starts[-1]:] == 9.0).all() and (gl[s.starts[-1]:] == 9.0).all()


def random_lists(s, k, seed, spoil=True):
    """Lists of different pages in any order, up to k of them, and entries that are none among and behind them."""
    rng = np.random.default_rng(seed)
    sel = np.full((s.n, s.H, k), -1)
    for r, (nq, kv) in enumerate(s.lens):
        for t in range(nq):
            own = max(kv - nq + t, 0) // s.ps
            for h in range(s.H):
                m = int(rng.integers(1, k + 1))
                pages = rng.permutation(own + 1)[:m]
                row = np.concatenate([pages, np.full(m - len(pages), -1)])
                if spoil:
                    rng.shuffle(row)
                    row[rng.random(m) < 0.1] = rng.choice([-1, -2 ** 31, s.table.shape[1], 2 ** 31 - 1])
                sel[s.starts[r] + t, h, :m] = row
    return sel


ATTEND = [
    # kind, lens, H, G, d, page, k
    ("bf16", [(1, 1)], 1, 1, 64, 16, 1),
    ("bf16", [(1, 300), (1, 77), (1, 16)], 2, 4, 128, 16, 5),
    ("bf16", [(3, 200), (0, 40), (5, 5)], 1, 2, 96, 7, 9),
    ("e4m3", [(1, 900), (2, 33)], 2, 8, 64, 16, 16),
    ("e4m3", [(4, 500)], 1, 16, 96, 32, 7),
    ("blocks", [(1, 1000), (2, 500)], 2, 5, 128, 16, 12),
    ("blocks", [(20, 800), (17, 17)], 1, 3, 96, 24, 6),
    ("bf16", [(10, 600)], 2, 1, 64, 1, 40),
    ("blocks", [(1, 2000)], 1, 33, 64, 100, 9),
    ("e4m3", [(2, 700)], 1, 40, 128, 64, 8),
]


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_selected_attention(cb, serve, case, ws):
    kind, lens, H, G, d, ps, k = ATTEND[case]
    s = make_step(cb, kind, lens, H, G, d, ps, pad=case % 3, seed=case)
    sel = random_lists(s, k, case)
    attend(cb, s, sel, ws=ws)
    check_attend(serve, s, sel)
    s.q = s.q * 3
    attend(cb, s, sel, ws=ws, scale=-0.1)
    check_attend(serve, s, sel, scale=-0.1)


@pytest.mark.parametrize("kind,d,ps,k", [("bf16", 128, 64, 100), ("blocks", 64, 16, 300), ("e4m3", 96, 128, 40), ("blocks", 128, 1000, 5)])
def test_selected_attention_in_parts(cb, serve, kind, d, ps, k):
    """Long lists of few tokens, divided among workgroups as the workspace allows; the same bits from call to call."""
    s = make_step(cb, kind, [(1, 9000), (2, 4001)], 2, 3, d, ps, pad=2, seed=k)
    sel = random_lists(s, k, k, spoil=False)
    assert cb.cb_attn_selected_workspace_bytes(s.n, 6, 2, d, ps, k) > 0
    attend(cb, s, sel)
    check_attend(serve, s, sel)
    a, al = s.out.clone(), s.lse.clone()
    attend(cb, s, sel)
    assert torch.equal(a, s.out) and torch.equal(al, s.lse)
    for ws in (16, 300000, 1000000):
        attend(cb, s, sel, ws=ws)
        check_attend(serve, s, sel)


def test_all_pages_selected_is_attention(cb, serve):
    """Every page in its order: attention over all visible keys."""
    for kind in ("bf16", "blocks"):
        s = make_step(cb, kind, [(1, 500), (3, 90), (12, 300)], 2, 4, 128, 16, seed=11)
        sel = np.broadcast_to(np.arange(s.table.shape[1]), (s.n, s.H, s.table.shape[1])).copy()
        attend(cb, s, sel)
        s.check(serve)


def test_selected_attention_sees_nothing(cb, serve):
    """Empty lists, lists of pages behind the token or outside the pool: zeros and -infinity."""
    s = make_step(cb, "bf16", [(1, 100), (2, 64), (1, 300)], 1, 2, 64, 16, seed=12)
    sel = np.full((s.n, 1, 5), -1)
    sel[1], sel[3] = 5, [3, 4, 3, 4, 3]
    table = s.table.copy()
    table[2, 3:5] = -1, s.pool.shape[2]
    for ws in (True, False):
        attend(cb, s, sel, table=table, ws=ws)
        assert (s.out == 0).all() and torch.isneginf(s.lse).all()


def test_selected_attention_counts_a_page_twice(cb, serve):
    s = make_step(cb, "bf16", [(1, 64)], 1, 2, 64, 16, seed=13)
    attend(cb, s, np.array([[[1, 3]]]))
    a, al = s.out.clone(), s.lse.clone()
    attend(cb, s, np.array([[[1, 3, 1, 3]]]))
    assert (f64(s.out) - f64(a) <= 2 * BF * np.abs(f64(a)) + 1e-3).all()
    assert np.allclose(f64(s.lse), f64(al) + np.log(2.0), atol=1e-5, rtol=0)


DIVIDED = [
    # kind, H, G, d, page, k: lists of about 10,000 keys, each row tile's in more than 16 parts
    ("bf16", 2, 3, 128, 64, 160),
    ("blocks", 2, 33, 64, 16, 640),
    ("e4m3", 1, 17, 96, 24, 430),
    ("blocks", 1, 40, 128, 32, 320),
]


def check_listed(serve, s, sel, table=None):
    """As check_attend, with pages that are listed more than once counted as often."""
    table = s.table if table is None else table
    got, gl, qd = f64(s.out), f64(s.lse), f64(s.q)
    for r, (nq, kv) in enumerate(s.lens):
        there = (table[r] >= 0) & (table[r] < s.pool.shape[2])
        for t in range(nq):
            p, at = kv - nq + t, s.starts[r] + t
            for h in range(s.H):
                pages = [int(i) for i in sel[at, h] if 0 <= i < len(there) and there[i]]
                keys = np.array([j for i in pages for j in range(i * s.ps, min((i + 1) * s.ps, p + 1))], dtype=int)
                hs, n = slice(h * s.G, (h + 1) * s.G), len(keys)
                o, l, mag, smag = serve.attention(qd[at:at + 1, hs], s.K[r][h][keys], s.V[r][h][keys], n, s.d ** -0.5)
                es, few = (s.d + 8) * 2 * F32 * smag, (n + 64) * 2 * F32
                tol = BF * np.abs(o) * 1.01 + mag * (BF * 1.01 + (2 * es + few)[..., None])
                assert (np.abs(got[at:at + 1, hs] - o) <= tol).all(), (r, t, h)
                assert np.array_equal(np.isneginf(gl[at:at + 1, hs]), np.isneginf(l)), (r, t, h)
                if n:
                    assert (np.abs(gl[at:at + 1, hs] - l) <= es + few + 8 * F32 * (np.abs(l) + 1)).all(), (r, t, h)


@pytest.mark.parametrize("case", range(len(DIVIDED)))
def test_selected_attention_in_many_parts(cb, serve, case):
    """Rows that a workgroup joins, beside rows whose lists are short, empty, of hidden pages or of later ones, so that some
    or all of their parts are."""
    kind, H, G, d, ps, k = DIVIDED[case]
    s = make_step(cb, kind, [(2, k * ps + 40), (1, 6 * ps + 1), (1, 3000), (1, 2 * ps), (2, 900)], H, G, d, ps, pad=1, seed=50 + case)
    # a part is a row of 16 query heads and its maximum and sum, in fp32
    row_tiles = s.n * -(-G // 16) * H
    need = cb.cb_attn_selected_workspace_bytes(s.n, H * G, H, d, ps, k)
    assert need > 16 * row_tiles * 16 * (d + 2) * 4
    sel, rng = random_lists(s, k, case), np.random.default_rng(case)
    sel[0] = rng.permutation(k)                                 # whole lists, beside a short one
    sel[1, :, 2:] = -1
    sel[3, 0] = -1
    sel[4] = 2 + np.arange(k) % 60                              # behind the token: pages of 2 ps keys are 0 and 1
    table = s.table.copy()
    table[3, 2:62] = table[0, :60]
    table[4, 1:4] = -1, s.pool.shape[2], 2 ** 31 - 1
    sel[5] = 1 + np.arange(k) % 3
    sel[5, :, k // 2:] = -1
    attend(cb, s, sel, table=table)
    check_listed(serve, s, sel, table=table)
    assert (s.out[4:6] == 0).all() and torch.isneginf(s.lse[4:6]).all()
    assert (s.out[s.starts[-1]:] == 9).all() and (s.lse[s.starts[-1]:] == 9).all()
    a, al = s.out.clone(), s.lse.clone()
    attend(cb, s, sel, table=table)
    assert torch.equal(a, s.out) and torch.equal(al, s.lse)
    # fewer parts: joined by waves, and just two
    for parts in (16, 2):
        attend(cb, s, sel, table=table, ws=parts * row_tiles * 16 * (d + 2) * 4)
        check_listed(serve, s, sel, table=table)


@pytest.mark.parametrize("kind,ps,pages", [("bf16", 16, 2), ("blocks", 32, 2), ("e4m3", 7, 3), ("bf16", 64, 30), ("blocks", 16, 100),
                                           ("e4m3", 24, 60)])
def test_selected_attention_counts_listed_pages(cb, serve, kind, ps, pages):
    """Lists in which every page stands twice, and some a third time, of rows that are not divided and that are."""
    s = make_step(cb, kind, [(1, pages * ps + 5), (1, 2 * pages * ps)], 2, 3, 64, ps, seed=60 + ps)
    rng = np.random.default_rng(ps)
    once = np.stack([[rng.permutation(pages) for _ in range(2)] for _ in range(2)])
    sel = np.concatenate([once, once[:, :, ::-1], once[:, :, :pages // 2]], 2)
    need = cb.cb_attn_selected_workspace_bytes(2, 6, 2, 64, ps, sel.shape[2])
    assert (need > 0) == (pages > 3)
    attend(cb, s, sel)
    check_listed(serve, s, sel)
    attend(cb, s, np.concatenate([once, once], 2))
    check_listed(serve, s, np.concatenate([once, once], 2))
    attend(cb, s, once)
    check_listed(serve, s, once)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_selected_attention_keeps_bad_values_from_rows_that_do_not_see_them(cb, serve, bad):
    """In a page that only some tokens list, and behind the position of the others; in keys and in values."""
    for z in range(2):
        s = make_step(cb, "bf16", [(6, 90)], 1, 2, 64, 16, seed=14)
        sel = np.tile(np.array([0, 2, 5]), (6, 1, 1))
        sel[:3, 0, 1] = 3                                        # tokens 0 .. 2 do not list page 2
        s.pool[s.layer, z, int(s.table[0, 2]), 0, 4, 3] = bad
        s.pool[s.layer, z, int(s.table[0, 5]), 0, 9, 5] = bad      # key 89: token 5's alone
        attend(cb, s, sel)
        check_attend(serve, s, sel, rows=[0, 1, 2])
        got = f64(s.out)
        if z == 1:
            assert not np.isfinite(got[3:, :, 3]).any() and np.isfinite(got[3:5, :, 5]).all() and not np.isfinite(got[5, :, 5]).any()
        elif np.isnan(bad):
            assert np.isnan(got[3:]).all()


SHARED = [
    # kind, lens, H, G, d, page, k: calls of enough tokens that several of a request share a row tile
    ("bf16", [(280, 700), (1, 300), (33, 33)], 8, 8, 128, 64, 5),
    ("blocks", [(300, 900), (1, 64), (0, 50), (77, 77), (129, 700)], 8, 2, 64, 32, 6),
    ("e4m3", [(40, 10), (399, 800)], 8, 5, 96, 32, 4),
    ("blocks", [(1100, 3300)], 16, 1, 128, 32, 70),
    ("bf16", [(517, 1000), (2, 1500)], 16, 3, 64, 96, 9),
    ("blocks", [(3, 70)] * 200, 8, 8, 64, 32, 2),
]


@pytest.mark.parametrize("case", range(len(SHARED)))
def test_selected_attention_of_many_tokens(cb, serve, case):
    kind, lens, H, G, d, ps, k = SHARED[case]
    s = make_step(cb, kind, lens, H, G, d, ps, pad=3, seed=20 + case)
    sel = random_lists(s, k, case)
    attend(cb, s, sel)
    first = s.out.clone()
    total, rng = int(s.starts[-1]), np.random.default_rng(case)
    rows = set(rng.choice(total, 24, replace=False)) | {0, 1, 2, total - 2, total - 1} | {int(a) for a in s.starts[1:4] if a < total}
    check_attend(serve, s, sel, rows=rows)
    assert (s.out[total:] == 9).all() and (s.lse[total:] == 9).all() and not (s.out[:total] == 9).all(-1).any()
    attend(cb, s, sel)
    assert torch.equal(s.out, first)


@pytest.mark.parametrize("G,k", [(8, 9), (1, 7)])
def test_selected_attention_of_many_tokens_counts_a_page_twice(cb, serve, G, k):
    """Lists in which pages stand up to three times, in any order."""
    s = make_step(cb, "bf16", [(700, 1000), (324, 500)], 8, G, 64, 32, seed=30)
    rng = np.random.default_rng(5)
    sel = rng.integers(0, 10, (s.n, s.H, k))
    attend(cb, s, sel)
    got, gl, qd = f64(s.out), f64(s.lse), f64(s.q)
    for t in list(rng.choice(s.n, 20, replace=False)) + [0, 699, 700, 1023]:
        r = 0 if t < 700 else 1
        nq, kv = s.lens[r]
        p = kv - nq + t - s.starts[r]
        for h in range(s.H):
            keys = np.array([32 * i + j for i in sel[t, h] for j in range(32) if 32 * i + j <= p], dtype=int)
            hs, n = slice(h * G, (h + 1) * G), len(keys)
            o, l, mag, smag = serve.attention(qd[t:t + 1, hs], s.K[r][h][keys], s.V[r][h][keys], n, s.d ** -0.5)
            es, few = (s.d + 8) * 2 * F32 * smag, (n + 64) * 2 * F32
            tol = BF * np.abs(o) * 1.01 + mag * (BF * 1.01 + (2 * es + few)[..., None])
            assert (np.abs(got[t:t + 1, hs] - o) <= tol).all() and (np.abs(gl[t:t + 1, hs] - l) <= es + few + 8 * F32 * (np.abs(l) + 1)).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "blocks"])
@pytest.mark.parametrize("z", [0, 1])
def test_bad_values_of_shared_tiles_reach_only_rows_that_see_them(cb, serve, kind, z):
    """NaN (bf16 V: infinity too) in a page that the odd tokens alone list, and behind the position of earlier tokens."""
    s = make_step(cb, kind, [(600, 700)], 8, 2, 64, 32, seed=31)
    sel = np.tile(np.array([0, 2, 21]), (s.n, s.H, 1))
    sel[::2, :, 1] = 3                                           # even tokens do not list page 2
    bad = float("nan")
    # pages 2 and 21 (keys 672 .. 699): places 4 and 9, key 681 is token 581's own
    s.pool[s.layer, z, int(s.table[0, 2]), :, 4, 3] = torch.tensor(bad, device="cuda").to(s.pool.dtype)
    s.pool[s.layer, z, int(s.table[0, 21]), :, 9, 5] = torch.tensor(float("inf") if kind == "bf16" and z else bad, device="cuda").to(s.pool.dtype)
    attend(cb, s, sel)
    check_attend(serve, s, sel, rows=[0, 2, 300, 302, 578, 580])
    got = f64(s.out)
    late = np.arange(s.n) >= 581
    odd = np.arange(s.n) % 2 == 1
    if z == 1:
        assert np.array_equal((~np.isfinite(got[:, :, 3])).any(1), odd) and np.array_equal((~np.isfinite(got[:, :, 3])).all(1), odd)
        assert np.array_equal((~np.isfinite(got[:, :, 5])).all(1), late) and np.array_equal((~np.isfinite(got[:, :, 5])).any(1), late)
        assert np.isfinite(np.delete(got, [3, 5], 2)).all()
    else:
        assert np.array_equal(np.isnan(got).all((1, 2)), odd | late) and np.array_equal(np.isnan(got).any((1, 2)), odd | late)


def test_selected_attention_strided_queries(cb, serve):
    s = make_step(cb, "blocks", [(2, 40), (1, 90)], 2, 2, 64, 16, seed=15)
    sel = random_lists(s, 3, 1)
    wide = torch.zeros((s.n, 8, 64), dtype=torch.bfloat16, device="cuda")
    wide[:, :4] = s.q
    attend(cb, s, sel)
    a = s.out.clone()
    attend(cb, s, sel, q=wide[:, :4])
    assert torch.equal(a, s.out)


# ------------------------------------------------------------------ together

class Server:
    """Steps of a receiver on 8-bit pages: tables, quantised writes with turned queries, bounds, choice, attention."""

    def __init__(self, cb, L, H, G, d, ps, P, R, n, width, k, n_pos=256):
        z = lambda *shape, t=torch.int32: torch.zeros(shape, dtype=t, device="cuda")  # noqa: E731
        self.cb, self.L, self.H, self.G, self.d, self.ps, self.n, self.k = cb, L, H, G, d, ps, n, k
        self.pool = torch.full((L, 2, P, H, ps, d), 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        self.scales = torch.full((L, P, H, 2), 2.0 ** 100, dtype=torch.float32, device="cuda")
        self.pages = cb.page_pool(self.pool, self.scales)
        self.bounds = torch.zeros((L, P, H, 2, d), device="cuda").to(torch.float8_e4m3fn)
        self.free, self.used = i32(np.random.default_rng(0).permutation(P)), z(1)
        self.table = i32(np.full((R, width), -1))
        self.ctx, self.new, self.starts, self.kv, self.info = z(R), z(R), z(R + 1), z(R), z(R)
        self.slots, self.pos = z(n), z(n)
        self.rope_table = torch.empty((n_pos, d // 2, 2), dtype=torch.float32, device="cuda")
        cb.cb_rope_table(THETA, d, n_pos, self.rope_table)
        self.rope = cb.rope_axes_spec(self.rope_table, self.pos)
        bf = torch.bfloat16
        self.rows, self.q = z(L, 2, 1, H, n, d, t=bf), z(L, n, H * G, d, t=bf)
        self.turned, self.out = z(L, n, H * G, d, t=bf), z(L, n, H * G, d, t=bf)
        self.selected = z(L, n, H, k)
        self.ws = z(cb.cb_page_select_workspace_bytes(n, H, width), t=torch.uint8)
        self.ws2 = z(cb.cb_attn_selected_workspace_bytes(n, H * G, H, d, ps, k), t=torch.uint8)

    def step(self, max_q):
        """One step of all layers; lengths are on the device."""
        cb, lens = self.cb, (self.starts[:-1], self.new, self.kv, self.table)
        cb.cb_page_tables(self.ctx, self.new, self.free, self.ps, self.table, self.starts, self.kv, self.slots, self.pos,
                          self.info, self.used)
        for l in range(self.L):
            cb.cb_page_quantize(self.rows[l:l + 1], self.pages, *lens, layer=l, rope=self.rope, q=self.q[l], q_out=self.turned[l])
            cb.cb_page_bounds(self.pages, self.bounds, *lens[1:], max_q, layer=l)
            cb.cb_page_select(self.turned[l], self.pages, l, self.bounds, self.starts, self.kv, self.table, self.selected[l],
                              first=1, last=1, workspace=self.ws)
            cb.cb_attn_selected(self.turned[l], self.pages, l, self.starts, self.kv, self.table, self.selected[l], self.out[l],
                                workspace=self.ws2)

    def advance(self):
        self.ctx.copy_(self.kv)
        self.free = self.free[int(self.used):].contiguous()


def test_steps_on_quantised_pages(cb, serve):
    """Three steps: what each layer holds, chooses and answers, against the definitions on what is stored; and the
    stored rows read back, turned back, near the rows that came."""
    L, H, G, d, ps, R, n, k = 2, 2, 4, 64, 8, 3, 40, 4
    s = Server(cb, L, H, G, d, ps, 40, R, n, 12, k)
    g = gen(21)
    came = [[[[] for _ in range(2)] for _ in range(L)] for _ in range(R)]
    for new in ([30, 9, 0], [1, 2, 17], [1, 0, 1]):
        s.new.copy_(i32(new))
        s.rows.copy_((randn(g, L, 2, 1, H, n, d) * 2.0).cuda())
        s.q.copy_((randn(g, L, n, H * G, d) * 2.0).cuda())
        s.step(max(new))
        torch.cuda.synchronize()
        starts, kv, table = s.starts.cpu().numpy(), s.kv.cpu().numpy(), s.table.cpu().numpy()
        assert s.info.tolist() == [0, 0, 0]
        codes, sc, bn = f64(s.pool), s.scales.double().cpu().numpy(), f64(s.bounds)
        for r in range(R):
            tok = slice(starts[r], starts[r] + new[r])
            for l in range(L):
                for z in range(2):
                    came[r][l][z].append(f64(s.rows[l, z, 0])[:, tok])
                if new[r] == 0:
                    continue
                pages = table[r, :-(-int(kv[r]) // ps)]
                K, V = (np.concatenate([codes[l, z, p] * sc[l, p, :, z][:, None, None] for p in pages], 1)[:, :kv[r]] for z in range(2))
                for t in range(new[r]):
                    p, at = int(kv[r]) - new[r] + t, starts[r] + t
                    for h in range(H):
                        hs = slice(h * G, (h + 1) * G)
                        q = f64(s.turned[l, at, hs])
                        m = p // ps + 1
                        scores = serve.page_scores(q, bn[l, pages[:m], h] * sc[l, pages[:m], h, 0][:, None, None])
                        want = serve.page_select(scores, [True] * m, 1, 1, k)
                        got = s.selected[l, at, h].tolist()
                        assert got == want + [-1] * (k - len(want))
                        keys = np.array([j for j in range(p + 1) if j // ps in want])
                        o, _, mag, smag = serve.attention(q[None], K[h][keys], V[h][keys], len(keys), d ** -0.5)
                        es, few = (d + 8) * 2 * F32 * smag, (len(keys) + 64) * 2 * F32
                        tol = BF * np.abs(o) * 1.01 + mag * (BF * 1.01 + (2 * es + few)[..., None])
                        assert (np.abs(f64(s.out[l, at, hs])[None] - o) <= tol).all()
        s.advance()
    back = torch.zeros((L, 2, R, H, 40, d), dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(40, dtype=torch.int32, device="cuda").repeat(R)
    cb.cb_page_read(s.pages, back, i32([0, 40, 80]), s.kv, s.kv, s.table, rope=cb.rope_axes_spec(s.rope_table, pos), inverse=True)
    for r in range(R):
        for l in range(L):
            x = np.concatenate(came[r][l][1], 1)
            y = f64(back[l, 1, r])[:, :x.shape[1]]
            assert (np.abs(x - y) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * np.abs(x).max() / 224).all()
            x = np.concatenate(came[r][l][0], 1)
            y = f64(back[l, 0, r])[:, :x.shape[1]]
            # keys: the rounding of both channels of a turned pair, turned back, and to bf16; a code that went over to
            # a larger scale was rounded twice
            pair = np.hypot(x[..., :d // 2], x[..., d // 2:])
            tol = np.concatenate([pair, pair], -1) * (2 * np.sqrt(2) * 2.0 ** -4 + 2 * BF) + 2.0 ** -8 * np.abs(x).max() / 158
            assert (np.abs(x - y) <= tol).all()


def test_steps_in_a_graph_with_other_lengths(cb):
    """A captured step replayed with other lengths and rows, and with eager work of the caller between: the eager step's
    bits every time."""
    make = lambda: Server(cb, 2, 2, 4, 64, 8, 60, 3, 24, 16, 5)  # noqa: E731
    eager, graph = make(), make()
    steps = [[20, 3, 1], [1, 1, 1], [5, 0, 9], [1, 1, 0], [2, 12, 1], [1, 1, 1]]
    side = torch.cuda.Stream()
    captured = None
    for i, new in enumerate(steps):
        for s in (eager, graph):
            g = gen(40 + i)
            s.new.copy_(i32(new))
            s.rows.copy_(randn(g, 2, 2, 1, 2, 24, 64).cuda())
            s.q.copy_(randn(g, 2, 24, 8, 64).cuda())
        # (the graph's free list keeps its place: the pages left are moved to its beginning)
        if i:
            rest = graph.free[int(graph.used):].clone()
            graph.free[:len(rest)] = rest
        eager.step(24)
        torch.cuda.synchronize()
        if captured is None:
            side.wait_stream(torch.cuda.current_stream())
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured, stream=side):
                graph.step(24)
        captured.replay()
        torch.cuda.synchronize()
        n = int(eager.starts[-1])
        for name in ("table", "starts", "kv", "scales", "bounds", "pool"):
            a, b = getattr(eager, name), getattr(graph, name)
            assert torch.equal(a.view(torch.uint8) if a.dtype == torch.float8_e4m3fn else a,
                               b.view(torch.uint8) if b.dtype == torch.float8_e4m3fn else b), (i, name)
        for name in ("selected", "out", "turned"):
            assert torch.equal(getattr(eager, name)[:, :n], getattr(graph, name)[:, :n]), (i, name)
        eager.advance()
        graph.ctx.copy_(graph.kv)
        torch.randn(1000, device="cuda").sort()


def test_choice_and_shared_tiles_in_a_graph(cb):
    """A captured choice and attention of many tokens, replayed with other lengths: the eager calls' bits every time, rows of
    no request as they were."""
    s = make_step(cb, "blocks", [(280, 700), (1, 300), (33, 33)], 8, 2, 64, 32, pad=3, seed=32)
    b, pages, k = all_bounds(cb, s), cb.page_pool(s.pool, s.scales), 6
    starts, kv, table = i32(s.starts), i32([n for _, n in s.lens]), i32(s.table)
    ws = torch.empty(cb.cb_page_select_workspace_bytes(s.n, 8, s.table.shape[1]), dtype=torch.uint8, device="cuda")

    def buffers():
        return (torch.full((s.n, 8, k), 7, dtype=torch.int32, device="cuda"),
                torch.full((s.n, 16, 64), 9.0, dtype=torch.bfloat16, device="cuda"),
                torch.full((s.n, 16), 9.0, dtype=torch.float32, device="cuda"))

    def run(sel, out, lse):
        cb.cb_page_select(s.q, pages, s.layer, b, starts, kv, table, sel, workspace=ws)
        cb.cb_attn_selected(s.q, pages, s.layer, starts, kv, table, sel, out, lse=lse)

    held = buffers()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    run(*buffers())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        run(*held)
    for lens in ([(280, 700), (1, 300), (33, 33)], [(100, 650), (150, 290), (60, 20)], [(0, 0), (314, 300), (0, 33)], [(1, 700), (0, 1), (2, 5)]):
        starts.copy_(i32(np.concatenate([[0], np.cumsum([q for q, _ in lens])])))
        kv.copy_(i32([n for _, n in lens]))
        s.q.copy_(randn(gen(len(lens) + lens[0][0]), *s.q.shape).cuda())
        for x, y in zip(held, buffers()):
            x.copy_(y)
        eager = buffers()
        run(*eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        n = int(starts[-1])
        for x, y, rest in zip(held, eager, (7, 9, 9)):
            assert torch.equal(x, y) and (x[n:] == rest).all() and not torch.equal(x[:n], torch.full_like(x[:n], rest))
        torch.randn(1000, device="cuda").sort()


def test_two_calls_at_once(cb, serve):
    """Choice and attention of two steps on two streams, a workspace each."""
    steps = [make_step(cb, "blocks", [(1, 4000), (2, 900)], 2, 4, 64, 16, seed=30 + i) for i in range(2)]
    want = []
    for s in steps:
        s.b = all_bounds(cb, s)
        sel = choose(cb, s, s.b, 80, 1, 2)
        attend(cb, s, sel)
        want.append((sel, s.out.clone()))
    streams, got = [torch.cuda.Stream() for _ in steps], []
    torch.cuda.synchronize()
    for s, st in zip(steps, streams):
        with torch.cuda.stream(st):
            sel = torch.full((s.n, s.H, 80), -7, dtype=torch.int32, device="cuda")
            out = torch.full_like(s.out, 9.0)
            args = (i32(s.starts), i32([k for _, k in s.lens]), i32(s.table))
            w1 = torch.empty((cb.cb_page_select_workspace_bytes(s.n, s.H, s.table.shape[1]),), dtype=torch.uint8, device="cuda")
            w2 = torch.empty((cb.cb_attn_selected_workspace_bytes(s.n, 8, 2, 64, 16, 80),), dtype=torch.uint8, device="cuda")
            pages = cb.page_pool(s.pool, s.scales)
            for _ in range(3):
                cb.cb_page_select(s.q, pages, s.layer, s.b, *args, sel, first=1, last=2, workspace=w1)
                cb.cb_attn_selected(s.q, pages, s.layer, *args, sel, out, workspace=w2)
            got.append((sel, out, args, w1, w2))
    torch.cuda.synchronize()
    for (sel, out, *_), (a, b) in zip(got, want):
        assert np.array_equal(sel.cpu().numpy(), a) and torch.equal(out, b)

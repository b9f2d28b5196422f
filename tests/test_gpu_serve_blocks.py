"""GPU tests of pages whose 8-bit rows have a scale for every page, head and K or V: rows written into them and read back,
against the plain fp64 forms of ``oracle.serve``.

Scales are powers of two found from the rows' own bits: they are exact, and so are the codes of rows that are not turned
and of old rows that go over to a larger scale.  A turned pair takes three fp32 roundings of terms no larger than
|a c| + |b s| and is rounded once to e4m3 (2^-4 of the value, 2^-10 below 2^-6) or bf16 (2^-8 of it).
"""
import numpy as np
import pytest
import torch

from test_gpu_serve import CASES, Step
from test_serve_blocks_host import build_span_cut

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


def by_row(x):
    """[layer][2][seq][head][token][d] as numbers [row][layer][2][head][d]."""
    L, _, B, H, T, d = x.shape
    return f64(x).transpose(2, 4, 0, 1, 3, 5).reshape(B * T, L, 2, H, d)


class Pool:
    """A pool of 8-bit pages with a scale for every page, head and K or V: bytes that are any, the NaN among them, and
    scales of different size where ``used``."""

    def __init__(self, cb, L, H, P, ps, d, token_major=False, seed=0):
        rng = np.random.default_rng(seed)
        shape = (L, 2, P, ps, H, d) if token_major else (L, 2, P, H, ps, d)
        raw = torch.tensor(rng.integers(0, 256, shape, dtype=np.uint8), device="cuda").view(torch.float8_e4m3fn)
        self.t = raw.permute(0, 1, 2, 4, 3, 5) if token_major else raw
        self.exps = rng.integers(-12, 3, (L, P, H, 2))
        self.scales = torch.tensor(2.0 ** self.exps, dtype=torch.float32, device="cuda")
        self.pages = cb.page_pool(self.t, self.scales)

    def codes(self):
        return f64(self.t)

    def raw(self):
        return self.t.view(torch.uint8).cpu().numpy()


def rope_of(cb, d, axes, n, seed, style, bad=()):
    rng = np.random.default_rng(seed)
    n_pos = 64
    pos = rng.integers(0, n_pos, (axes, n)).astype(np.int32)
    for t in bad:
        pos[0, t] = n_pos if t % 2 else -1
    table = torch.empty((n_pos, d // 2, 2), dtype=torch.float32, device="cuda")
    cb.cb_rope_table(THETA, d, n_pos, table)
    axis = [(i * 7 // 3) % axes for i in range(d // 2)]
    return cb.rope_axes_spec(table, i32(pos), axis, style), table.cpu().numpy(), pos, axis


def turned_keys(serve, rows, rope, inverse=False):
    """The rows with their keys turned, and the products' magnitudes behind every element."""
    _, table, pos, axis, style = rope
    y, mag = rows.copy(), np.zeros_like(rows)
    y[:, :, 0], mag[:, :, 0] = serve.turn(rows[:, :, 0], table, pos, axis, style, inverse)
    return y, mag


def make_step(lens, ps, P, seed, packed, T=None):
    """Requests (new tokens, tokens with them) in a shuffled pool: starts, lengths, table."""
    rng = np.random.default_rng(seed)
    q = np.array([a for a, _ in lens])
    kv = np.array([b for _, b in lens])
    width = max(1, max(-(-int(k) // ps) for k in kv)) + 1
    order, at = rng.permutation(P), 0
    table = np.full((len(lens), width), -1, np.int64)
    for r, k in enumerate(kv):
        n = -(-int(k) // ps)
        table[r, :n] = order[at:at + n]
        at += n
    starts = np.concatenate([[0], np.cumsum(np.maximum(q, 0))[:-1]]) if packed else np.arange(len(lens)) * T
    return starts, q, kv, table, width


def check_codes(serve, got, want, mag, turned, written):
    """Codes that the call wrote: exact where nothing was turned, else within the roundings of a turn and of e4m3."""
    got, want, mag, turned = got[written], want[written], mag[written], turned[written]
    plain = serve.e4m3(want[~turned])
    assert np.array_equal(got[~turned], plain, equal_nan=True)
    got, want, mag = got[turned], want[turned], mag[turned]
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), ~fine)
    tol = np.maximum(2.0 ** -4 * np.abs(want[fine]), 2.0 ** -10) + 5 * F32 * (mag[fine] + np.abs(want[fine]))
    assert (np.abs(got[fine] - want[fine]) <= tol).all()


QUANT = [
    # lens (new, with them), L, H, G, d, page, axes, style, packed, token major, odd value
    ([(1, 1)], 1, 1, 0, 64, 16, 0, 0, True, False),
    ([(1, 17), (1, 16), (1, 32), (1, 1)], 1, 8, 8, 128, 16, 1, 0, True, True),
    ([(3, 40), (0, 9), (5, 5), (1, 100)], 2, 2, 3, 96, 24, 3, 1, True, False),
    ([(40, 40), (17, 17), (33, 33)], 3, 2, 0, 128, 16, 3, 0, False, False),
    ([(64, 64), (200, 263)], 2, 4, 0, 128, 64, 0, 0, False, True),
    ([(130, 131), (1, 65)], 1, 2, 2, 64, 64, 1, 1, True, False),
    ([(7, 30), (9, 9)], 1, 3, 1, 80, 7, 2, 0, True, False),
    ([(5, 5), (2, 9)], 2, 1, 0, 16, 1, 1, 0, True, False),
    ([(90, 300)], 1, 2, 0, 256, 100, 3, 1, True, True),
    ([(300, 700), (300, 300)], 1, 1, 2, 128, 256, 1, 0, True, False),
    ([(1000, 1003)], 2, 2, 0, 64, 1024, 3, 0, True, False),
    ([(128, 128)], 1, 2, 0, 128, 128, 1, 0, True, False),
]


@pytest.mark.parametrize("case", range(len(QUANT)))
def test_quantize(cb, serve, case):
    lens, L, H, G, d, ps, axes, style, packed, tm = QUANT[case]
    T = max(q for q, _ in lens)
    B, T = (1, sum(q for q, _ in lens)) if packed else (len(lens), T)
    P = sum(-(-k // ps) for _, k in lens) + 2
    starts, q, kv, table, width = make_step(lens, ps, P, case, packed, T)
    g, n = gen(case), B * T
    x = randn(g, L, 2, B, T, H, d) if tm else randn(g, L, 2, B, H, T, d)
    x = x.permute(0, 1, 2, 4, 3, 5) if tm else x
    x = x * torch.exp(2 * torch.randn((L, 2, B, H, T, 1), generator=g)).to(torch.bfloat16)
    if case % 3 == 2:
        x[0, 0, 0, 0, 0, 3], x[0, 1, 0, 0, 0, 5], x[-1, 1, 0, -1, -1, 0] = float("nan"), -float("inf"), float("inf")
    x = x.contiguous().cuda() if not tm else x.permute(0, 1, 2, 4, 3, 5).contiguous().cuda().permute(0, 1, 2, 4, 3, 5)
    pool = Pool(cb, L + 1, H, P, ps, d, tm, seed=case)
    rope, tables = None, None
    if axes:
        rope, *rest = rope_of(cb, d, axes, n, case, style, bad=[n // 2] if n > 30 else [])
        tables = (rope, *rest, style)
    qx = qo = None
    if G:
        qx = randn(g, n, H * G, d).cuda()
        qo = torch.full_like(qx, 5.0)
    before, raw0 = pool.codes(), pool.raw()
    cb.cb_page_quantize(x, pool.pages, i32(starts), i32(q), i32(kv), i32(table), layer=1, rope=rope, q=qx, q_out=qo)
    torch.cuda.synchronize()
    rows = by_row(x)
    y, mag = turned_keys(serve, rows, tables) if axes else (rows, np.zeros_like(rows))
    spans = serve.page_spans(starts, q, kv, ps, n, width)
    want, exps = before[1:].copy(), pool.exps[1:].copy()
    wmag = np.zeros_like(want)
    serve.page_quantize(rows, y if axes else None, want, exps, spans, table)
    assert np.array_equal(pool.scales[1:].cpu().numpy(), (2.0 ** exps).astype(np.float32))
    assert np.array_equal(pool.scales[:1].cpu().numpy(), (2.0 ** pool.exps[:1]).astype(np.float32))
    new, old = np.zeros(want.shape, bool), np.zeros(want.shape, bool)
    for r, entry, at, m, t in spans:
        p = int(table[r, entry])
        new[:, :, p, :, at:at + m] = True
        old[:, :, p, :, :at] = True
        s = (2.0 ** -exps[:, p].astype(float)).transpose(0, 2, 1)[..., None, None]     # [layer][2][head]
        wmag[:, :, p, :, at:at + m] = mag[t:t + m].transpose(1, 2, 3, 0, 4) * s
    got, raw = pool.codes()[1:], pool.raw()[1:]
    is_k = np.zeros(want.shape, bool)
    is_k[:, 0] = bool(axes)
    check_codes(serve, got, want, wmag, is_k, new)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    assert same[old].all()
    rest = ~new & ~old
    assert np.array_equal(raw[rest], raw0[1:][rest]) and np.array_equal(pool.raw()[:1], raw0[:1])
    if G:
        keep = np.concatenate([np.arange(t, t + m) for *_, m, t in spans])
        yq, mq = serve.turn(f64(qx), tables[1], tables[2], tables[3], style)
        gq = f64(qo)
        assert np.array_equal(np.isnan(gq[keep]), np.isnan(yq[keep]))
        fine = ~np.isnan(yq[keep])
        assert (np.abs(gq[keep] - yq[keep])[fine] <= (BF * np.abs(yq[keep]) + 4 * F32 * mq[keep])[fine]).all()
        q2 = qx.clone()
        cb.cb_page_quantize(x, pool.pages, i32(starts), i32(q), i32(kv), i32(table), layer=1, rope=rope, q=q2, q_out=q2)
        assert torch.equal(q2[keep].nan_to_num(1.0), qo[keep].nan_to_num(1.0))
    # the same call again changes nothing: the larger scales are there already
    cb.cb_page_quantize(x, pool.pages, i32(starts), i32(q), i32(kv), i32(table), layer=1, rope=rope)
    assert np.array_equal(pool.raw()[1:], raw) and np.array_equal(pool.scales[1:].cpu().numpy(), (2.0 ** exps).astype(np.float32))


@pytest.mark.parametrize("kind", ["blocks", "e4m3", "bf16"])
@pytest.mark.parametrize("case", range(len(QUANT)))
def test_read(cb, serve, case, kind):
    lens, L, H, _, d, ps, axes, style, packed, tm = QUANT[case]
    B, T = (1, sum(q for q, _ in lens)) if packed else (len(lens), max(q for q, _ in lens))
    P = sum(-(-k // ps) for _, k in lens) + 2
    starts, q, kv, table, width = make_step(lens, ps, P, case, packed, T)
    n, inverse = B * T, bool(case % 2)
    if kind == "blocks":
        pool = Pool(cb, L + 1, H, P, ps, d, tm, seed=case)
        pages = pool.pages
        value = pool.codes() * (2.0 ** pool.exps.astype(float)).transpose(0, 3, 1, 2)[..., None, None]
    else:
        shape = (L + 1, 2, P, ps, H, d) if tm else (L + 1, 2, P, H, ps, d)
        t = randn(gen(case), *shape).cuda()
        t = t.to(torch.float8_e4m3fn) if kind == "e4m3" else t
        t = t.permute(0, 1, 2, 4, 3, 5) if tm else t
        scales = 0.01 + torch.rand((L + 1, 2, H), generator=gen(case + 1)) if kind == "e4m3" else None
        value = f64(t) * (scales.double().numpy()[:, :, None, :, None, None] if kind == "e4m3" else 1.0)
        pages = cb.page_pool(t, None if scales is None else scales.cuda())
    out = torch.full((L, 2, B, T, H, d) if tm else (L, 2, B, H, T, d), 7.0, dtype=torch.bfloat16, device="cuda")
    out = out.permute(0, 1, 2, 4, 3, 5) if tm else out
    rope, tables = None, None
    if axes:
        rope, *rest = rope_of(cb, d, axes, n, case, style, bad=[n // 2] if n > 30 else [])
        tables = (rope, *rest, style)
    cb.cb_page_read(pages, out, i32(starts), i32(q), i32(kv), i32(table), layer=1, rope=rope, inverse=inverse)
    torch.cuda.synchronize()
    want, read = np.full((n, L, 2, H, d), 7.0), np.zeros(n, bool)
    for r, entry, at, m, t in serve.page_spans(starts, q, kv, ps, n, width):
        want[t:t + m] = value[1:, :, int(table[r, entry]), :, at:at + m].transpose(3, 0, 1, 2, 4)
        read[t:t + m] = True
    mag = np.abs(want)
    if axes:
        want, tmag = turned_keys(serve, want, tables, inverse)
        mag[:, :, 0] = tmag[:, :, 0]
    got = by_row(out)
    assert (got[~read] == 7.0).all()
    got, want, mag = got[read], want[read], mag[read]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    if kind != "e4m3":
        exact = fine.copy()
        if axes:
            exact[:, :, 0] = False
        assert np.array_equal(got[exact], want[exact])
    assert (np.abs(got - want)[fine] <= (BF * np.abs(want) + 6 * F32 * mag)[fine]).all()


MIXED = [
    # single tokens, the chunk among them (new, with them), L, H, G, d, page, axes, style
    (63, (200, 237), 1, 2, 0, 128, 64, 0, 0),
    (63, (200, 237), 2, 2, 2, 128, 64, 3, 1),
    (63, (230, 260), 1, 3, 2, 128, 16, 1, 0),
    (40, (150, 170), 2, 2, 0, 64, 64, 3, 0),
    (90, (300, 333), 1, 1, 3, 96, 64, 2, 1),
    (120, (200, 250), 1, 2, 0, 256, 32, 1, 0),
    (200, (500, 700), 1, 1, 1, 64, 256, 1, 0),
]


def mixed_step(tmp_path, case):
    """A step of many single tokens and one chunk that begins inside a page, and the rule that gives its rows teams made for
    single tokens, while the chunk's whole pages have more units than a wave."""
    singles, chunk, L, H, G, d, ps, axes, style = MIXED[case]
    rng = np.random.default_rng(case)
    lens = [(1, int(k)) for k in rng.integers(1, 3 * ps, singles)]
    lens.insert(singles // 2, chunk)
    n = singles + chunk[0]
    cut = build_span_cut(tmp_path)(n, len(lens), ps, d, 2 * L * H + H * G)
    assert not cut["wide"] and ps << cut["lgc"] > 64 and (chunk[1] - chunk[0]) % ps
    P = sum(-(-k // ps) for _, k in lens) + 2
    return n, P, make_step(lens, ps, P, case, True)


@pytest.mark.parametrize("case", range(len(MIXED)))
def test_quantize_single_tokens_and_a_chunk(cb, serve, tmp_path, case):
    """Scales that grow and others that stay, a NaN and an infinity in the chunk's whole pages; queries beside the rows."""
    singles, chunk, L, H, G, d, ps, axes, style = MIXED[case]
    n, P, (starts, q, kv, table, width) = mixed_step(tmp_path, case)
    g = gen(100 + case)
    x = (randn(g, L, 2, 1, H, n, d) * torch.exp(2 * torch.randn((L, 2, 1, H, n, 1), generator=g)).to(torch.bfloat16)).cuda()
    whole = singles // 2 + chunk[0] // 2                           # a token of a whole page of the chunk
    x[0, 0, 0, 0, whole, 3], x[-1, 1, 0, -1, whole, 5] = float("nan"), float("inf")
    pool = Pool(cb, L + 1, H, P, ps, d, seed=case)
    rope = tables = qx = qo = None
    if axes:
        rope, *rest = rope_of(cb, d, axes, n, case, style, bad=[singles // 2 + 7])
        tables = (rope, *rest, style)
    if G:
        qx = randn(g, n, H * G, d).cuda()
        qo = torch.full_like(qx, 5.0)
    before, raw0 = pool.codes()[1:], pool.raw()
    cb.cb_page_quantize(x, pool.pages, i32(starts), i32(q), i32(kv), i32(table), layer=1, rope=rope, q=qx, q_out=qo)
    torch.cuda.synchronize()
    rows = by_row(x)
    y, mag = turned_keys(serve, rows, tables) if axes else (rows, np.zeros_like(rows))
    spans = serve.page_spans(starts, q, kv, ps, n, width)
    want, exps, wmag = before.copy(), pool.exps[1:].copy(), np.zeros_like(before)
    serve.page_quantize(rows, y if axes else None, want, exps, spans, table)
    assert np.array_equal(pool.scales[1:].cpu().numpy(), (2.0 ** exps).astype(np.float32))
    new, old, grown = np.zeros(want.shape, bool), np.zeros(want.shape, bool), 0
    for r, entry, at, m, t in spans:
        p = int(table[r, entry])
        new[:, :, p, :, at:at + m] = True
        old[:, :, p, :, :at] = True
        grown += int((exps[:, p] > pool.exps[1:, p]).sum()) if r == singles // 2 and at else 0
        wmag[:, :, p, :, at:at + m] = mag[t:t + m].transpose(1, 2, 3, 0, 4) * (2.0 ** -exps[:, p].astype(float)).transpose(0, 2, 1)[..., None, None]
    assert grown > 0
    got, raw = pool.codes()[1:], pool.raw()
    is_k = np.zeros(want.shape, bool)
    is_k[:, 0] = bool(axes)
    check_codes(serve, got, want, wmag, is_k, new)
    assert ((got == want) | (np.isnan(got) & np.isnan(want)))[old].all()
    rest = ~new & ~old
    assert np.array_equal(raw[1:][rest], raw0[1:][rest]) and np.array_equal(raw[:1], raw0[:1])
    if G:
        yq, mq = serve.turn(f64(qx), *tables[1:4], style)
        gq, fine = f64(qo), ~np.isnan(yq)
        assert np.array_equal(np.isnan(gq), ~fine)
        assert (np.abs(gq - yq)[fine] <= (BF * np.abs(yq) + 4 * F32 * mq)[fine]).all()
    cb.cb_page_quantize(x, pool.pages, i32(starts), i32(q), i32(kv), i32(table), layer=1, rope=rope, q=qx, q_out=qo)
    assert np.array_equal(pool.raw(), raw)


@pytest.mark.parametrize("kind", ["blocks", "e4m3", "bf16"])
@pytest.mark.parametrize("case", range(len(MIXED)))
def test_read_single_tokens_and_a_chunk(cb, serve, tmp_path, case, kind):
    singles, chunk, L, H, _, d, ps, axes, style = MIXED[case]
    n, P, (starts, q, kv, table, width) = mixed_step(tmp_path, case)
    scales = None
    if kind == "blocks":
        pool = Pool(cb, L + 1, H, P, ps, d, seed=case)
        pages, value = pool.pages, pool.codes() * (2.0 ** pool.exps.astype(float)).transpose(0, 3, 1, 2)[..., None, None]
    else:
        t = randn(gen(case), L + 1, 2, P, H, ps, d).cuda()
        value = None
        if kind == "e4m3":
            t, scales = t.to(torch.float8_e4m3fn), (0.01 + torch.rand((L + 1, 2, H), generator=gen(case + 1)))
            value = f64(t) * scales.double().numpy()[:, :, None, :, None, None]
        pages, value = cb.page_pool(t, None if scales is None else scales.cuda()), f64(t) if value is None else value
    rope = tables = None
    if axes:
        rope, *rest = rope_of(cb, d, axes, n, case, style, bad=[singles // 2 + 7])
        tables = (rope, *rest, style)
    out = torch.full((L, 2, 1, H, n, d), 7.0, dtype=torch.bfloat16, device="cuda")
    cb.cb_page_read(pages, out, i32(starts), i32(q), i32(kv), i32(table), layer=1, rope=rope, inverse=bool(case % 2))
    torch.cuda.synchronize()
    want = np.full((n, L, 2, H, d), 7.0)
    for r, entry, at, m, t in serve.page_spans(starts, q, kv, ps, n, width):
        want[t:t + m] = value[1:, :, int(table[r, entry]), :, at:at + m].transpose(3, 0, 1, 2, 4)
    mag = np.abs(want)
    if axes:
        want, turned = turned_keys(serve, want, tables, bool(case % 2))
        mag[:, :, 0] = turned[:, :, 0]
    got, fine = by_row(out), ~np.isnan(want)
    assert np.array_equal(np.isnan(got), ~fine)
    if kind != "e4m3":
        exact = fine.copy()
        exact[:, :, 0] &= not axes
        assert np.array_equal(got[exact], want[exact])
    assert (np.abs(got - want)[fine] <= (BF * np.abs(want) + 6 * F32 * mag)[fine]).all()


def test_read_of_what_was_written_is_near(cb):
    """Through pages and back: off by a rounding to e4m3 of every element, 2^-4 of it, 2^-10 of the scale where that is
    more.  The scale is the least power of two that is max / 448 or more, so less than max / 224."""
    g = gen(3)
    x = (randn(g, 2, 2, 3, 2, 50, 128) * torch.exp(3 * torch.randn((2, 2, 3, 2, 50, 1), generator=g)).to(torch.bfloat16)).cuda()
    pool = Pool(cb, 2, 2, 12, 16, 128)
    table = i32(np.arange(12).reshape(3, 4))
    starts, lens = i32([0, 50, 100]), i32([50, 33, 1])
    cb.cb_page_quantize(x, pool.pages, starts, lens, lens, table)
    y = torch.zeros_like(x)
    cb.cb_page_read(pool.pages, y, starts, lens, lens, table)
    for b, n in enumerate((50, 33, 1)):
        a, z = f64(x[:, :, b, :, :n]), f64(y[:, :, b, :, :n])
        for p in range(0, n, 16):
            s = np.abs(a[..., p:p + 16, :]).max((-2, -1), keepdims=True) / 224
            assert (np.abs(a - z)[..., p:p + 16, :] <= np.maximum(2.0 ** -4 * np.abs(a[..., p:p + 16, :]), 2.0 ** -10 * s)).all()
    assert (y[:, :, 1, :, 33:] == 0).all() and (y[:, :, 2, :, 1:] == 0).all()


def test_pages_filled_token_by_token(cb, serve):
    """Sixty steps of one token: rows of ever different size, scales that grow, old codes that go over to them."""
    H, d, ps, P = 2, 64, 16, 8
    pool = Pool(cb, 1, H, P, ps, d, seed=5)
    table = np.array([[3, 1, 6, 0, -1], [2, 7, 4, 5, -1]])
    codes, exps = pool.codes(), pool.exps.copy()
    rng = np.random.default_rng(2)
    for step in range(60):
        x = (torch.randn((1, 2, 1, H, 2, d), generator=gen(step)) * float(2.0 ** rng.integers(-9, 9))).to(torch.bfloat16).cuda()
        q, kv = [1, int(step < 50)], [step + 1, min(step, 49) + 1]
        cb.cb_page_quantize(x, pool.pages, i32([0, 1]), i32(q), i32(kv), i32(table))
        spans = serve.page_spans([0, 1], q, kv, ps, 2, 5)
        serve.page_quantize(by_row(x), None, codes, exps, spans, table)
        for r, entry, at, m, _ in spans:
            p = table[r, entry]
            codes[:, :, p, :, at:at + m] = serve.e4m3(codes[:, :, p, :, at:at + m])
    got = pool.codes()
    assert np.array_equal(pool.scales.cpu().numpy(), (2.0 ** exps).astype(np.float32))
    assert ((got == codes) | (np.isnan(got) & np.isnan(codes))).all()


def test_scales_at_their_borders(cb, serve):
    """Blocks whose largest magnitude is 448 or 316 times a power of two, just above it, the least and the largest numbers."""
    H, d, ps = 1, 64, 8
    tops = []
    for top in (448.0, 450.0, 446.0, 316.0, 318.0, 314.0):
        tops += [top, top * 2.0 ** -30, top * 2.0 ** 60]
    tops += [0.0, 1e-38, 2.0 ** -56, 2.0 ** -55, 3.38e38, 2.0 ** 127, 448 * 2.0 ** -64, 450 * 2.0 ** -64]
    n = len(tops)
    x = torch.zeros((1, 2, n, H, 1, d))
    for i, t in enumerate(tops):
        x[0, :, i, 0, 0, 5] = -t
        x[0, :, i, 0, 0, 6] = t / 3
    x = x.to(torch.bfloat16).cuda()
    table = np.arange(n)[:, None]
    for axes in (0, 1):
        pool = Pool(cb, 1, H, n, ps, d, seed=7)
        rope = tables = None
        if axes:
            rope, *rest = rope_of(cb, d, 1, n, 3, 0)
            tables = (rope, *rest, 0)
        cb.cb_page_quantize(x, pool.pages, i32(np.arange(n)), i32([1] * n), i32([1] * n), i32(table), rope=rope)
        rows = by_row(x)
        codes, exps = np.zeros((1, 2, n, H, ps, d)), pool.exps.copy()
        y, mag = turned_keys(serve, rows, tables) if axes else (rows, None)
        serve.page_quantize(rows, y if axes else None, codes, exps, serve.page_spans(np.arange(n), [1] * n, [1] * n, ps, n, 1), table)
        assert np.array_equal(pool.scales.cpu().numpy(), (2.0 ** exps.astype(float)).astype(np.float32))
        got = pool.codes()
        far = tops.index(3.38e38)                               # beyond the largest scale's largest number
        assert np.isnan(got[0, 1, far, 0, 0, 5]) and np.isfinite(np.delete(got[:, :, :, :, 0], far, 2)).all()
        assert np.array_equal(got[:, 1, :, :, 0], serve.e4m3(codes[:, 1, :, :, 0]), equal_nan=True)


@pytest.mark.parametrize("style", [0, 1])
def test_turned_keys_fit_their_scale(cb, style):
    """Pairs of the largest size turned by an eighth of a circle, in one channel sqrt 2 larger, by a table that is 1.03 too
    long as well: 316 sqrt 2 1.03 = 460.3 is 448, the nearest number."""
    d, ps = 64, 4
    x = torch.full((1, 2, 1, 1, ps, d), 316.0, dtype=torch.bfloat16, device="cuda")
    x[0, :, 0, 0, 1] *= -1
    x[0, :, 0, 0, 2] = 0
    for size in (1.0, 1.03):
        table = torch.full((1, d // 2, 2), size * 0.5 ** 0.5, dtype=torch.float32, device="cuda")
        pool = Pool(cb, 1, 1, 1, ps, d)
        rope = cb.rope_axes_spec(table, i32(np.zeros(ps)), None, style)
        cb.cb_page_quantize(x, pool.pages, i32([0]), i32([ps]), i32([ps]), i32([[0]]), rope=rope)
        assert pool.scales[0, 0, 0, 0] == 1.0 and pool.scales[0, 0, 0, 1] == 1.0
        k = pool.codes()[0, 0, 0, 0]
        first = np.r_[0:d // 2] if style == 0 else np.r_[0:d:2]       # a c - a s = 0, a c + a s
        assert (k[:, first] == 0).all()
        other = np.setdiff1d(np.arange(d), first)
        assert (k[[0, 3]][:, other] == 448).all() and (k[1, other] == -448).all() and (k[2] == 0).all()


def test_requests_that_take_no_part(cb):
    """Lengths out of range, rows outside the tensor, pages outside the pool: nothing of theirs is written."""
    H, d, ps, P = 2, 64, 4, 6
    x = randn(gen(1), 1, 2, 1, H, 12, d).cuda()
    table = np.array([[0, -1], [1, 1], [2, 2], [3, 3], [4, P], [5, 2 ** 31 - 1], [0, 0], [1, 0]])
    starts = [0, 1, 10, -1, 0, 0, 0, 0]
    q = [0, 3, 3, 2, 4, 4, -2, 9]
    kv = [0, 2, 3, 2, 8, 8, 5, 9]
    for f in ("write", "read"):
        pool = Pool(cb, 1, H, P, ps, d, seed=9)
        raw, sc = pool.raw(), pool.scales.clone()
        out = torch.full_like(x, 3.0)
        args = (i32(starts), i32(q), i32(kv), i32(table))
        if f == "write":
            cb.cb_page_quantize(x, pool.pages, *args)
        else:
            cb.cb_page_read(pool.pages, out, *args)
        torch.cuda.synchronize()
        assert np.array_equal(pool.raw(), raw) and torch.equal(sc, pool.scales) and (out == 3.0).all()


def test_rows_that_serve_several_requests(cb):
    """One prompt written for five requests: more pages than its rows alone have; each gets what one would."""
    H, d, ps, n = 2, 64, 16, 40
    x = randn(gen(2), 2, 2, 1, H, n, d).cuda()
    one, many = Pool(cb, 2, H, 3, ps, d, seed=3), Pool(cb, 2, H, 15, ps, d, seed=4)
    cb.cb_page_quantize(x, one.pages, i32([0]), i32([n]), i32([n]), i32([[0, 1, 2]]))
    cb.cb_page_quantize(x, many.pages, i32([0] * 5), i32([n] * 5), i32([n] * 5), i32(np.arange(15).reshape(5, 3)))
    for r in range(5):
        a, b = one.t.view(torch.uint8), many.t.view(torch.uint8)[:, :, 3 * r:3 * r + 3]
        assert torch.equal(a[:, :, :2], b[:, :, :2]) and torch.equal(a[:, :, 2, :, :8], b[:, :, 2, :, :8])
        assert torch.equal(one.scales, many.scales[:, 3 * r:3 * r + 3])


@pytest.mark.parametrize("n", [300, 3000])
def test_many_requests(cb, serve, n):
    """More requests than a wave looks at in one round, some without tokens."""
    H, d, ps = 1, 64, 4
    rng = np.random.default_rng(n)
    q = rng.integers(0, 6, n)
    kv = np.where(q > 0, q + rng.integers(0, 5, n), 0)
    starts = np.concatenate([[0], np.cumsum(q)[:-1]])
    used = -(-kv // ps)
    P = int(used.sum())
    table, at = np.full((n, 3), -1), 0
    for r in range(n):
        table[r, :used[r]] = np.arange(at, at + used[r])
        at += used[r]
    total = int(q.sum())
    x = randn(gen(n), 1, 2, 1, H, total, d).cuda()
    pool = Pool(cb, 1, H, P, ps, d, seed=n)
    codes, exps = pool.codes(), pool.exps.copy()
    cb.cb_page_quantize(x, pool.pages, i32(starts), i32(q), i32(kv), i32(table))
    y = torch.zeros_like(x)
    cb.cb_page_read(pool.pages, y, i32(starts), i32(q), i32(kv), i32(table))
    spans = serve.page_spans(starts, q, kv, ps, total, 3)
    serve.page_quantize(by_row(x), None, codes, exps, spans, table)
    assert np.array_equal(pool.scales.cpu().numpy(), (2.0 ** exps).astype(np.float32))
    back, got = by_row(y), pool.codes()
    for r, entry, a, m, t in spans:
        p = table[r, entry]
        want = serve.e4m3(codes[0, :, p, 0, a:a + m])
        assert np.array_equal(got[0, :, p, 0, a:a + m], want)
        assert np.array_equal(back[t:t + m, 0, :, 0], (want * 2.0 ** exps[0, p, 0, :, None, None]).transpose(1, 0, 2))


def test_pool_beyond_32_bits(cb):
    """Rows more than 2^32 bytes apart, of the pool and of the cache that they are read into."""
    ps, H, d = 64, 8, 128
    P = (5 << 30) // (ps * H * d)
    raw = torch.empty((1, 2, P, H, ps, d), dtype=torch.uint8, device="cuda")
    scales = torch.ones((1, P, H, 2), dtype=torch.float32, device="cuda")
    pages = cb.page_pool(raw.view(torch.float8_e4m3fn), scales)
    x = randn(gen(14), 1, 2, 1, H, 150, d).cuda()
    ids = i32([[P - 1, 3, P - 2]])
    cb.cb_page_quantize(x, pages, i32([0]), i32([150]), i32([150]), ids)
    B = 5 * (1 << 30) // (2 * H * 200 * d * 2)
    out = torch.empty((1, 2, B, H, 200, d), dtype=torch.bfloat16, device="cuda")
    cb.cb_page_read(pages, out, i32([(B - 1) * 200]), i32([150]), i32([150]), ids)
    a, z = f64(x[:, :, 0]), f64(out[:, :, B - 1, :, :150])
    assert (np.abs(a - z) <= np.maximum(2.0 ** -4 * np.abs(a), 2.0 ** -10)).all()
    del raw, out, pages
    torch.cuda.empty_cache()


def test_more_pages_than_a_launch_has_workgroups(cb):
    """2^24 pages of one token and a few: back come numbers within half a step (2^-4 of the number; below 2^-6 of the
    scale 2^-10 of it, and 2^e < max / 224)."""
    n, d = (1 << 24) + 5, 16
    x = torch.randn((1, 2, 1, 1, n, d), generator=torch.Generator(device="cuda").manual_seed(15), device="cuda").bfloat16()
    raw = torch.empty((1, 2, n, 1, 1, d), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((1, n, 1, 2), dtype=torch.float32, device="cuda")
    pages = cb.page_pool(raw.view(torch.float8_e4m3fn), scales)
    span = (i32([0]), i32([n]), i32([n]), torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda")[None])
    cb.cb_page_quantize(x, pages, *span)
    most = x.abs().amax(-1).float()[0, :, 0, 0]                    # [2][token]
    sc = scales[0, :, 0].flip(0).T
    assert bool(((most <= 448 * sc) & (most > 224 * sc)).all())
    y = torch.full_like(x, 9.0)
    cb.cb_page_read(pages, y, *span)
    tol = torch.maximum(x.abs().float() * 2.0 ** -4, (most * (2.0 ** -10 / 224))[None, :, None, None, :, None])
    assert bool(((y.float() - x.float()).abs() <= tol).all())
    del x, y, tol, raw, scales, pages
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ attention

class BlockStep(Step):
    """Step over pages with scales of their own; the numbers that its keys and values stand for.  Unused places hold the
    NaN of e4m3, unused pages' scales are the largest."""

    def __init__(self, cb, lens, H, G, d, ps, token_major=False, pad=0, seed=0, layers=2, layer=1, lo=-4, hi=5):
        Step.__init__(self, cb, lens, H, G, d, ps, True, token_major, pad, seed, layers, layer)
        P, rng = self.pool.shape[2], np.random.default_rng(seed + 1)
        exps = np.full((layers, P, H, 2), 119)
        static = self.scales[layer].double().cpu().numpy()             # Step's numbers have these in them
        for r, (_, kv) in enumerate(lens):
            k, v = self.K[r] / static[0][:, None, None], self.V[r] / static[1][:, None, None]
            e = rng.integers(lo - 5, hi - 5, (-(-kv // ps), H, 2))
            exps[layer, self.table[r, :len(e)]] = e
            f = 2.0 ** np.repeat(e, ps, 0)[:kv].astype(float)               # [key][head][2]
            self.K[r], self.V[r] = (np.round(x * 512) / 512 * f[:, :, z].T[..., None] for z, x in enumerate((k, v)))
        self.scales = torch.tensor(2.0 ** exps.astype(float), dtype=torch.float32, device="cuda")


BLOCKS = [(lens, H, G, d, ps, tm) for lens, H, G, d, ps, _, tm in CASES]


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("case", range(len(BLOCKS)))
def test_attention(cb, serve, case, ws):
    lens, H, G, d, ps, tm = BLOCKS[case]
    s = BlockStep(cb, lens, H, G, d, ps, tm, pad=case % 3, seed=case)
    s.run(ws=ws)
    s.check(serve)


@pytest.mark.parametrize("window,sinks", [(1, 0), (33, 4), (64, 70), (2 ** 31 - 1, 0)])
@pytest.mark.parametrize("case", [2, 3, 5, 7, 10, 11])
def test_attention_window(cb, serve, case, window, sinks):
    lens, H, G, d, ps, tm = BLOCKS[case]
    s = BlockStep(cb, lens, H, G, d, ps, tm, pad=1, seed=case)
    s.run(window, sinks)
    s.check(serve, window, sinks)


@pytest.mark.parametrize("d,ps", [(64, 16), (96, 24), (128, 64), (128, 7)])
def test_attention_rows_in_many_parts(cb, serve, d, ps):
    """Rows in dozens of parts, of single tokens and of chunks; the same bits every time."""
    s = BlockStep(cb, [(1, 20000), (40, 12000), (3, 5000), (2, 300)], 2, 2, d, ps, pad=1, seed=80)
    s.run()
    s.check(serve)
    a, al = s.out.clone(), s.lse.clone()
    s.run()
    assert torch.equal(a, s.out) and torch.equal(al, s.lse)
    s.run(max_q=1)
    s.check(serve)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_large_alike_chunks(cb, serve, d):
    """Chunks that fill the chip with row tiles of 256: eight waves share K and V."""
    s = BlockStep(cb, [(512, 700), (512, 512)], 16, 8, d, 32, seed=5)
    s.run()
    s.check(serve, rows=[1])


def test_attention_of_scales_far_apart(cb, serve):
    """Blocks 2^40 apart: the values' sizes, and scores of hundreds."""
    for lens, G in (([(1, 100), (2, 60)], 2), ([(40, 90)], 4)):
        s = BlockStep(cb, lens, 2, G, 64, 16, seed=6, lo=-36, hi=4)
        s.run()
        s.check(serve)


@pytest.mark.parametrize("G,q,kv", [(2, 3, 60), (4, 40, 90), (1, 130, 130)])
def test_attention_nan_stays_with_its_rows(cb, serve, G, q, kv):
    """The NaN of e4m3 in a key or value that later rows see does not reach the rows before it."""
    for z in range(2):
        s = BlockStep(cb, [(q, kv)], 1, G, 64, 16, seed=8)
        j = kv - q + q // 2
        s.pool.view(torch.uint8)[s.layer, z, int(s.table[0, j // 16]), 0, j % 16, 3] = 0x7f
        s.run()
        got = f64(s.out)
        early, late = got[:q // 2], got[q // 2:]
        o, _, mag, smag = serve.attention(f64(s.q), s.K[0][0], s.V[0][0], kv, 64 ** -0.5)
        tol = BF * 1.01 * np.abs(o) + mag * (BF * 1.01 + (2 * 72 * 2 * F32 * smag + (kv + 64) * 2 * F32)[..., None])
        assert (np.abs(early - o[:q // 2]) <= tol[:q // 2]).all(), z
        if z == 1:
            assert np.isnan(late[..., 3]).all()
            keep = [c for c in range(64) if c != 3]
            assert (np.abs(late - o[q // 2:]) <= tol[q // 2:])[..., keep].all()
        else:
            assert np.isnan(late).all()


@pytest.mark.parametrize("lens,G", [([(1, 100), (1, 70)], 4), ([(70, 200)], 2)])
def test_attention_hidden_pages(cb, serve, lens, G):
    """Entries outside the pool hide their keys; all of them: zeros and -inf."""
    s = BlockStep(cb, lens, 1, G, 128, 16, seed=6)
    table = s.table.copy()
    table[0, 0], table[0, 3] = -1, s.pool.shape[2]
    s.run(table=table)
    s.check(serve, hidden=[set(range(16)) | set(range(48, 64))] + [set()] * (len(lens) - 1))
    table[0, :] = 2 ** 31 - 1
    s.run(table=table)
    s.check(serve, hidden=[set(range(lens[0][1]))] + [set()] * (len(lens) - 1))

"""Serving a receiver model from a transferred cache: the operators on pages, case by case, in plain form and as calls.

* ``tables``  block tables, slot maps and positions of a step from the requests' lengths (``cb_page_tables``);
* ``rope``    keys turned by positions of several axes, time, height and width (``cb_rope_axes``);
* ``write``   rows of a cache into the pages of a pool, keys turned on the way, bf16 or e4m3 pages, with the step's
              queries turned beside them (``cb_page_write``);
* ``attn``    attention of the new tokens of every request over its pages, whole or with a sliding window and first
              tokens that stay visible (``cb_attn_paged``).

With ``own`` false every operator is computed from elementary torch operations in 32 bits.  Geometries are the
repository's own: 64 layers x 8 KV heads x 128 with 64 query heads (the receiver), 40 query heads over 8 (the sender),
heads of 96 and of 64.
"""
import math
import random

import torch

own = False

DEV = "cuda"
E4M3_MAX = 448.0
THETA = 1e6


# ---------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the smallest decode step: four short conversations of a small model, where only latency counts
        dict(name="attn_decode_tiny", kind="attn", decode=4, chunks=0, q_len=1, kv_min=40, kv_max=300, H=2, G=2, d=64,
             page=16, e4m3=False, window=0, sinks=0, pad=0, token_major=False),
        # one layer's attention of a decode step over 64 requests of very different lengths, padded for a graph
        dict(name="attn_decode_batch", kind="attn", decode=64, chunks=0, q_len=1, kv_min=512, kv_max=16384, H=8, G=8,
             d=128, page=16, e4m3=False, window=0, sinks=0, pad=8, token_major=False),
        # decode over long contexts held in 8 bits, five query heads to a KV head: bandwidth
        dict(name="attn_decode_long_e4m3", kind="attn", decode=8, chunks=0, q_len=1, kv_min=65536, kv_max=131072, H=8,
             G=5, d=128, page=64, e4m3=True, window=0, sinks=0, pad=0, token_major=True),
        # the receiver reads 2,048 new tokens behind a transferred context: matrix products
        dict(name="attn_chunk", kind="attn", decode=0, chunks=1, q_len=2048, kv_min=32768, kv_max=32768, H=8, G=8,
             d=128, page=64, e4m3=False, window=0, sinks=0, pad=0, token_major=False),
        # decode requests and prompt chunks in one step of a windowed model with four sinks, heads of 96
        dict(name="attn_mixed_window", kind="attn", decode=24, chunks=3, q_len=515, kv_min=900, kv_max=9000, H=8, G=4,
             d=96, page=32, e4m3=False, window=1024, sinks=4, pad=5, token_major=True),
        # an ordinary decode step's tables: 64 requests, one new token each
        dict(name="tables_decode", kind="tables", reqs=64, q_min=1, q_max=1, ctx_max=16384, page=16, spare=64, pad=8),
        # tables of a bulk handoff: 512 contexts of up to 4,096 tokens that get their pages at once
        dict(name="tables_handoff", kind="tables", reqs=512, q_min=1, q_max=4096, ctx_max=0, page=16, spare=100, pad=0),
        # keys of one layer of a decode step
        dict(name="rope_step", kind="rope", layers=1, heads=8, d=128, seqs=1, seq_len=64, axes=3, style=0, inverse=False,
             token_major=True),
        # a sender's cache of image and text tokens turned back to content coordinates
        dict(name="rope_cache_inverse", kind="rope", layers=40, heads=8, d=128, seqs=6, seq_len=2047, axes=3, style=1,
             inverse=True, token_major=False),
        # one layer's write of a decode step: 64 tokens' keys and values, and their queries
        dict(name="write_decode", kind="write", layers=1, heads=8, G=8, d=128, seqs=1, seq_len=64, fill=1.0, page=16,
             e4m3=False, axes=1, style=0, token_major=True),
        # four mapped caches of up to 2,048 tokens into 8-bit pages, all layers, positions of three axes
        dict(name="write_handoff_e4m3", kind="write", layers=64, heads=8, G=0, d=128, seqs=4, seq_len=2048, fill=0.6,
             page=64, e4m3=True, axes=3, style=0, token_major=False),
        # a mapped cache whose keys are turned already, into 16-bit pages
        dict(name="write_handoff", kind="write", layers=64, heads=8, G=0, d=128, seqs=1, seq_len=4096, fill=1.0, page=16,
             e4m3=False, axes=0, style=0, token_major=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "attn", "tables", "rope", "write", "write"])
    page = rng.choice([8, 16, 24, 32, 64, 100, 128])
    d = rng.choice([64, 96, 128, 128])
    if kind == "attn":
        H, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8, 16])
        window = rng.choice([0, 0, _log(rng, 16, 8192)])
        c = dict(kind=kind, H=H, G=G, d=d, page=page, e4m3=rng.random() < 0.4, window=window,
                 sinks=rng.choice([0, 1, 4, 70]) if window else 0, pad=rng.choice([0, 0, 3, 17]),
                 token_major=rng.random() < 0.5)
        form = rng.choice(["decode", "few", "chunk", "mixed"])
        if form == "decode":
            n = _log(rng, 1, 256)
            top = _log(rng, 64, min(131072, 1048576 // n))
            return dict(c, decode=n, chunks=0, q_len=1, kv_min=rng.choice([1, max(1, top // 8)]), kv_max=top)
        if form == "few":                                     # a few tokens checked at once
            n = _log(rng, 1, 64)
            top = _log(rng, 64, 32768)
            return dict(c, decode=0, chunks=n, q_len=rng.randint(2, 9), kv_min=max(1, top // 4), kv_max=top)
        q = _log(rng, 10, 2048)
        top = max(q, _log(rng, 64, 16384))
        n = rng.randint(1, 3)
        return dict(c, decode=rng.randint(1, 40) if form == "mixed" else 0, chunks=n, q_len=q, kv_min=max(1, top // 3),
                    kv_max=top)
    if kind == "tables":
        q_max = _log(rng, 1, 4096)
        return dict(kind=kind, reqs=_log(rng, 1, 512), q_min=rng.choice([0, 1, q_max]), q_max=q_max,
                    ctx_max=rng.choice([0, _log(rng, 1, 60000)]), page=page, spare=rng.choice([-3, 0, 1, 500]),
                    pad=rng.choice([0, 1, 50]))
    seqs, seq_len = _log(rng, 1, 8), _log(rng, 1, 2048)
    layers = _log(rng, 1, 64 if kind == "write" else 40)
    if kind == "rope":
        return dict(kind=kind, layers=layers, heads=rng.choice([1, 2, 4, 8]), d=d, seqs=min(seqs, 6), seq_len=seq_len,
                    axes=rng.choice([1, 2, 3]), style=rng.choice([0, 1]), inverse=rng.random() < 0.5,
                    token_major=rng.random() < 0.5)
    axes = rng.choice([0, 1, 3])
    return dict(kind=kind, layers=layers, heads=rng.choice([1, 2, 4, 8]), G=rng.choice([0, 1, 5, 8]) if axes else 0, d=d,
                seqs=min(seqs, 4), seq_len=seq_len, fill=rng.choice([1.0, 0.5]), page=page, e4m3=rng.random() < 0.5,
                axes=axes, style=rng.choice([0, 1]), token_major=rng.random() < 0.5)


# --------------------------------------------------------------------------------------------------------- lengths

def _rng(case):
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _attn_lengths(case):
    """(new tokens, cached and new tokens) of every request, in a mixed order."""
    rng = _rng(case)
    out = []
    for i in range(case["decode"] + case["chunks"]):
        lo, hi = case["kv_min"], case["kv_max"]
        kv = _log(rng, lo, hi) if hi > lo else hi
        q = 1 if i < case["decode"] else case["q_len"]
        out.append((q, max(kv, q)))
    rng.shuffle(out)
    return out


def _table_lengths(case):
    rng = _rng(case)
    return [(rng.randint(0, case["ctx_max"]), _log(rng, max(1, case["q_min"]), max(1, case["q_max"]))
             if rng.random() < 0.95 or case["q_min"] else 0) for _ in range(case["reqs"])]


def _row_lengths(case):
    """Tokens of every sequence of a padded batch that are there."""
    rng = _rng(case)
    lo = max(1, int(case["fill"] * case["seq_len"]))
    return [rng.randint(lo, case["seq_len"]) for _ in range(case["seqs"])]


def _visible(q, kv, window, sinks):
    """(row, key) pairs that are visible, and keys that some row sees."""
    pairs = 0
    for i in range(q):
        p = kv - q + i
        pairs += p + 1 if not window or window > p else window + min(sinks, p + 1 - window)
    first = max(0, kv - q - window + 1) if window else 0
    return pairs, kv - first + min(sinks, first)


def work(case):
    kind, d = case["kind"], case.get("d", 0)
    if kind == "attn":
        el = 1 if case["e4m3"] else 2
        bytes_ = flops = 0
        for q, kv in _attn_lengths(case):
            pairs, keys = _visible(q, kv, case["window"], case["sinks"])
            rows = q * case["H"] * case["G"]
            bytes_ += rows * (4 * d + 4) + 2 * keys * case["H"] * d * el + 4 * (kv // case["page"])
            flops += 4 * d * pairs * case["H"] * case["G"]
        return {"bytes": bytes_, "flops": flops}
    if kind == "tables":
        lens = _table_lengths(case)
        new = sum(-(-(c + q) // case["page"]) - -(-c // case["page"]) for c, q in lens)
        return {"bytes": 20 * len(lens) + 8 * new + 8 * sum(q for _, q in lens), "flops": sum(q for _, q in lens)}
    rows = case["layers"] * case["heads"]
    if kind == "rope":                                        # out of place: values are copied
        tok = case["seqs"] * case["seq_len"]
        return {"bytes": tok * (rows * 8 * d + 4 * case["axes"]), "flops": 3 * tok * rows * d}
    tok = sum(_row_lengths(case))
    el = 1 if case["e4m3"] else 2
    qh = case["heads"] * case["G"]
    return {"bytes": tok * (2 * rows * d * (2 + el) + 4 * qh * d + 4 * (1 + case["axes"])),
            "flops": tok * d * (3 * (rows + qh) if case["axes"] else 0) + (2 * tok * rows * d if case["e4m3"] else 0) + 1}


# ---------------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _pool_shape(case, layers, n_pages, heads):
    """A pool [layer][2][page][head][token][channel], stored by head or by token inside a page."""
    page, d = case["page"], case["d"]
    if case["token_major"]:
        return (layers, 2, n_pages, page, heads, d), (0, 1, 2, 4, 3, 5)
    return (layers, 2, n_pages, heads, page, d), (0, 1, 2, 3, 4, 5)


def _rows(case, g):
    """A cache [layer][2][seq][head][token][channel]: channels of different size, keys with offsets."""
    L, H, d, B, T = case["layers"], case["heads"], case["d"], case["seqs"], case["seq_len"]
    shape = (L, 2, B, T, H, d) if case["token_major"] else (L, 2, B, H, T, d)
    x = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    size = torch.exp(0.5 * torch.randn(d, generator=g, device=DEV))
    for l in range(L):
        x[l] = torch.randn(shape[1:], generator=g, device=DEV, dtype=torch.bfloat16) * size.to(torch.bfloat16)
    return x.permute(0, 1, 2, 4, 3, 5) if case["token_major"] else x


def _positions(case, n):
    """Text and images in turn: text counts on in every axis, an image of 16 x 24 stands at one time."""
    axes = max(1, case["axes"])
    pos, at, i = [[], [], []], 0, 0
    while len(pos[0]) < n:
        for _ in range(min(96, n - len(pos[0]))):
            for a in range(3):
                pos[a].append(at)
            at += 1
        for j in range(min(384, n - len(pos[0]))):
            pos[0].append(at)
            pos[1].append(at + j // 24)
            pos[2].append(at + j % 24)
        at += 24
    if axes == 1:
        pos = [list(range(n))]
    return torch.tensor(pos[:axes], dtype=torch.int32, device=DEV)


def _axis(d, axes):
    """The axis of each of the d / 2 pairs: a quarter to time, the rest shared."""
    h = d // 2
    if axes <= 1:
        return [0] * h
    if axes == 2:
        return [0] * (h // 2) + [1] * (h - h // 2)
    a, b = h // 4, (h - h // 4) // 2
    return [0] * a + [1] * b + [2] * (h - a - b)


def _table(d, n_pos):
    f = THETA ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d)
    ang = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * f
    return torch.stack([ang.cos(), ang.sin()], dim=-1).to(torch.float32).contiguous()


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind == "attn":
        lens = _attn_lengths(case)
        H, G, d, page = case["H"], case["G"], case["d"], case["page"]
        width = max(-(-kv // page) for _, kv in lens)
        used = [-(-kv // page) for _, kv in lens]
        n_pages = sum(used) + 3
        perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
        at = 0
        for r, u in enumerate(used):
            table[r, :u] = perm[at:at + u]
            at += u
        n = sum(q for q, _ in lens) + case["pad"]
        shape, order = _pool_shape(case, 1, n_pages, H)
        size = torch.exp(0.3 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
        pool = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
        pool *= size
        s["scales"] = None
        if case["e4m3"]:
            s["scales"] = (0.01 + 0.02 * torch.rand((1, 2, H), generator=g, device=DEV))
            pool = (pool * 40.0).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        s["pool"] = pool.permute(order)
        s["q"] = 2.0 * torch.randn((n, H * G, d), generator=g, device=DEV, dtype=torch.bfloat16)
        starts = [0]
        for q, _ in lens:
            starts.append(starts[-1] + q)
        s["lens"] = lens
        s["max_q"] = max(q for q, _ in lens)
        s["q_starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
        s["kv_lens"] = torch.tensor([kv for _, kv in lens], dtype=torch.int32, device=DEV)
        s["block_table"] = table
        s["out"] = torch.zeros((n, H * G, d), dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.zeros((n, H * G), dtype=torch.float32, device=DEV)
        if own:
            import paper_2609_00891_amd as cb
            s["cb"] = cb
            s["pages"] = cb.page_pool(s["pool"], s["scales"])
            need = cb.cb_attn_paged_workspace_bytes(n, len(lens), H * G, H, d, s["max_q"])
            s["workspace"] = torch.empty((need,), dtype=torch.uint8, device=DEV)
    elif kind == "tables":
        lens, page = _table_lengths(case), case["page"]
        have = [-(-c // page) for c, _ in lens]
        total = [-(-(c + q) // page) for c, q in lens]
        new = sum(total) - sum(have)
        n_free = max(0, new + case["spare"])
        perm = torch.randperm(sum(have) + n_free, generator=g, device=DEV).to(torch.int32)
        table = torch.full((len(lens), max(1, max(total))), -1, dtype=torch.int32, device=DEV)
        at = 0
        for r, u in enumerate(have):
            table[r, :u] = perm[at:at + u]
            at += u
        n = sum(q for _, q in lens) + case["pad"]
        s["ctx_lens"] = torch.tensor([c for c, _ in lens], dtype=torch.int32, device=DEV)
        s["q_lens"] = torch.tensor([q for _, q in lens], dtype=torch.int32, device=DEV)
        s["free"] = perm[at:].contiguous()
        s["block_table"] = table
        for name, m in (("q_starts", len(lens) + 1), ("kv_lens", len(lens)), ("info", len(lens)), ("n_used", 1),
                        ("slots", n), ("positions", n)):
            s[name] = torch.zeros((m,), dtype=torch.int32, device=DEV)
        if own:
            import paper_2609_00891_amd as cb
            s["cb"] = cb
    else:
        n = case["seqs"] * case["seq_len"]
        s["rows"] = _rows(case, g)
        axes = case["axes"]
        if axes:
            s["positions"] = _positions(case, n)
            s["table"] = _table(case["d"], int(s["positions"].max()) + 1)
            s["axis"] = _axis(case["d"], axes)
        if kind == "rope":
            s["out"] = torch.empty_like(s["rows"])
        else:
            page = case["page"]
            lens = _row_lengths(case)
            used = [-(-t // page) for t in lens]
            n_pages = sum(used) + 2
            perm = torch.randperm(n_pages, generator=g, device=DEV)
            slots = torch.full((case["seqs"], case["seq_len"]), -1, dtype=torch.int64, device=DEV)
            at = 0
            for b, (t, u) in enumerate(zip(lens, used)):
                tok = torch.arange(t, device=DEV)
                slots[b, :t] = perm[at:at + u][tok // page] * page + tok % page
                at += u
            s["slots"] = slots.reshape(-1).to(torch.int32)
            shape, order = _pool_shape(case, case["layers"], n_pages, case["heads"])
            pool = torch.full(shape, 0.5, dtype=torch.bfloat16, device=DEV)
            s["scales"] = None
            if case["e4m3"]:
                pool = pool.to(torch.float8_e4m3fn)
                s["scales"] = 0.02 + 0.03 * torch.rand((case["layers"], 2, case["heads"]), generator=g, device=DEV)
            s["pool"] = pool.permute(order)
            if case["G"]:
                s["q"] = torch.randn((n, case["heads"] * case["G"], case["d"]), generator=g, device=DEV,
                                     dtype=torch.bfloat16)
                s["q_out"] = torch.zeros_like(s["q"])
        if own:
            import paper_2609_00891_amd as cb
            s["cb"] = cb
            s["rope"] = cb.rope_axes_spec(s["table"], s["positions"], s["axis"], case["style"]) if axes else None
            if kind == "write":
                s["pages"] = cb.page_pool(s["pool"], s["scales"])
    return s


# ------------------------------------------------------------------------------------------------------------- run

def run(s):
    c = s["case"]
    if c["kind"] == "attn":
        if own:
            s["cb"].cb_attn_paged(s["q"], s["pages"], 0, s["q_starts"], s["kv_lens"], s["block_table"], s["out"],
                                  s["max_q"], window=c["window"], sinks=c["sinks"], lse=s["lse"],
                                  workspace=s["workspace"])
        else:
            _plain_attn(s)
        return {"out": s["out"], "lse": s["lse"]}
    if c["kind"] == "tables":
        if own:
            s["cb"].cb_page_tables(s["ctx_lens"], s["q_lens"], s["free"], c["page"], s["block_table"], s["q_starts"],
                                   s["kv_lens"], s["slots"], s["positions"], s["info"], s["n_used"])
        else:
            _plain_tables(s)
        return {k: s[k] for k in ("block_table", "q_starts", "kv_lens", "slots", "positions", "info", "n_used")}
    if c["kind"] == "rope":
        if own:
            s["cb"].cb_rope_axes(s["rows"], s["out"], s["rope"], inverse=c["inverse"])
        else:
            _plain_rope(s)
        return {"out": s["out"]}
    if own:
        s["cb"].cb_page_write(s["rows"], s["pages"], s["slots"], rope=s["rope"], q=s.get("q"), q_out=s.get("q_out"))
    else:
        _plain_write(s)
    out = {"pool": s["pool"]}
    if c["G"]:
        out["q_out"] = s["q_out"]
    return out


def _mask(q, kv, window, sinks):
    p = torch.arange(kv - q, kv, device=DEV)[:, None]
    j = torch.arange(kv, device=DEV)[None, :]
    see = j <= p
    if window:
        see &= (j > p - window) | (j < sinks)
    return see


def _plain_attn(s):
    c = s["case"]
    H, G, d, page = c["H"], c["G"], c["d"], c["page"]
    at = 0
    for r, (q, kv) in enumerate(s["lens"]):
        pages = s["block_table"][r, :-(-kv // page)].long()
        K, V = (s["pool"][0, z].view(torch.uint8 if c["e4m3"] else torch.bfloat16)[pages].view(s["pool"].dtype)
                for z in range(2))
        K, V = (x.permute(1, 0, 2, 3).reshape(H, -1, d)[:, :kv].float() for x in (K, V))
        if c["e4m3"]:
            K, V = K * s["scales"][0, 0][:, None, None], V * s["scales"][0, 1][:, None, None]
        Q = s["q"][at:at + q].float().view(q, H, G, d).permute(1, 2, 0, 3).reshape(H, G * q, d) / math.sqrt(d)
        hide = ~_mask(q, kv, c["window"], c["sinks"]).repeat(G, 1)
        step = H if H * G * q * kv < 1 << 26 else 1           # heads at a time
        for h in range(0, H, step):
            S = torch.matmul(Q[h:h + step], K[h:h + step].transpose(1, 2).contiguous())
            S.masked_fill_(hide, -math.inf)
            m = S.amax(-1, keepdim=True)
            S.sub_(m).exp_()
            l = S.sum(-1, keepdim=True)
            o = torch.matmul(S, V[h:h + step]) / l
            n = o.shape[0]
            s["out"][at:at + q, h * G:(h + n) * G] = o.view(n * G, q, d).transpose(0, 1).to(torch.bfloat16)
            s["lse"][at:at + q, h * G:(h + n) * G] = (m + l.log()).view(n * G, q).transpose(0, 1)
        at += q


def _plain_tables(s):
    c = s["case"]
    page, table = c["page"], s["block_table"]
    ctx, q = s["ctx_lens"].long(), s["q_lens"].long()
    R, width = table.shape
    n, n_free = s["slots"].numel(), s["free"].numel()
    have, total = (ctx + page - 1) // page, (ctx + q + page - 1) // page
    need = torch.where(total > width, 0, total - have)
    base = need.cumsum(0) - need
    start = q.cumsum(0) - q
    info = torch.where(total > width, 2, torch.where((need > 0) & (base + need > n_free), 1, 0))
    fits = info == 0
    j = torch.arange(width, device=DEV)[None, :]
    new = fits[:, None] & (j >= have[:, None]) & (j < total[:, None])
    at = base[:, None] + j - have[:, None]
    if n_free:
        table.copy_(torch.where(new, s["free"][at.clamp(0, n_free - 1)], table))
    s["n_used"].copy_((need * fits).sum())
    s["q_starts"][0] = 0
    s["q_starts"][1:] = q.cumsum(0)
    s["kv_lens"].copy_(torch.where(fits, ctx + q, 0))
    s["info"].copy_(info)
    t = torch.arange(n, device=DEV)
    r = torch.searchsorted(q.cumsum(0), t, right=True)
    there = r < R
    r = r.clamp(max=R - 1)
    pos = ctx[r] + t - start[r]
    ok = there & fits[r]
    page_id = table[r, (pos // page).clamp(0, width - 1)].long()
    s["slots"].copy_(torch.where(ok, page_id * page + pos % page, -1))
    s["positions"].copy_(torch.where(ok, pos, -1))


def _turn(x, table, positions, axis, style, inverse):
    """x [..., token, channel] in 32 or 64 bits, turned by its positions' angles."""
    h = x.shape[-1] // 2
    pos = positions[torch.tensor(axis, device=DEV)].long()                       # [pair][token]
    cs = table.to(x.dtype)[pos, torch.arange(h, device=DEV)[:, None]]            # [pair][token][2]
    co, si = cs[..., 0].T, cs[..., 1].T
    if inverse:
        si = -si
    if style == 0:
        a, b = x[..., :h], x[..., h:]
        return torch.cat([a * co - b * si, b * co + a * si], dim=-1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * co - b * si, b * co + a * si], dim=-1).flatten(-2)


def _plain_rope(s):
    c, x = s["case"], s["rows"]
    L, _, B, H, T, d = x.shape
    s["out"][:, 1] = x[:, 1]
    for l in range(L):
        for b in range(B):
            pos = s["positions"][:, b * T:(b + 1) * T]
            y = _turn(x[l, 0, b].float(), s["table"], pos, s["axis"], c["style"], c["inverse"])
            s["out"][l, 0, b] = y.to(torch.bfloat16)


def _plain_write(s):
    c, x = s["case"], s["rows"]
    L, _, B, H, T, d = x.shape
    page = c["page"]
    keep = (s["slots"] >= 0).nonzero()[:, 0]
    slot = s["slots"][keep].long()
    raw = s["pool"].view(torch.uint8) if c["e4m3"] else s["pool"]
    pos = s["positions"][:, keep] if c["axes"] else None
    for l in range(L):
        for z in range(2):
            y = x[l, z].transpose(0, 1).reshape(H, B * T, d)[:, keep].float()
            if z == 0 and c["axes"]:
                y = _turn(y, s["table"], pos, s["axis"], c["style"], False)
            if c["e4m3"]:
                y = (y * (1.0 / s["scales"][l, z])[:, None, None]).clamp(-E4M3_MAX, E4M3_MAX)
                y = y.to(torch.float8_e4m3fn).view(torch.uint8)
            else:
                y = y.to(torch.bfloat16)
            raw[l, z][slot // page, :, slot % page] = y.transpose(0, 1)
    if c["G"]:
        y = _turn(s["q"][keep].transpose(0, 1).float(), s["table"], pos, s["axis"], c["style"], False)
        s["q_out"][keep] = y.transpose(0, 1).to(torch.bfloat16)


# ----------------------------------------------------------------------------------------------------------- exact

def exact(case, seed):
    """The outputs in 64 bits from the definitions, head by head and token by token's position."""
    s = prepare(case, seed)
    if case["kind"] == "tables":
        return None
    if case["kind"] == "attn":
        return _exact_attn(s)
    c = case
    x = s["rows"]
    L, _, B, H, T, d = x.shape
    h = d // 2
    if c["axes"]:
        i = torch.arange(h, device=DEV)
        which = s["positions"].long()[torch.tensor(s["axis"], device=DEV)]       # [pair][token]
        ang = s["table"].double()[which.T, i]                                    # [token][pair][2]
        z = torch.complex(ang[..., 0], ang[..., 1])
        if c.get("inverse"):
            z = z.conj()

    def turned(rows, zt):                                                        # rows [..., channel], zt [..., pair]
        pairs = torch.stack([rows[..., :h], rows[..., h:]], -1) if c["style"] == 0 else rows.unflatten(-1, (h, 2))
        w = torch.view_as_real(torch.view_as_complex(pairs.double().contiguous()) * zt)
        return torch.cat([w[..., 0], w[..., 1]], -1) if c["style"] == 0 else w.flatten(-2)

    if c["kind"] == "rope":
        out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
        for l in range(L):
            out[l, 1] = x[l, 1].double()
            out[l, 0] = turned(x[l, 0], z.view(B, 1, T, h))
        return {"out": out}
    pool = s["pool"].double()
    ok = s["slots"] >= 0
    slot = s["slots"].long()[ok]
    pg, off = slot // c["page"], slot % c["page"]
    for l in range(L):
        for k in range(2):
            y = x[l, k].permute(0, 2, 1, 3).reshape(B * T, H, d)[ok].double()
            if k == 0 and c["axes"]:
                y = turned(y, z[ok][:, None])
            if c["e4m3"]:
                y = (y / s["scales"][l, k].double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
            pool[l, k, pg, :, off] = y
    out = {"pool": pool}
    if c["G"]:
        qo = s["q_out"].double()
        qo[ok] = turned(s["q"][ok], z[ok][:, None])
        out["q_out"] = qo
    return out


def _exact_attn(s):
    c = s["case"]
    H, G, d, page = c["H"], c["G"], c["d"], c["page"]
    if work(c)["flops"] > 5e12:
        return None
    out, lse = s["out"].double(), s["lse"].double()
    starts = s["q_starts"].tolist()
    for r, (q, kv) in enumerate(s["lens"]):
        tok = torch.arange(kv, device=DEV)
        pg, off = s["block_table"][r].long()[tok // page], tok % page
        for h in range(H):
            kr, vr = (s["pool"][0, z, :, h].contiguous().view(torch.uint8 if c["e4m3"] else torch.int16)[pg, off]
                      .view(s["pool"].dtype).double() for z in range(2))
            if c["e4m3"]:
                kr, vr = kr * s["scales"][0, 0, h].double(), vr * s["scales"][0, 1, h].double()
            rows = s["q"][starts[r]:starts[r + 1], h * G:(h + 1) * G].double().reshape(q * G, d)
            block = max(1, (1 << 27) // kv)
            for a in range(0, q * G, block):
                z = rows[a:a + block] @ kr.T * d ** -0.5
                p = kv - q + torch.arange(a, a + z.shape[0], device=DEV)[:, None] // G
                gone = tok > p
                if c["window"]:
                    gone = gone | ((tok <= p - c["window"]) & (tok >= c["sinks"]))
                z = z.masked_fill(gone, -math.inf)
                e = torch.logsumexp(z, -1)
                o = torch.exp(z - e[:, None]) @ vr
                t = starts[r] + torch.arange(a, a + z.shape[0], device=DEV) // G
                u = h * G + torch.arange(a, a + z.shape[0], device=DEV) % G
                out[t, u], lse[t, u] = o, e
    return {"out": out, "lse": lse}

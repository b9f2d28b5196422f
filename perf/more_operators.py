"""Serving a receiver from 8-bit pages whose scales are found as they are written, and attending to selected pages only:
the operators case by case, in plain form and as calls.

* ``quant``   rows of a cache into 8-bit pages, a scale found for every page, head and K or V, keys turned on the way
              with the step's queries beside them (``cb_page_quantize``);
* ``read``    pages back into a cache of rows, keys turned back (``cb_page_read``);
* ``attn``    attention over pages whose scales belong to a page and head (``cb_attn_paged``);
* ``select``  least and greatest key channels of the pages that a step changed, and the pages that every query of the
              step attends to, by a bound on their scores (``cb_page_bounds``, ``cb_page_select``);
* ``sparse``  attention of every query over its selected pages (``cb_attn_selected``).

With ``own`` false every operator is computed from elementary torch operations in 32 bits, the scores that decide a
selection in 64.  Geometries are the repository's own: 64 layers x 8 KV heads x 128 with 64 query heads (the receiver),
40 layers (the sender), heads of 96 and of 64.
"""
import math
import random

import torch

own = False

DEV = "cuda"
THETA = 1e6
E4M3_MAX = 448.0
TURNED_MAX = 316.0             # keys that will be turned: a turn makes a channel larger by up to sqrt(2)
E_MIN = -64                    # exponent of the smallest scale


# ---------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one layer's write of a decode step: 64 requests, their queries turned beside
        dict(name="quant_decode", kind="quant", layers=1, heads=8, G=8, d=128, reqs=64, q_min=1, q_max=1, ctx_max=2048,
             page=16, axes=1, style=0, token_major=True),
        # one layer of a prompt step: three chunks that begin inside a page, images among the text, heads of 96
        dict(name="quant_chunks", kind="quant", layers=1, heads=8, G=5, d=96, reqs=3, q_min=515, q_max=700, ctx_max=4000,
             page=64, axes=3, style=1, token_major=True),
        # four mapped caches of up to 2,048 tokens into pages, every layer, keys turned
        dict(name="quant_handoff", kind="quant", layers=64, heads=8, G=0, d=128, reqs=4, q_min=1229, q_max=2048, ctx_max=0,
             page=64, axes=3, style=0, token_major=False),
        # one layer of four short conversations of a small model read back
        dict(name="read_small", kind="read", layers=1, heads=2, d=64, reqs=4, q_min=40, q_max=300, page=16, pool="blocks",
             axes=0, style=0, token_major=False),
        # a sender's context read from its pages for the mapping, keys turned back to content coordinates
        dict(name="read_context", kind="read", layers=40, heads=8, d=128, reqs=1, q_min=8191, q_max=8191, page=64,
             pool="blocks", axes=1, style=0, token_major=False),
        # the smallest decode step, where only latency counts
        dict(name="attn_decode_tiny", kind="attn", decode=4, chunks=0, q_len=1, kv_min=40, kv_max=300, H=2, G=2, d=64,
             page=16, window=0, sinks=0, pad=0, token_major=False),
        # one layer's attention of a decode step over 64 requests of very different lengths: bandwidth
        dict(name="attn_decode_batch", kind="attn", decode=64, chunks=0, q_len=1, kv_min=512, kv_max=16384, H=8, G=8,
             d=128, page=16, window=0, sinks=0, pad=8, token_major=False),
        # the receiver reads 2,048 new tokens behind a transferred context: matrix products
        dict(name="attn_chunk", kind="attn", decode=0, chunks=1, q_len=2048, kv_min=32768, kv_max=32768, H=8, G=8,
             d=128, page=64, window=0, sinks=0, pad=0, token_major=False),
        # a decode step's choice of 64 pages in contexts of 4,096 to 65,536 tokens
        dict(name="select_decode", kind="select", reqs=48, q_len=1, kv_min=4096, kv_max=65536, H=8, G=8, d=128, page=32,
             pool="bf16", first=1, last=2, n_selected=64, token_major=False),
        # the choices of a chunk of 1,024 new tokens behind a long context
        dict(name="select_chunk", kind="select", reqs=1, q_len=1024, kv_min=32768, kv_max=32768, H=8, G=8, d=128, page=64,
             pool="blocks", first=1, last=2, n_selected=64, token_major=False),
        # the decode step's attention over the chosen pages
        dict(name="sparse_decode", kind="sparse", reqs=48, q_len=1, kv_min=4096, kv_max=65536, H=8, G=8, d=128, page=32,
             pool="bf16", first=1, last=2, n_selected=64, token_major=False),
        # a chunk's attention over the chosen 8-bit pages
        dict(name="sparse_chunk", kind="sparse", reqs=1, q_len=512, kv_min=32768, kv_max=32768, H=8, G=8, d=128, page=64,
             pool="blocks", first=1, last=2, n_selected=64, token_major=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["quant", "quant", "read", "attn", "attn", "select", "sparse", "sparse"])
    page = rng.choice([8, 16, 24, 32, 64, 100, 128])
    d = rng.choice([64, 96, 128, 128])
    heads = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 4, 5, 7, 8, 16])
    c = dict(kind=kind, d=d, page=page, token_major=rng.random() < 0.5)
    if kind in ("quant", "read"):
        axes = rng.choice([0, 1, 3])
        c.update(heads=heads, layers=_log(rng, 1, 64 if kind == "quant" else 40), axes=axes, style=rng.choice([0, 1]),
                 q_max=_log(rng, 1, 2048 if kind == "quant" else 4096))
        c["q_min"] = rng.choice([1, c["q_max"]])
        c["reqs"] = _log(rng, 1, max(1, min(256, 8192 // c["q_max"])))
        if kind == "quant":
            c.update(G=rng.choice([0, 1, 5, 8]) if axes else 0, ctx_max=rng.choice([0, _log(rng, 1, 2048)]))
            if c["ctx_max"] and c["layers"] * c["reqs"] > 256:               # the pool of the contexts has to fit
                c["layers"] = max(1, 256 // c["reqs"])
        else:
            c["pool"] = rng.choice(["blocks", "blocks", "e4m3", "bf16"])
        return c
    if kind == "attn":
        window = rng.choice([0, 0, _log(rng, 16, 8192)])
        c.update(H=heads, G=G, window=window, sinks=rng.choice([0, 1, 4, 70]) if window else 0, pad=rng.choice([0, 0, 3, 17]))
        form = rng.choice(["decode", "few", "chunk", "mixed"])
        if form == "decode":
            n = _log(rng, 1, 256)
            top = _log(rng, 64, min(131072, 1048576 // n))
            return dict(c, decode=n, chunks=0, q_len=1, kv_min=rng.choice([1, max(1, top // 8)]), kv_max=top)
        if form == "few":                                     # a few tokens checked at once
            n = _log(rng, 1, 64)
            top = _log(rng, 64, min(32768, 1048576 // n))
            return dict(c, decode=0, chunks=n, q_len=rng.randint(2, 9), kv_min=max(1, top // 4), kv_max=top)
        q = _log(rng, 10, 2048)
        top = max(q, _log(rng, 64, 16384))
        return dict(c, decode=rng.randint(1, 40) if form == "mixed" else 0, chunks=rng.randint(1, 3), q_len=q,
                    kv_min=max(1, top // 3), kv_max=top)
    q = rng.choice([1, 1, rng.randint(2, 9), _log(rng, 10, 512)])
    n = _log(rng, 1, 64) if q < 10 else rng.randint(1, 2)
    top = max(q, _log(rng, 64, min(65536, 1048576 // n)))
    k = _log(rng, 4, 128)
    k = max(4, min(k, 2 ** 30 // (n * q * heads * page * d)))
    first = rng.randint(0, 2)
    return dict(c, H=heads, G=G, reqs=n, q_len=q, kv_min=max(1, top // 4), kv_max=top, n_selected=k, first=first,
                last=rng.randint(1, 2), pool=rng.choice(["bf16", "blocks", "e4m3"]))


# --------------------------------------------------------------------------------------------------------- lengths

def _rng(case):
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lengths(case):
    """(new tokens, cached and new tokens) of every request of a step, in a mixed order."""
    rng = _rng(case)
    n = case["decode"] + case["chunks"] if case["kind"] == "attn" else case["reqs"]
    out = []
    for i in range(n):
        if case["kind"] in ("quant", "read"):
            q = _log(rng, case["q_min"], case["q_max"])
            kv = q + (rng.randint(0, case["ctx_max"]) if case["kind"] == "quant" else 0)
        else:
            kv = _log(rng, case["kv_min"], case["kv_max"])
            q = 1 if case["kind"] == "attn" and i < case["decode"] else case["q_len"]
        out.append((q, max(kv, q)))
    rng.shuffle(out)
    return out


def _visible(q, kv, window, sinks):
    """(row, key) pairs that are visible, and keys that some row sees."""
    pairs = 0
    for i in range(q):
        p = kv - q + i
        pairs += p + 1 if not window or window > p else window + min(sinks, p + 1 - window)
    first = max(0, kv - q - window + 1) if window else 0
    return pairs, kv - first + min(sinks, first)


def work(case):
    kind, d, page = case["kind"], case["d"], case["page"]
    lens = _lengths(case)
    n = sum(q for q, _ in lens)
    if kind in ("quant", "read"):
        rows = case["layers"] * case["heads"]
        el = 2 if case.get("pool") == "bf16" else 1
        pages = sum((kv - 1) // page - (kv - q) // page + 1 for q, kv in lens) if case.get("pool", "blocks") == "blocks" else 0
        qh = case["heads"] * case.get("G", 0)
        return {"bytes": n * (2 * rows * d * (2 + el) + 4 * qh * d + 4 * case["axes"]) + 8 * pages * rows,
                "flops": n * d * (3 * (rows + qh) if case["axes"] else 0) + 2 * n * rows * d}
    H, G = case["H"], case["G"]
    if kind == "attn":
        bytes_ = flops = 0
        for q, kv in lens:
            pairs, keys = _visible(q, kv, case["window"], case["sinks"])
            bytes_ += q * H * G * (4 * d + 4) + keys * H * (2 * d + 8 / page) + 4 * (kv // page)
            flops += 4 * d * pairs * H * G
        return {"bytes": bytes_, "flops": flops}
    el, k = 2 if case["pool"] == "bf16" else 1, case["n_selected"]
    bytes_ = flops = 0
    for q, kv in lens:
        if kind == "select":
            every, new = (kv - 1) // page + 1, (kv - 1) // page - (kv - q) // page + 1
            bytes_ += H * d * el * (2 * every + new * page + 2 * new) + q * H * (2 * G * d + 4 * k)
            flops += sum(((kv - q + i) // page + 1) * 4 * d * H for i in range(q)) + 2 * new * page * H * d
        else:
            keys = sum(min(k * page, kv - q + i + 1) for i in range(q))
            bytes_ += H * (2 * d * el * min(keys, kv) + q * (G * (4 * d + 4) + 4 * k))
            flops += 4 * d * G * H * keys
    return {"bytes": bytes_, "flops": flops}


# ---------------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _pages(case, lens, g, spare):
    """A block table in which every request's pages lie anywhere in the pool, and the pool's pages."""
    page = case["page"]
    used = torch.tensor([-(-kv // page) for _, kv in lens], device=DEV)
    width, total = int(used.max()), int(used.sum())
    perm = torch.randperm(total + spare, generator=g, device=DEV).to(torch.int32)
    j = torch.arange(width, device=DEV)[None, :]
    at = (used.cumsum(0) - used)[:, None] + j
    return torch.where(j < used[:, None], perm[at.clamp(max=total + spare - 1)], -1).to(torch.int32), total + spare


def _stored(case, shape, make):
    """make(shape) stored [.., head, token, channel] or [.., token, head, channel], seen as the former."""
    if not case["token_major"]:
        return make(shape)
    return make(shape[:-3] + (shape[-2], shape[-3], shape[-1])).transpose(-3, -2)


def _exponents(amax, limit):
    """The least e >= E_MIN with amax <= limit 2^e."""
    m, e = torch.frexp(amax.double() / limit)
    return torch.where(amax > 0, torch.where(m == 0.5, e - 1, e), E_MIN).clamp(min=E_MIN)


def _power(e):
    """2^e in 32 bits."""
    return torch.ldexp(torch.ones_like(e, dtype=torch.float64), e).float()


def _pool(case, layers, n_pages, heads, kind, g):
    """A pool in use [layer][2][page][head][token][channel] and its scales."""
    d, page = case["d"], case["page"]
    shape = (layers, 2, n_pages, heads, page, d)
    size = torch.exp(0.3 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
    x = _stored(case, shape, lambda s: torch.randn(s, generator=g, device=DEV, dtype=torch.bfloat16).mul_(size))
    if kind == "bf16":
        return x, None
    # pages differ in size: their scales do
    x *= torch.exp(0.7 * torch.randn((layers, 2, n_pages, heads, 1, 1), generator=g, device=DEV)).to(torch.bfloat16)
    if kind == "e4m3":
        scales = 0.02 + 0.02 * torch.rand((layers, 2, heads), generator=g, device=DEV)
        x /= scales[:, :, None, :, None, None].to(torch.bfloat16)
        return x.clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scales
    e = _exponents(torch.maximum(x.amax((-2, -1)), -x.amin((-2, -1))), E4M3_MAX)
    x *= _power(-e)[..., None, None].to(torch.bfloat16)
    return x.to(torch.float8_e4m3fn), _power(e).permute(0, 2, 3, 1).contiguous()


def _rope(case, n):
    """Positions of n tokens, the angles' table and the axis of each of the d / 2 pairs: text, or text and images of
    16 x 24 in turn."""
    d, t = case["d"], torch.arange(n, device=DEV)
    if case["axes"] == 1:
        pos, axis = t[None], [0] * (d // 2)
    else:
        part, i = t // 480, t % 480                           # 96 tokens of text, 384 of an image that takes 24 positions
        img = (i - 96).clamp(min=0)
        base = part * 120 + i.clamp(max=96)
        pos = torch.stack([base, base + img // 24, base + img % 24])
        a, b = d // 8, 3 * d // 16
        axis = [0] * a + [1] * b + [2] * (d // 2 - a - b)
    n_pos = int(pos.max()) + 1
    f = THETA ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d)
    ang = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * f
    return pos.to(torch.int32).contiguous(), torch.stack([ang.cos(), ang.sin()], dim=-1).to(torch.float32).contiguous(), axis


def _touched(s):
    """Pages that the step's new tokens lie in: request and index of each, in the requests' order."""
    page = s["case"]["page"]
    q, kv = s["q_lens"].long(), s["kv_lens"].long()
    lo, n = (kv - q) // page, (kv - 1) // page - (kv - q) // page + 1
    r = torch.repeat_interleave(torch.arange(len(q), device=DEV), n)
    return r, lo[r] + torch.arange(len(r), device=DEV) - (n.cumsum(0) - n)[r]


def _bounds_of(s, r, i):
    """Least and greatest key channels over the tokens of page i of request r: [item][head][2][channel]."""
    c = s["case"]
    x = s["pool"][0, 0] if c["pool"] == "bf16" else s["pool"][0, 0].view(torch.uint8)
    x = x[s["block_table"][r, i].long()].view(s["pool"].dtype).float()
    there = i[:, None] * c["page"] + torch.arange(c["page"], device=DEV) < s["kv_lens"].long()[r][:, None]
    there = there[:, None, :, None]
    lo, hi = x.masked_fill(~there, math.inf).amin(2), x.masked_fill(~there, -math.inf).amax(2)
    return torch.stack([lo, hi], 2).to(s["pool"].dtype)


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    kind, d, page = case["kind"], case["d"], case["page"]
    lens = _lengths(case)
    n = sum(q for q, _ in lens)
    s["lens"] = lens
    s["q_lens"], s["kv_lens"] = _ints([q for q, _ in lens]), _ints([kv for _, kv in lens])
    s["block_table"], n_pages = _pages(case, lens, g, 3)
    if kind in ("quant", "read"):
        L, H = case["layers"], case["heads"]
        # the step's tokens packed, or a batch of caches padded to one length
        packed = kind == "quant" and case["ctx_max"] > 0
        B, T = (1, n) if packed else (len(lens), max(q for q, _ in lens))
        starts = [0]
        for q, _ in lens:
            starts.append(starts[-1] + q)
        s["row_starts"] = _ints(starts[:-1] if packed else [b * T for b in range(B)])
        size = torch.exp(0.5 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
        make = lambda shape: torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16).mul_(size)  # noqa: E731
        if kind == "quant":
            s["rows"] = _stored(case, (L, 2, B, H, T, d), make)
            s["pool"], s["scales"] = _pool(case, L, n_pages, H, "blocks", g)
            if case["G"]:
                s["q"] = torch.randn((n if packed else B * T, H * case["G"], d), generator=g, device=DEV, dtype=torch.bfloat16)
                s["q_out"] = torch.zeros_like(s["q"])
        else:
            s["rows"] = _stored(case, (L, 2, B, H, T, d), lambda shape: torch.zeros(shape, dtype=torch.bfloat16, device=DEV))
            s["pool"], s["scales"] = _pool(case, L, n_pages, H, case["pool"], g)
        if case["axes"]:
            s["positions"], s["table"], s["axis"] = _rope(case, B * T)
    else:
        H, G = case["H"], case["G"]
        s["pool"], s["scales"] = _pool(case, 1, n_pages, H, "blocks" if kind == "attn" else case["pool"], g)
        s["q"] = 2.0 * torch.randn((n + case.get("pad", 0), H * G, d), generator=g, device=DEV, dtype=torch.bfloat16)
        starts = [0]
        for q, _ in lens:
            starts.append(starts[-1] + q)
        s["q_starts"] = _ints(starts)
        s["max_q"] = max(q for q, _ in lens)
        if kind == "select":
            # the bounds of every page but the step's own
            every = -(-s["kv_lens"].long() // page)
            r = torch.repeat_interleave(torch.arange(len(lens), device=DEV), every)
            i = torch.arange(len(r), device=DEV) - (every.cumsum(0) - every)[r]
            s["bounds"] = torch.zeros((1, n_pages, H, 2, d), device=DEV).to(s["pool"].dtype)
            raw = s["bounds"].view(torch.uint8) if case["pool"] != "bf16" else s["bounds"]
            for a in range(0, len(r), 4096):
                got = _bounds_of(s, r[a:a + 4096], i[a:a + 4096])
                raw[0, s["block_table"][r[a:a + 4096], i[a:a + 4096]].long()] = got.view(raw.dtype)
            r, i = _touched(s)
            raw[0, s["block_table"][r, i].long()] = 0
        else:
            s["out"] = torch.zeros_like(s["q"])
            s["lse"] = torch.zeros(s["q"].shape[:2], dtype=torch.float32, device=DEV)
        if kind == "select":
            s["selected"] = torch.zeros((n, H, case["n_selected"]), dtype=torch.int32, device=DEV)
        if kind == "sparse":
            # neighbouring tokens want much the same pages
            own_page, r = _own_pages(s)
            width = s["block_table"].shape[1]
            drift = torch.randn((len(lens), H, width), generator=g, device=DEV)
            s["selected"] = _choose(s, drift[r] + 0.4 * torch.randn((n, H, width), generator=g, device=DEV), own_page)
    if own:
        import paper_2609_00891_amd as cb
        s["cb"] = cb
        s["pages"] = cb.page_pool(s["pool"], s["scales"])
        if kind in ("quant", "read"):
            s["rope"] = cb.rope_axes_spec(s["table"], s["positions"], s["axis"], case["style"]) if case["axes"] else None
        else:
            qh = case["H"] * case["G"]
            if kind == "attn":
                need = cb.cb_attn_paged_workspace_bytes(s["q"].shape[0], len(lens), qh, case["H"], d, s["max_q"])
            elif kind == "select":
                need = cb.cb_page_select_workspace_bytes(n, case["H"], s["block_table"].shape[1])
            else:
                need = cb.cb_attn_selected_workspace_bytes(n, qh, case["H"], d, page, case["n_selected"])
            s["workspace"] = torch.empty((need,), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------------------- run

def run(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "quant":
        if own:
            s["cb"].cb_page_quantize(s["rows"], s["pages"], s["row_starts"], s["q_lens"], s["kv_lens"], s["block_table"],
                                     rope=s["rope"], q=s.get("q"), q_out=s.get("q_out"))
        else:
            _plain_quant(s)
        # codes are e4m3 numbers, scales powers of two: both are exactly defined, and every stored value is their product
        return {k: s[k] for k in ("pool", "scales", "q_out") if k in s}
    if kind == "read":
        if own:
            s["cb"].cb_page_read(s["pages"], s["rows"], s["row_starts"], s["q_lens"], s["kv_lens"], s["block_table"],
                                 rope=s["rope"], inverse=True)
        else:
            _plain_read(s)
        return {"rows": s["rows"]}
    if kind == "select":
        if own:
            s["cb"].cb_page_bounds(s["pages"], s["bounds"], s["q_lens"], s["kv_lens"], s["block_table"], s["max_q"])
            s["cb"].cb_page_select(s["q"], s["pages"], 0, s["bounds"], s["q_starts"], s["kv_lens"], s["block_table"],
                                   s["selected"], first=c["first"], last=c["last"], workspace=s["workspace"])
        else:
            _plain_select(s)
        return {"bounds": s["bounds"], "selected": s["selected"]}
    if kind == "attn":
        if own:
            s["cb"].cb_attn_paged(s["q"], s["pages"], 0, s["q_starts"], s["kv_lens"], s["block_table"], s["out"],
                                  s["max_q"], window=c["window"], sinks=c["sinks"], lse=s["lse"],
                                  workspace=s["workspace"])
        else:
            _plain_attn(s)
    elif own:
        s["cb"].cb_attn_selected(s["q"], s["pages"], 0, s["q_starts"], s["kv_lens"], s["block_table"], s["selected"],
                                 s["out"], lse=s["lse"], workspace=s["workspace"])
    else:
        _plain_sparse(s)
    return {"out": s["out"], "lse": s["lse"]}


def _turn(x, cs, style):
    """x [.., token, .., channel] turned by cs (cos and sin) [.., token, .., pair]."""
    co, si = cs
    if style == 0:
        a, b = x.chunk(2, -1)
        return torch.cat([a * co - b * si, b * co + a * si], dim=-1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * co - b * si, b * co + a * si], dim=-1).flatten(-2)


def _angles(s, tok):
    """cos and sin [token][pair] of the tokens' positions."""
    pos = s["positions"].long()[torch.tensor(s["axis"], device=DEV)][:, tok]      # [pair][token]
    cs = s["table"][pos, torch.arange(pos.shape[0], device=DEV)[:, None]]
    return cs[..., 0].T, cs[..., 1].T


def _tokens(s):
    """Of every new token: its request, row, position, page and place in it."""
    q, kv = s["q_lens"].long(), s["kv_lens"].long()
    r = torch.repeat_interleave(torch.arange(len(q), device=DEV), q)
    i = torch.arange(len(r), device=DEV) - (q.cumsum(0) - q)[r]
    pos = kv[r] - q[r] + i
    page = s["case"]["page"]
    return r, s["row_starts"].long()[r] + i, pos, s["block_table"][r, pos // page].long(), pos % page


def _plain_quant(s):
    c = s["case"]
    x = s["rows"]
    L, _, B, H, T, d = x.shape
    _, tok, pos, page, off = _tokens(s)
    x = x.permute(2, 4, 0, 1, 3, 5).reshape(B * T, L, 2, H, d)[tok].float()     # [token][layer][2][head][channel]
    # the scales: of pages that this step begins from its rows alone, of the others at least what they were
    n_pages = s["pool"].shape[2]
    amax = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    top = torch.zeros((n_pages, L, 2, H), device=DEV)
    top.scatter_reduce_(0, page[:, None, None, None].expand_as(amax), amax, "amax")
    e_k = _exponents(top[:, :, 0], TURNED_MAX if c["axes"] else E4M3_MAX)
    e = torch.stack([e_k, _exponents(top[:, :, 1], E4M3_MAX)], 2)                # [page][layer][2][head]
    old = torch.frexp(s["scales"].permute(1, 0, 3, 2))[1] - 1
    written, begun = (torch.zeros(n_pages, dtype=torch.bool, device=DEV) for _ in range(2))
    written[page] = True
    begun[page[off == 0]] = True
    e = torch.where(begun[:, None, None, None], e, torch.maximum(e, old))
    e = torch.where(written[:, None, None, None], e, old)
    # what the pages hold already goes over to the larger scale
    raw = s["pool"].view(torch.uint8)
    r0 = (s["kv_lens"] - s["q_lens"]).long()
    there = (r0 % c["page"] > 0).nonzero()[:, 0]
    p0, n0 = s["block_table"][there, r0[there] // c["page"]].long(), r0[there] % c["page"]
    y = raw[:, :, p0].view(torch.float8_e4m3fn).float()                          # [layer][2][request][head][token][channel]
    f = _power((old - e)[p0]).permute(1, 2, 0, 3)[..., None, None]
    keep = (torch.arange(c["page"], device=DEV) < n0[:, None])[:, None, :, None]
    raw[:, :, p0] = torch.where(keep, (y * f).to(torch.float8_e4m3fn).view(torch.uint8), raw[:, :, p0])
    # the new rows
    if c["axes"]:
        cs = [v[:, None, None] for v in _angles(s, tok)]
        x[:, :, 0] = _turn(x[:, :, 0], cs, c["style"])
    x = x * _power(-e)[page][..., None]
    raw[:, :, page, :, off] = x.to(torch.float8_e4m3fn).view(torch.uint8)
    s["scales"].copy_(_power(e).permute(1, 0, 3, 2))
    if c["G"]:
        y = _turn(s["q"][tok].float(), [v[:, None] for v in _angles(s, tok)], c["style"])
        s["q_out"][tok] = y.to(torch.bfloat16)


def _plain_read(s):
    c = s["case"]
    L, _, B, H, T, d = s["rows"].shape
    _, tok, pos, page, off = _tokens(s)
    raw = s["pool"] if c["pool"] == "bf16" else s["pool"].view(torch.uint8)
    x = raw[:, :, page, :, off].view(s["pool"].dtype).float()                    # [token][layer][2][head][channel]
    if c["pool"] == "e4m3":
        x *= s["scales"][None, ..., None]
    if c["pool"] == "blocks":
        x *= s["scales"][:, page].permute(1, 0, 3, 2)[..., None]
    if c["axes"]:
        co, si = _angles(s, tok)
        x[:, :, 0] = _turn(x[:, :, 0], (co[:, None, None], -si[:, None, None]), c["style"])
    s["rows"][:, :, tok // T, :, tok % T] = x.to(torch.bfloat16)


def _keys_and_values(s, pages, heads, dt=torch.float32):
    """K and V [.., head, token, channel] of pages [..] as the numbers that they stand for."""
    kind = s["case"].get("pool", "blocks")
    out = []
    for z in range(2):
        raw = s["pool"][0, z, :, heads]
        x = (raw if kind == "bf16" else raw.view(torch.uint8))[pages].view(s["pool"].dtype).to(dt)
        if kind == "e4m3":
            x *= s["scales"][0, z, heads][:, None, None]
        if kind == "blocks":
            x *= s["scales"][0, :, heads, z][pages][..., None, None]
        out.append(x)
    return out


def _plain_attn(s):
    """Requests of equal numbers of new tokens together, padded to the longest."""
    c = s["case"]
    H, G, d, page = c["H"], c["G"], c["d"], c["page"]
    q_lens, kv_lens = s["q_lens"].long(), s["kv_lens"].long()
    for n in sorted({q for q, _ in s["lens"]}):
        r = (q_lens == n).nonzero()[:, 0]
        kv, width = kv_lens[r], -(-max(k for q, k in s["lens"] if q == n) // page)
        tok = s["q_starts"].long()[r][:, None] + torch.arange(n, device=DEV)     # [request][new token]
        pages = s["block_table"][r, :width].long().clamp(min=0)
        j = torch.arange(width * page, device=DEV)
        p = (kv[:, None] - n + torch.arange(n, device=DEV))[..., None]
        see = (j <= p) & ((j > p - c["window"]) | (j < c["sinks"]) if c["window"] else True)
        hide = ~see[:, None].repeat(1, 1, G, 1)                                  # [request][1][G x new token][key]
        step = max(1, min(H, (1 << 31) // (len(r) * G * n * width * page)))      # heads at a time
        for h in range(0, H, step):
            hs = slice(h, min(h + step, H))
            K, V = (x.transpose(1, 2).reshape(len(r), -1, width * page, d) for x in _keys_and_values(s, pages, hs))
            V.masked_fill_((j >= kv[:, None])[:, None, :, None], 0.0)
            m = K.shape[1]
            Q = s["q"].view(-1, H, G, d)[tok][:, :, hs].float().permute(0, 2, 3, 1, 4).reshape(len(r), m, G * n, d)
            S = torch.matmul(Q / math.sqrt(d), K.transpose(2, 3).contiguous()).masked_fill_(hide, -math.inf)
            top = S.amax(-1, keepdim=True)
            S.sub_(top).exp_()
            sums = S.sum(-1, keepdim=True)
            o = (torch.matmul(S, V) / sums).view(len(r), m, G, n, d).permute(0, 3, 1, 2, 4)
            s["out"].view(-1, H, G, d)[tok, hs] = o.to(torch.bfloat16)
            s["lse"].view(-1, H, G)[tok, hs] = (top + sums.log()).view(len(r), m, G, n).permute(0, 3, 1, 2)


def _own_pages(s):
    """Of every new token of a step its own page's index and its request."""
    q, kv = s["q_lens"].long(), s["kv_lens"].long()
    r = torch.repeat_interleave(torch.arange(len(q), device=DEV), q)
    i = torch.arange(len(r), device=DEV) - (q.cumsum(0) - q)[r]
    return (kv[r] - q[r] + i) // s["case"]["page"], r


def _choose(s, score, own_page):
    """The pages of the highest scores [token][head][page] among those up to the token's own, the first and the last
    ones always; equal scores go to the lower page.  In the pages' order, -1 behind them."""
    c = s["case"]
    k, width = c["n_selected"], score.shape[-1]
    j = torch.arange(width, device=DEV)
    last = own_page[:, None, None]
    key = score.float().double()
    key = torch.where(key.isnan() | (key == math.inf), 1e39, key)
    key = torch.where((j < c["first"]) | (j > last - c["last"]), math.inf, key)
    there = (j <= last).expand_as(key)
    # (a score of -infinity still comes before what is not there)
    order = torch.argsort(torch.where(there, key.clamp(min=-1e39), -math.inf), dim=-1, descending=True, stable=True)[..., :k]
    got = torch.where(torch.gather(there, -1, order), order, width).sort(-1).values
    out = torch.full(key.shape[:-1] + (k,), -1, dtype=torch.int32, device=DEV)
    out[..., :got.shape[-1]] = torch.where(got < width, got, -1)
    return out


def _plain_select(s):
    c = s["case"]
    H, G, d = c["H"], c["G"], c["d"]
    r, i = _touched(s)
    raw = s["bounds"] if c["pool"] == "bf16" else s["bounds"].view(torch.uint8)
    raw[0, s["block_table"][r, i].long()] = _bounds_of(s, r, i).view(raw.dtype)
    own_page, _ = _own_pages(s)
    R, n, table = len(s["lens"]), c["q_len"], s["block_table"]
    Q = s["q"].double().view(R, n, H, G, d)
    lo, hi = raw[0][table.long().clamp(min=0)].view(s["bounds"].dtype).double().permute(3, 0, 2, 4, 1)   # [request][head][channel][page]
    score = torch.matmul(Q.clamp(min=0).sum(3).transpose(1, 2), hi.contiguous())
    score += torch.matmul(Q.clamp(max=0).sum(3).transpose(1, 2), lo.contiguous())
    if c["pool"] == "blocks":
        score *= s["scales"][0][table.long().clamp(min=0)][..., 0].double().transpose(1, 2)[:, :, None]
    s["selected"].copy_(_choose(s, score.transpose(1, 2).reshape(R * n, H, -1), own_page))


def _plain_sparse(s):
    c = s["case"]
    H, G, d, page = c["H"], c["G"], c["d"], c["page"]
    n, _, k = s["selected"].shape
    q, kv = s["q_lens"].long(), s["kv_lens"].long()
    _, r = _own_pages(s)
    p = kv[r] - q[r] + torch.arange(n, device=DEV) - (q.cumsum(0) - q)[r]
    step = max(1, min(H, (1 << 29) // (n * k * page * d)))                       # heads at a time
    for h in range(0, H, step):
        hs = torch.arange(h, min(h + step, H), device=DEV)
        sel = s["selected"][:, hs].long()                                       # [token][head][place]
        pages = s["block_table"][r[:, None, None], sel.clamp(min=0)].long()
        K, V = _of_heads(s, pages, hs[None, :, None])
        j = (sel[..., None] * page + torch.arange(page, device=DEV)).flatten(2)
        hide = ((sel < 0).repeat_interleave(page, -1) | (j > p[:, None, None]))[:, :, None]
        K, V = (x.reshape(n, len(hs), k * page, d) for x in (K, V))
        Q = s["q"].view(n, H, G, d)[:, hs].float() / math.sqrt(d)
        S = torch.matmul(Q, K.transpose(2, 3).contiguous()).masked_fill_(hide, -math.inf)
        top = S.amax(-1, keepdim=True)
        S.sub_(top).exp_()
        sums = S.sum(-1, keepdim=True)
        s["out"].view(n, H, G, d)[:, hs] = (torch.matmul(S, V) / sums).to(torch.bfloat16)
        s["lse"].view(n, H, G)[:, hs] = (top + sums.log())[..., 0]


def _of_heads(s, pages, heads, dt=torch.float32):
    """K and V [.., token, channel] of (page, head) pairs as the numbers that they stand for."""
    kind = s["case"]["pool"]
    out = []
    for z in range(2):
        raw = s["pool"][0, z]
        x = (raw if kind == "bf16" else raw.view(torch.uint8))[pages, heads].view(s["pool"].dtype).to(dt)
        if kind == "e4m3":
            x *= s["scales"][0, z][heads][..., None, None]
        if kind == "blocks":
            x *= s["scales"][0][pages, heads][..., z][..., None, None]
        out.append(x)
    return out


# ----------------------------------------------------------------------------------------------------------- exact

def exact(case, seed):
    """The outputs in 64 bits from the definitions, request by request."""
    s = prepare(case, seed)
    if case["kind"] in ("quant", "read"):
        return _exact_rows(s)
    if work(case)["flops"] > 5e12:
        return None
    return _exact_select(s) if case["kind"] == "select" else _exact_attn(s)


def _exact_rows(s):
    c = s["case"]
    page, quant = c["page"], c["kind"] == "quant"
    L, _, B, H, T, d = s["rows"].shape
    z = None
    if c["axes"]:
        i = torch.arange(d // 2, device=DEV)
        cs = s["table"].double()[s["positions"].long()[torch.tensor(s["axis"], device=DEV)].T, i]
        z = torch.complex(cs[..., 0], cs[..., 1])                                # [row][pair]

    def turned(x, zt):                                                           # x [.., token, channel], zt [token][pair]
        pairs = torch.stack(x.chunk(2, -1), -1) if c["style"] == 0 else x.unflatten(-1, (d // 2, 2))
        w = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * zt)
        return torch.cat([w[..., 0], w[..., 1]], -1) if c["style"] == 0 else w.flatten(-2)

    def two(e):                                                                  # 2^e, which pow() may miss by an ulp
        return (2.0 ** e).float().double()

    pool = s["pool"].double()
    scales = s["scales"].double() if s["scales"] is not None else None
    q_out = s["q_out"].double() if quant and c["G"] else None
    rows = None if quant else s["rows"].double()
    starts, table = s["row_starts"].tolist(), s["block_table"].tolist()
    for r, (q, kv) in enumerate(s["lens"]):
        pos = kv - q
        if q_out is not None:
            t = slice(starts[r], starts[r] + q)
            q_out[t] = turned(s["q"][t].double().transpose(0, 1), z[t]).transpose(0, 1)
        while pos < kv:
            n = min(kv - pos, page - pos % page)
            t, P, at = starts[r] + pos - (kv - q), table[r][pos // page], pos % page
            b, u = slice(t // T, t // T + 1), slice(t % T, t % T + n)
            if quant:
                x = s["rows"][:, :, b, :, u].double()[:, :, 0]                   # [layer][2][head][token][channel]
                fin = torch.where(x.isfinite(), x.abs(), 0.0).flatten(-2).amax(-1)
                lim = torch.tensor([TURNED_MAX if z is not None else E4M3_MAX, E4M3_MAX], device=DEV, dtype=torch.float64)
                e = torch.log2(fin / lim[:, None]).ceil().clamp(min=E_MIN)       # [layer][2][head], perhaps one off
                e = torch.where(fin > lim[:, None] * two(e), e + 1, torch.where(fin <= lim[:, None] * two(e - 1), e - 1, e))
                e = e.clamp(min=E_MIN)
                if at:
                    was = scales[:, P].permute(0, 2, 1)
                    e = torch.maximum(e, torch.log2(was).round())
                    y = pool[:, :, P, :, :at] * (was / two(e))[..., None, None]
                    # (what goes over to a larger scale is rounded to 8 bits once more)
                    pool[:, :, P, :, :at] = y.float().to(torch.float8_e4m3fn).double()
                if z is not None:
                    x[:, 0] = turned(x[:, 0], z[t:t + n])
                pool[:, :, P, :, at:at + n] = x / two(e)[..., None, None]
                scales[:, P] = two(e).permute(0, 2, 1)
            else:
                x = pool[:, :, P, :, at:at + n]
                if c["pool"] == "e4m3":
                    x = x * scales[:, :, :, None, None]
                if c["pool"] == "blocks":
                    x = x * scales[:, P].permute(0, 2, 1)[..., None, None]
                if z is not None:
                    x = torch.stack([turned(x[:, 0], z[t:t + n].conj()), x[:, 1]], 1)
                rows[:, :, b, :, u] = x[:, :, None]
            pos += n
    if not quant:
        return {"rows": rows}
    return {k: v for k, v in (("pool", pool), ("scales", scales), ("q_out", q_out)) if v is not None}


def _exact_kv(s, r, h, keys):
    """K and V [key][channel] of keys of request r in head h."""
    c = s["case"]
    kind = c.get("pool", "blocks")
    P, at = s["block_table"][r].long()[keys // c["page"]], keys % c["page"]
    out = []
    for z in range(2):
        head = s["pool"][0, z, :, h]
        x = (head if kind == "bf16" else head.view(torch.uint8))[P, at].view(s["pool"].dtype).double()
        if kind == "e4m3":
            x = x * s["scales"][0, z, h].double()
        if kind == "blocks":
            x = x * s["scales"][0, P, h, z].double()[:, None]
        out.append(x)
    return out


def _exact_attn(s):
    c = s["case"]
    H, G, d, page = c["H"], c["G"], c["d"], c["page"]
    sparse = c["kind"] == "sparse"
    out, lse = s["out"].double(), s["lse"].double()
    starts = s["q_starts"].tolist()
    for r, (q, kv) in enumerate(s["lens"]):
        every = torch.arange(kv, device=DEV)
        for h in range(H):
            k, v = _exact_kv(s, r, h, every)
            rows = s["q"][starts[r]:starts[r + 1], h * G:(h + 1) * G].double().reshape(q * G, d)
            block = max(G, (1 << 26) // kv // G * G)
            for a in range(0, q * G, block):
                z = rows[a:a + block] @ k.T * d ** -0.5
                row = torch.arange(a, a + z.shape[0], device=DEV)
                p = kv - q + row[:, None] // G
                gone = every > p
                if sparse:
                    listed_ = s["selected"][starts[r] + a // G:starts[r] + (a + z.shape[0]) // G, h].long()
                    chosen = torch.zeros((listed_.shape[0], -(-kv // page) + 1), dtype=torch.bool, device=DEV)
                    chosen.scatter_(1, torch.where(listed_ < 0, chosen.shape[1] - 1, listed_), True)
                    gone = gone | ~chosen[:, :-1].repeat_interleave(page, 1)[:, :kv].repeat_interleave(G, 0)
                elif c["window"]:
                    gone = gone | ((every <= p - c["window"]) & (every >= c["sinks"]))
                z = z.masked_fill(gone, -math.inf)
                e = torch.logsumexp(z, -1)
                o = torch.exp(z - e[:, None]) @ v
                t, u = starts[r] + row // G, h * G + row % G
                out[t, u], lse[t, u] = o, e
    return {"out": out, "lse": lse}


def _exact_select(s):
    c = s["case"]
    H, G, d, page, k = c["H"], c["G"], c["d"], c["page"], c["n_selected"]
    bounds, selected = s["bounds"].double(), s["selected"].clone()
    starts, table = s["q_starts"].tolist(), s["block_table"].long()
    for r, (q, kv) in enumerate(s["lens"]):
        for i in range((kv - q) // page, (kv - 1) // page + 1):
            x = s["pool"][0, 0, table[r, i], :, :min(page, kv - i * page)].double()
            bounds[0, table[r, i], :, 0], bounds[0, table[r, i], :, 1] = x.amin(1), x.amax(1)
        pages = table[r, :(kv - 1) // page + 1]
        for h in range(H):
            lo, hi = bounds[0, pages, h].unbind(1)
            rows = s["q"][starts[r]:starts[r + 1], h * G:(h + 1) * G].double()
            score = sum((rows[:, g].clamp(min=0) @ hi.T) + (rows[:, g].clamp(max=0) @ lo.T) for g in range(G))
            if c["pool"] == "blocks":
                score = score * s["scales"][0, pages, h, 0].double()
            score = score.float()
            for t in range(q):
                own_page = (kv - q + t) // page
                always = {i for i in range(own_page + 1) if i < c["first"] or i > own_page - c["last"]}
                order = torch.sort(score[t, :own_page + 1], descending=True, stable=True).indices.tolist()
                best = [i for i in order if i not in always][:k - len(always)]
                got = sorted(always | set(best))
                selected[starts[r] + t, h] = torch.tensor(got + [-1] * (k - len(got)), dtype=torch.int32)
    return {"bounds": bounds, "selected": selected}

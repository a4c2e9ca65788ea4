"""The measured cases of the paged cache: what they are, how their inputs are made, the
operators in plain torch and the same pass through the library.

``append``  norms of queries and keys per head and the position rotation, from one projection
            row per token into q and into the pages of a layer.
``attend``  attention of new tokens over one layer of a paged cache.
``stage``   a paged cache into the contiguous layout of the eviction calls, and from there into
            other pages.

A cache's slot t of sequence s lies in page ``table[s, t // page]`` at ``t % page``.  Pages
hold bf16 values, or e4m3 ones with an fp32 scale for each layer and KV head.
"""
from __future__ import annotations

import math

import torch

own = False

BASE = dict(n_seq=1, n_layer=1, layer=0, n_kv=8, group=4, d=128, page=16, dtype="bf16", by_token=False,
            lens="even")
APPEND = dict(BASE, op="append", len0=0, B=1, rd=128, interleaved=False, norm=True, theta=1.0e6,
              evicted=False, padded=False)
ATTEND = dict(BASE, op="attend", len0=4096, B=1, causal=True, padded=False)
STAGE = dict(BASE, op="stage", len0=4096, B=0, padded=False)


def listed():
    return [
        # one user's decode step: one token of an 8B-class GQA model (latency)
        dict(APPEND, name="append_one", len0=4096, evicted=True),
        # two long prompts at once into empty pages
        dict(APPEND, name="append_prompt", n_seq=2, B=8192, page=64),
        # a decode step of a fixed batch of 256 places, some of them idle, into 8-bit pages
        dict(APPEND, name="append_batch_8bit", n_seq=256, len0=250, lens="near", page=32,
             dtype="e4m3", by_token=True, padded=True, evicted=True),
        # one user's decode step over 4096 cached tokens, one layer (latency)
        dict(ATTEND, name="attend_one"),
        # batched decode of 64 sequences around a budget of 4096
        dict(ATTEND, name="attend_batch", n_seq=64, lens="near"),
        # the same batch size over 8-bit pages, whose heads lie token by token
        dict(ATTEND, name="attend_batch_8bit", n_seq=64, lens="near", dtype="e4m3", page=32,
             by_token=True),
        # two long contexts that are not evicted: offsets beyond 32 bits
        dict(ATTEND, name="attend_long", n_seq=2, n_layer=18, layer=17, len0=131000, page=64),
        # a few long sequences among many short and empty ones, one KV head for all query heads
        dict(ATTEND, name="attend_skew", n_seq=24, n_kv=1, group=8, len0=65000, lens="skew"),
        # drafted tokens, odd head counts, a head dim that is no power of two, ragged lengths
        dict(ATTEND, name="attend_draft", n_seq=5, n_layer=2, layer=1, n_kv=3, group=5, d=96, B=4,
             len0=2500, lens="skew", page=24, padded=True),
        # a block of 128 tokens of block prompt processing at budget 2048
        dict(ATTEND, name="attend_block", B=128, len0=2048, page=128),
        # the cache of a prompt, 4096 tokens, all 36 layers
        dict(STAGE, name="stage_cache", n_layer=36),
        # ragged 8-bit sequences, a head dim that is no power of two
        dict(STAGE, name="stage_odd", n_seq=3, n_layer=24, n_kv=6, d=96, len0=1100, lens="skew",
             page=24, dtype="e4m3", by_token=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "stage", "attend", "attend", "attend"])
    c = dict(n_kv=_log_int(rng, 1, 16), group=rng.randint(1, 8),
             d=rng.choice([64, 80, 96, 128, 128, 128, 192, 256]),
             page=rng.choice([8, 16, 16, 24, 32, 64, 128]), dtype=rng.choice(["bf16", "bf16", "e4m3"]),
             by_token=rng.random() < 0.4)
    row = c["n_kv"] * c["d"]
    if op == "append":
        c["n_seq"] = _log_int(rng, 1, 256)
        heads = c["n_kv"] * (c["group"] + 2) * c["d"]
        most = max(1, (1 << 26) // (c["n_seq"] * heads))
        c["B"] = _log_int(rng, 1, min(most, 4 if c["n_seq"] > 32 else 8192))
        c["len0"] = _log_int(rng, 1, max(2, min(100000, (1 << 26) // (c["n_seq"] * row)))) - 1
        c.update(rd=rng.choice([c["d"], c["d"], c["d"] // 32 * 16]), norm=rng.random() < 0.8,
                 interleaved=rng.random() < 0.3, theta=rng.choice([1.0e4, 5.0e5, 1.0e6]),
                 evicted=rng.random() < 0.6)
        base = APPEND
    elif op == "stage":
        c.update(n_seq=_log_int(rng, 1, 16), n_layer=_log_int(rng, 1, 36))
        c["len0"] = _log_int(rng, 1, max(16, min(8192, (1 << 27) // (c["n_seq"] * c["n_layer"] * row))))
        base = STAGE
    else:
        kind = rng.random()
        c["n_seq"] = _log_int(rng, 1, 96 if kind < 0.6 else 16)
        c["B"] = 1 if kind < 0.6 else rng.randint(2, 8) if kind < 0.9 else _log_int(rng, 9, 128)
        rows = c["n_seq"] * row  # values a token of every sequence
        flops = (1 << 30) // (rows * c["group"] * c["B"])
        c["len0"] = _log_int(rng, 1, max(2, min(131000, (1 << 27) // rows, flops)))
        c.update(n_layer=rng.choice([1, 1, 2]), causal=rng.random() < 0.85)
        c["layer"] = c["n_layer"] - 1
        base = ATTEND
    more = c["n_seq"] > 1
    c["lens"] = rng.choice(["even", "near", "skew"]) if more else "even"
    c["padded"] = op != "stage" and more and rng.random() < 0.4
    return dict(base, **c)


def _lens(c):
    """Cached tokens of each sequence: len0, a little below it, or anything from none to it."""
    n, top = c["n_seq"], c["len0"]
    if c["lens"] == "even":
        return [top] * n
    if c["lens"] == "near":  # sequences around one budget
        return [top - (s * 7919 % 97) * top // 200 for s in range(n)]
    part = lambda s: int(top * ((s * 61 % 97) / 97.0) ** 3)  # noqa: E731
    return [(top, 0, 1)[s] if s < 3 else part(s) for s in range(n)]


def _news(c):
    """New tokens of each sequence: B, or down to none where the batch is padded."""
    return [(s * 5 + 1) % (c["B"] + 1) if c["padded"] and s else c["B"] for s in range(c["n_seq"])]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _rows(g, shape, channels):
    """Key- or value-like rows: per-channel spread with a few large channels
    (keys), a common offset, and some tokens with larger norms."""
    d = shape[-1]
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    spread = torch.exp(0.4 * torch.randn(d, generator=g, device="cuda"))
    spread[torch.randperm(d, generator=g, device="cuda")[:channels]] *= 4.0
    x *= spread.to(torch.bfloat16)
    x += (0.5 * torch.randn(d, generator=g, device="cuda")).to(torch.bfloat16)
    x *= 1.0 + 3.0 * (torch.rand(shape[:-1] + (1,), generator=g, device="cuda") < 0.02)
    return x


def _inputs(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    n, L, h, d, page, B = c["n_seq"], c["n_layer"], c["n_kv"], c["d"], c["page"], c["B"]
    lens, news = _lens(c), _news(c)
    x = {"len": torch.tensor(lens, dtype=torch.int32, device="cuda"), "new": None}
    if c["padded"]:
        x["new"] = torch.tensor(news, dtype=torch.int32, device="cuda")
    # pages of the pool in a random order; places of the table behind a sequence's pages hold -1
    need = [-(-(m + B) // page) for m in lens]
    P, width = sum(need) + 3, max(need) + 2
    order = torch.randperm(P, generator=g, device="cuda").int()
    at = torch.arange(width, device="cuda")[None, :]
    first = torch.tensor([sum(need[:s]) for s in range(n)], device="cuda")[:, None]
    used = at < torch.tensor(need, device="cuda")[:, None]
    x["table"] = torch.where(used, order[(first + at).clamp_max(P - 1)], -1).int()
    shape = (L, P, page, h, d) if c["by_token"] else (L, P, h, page, d)
    # the layers that the pass reads, as rows of a model; the others stay empty
    layers = slice(c["layer"], c["layer"] + 1) if c["op"] != "stage" else slice(0, L)
    for t, channels in (("k", 4), ("v", 0)):
        rows = _rows(g, (layers.stop - layers.start,) + shape[1:], channels)
        if c["dtype"] == "e4m3":
            scale = 0.25 * (0.8 + 0.4 * torch.rand((L, h), generator=g, device="cuda"))
            by = scale[layers, None, None, :, None] if c["by_token"] else scale[layers, None, :, None, None]
            rows = (rows.float() / by).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
            x[t + "_scale"] = scale
        else:
            x[t + "_scale"] = None
        if L == layers.stop - layers.start:
            pool = rows
        else:
            pool = torch.zeros(shape, dtype=torch.uint8 if c["dtype"] == "e4m3" else torch.bfloat16,
                               device="cuda").view(rows.dtype)
            pool[layers].copy_(rows)
        x[t] = pool.transpose(2, 3) if c["by_token"] else pool  # [L, P, h, page, d]
    if c["op"] == "append":
        n_q = h * c["group"]
        x["qkv"] = _rows(g, (n, B, n_q + 2 * h, d), 2)
        x["qw"] = x["kw"] = x["freq"] = x["first"] = None
        if c["norm"]:
            x["qw"] = (1.0 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(torch.bfloat16)
            x["kw"] = (1.0 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(torch.bfloat16)
        if c["rd"]:
            e = torch.arange(0, c["rd"], 2, dtype=torch.float64, device="cuda") / c["rd"]
            x["freq"] = (c["theta"] ** -e).float()
        if c["evicted"]:  # positions run ahead of the slots
            x["first"] = x["len"] + torch.randint(0, 30000, (n,), generator=g, device="cuda").int()
    elif c["op"] == "attend":
        x["q"] = _rows(g, (n, B, h * c["group"], d), 0)
    return x


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _raw(pool):
    """A pool with elements that torch can index: 8-bit floats as bytes."""
    return pool if pool.dtype == torch.bfloat16 else pool.view(torch.uint8)


def _take(pool, page, at, scale):
    """fp32 values [..., L, h, d] of the slots at (page, at) of a pool [L, P, h, page, d]."""
    rows = _raw(pool)[:, page, :, at]
    if pool.dtype == torch.bfloat16:
        return rows.float()
    return rows.view(torch.float8_e4m3fn).float() * scale[..., None]


def _put(pool, page, at, rows, scale):
    """fp32 rows [..., L, h, d] into the slots at (page, at), rounded once."""
    if pool.dtype == torch.bfloat16:
        pool[:, page, :, at] = rows.to(torch.bfloat16)
    else:
        rows = (rows / scale[..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
        _raw(pool)[:, page, :, at] = rows.view(torch.uint8)


def _turn(part, w, x, c, pos):
    """Heads [tokens, heads, d] in fp32, normed and rotated to positions [tokens]."""
    half = c["rd"] // 2
    if w is not None:
        part = part / torch.sqrt(part.square().mean(-1, keepdim=True) + 1.0e-6) * w.float()
    if not half:
        return part
    angle = pos.double()[:, None, None] * x["freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if c["interleaved"]:
        a, b = part[..., 0:2 * half:2], part[..., 1:2 * half:2]
    else:
        a, b = part[..., :half], part[..., half:2 * half]
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((ra, rb), -1).flatten(-2) if c["interleaved"] else torch.cat((ra, rb), -1)
    return torch.cat((turned, part[..., 2 * half:]), -1)


def _plain_append(s, x, c):
    n_q, h, page, layer = c["n_kv"] * c["group"], c["n_kv"], c["page"], c["layer"]
    seq, tok = s["tokens"]
    slot = x["len"].long()[seq] + tok
    pos = slot if x["first"] is None else x["first"].long()[seq] + tok
    rows = x["qkv"][seq, tok].float()
    s["q"][seq, tok] = _turn(rows[:, :n_q], x["qw"], x, c, pos).to(torch.bfloat16)
    new = (_turn(rows[:, n_q:n_q + h], x["kw"], x, c, pos), rows[:, n_q + h:])
    where = x["table"][seq, slot // page].long()
    for t, r in zip(("k", "v"), new):
        scale = None if x[t + "_scale"] is None else x[t + "_scale"][layer:layer + 1]
        _put(x[t][layer:layer + 1], where, slot % page, r[:, None], scale)
    return [s["q"], x["k"], x["v"]]


def _plain_attend(s, x, c):
    n, h, G, d, B, page, layer = (c[t] for t in ("n_seq", "n_kv", "group", "d", "B", "page", "layer"))
    cols = max(_lens(c)) + (B if c["causal"] else 0)
    t = torch.arange(cols, device="cuda")
    where = x["table"][:, t // page].long().clamp_min(0)
    keys, vals = (_take(x[m][layer:layer + 1], where, (t % page).expand(n, cols),
                        None if x[m + "_scale"] is None else x[m + "_scale"][layer:layer + 1])[:, :, 0]
                  for m in ("k", "v"))                                  # [n, cols, h, d]
    q = x["q"].float().view(n, B, h, G, d).permute(0, 2, 1, 3, 4).reshape(n, h, B * G, d)
    p = torch.matmul(q, keys.permute(0, 2, 3, 1)).view(n, h, B, G, cols) * (1.0 / math.sqrt(d))
    ends = x["len"][:, None] + (torch.arange(1, B + 1, device="cuda") if c["causal"] else
                                torch.zeros(B, dtype=torch.long, device="cuda"))
    p.masked_fill_((t >= ends[:, :, None])[:, None, :, None], -math.inf)
    top = p.amax(-1, keepdim=True) if cols else p.new_full(p.shape[:-1] + (1,), -math.inf)
    p = torch.exp(p - torch.where(torch.isinf(top), 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, h, B * G, cols), vals.permute(0, 2, 1, 3)).view(n, h, B, G, d)
    o = o / torch.where(total > 0, total, 1.0)
    e = (top + torch.log(total)).squeeze(-1)
    seq, tok = s["tokens"]
    s["out"][seq, tok] = o.permute(0, 2, 1, 3, 4).reshape(n, B, h * G, d)[seq, tok].to(torch.bfloat16)
    s["lse"][seq, tok] = e.permute(0, 2, 1, 3).reshape(n, B, h * G)[seq, tok]
    return [s["out"], s["lse"]]


def _plain_stage(s, x, c):
    page = c["page"]
    seq, t = s["tokens"]
    src, dst = (table[seq, t // page].long() for table in (x["table"], s["table2"]))
    for m in ("k", "v"):
        rows = _take(x[m], src, t % page, x[m + "_scale"])             # [tokens, L, h, d]
        s[m + "1"][seq, :, :, t] = rows.to(torch.bfloat16)
        _put(s[m + "2"], dst, t % page, s[m + "1"][seq, :, :, t].float(), x[m + "_scale"])
    s["len1"].copy_(x["len"])
    s["len2"].copy_(s["len1"])
    return [s[t] for t in ("k1", "v1", "len1", "k2", "v2", "len2")]


# ---------------------------------------------------------------------------
# one state, one pass
# ---------------------------------------------------------------------------
def prepare(case, seed):
    c, x = case, _inputs(case, seed)
    n, L, h, d, B = c["n_seq"], c["n_layer"], c["n_kv"], c["d"], c["B"]
    n_q = h * c["group"]
    s = dict(case=c, x=x)
    # the scheduler's list of tokens: (sequence, number in it) of each
    counts = torch.tensor(_lens(c) if c["op"] == "stage" else _news(c))
    seq = torch.repeat_interleave(torch.arange(n), counts)
    tok = torch.arange(int(counts.sum())) - (torch.cumsum(counts, 0) - counts)[seq]
    s["tokens"] = (seq.cuda(), tok.cuda())
    if c["op"] == "append":
        s["q"] = torch.zeros((n, B, n_q, d), dtype=torch.bfloat16, device="cuda")
    elif c["op"] == "attend":
        s["out"] = torch.zeros((n, B, n_q, d), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros((n, B, n_q), dtype=torch.float32, device="cuda")
    else:
        for t in ("k", "v"):
            s[t + "1"] = torch.zeros((n, L, h, c["len0"], d), dtype=torch.bfloat16, device="cuda")
            s[t + "2"] = _raw(torch.empty_like(x[t])).zero_().view(x[t].dtype)
        s["len1"], s["len2"] = torch.zeros((2, n), dtype=torch.int32, device="cuda").unbind(0)
        s["table2"] = torch.where(x["table"] >= 0, x["k"].shape[1] - 1 - x["table"], -1).int()
    if own:
        import paper_2609_23314_gb300 as vd
        s["cache"] = vd.PagedCache(x["k"], x["v"], x["table"], x["len"], x["k_scale"], x["v_scale"])
        if c["op"] == "attend":
            size = vd.vd_paged_attend_workspace(s["cache"], n_q, B)
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        elif c["op"] == "stage":
            s["stage"] = vd.Cache(s["k1"], s["v1"], s["len1"])
            s["other"] = vd.PagedCache(s["k2"], s["v2"], s["table2"], s["len2"], x["k_scale"],
                                       x["v_scale"])
    return s


def run(state):
    s, c, x = state, state["case"], state["x"]
    if not own:
        plain = {"append": _plain_append, "attend": _plain_attend, "stage": _plain_stage}
        return plain[c["op"]](s, x, c)
    import paper_2609_23314_gb300 as vd
    if c["op"] == "append":
        vd.vd_paged_append(s["cache"], x["qkv"], s["q"], layer=c["layer"], q_weight=x["qw"],
                           k_weight=x["kw"], eps=1.0e-6, inv_freq=x["freq"],
                           pos_first_new=x["first"], interleaved=c["interleaved"], n_new=x["new"])
        return [s["q"], x["k"], x["v"]]
    if c["op"] == "attend":
        vd.vd_paged_attend(s["cache"], x["q"], s["out"], s["workspace"], layer=c["layer"],
                           causal=c["causal"], n_new=x["new"], lse_out=s["lse"])
        return [s["out"], s["lse"]]
    vd.vd_paged_unpack(s["cache"], s["stage"], layer0=0)
    vd.vd_paged_pack(s["other"], s["stage"], layer0=0)
    return [s[t] for t in ("k1", "v1", "len1", "k2", "v2", "len2")]


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    """Bytes: each input and output once.  Flops: two per multiply-add of the two products, a
    handful per value elsewhere."""
    c = case
    h, G, d, B = c["n_kv"], c["group"], c["d"], c["B"]
    size = 1 if c["dtype"] == "e4m3" else 2
    lens, news = _lens(c), _news(c)
    if c["op"] == "append":
        tokens = sum(news)
        return {"bytes": tokens * h * d * (2 * (G + 2) + 2 * G + 2 * size) + 2 * c["rd"] + 12 * c["n_seq"],
                "flops": 8 * tokens * h * (G + 2) * d}
    if c["op"] == "stage":
        values = 2 * sum(lens) * c["n_layer"] * h * d
        return {"bytes": values * (2 * size + 4), "flops": 2 * values}
    grow = 1 if c["causal"] else 0
    slots = sum(m + grow * b for m, b in zip(lens, news) if b)
    pairs = sum(m * b + grow * b * (b + 1) // 2 for m, b in zip(lens, news))
    return {"bytes": h * d * (2 * size * slots + 4 * G * sum(news)) + 4 * h * G * sum(news),
            "flops": 4 * d * h * G * pairs}


# ---------------------------------------------------------------------------
# the same outputs from the definition, in 64 bits
# ---------------------------------------------------------------------------
# what the bytes 0 .. 126 of an e4m3 value stand for
_E4M3 = [m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127]


def _held64(y, scale):
    """What a page holds for values in 64 bits: bf16 pages leave them as they are, e4m3 ones
    hold the nearest value times scale, the even one of two equally near."""
    if scale is None:
        return y
    grid = torch.tensor(_E4M3, dtype=torch.float64, device=y.device)
    t = (y / scale.double()).abs().contiguous()
    hi = torch.searchsorted(grid, t).clamp_max(126)
    lo = (hi - 1).clamp_min(0)
    up, down = grid[hi] - t, t - grid[lo]
    near = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.sign(y) * grid[near]


def _slots64(x, c, name, layer, s, m):
    """Rows [h, m, d] in 64 bits of the first m slots of one sequence."""
    pages = x["table"][s, :-(-m // c["page"])].long()
    pool = x[name][layer]
    if c["dtype"] == "e4m3":
        pool = pool.view(torch.uint8)
    rows = pool[pages].view(x[name].dtype).float().double().transpose(0, 1)  # [h, pages, page, d]
    rows = rows.reshape(rows.shape[0], -1, rows.shape[-1])[:, :m]
    scale = x[name + "_scale"]
    return rows if scale is None else rows * scale[layer].double()[:, None, None]


def exact(case, seed):
    c = case
    n, L, h, G, d, page, B, layer = (c[t] for t in ("n_seq", "n_layer", "n_kv", "group", "d", "page",
                                                    "B", "layer"))
    lens, news = _lens(c), _news(c)
    x = _inputs(c, seed)
    if c["op"] == "append":
        n_q = h * G
        q = torch.zeros((n, B, n_q, d), dtype=torch.float64, device="cuda")
        pools = {t: x[t].float().double().contiguous() for t in ("k", "v")}
        for s in range(n):
            for b0 in range(0, news[s], 2048):
                b = torch.arange(b0, min(news[s], b0 + 2048), device="cuda")
                slot = lens[s] + b
                pos = slot if x["first"] is None else int(x["first"][s]) + b
                y = x["qkv"][s, b].double()
                for lo, hi, w in ((0, n_q, x["qw"]), (n_q, n_q + h, x["kw"])):
                    z = y[:, lo:hi]
                    if w is not None:
                        z = z * torch.rsqrt((z * z).sum(-1, keepdim=True) / d + 1.0e-6) * w.double()
                    if c["rd"]:
                        i = torch.arange(c["rd"] // 2, device="cuda")
                        i, j = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + c["rd"] // 2)
                        angle = pos.double()[:, None, None] * x["freq"].double()
                        turned = torch.complex(z[..., i], z[..., j]) * \
                            torch.polar(torch.ones_like(angle), angle)
                        z[..., i], z[..., j] = turned.real, turned.imag
                    y[:, lo:hi] = z
                q[s, b] = y[:, :n_q]
                where = x["table"][s, slot // page].long()
                for t, r in (("k", y[:, n_q:n_q + h]), ("v", y[:, n_q + h:])):
                    scale = x[t + "_scale"]
                    held = _held64(r, None if scale is None else scale[layer][:, None])
                    pools[t][layer, where, :, slot % page] = held
        return [q, pools["k"], pools["v"]]
    if c["op"] == "stage":
        outs = []
        for t in ("k", "v"):
            first = torch.zeros((n, L, h, c["len0"], d), dtype=torch.float64, device="cuda")
            second = torch.zeros(x[t].shape, dtype=torch.float64, device="cuda")
            for s in range(n):
                if not lens[s]:
                    continue
                at = torch.arange(lens[s], device="cuda")
                where = (x["k"].shape[1] - 1 - x["table"][s, at // page]).long()
                for i in range(L):
                    rows = _slots64(x, c, t, i, s, lens[s])
                    first[s, i, :, :lens[s]] = rows
                    scale = x[t + "_scale"]
                    held = rows if scale is None else rows / scale[i].double()[:, None, None]
                    second[i, where, :, at % page] = held.transpose(0, 1)
            outs.append((first, second))
        return [outs[0][0], outs[1][0], None, outs[0][1], outs[1][1], None]
    out = torch.zeros((n, B, h * G, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((n, B, h * G), dtype=torch.float64, device="cuda")
    for s in range(n):
        if not news[s]:
            continue
        total = lens[s] + (news[s] if c["causal"] else 0)
        if total == 0:
            lse[s, :news[s]] = -math.inf
            continue
        ks, vs = (_slots64(x, c, t, layer, s, total) for t in ("k", "v"))
        for j in range(h):
            z = torch.einsum("bgd,td->gbt", x["q"][s, :news[s], j * G:(j + 1) * G].double(), ks[j])
            z = z / math.sqrt(d)
            if c["causal"]:
                last = lens[s] + torch.arange(news[s], device="cuda")
                z.masked_fill_(torch.arange(total, device="cuda") > last[:, None], -math.inf)
            lse[s, :news[s], j * G:(j + 1) * G] = torch.logsumexp(z, -1).T
            out[s, :news[s], j * G:(j + 1) * G] = (torch.softmax(z, -1) @ vs[j]).transpose(0, 1)
    return [out, lse]

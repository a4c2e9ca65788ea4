"""The measured cases of the 4-bit cache and of the pass that makes its rows:
what they are, how their inputs are made, the operators in plain torch and the
same pass through the library.

``rope``    norms of queries and keys per head and the position rotation, from
            one projection row per token into q and the new rows of a layer.
``append``  new bf16 rows into a cache held in 4 bits, read back as bf16.
``pack``    a bf16 cache (an evicted one) into 4 bits, read back as bf16.
``attend``  attention of new tokens over one layer of the 4-bit cache and over
            the new rows themselves.

The 4-bit format: 16 values along the head share a scale s, amax / 6 rounded to
an unsigned float of 5 exponent bits (bias 15) and 3 mantissa bits, at most
10240; a value is a sign and one of 0, .5, 1, 1.5, 2, 3, 4, 6 times s, rounded to
nearest, ties to the even code.
"""
from __future__ import annotations

import math

import torch

own = False

BASE = dict(n_seq=1, n_layer=1, n_kv=8, d=128)
ROPE = dict(BASE, op="rope", n_q=32, B=1, rd=128, interleaved=False, norm=True, theta=1.0e6,
            first=30000)
ROWS = dict(BASE, op="append", cap=256, len0=128, B=128, ragged=False)
PACK = dict(BASE, op="pack", cap=4096, len0=4096, ragged=False)
ATTEND = dict(BASE, op="attend", group=4, layer=0, cap=4224, len0=4096, B=1, ragged=False,
              new=True)


def listed():
    return [
        # one user's decode step: the projection row of one token of an 8B-class GQA model (latency)
        dict(ROPE, name="rope_one"),
        # two long prompts at once
        dict(ROPE, name="rope_prompt", n_seq=2, B=8192, first=0),
        # one decode token of 16 sequences into short caches of all layers, ragged lengths
        dict(ROWS, name="append_decode_ragged", n_seq=16, n_layer=28, n_kv=4, cap=320, len0=300,
             B=1, ragged=True),
        # the second block of a prompt, all 36 layers at once
        dict(ROWS, name="append_block", n_layer=36),
        # the evicted cache of a prompt, budget 4096, all 36 layers
        dict(PACK, name="pack_cache", n_layer=36),
        # three ragged sequences, a head dim that is no power of two
        dict(PACK, name="pack_odd", n_seq=3, n_layer=24, n_kv=6, d=96, cap=1104, len0=1100,
             ragged=True),
        # one user's decode step over an evicted cache of 4096 tokens, one layer (latency)
        dict(ATTEND, name="attend_one"),
        # batched decode of 64 sequences around that budget
        dict(ATTEND, name="attend_batch", n_seq=64, ragged=True),
        # two long contexts that are not evicted: offsets beyond 32 bits
        dict(ATTEND, name="attend_long", n_seq=2, n_layer=18, layer=17, cap=131072, len0=131000),
        # a block of 128 tokens of block prompt processing at budget 2048
        dict(ATTEND, name="attend_block", B=128, cap=2176, len0=2048),
        # a chunk of 512 tokens of a long prompt
        dict(ATTEND, name="attend_chunk", B=512, cap=33280, len0=32768),
        # a few drafted tokens, odd head counts, lengths from nothing to a few thousand
        dict(ATTEND, name="attend_odd", n_seq=5, n_layer=2, layer=1, n_kv=3, group=5, d=96, B=3,
             cap=2504, len0=2500, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "pack", "attend", "attend", "attend"])
    d = rng.choice([64, 96, 128, 128, 128, 192, 256])
    n_kv = _log_int(rng, 1, 16)
    if op == "rope":
        n_seq = _log_int(rng, 1, 32)
        d = rng.choice([64, 80, 96, 128, 128, 192, 256])
        return dict(ROPE, n_seq=n_seq, n_kv=n_kv, n_q=n_kv * rng.randint(1, 8), d=d,
                    B=_log_int(rng, 1, max(1, 200000 // (n_seq * n_kv * d // 64))),
                    rd=rng.choice([d, d, d // 32 * 16]), interleaved=rng.random() < 0.3,
                    norm=rng.random() < 0.8, theta=rng.choice([1.0e4, 5.0e5, 1.0e6]),
                    first=rng.choice([0, _log_int(rng, 1, 1000000)]))
    if op in ("append", "pack"):
        n_seq, n_layer = _log_int(rng, 1, 16), _log_int(rng, 1, 36)
        most = max(16, min(8192, (1 << 30) // (n_seq * n_layer * n_kv * d * 2)))
        rows = _log_int(rng, 2, most)
        new = _log_int(rng, 1, max(1, rows // 2)) if op == "append" else 0
        return dict(ROWS if op == "append" else PACK, n_seq=n_seq, n_layer=n_layer, n_kv=n_kv, d=d,
                    cap=(rows + 7) // 8 * 8 + 8 * rng.randint(0, 4), len0=rows - new, B=new,
                    ragged=n_seq > 1 and rng.random() < 0.5)
    new = rng.random() < 0.85
    long = rng.random() < 0.35  # many new tokens, or many sequences
    group = rng.randint(1, 8)
    n_seq = _log_int(rng, 1, 4 if long else 64)
    B = _log_int(rng, 16, 700) if long else _log_int(rng, 1, 8)
    work = n_seq * n_kv * group * B * d
    len0 = _log_int(rng, 1, max(2, min(60000, (1 << 37) // work, (3 << 30) // (n_seq * n_kv * d))))
    return dict(ATTEND, n_seq=n_seq, n_kv=n_kv, group=group, d=d, B=B, len0=len0,
                cap=(len0 + B + 7) // 8 * 8 + 8 * rng.randint(0, 3), n_layer=rng.choice([1, 1, 2]),
                ragged=n_seq > 1 and rng.random() < 0.5, new=new)


def _lens(c):
    """Cached tokens of each sequence: len0, or spread below it where ragged: around
    one budget in large attention batches, down to one and zero elsewhere."""
    n, top = c["n_seq"], c["len0"]
    if not c["ragged"]:
        return [top] * n
    if c["op"] == "attend" and n >= 16:  # sequences around one budget
        return [max(1, top - (s * 7919 % 97) * top // 200) for s in range(n)]
    low = 0 if c["op"] != "attend" or c["new"] else 1
    return [max(low, min(top, [top, 1, low, top // 3, top - 1][s % 5])) for s in range(n)]


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
    n, L, h, d = c["n_seq"], c["n_layer"], c["n_kv"], c["d"]
    x = {}
    if c["op"] == "rope":
        n_q = c["n_q"]
        x["qkv"] = _rows(g, (n, c["B"], n_q + 2 * h, d), 2)
        x["qw"] = x["kw"] = x["freq"] = None
        if c["norm"]:
            x["qw"] = (1.0 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(torch.bfloat16)
            x["kw"] = (1.0 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(torch.bfloat16)
        if c["rd"]:
            e = torch.arange(0, c["rd"], 2, dtype=torch.float64, device="cuda") / c["rd"]
            x["freq"] = (c["theta"] ** -e).float()
        x["first"] = (c["first"] + torch.randint(0, 1000, (n,), generator=g, device="cuda")).int()
        return x
    x["len0"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda")
    if c["op"] == "pack":
        x["k"], x["v"] = (_rows(g, (n, L, h, c["cap"], d), m) for m in (4, 0))
    elif c["op"] == "append":
        x["k"], x["v"] = (_rows(g, (n, L, h, max(c["len0"], 1), d), m) for m in (4, 0))
        x["k_new"], x["v_new"] = (_rows(g, (n, L, h, c["B"], d), m) for m in (4, 0))
    else:
        x["k"], x["v"] = (_rows(g, (n, h, c["len0"], d), m) for m in (4, 0))
        x["k_new"], x["v_new"] = (_rows(g, (n, L, h, c["B"], d), m) for m in (4, 0))
        x["q"] = _rows(g, (n, c["B"], h * c["group"], d), 0)
    return x


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantise(rows, codes, scales):
    """bf16 rows [..., d] into packed codes [..., d/2] and scale bytes [..., d/16]."""
    x = rows.float().unflatten(-1, (-1, 16))
    # true quotients: a division by a Python number becomes a product on the GPU
    top = x.abs().amax(-1)
    t = top / torch.full_like(top, 6.0)
    power = torch.tensor([2.0 ** e for e in range(-17, 128)], device=x.device)  # exact ones
    ulp = power[(torch.frexp(t.clamp_min(2.0 ** -14))[1] + 13).long()]
    s = (torch.round(t / ulp) * ulp).clamp_max(10240.0)
    scales.copy_((s.half().view(torch.int16) >> 7).to(torch.uint8))
    y = x.abs() / torch.where(s > 0, s, torch.ones_like(s))[..., None]
    c = (y > 0.25).byte()
    for edge, even in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True),
                       (5.0, False)):
        c += (y >= edge) if even else (y > edge)
    c += 8 * (x < 0).byte()
    c = c.flatten(-2)
    codes.copy_(c[..., 0::2] | (c[..., 1::2] << 4))


def _values(codes, scales):
    """The fp32 values of packed codes [..., d/2] with scale bytes [..., d/16]."""
    table = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), device=codes.device)
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()
    s = (scales.short() << 7).view(torch.float16).float()
    return (table[c].unflatten(-1, (-1, 16)) * s[..., None]).flatten(-2)


def _by_unit(shape, rows, d):
    """Slices of the leading dimension of [units, rows, d] that stay near 256 MB in fp32."""
    step = max(1, (64 << 20) // max(1, rows * d))
    return [slice(u, min(shape, u + step)) for u in range(0, shape, step)]


def _plain_rope(s, x, c):
    n_q, h, d, half = c["n_q"], c["n_kv"], c["d"], c["rd"] // 2
    xs = x["qkv"].float()
    out = []
    for part, w in ((xs[:, :, :n_q], x["qw"]), (xs[:, :, n_q:n_q + h], x["kw"])):
        if w is not None:
            part = part / torch.sqrt(part.square().mean(-1, keepdim=True) + s["eps"]) * w.float()
        if half:
            pos = x["first"][:, None] + torch.arange(c["B"], device="cuda", dtype=torch.int32)
            angle = pos.double()[:, :, None, None] * x["freq"].double()
            cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
            if c["interleaved"]:
                a, b = part[..., 0:2 * half:2], part[..., 1:2 * half:2]
            else:
                a, b = part[..., :half], part[..., half:2 * half]
            ra, rb = a * cos - b * sin, b * cos + a * sin
            turned = torch.stack((ra, rb), -1).flatten(-2) if c["interleaved"] else \
                torch.cat((ra, rb), -1)
            part = torch.cat((turned, part[..., 2 * half:]), -1)
        out.append(part.to(torch.bfloat16))
    swap = [t.transpose(1, 2).unsqueeze(1).contiguous() for t in (out[1], x["qkv"][:, :, n_q + h:])]
    return [out[0]] + swap


def _plain_rows(s, x, c):
    d, cap, U = c["d"], c["cap"], c["n_seq"] * c["n_layer"] * c["n_kv"]
    per = c["n_layer"] * c["n_kv"]
    s["len"].copy_(x["len0"])
    outs = []
    for name in ("k", "v"):
        codes, scales = s["q4"][name].view(U, cap, d // 2), s["q4"][name + "s"].view(U, cap, d // 16)
        back = torch.zeros((U, cap, d), dtype=torch.bfloat16, device="cuda")
        src = x[name].view(U, -1, d) if c["op"] == "pack" else x[name + "_new"].view(U, c["B"], d)
        for i, n in enumerate(_lens(c)):
            lo, hi = (0, n) if c["op"] == "pack" else (n, n + c["B"])
            for sl in _by_unit(per, max(hi, 1), d):
                u = slice(i * per + sl.start, i * per + sl.stop)
                _quantise(src[u, :hi - lo], codes[u, lo:hi], scales[u, lo:hi])
                back[u, :hi] = _values(codes[u, :hi], scales[u, :hi])
        outs.append(back.view(c["n_seq"], c["n_layer"], c["n_kv"], cap, d))
    if c["op"] == "append":
        s["len"] += c["B"]
    return outs + [s["len"]]


def _plain_attend(s, x, c):
    n, h, d, B, G, layer = c["n_seq"], c["n_kv"], c["d"], c["B"], c["group"], c["layer"]
    scale = 1.0 / math.sqrt(d)
    out = torch.empty((n, B, h * G, d), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((n, B, h * G), dtype=torch.float32, device="cuda")
    lens = _lens(c)
    for i in range(n):
        m = lens[i]
        keys, vals = ([_values(s["q4"][t][i, layer, :, :m], s["q4"][t + "s"][i, layer, :, :m])]
                      for t in ("k", "v"))
        if c["new"]:
            keys.append(x["k_new"][i, layer].float())
            vals.append(x["v_new"][i, layer].float())
        keys, vals = torch.cat(keys, 1), torch.cat(vals, 1)
        cols = keys.shape[1]
        q = x["q"][i].float().view(B, h, G, d).permute(1, 0, 2, 3).reshape(h, B * G, d)
        heads = max(1, (1 << 29) // (B * G * cols))
        for a in range(0, h, heads):
            b = min(h, a + heads)
            p = torch.matmul(q[a:b], keys[a:b].transpose(1, 2))
            p *= scale
            if c["new"] and B > 1:
                seen = torch.arange(cols, device="cuda")[None, :] <= \
                    m + torch.arange(B, device="cuda")[:, None]
                p = p.view(b - a, B, G, cols).masked_fill_(~seen[:, None, :], -math.inf)
                p = p.view(b - a, B * G, cols)
            top = p.amax(-1, keepdim=True)
            p -= top
            torch.exp(p, out=p)
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p, vals[a:b]) / total
            e = (top + torch.log(total)).squeeze(-1)
            out[i].view(B, h, G, d)[:, a:b] = o.view(b - a, B, G, d).transpose(0, 1)
            lse[i].view(B, h, G)[:, a:b] = e.view(b - a, B, G).transpose(0, 1)
    return [out, lse]


# ---------------------------------------------------------------------------
# one state, one pass
# ---------------------------------------------------------------------------
def prepare(case, seed):
    c, x = case, _inputs(case, seed)
    n, L, h, d = c["n_seq"], c["n_layer"], c["n_kv"], c["d"]
    s = dict(case=c, x=x, eps=1.0e-6)
    if c["op"] == "rope":
        if own:
            s["out"] = [torch.empty((n, c["B"], c["n_q"], d), dtype=torch.bfloat16, device="cuda")]
            s["out"] += [torch.empty((n, 1, h, c["B"], d), dtype=torch.bfloat16, device="cuda")
                         for _ in range(2)]
        return s
    cap, m = c["cap"], c["len0"]
    s["len"] = x["len0"].clone()
    s["q4"] = {t + e: torch.zeros((n, L, h, cap, d // k), dtype=torch.uint8, device="cuda")
               for t in ("k", "v") for e, k in (("", 2), ("s", 16))}
    if c["op"] != "pack":  # the rows that the cache holds already
        for t in ("k", "v"):
            rows = x.pop(t)
            if c["op"] == "attend":
                rows = rows.view(n * h, m, d)
                codes, scales = ((s["q4"][t + e][:, c["layer"], :, :m]) for e in ("", "s"))
                for u in range(n * h):
                    for r in range(0, m, 1 << 18):
                        part = slice(r, min(m, r + (1 << 18)))
                        _quantise(rows[u, part], codes[u // h, u % h, part],
                                  scales[u // h, u % h, part])
            elif m:
                U = n * L * h
                codes, scales = (s["q4"][t + e].view(U, cap, -1)[:, :m] for e in ("", "s"))
                for u in _by_unit(U, m, d):
                    _quantise(rows.view(U, m, d)[u], codes[u], scales[u])
    if own:
        import paper_2609_23314_gb300 as vd
        q4 = s["q4"]
        s["cache4"] = vd.Q4Cache(q4["k"], q4["v"], q4["ks"], q4["vs"], s["len"])
        if c["op"] == "attend":
            s["out"] = [torch.empty_like(x["q"]),
                        torch.empty(x["q"].shape[:-1], dtype=torch.float32, device="cuda")]
        else:
            s["back"] = vd.Cache.empty(n, L, h, cap, d)
            if c["op"] == "pack":
                s["cache"] = vd.Cache(x["k"], x["v"], x["len0"])
    return s


def run(state):
    s, c, x = state, state["case"], state["x"]
    if not own:
        plain = {"rope": _plain_rope, "append": _plain_rows, "pack": _plain_rows,
                 "attend": _plain_attend}
        return plain[c["op"]](s, x, c)
    import paper_2609_23314_gb300 as vd
    if c["op"] == "rope":
        q, k_new, v_new = s["out"]
        vd.vd_qkv_norm_rope(x["qkv"], q, k_new, v_new, layer=0, q_weight=x["qw"],
                            k_weight=x["kw"], eps=s["eps"], inv_freq=x["freq"],
                            pos_first_new=x["first"], interleaved=c["interleaved"])
        return s["out"]
    if c["op"] == "attend":
        new = (x["k_new"], x["v_new"]) if c["new"] else (None, None)
        vd.vd_q4_attend(s["cache4"], x["q"], s["out"][0], k_new=new[0], v_new=new[1],
                        layer=c["layer"], lse_out=s["out"][1])
        return s["out"]
    if c["op"] == "append":
        s["len"].copy_(x["len0"])
        vd.vd_q4_append(s["cache4"], x["k_new"], x["v_new"], c["B"])
    else:
        vd.vd_q4_pack(s["cache4"], s["cache"], layer0=0)
    back = s["back"]
    vd.vd_q4_unpack(s["cache4"], back, layer0=0)
    return [back.k, back.v, back.len]


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    """Bytes: each input and output once (a 4-bit value with its share of the
    scale is 0.5625 bytes).  Flops: two per multiply-add of the two products, a
    handful per value elsewhere."""
    c = case
    h, d = c["n_kv"], c["d"]
    if c["op"] == "rope":
        values = c["n_seq"] * c["B"] * (c["n_q"] + 2 * h) * d
        return {"bytes": 4 * values + 2 * c["rd"] + 4 * c["n_seq"] + (4 * d if c["norm"] else 0),
                "flops": 8 * values}
    total = sum(_lens(c))
    if c["op"] in ("append", "pack"):
        per = 2 * c["n_layer"] * h * d
        new = total if c["op"] == "pack" else c["n_seq"] * c["B"]
        held = total if c["op"] == "pack" else total + new
        return {"bytes": int(per * (new * 2.5625 + held * 2.5625)), "flops": 8 * per * new}
    B, G = c["B"], c["group"]
    pairs = G * (B * total + (c["n_seq"] * B * (B + 1) // 2 if c["new"] else 0))
    rows = c["n_seq"] * h * B
    return {"bytes": int(1.125 * h * d * total + rows * (4 * G * d + 4 * G + 4 * d * c["new"])),
            "flops": 4 * d * h * pairs}


# ---------------------------------------------------------------------------
# the same outputs from the definition, in 64 bits
# ---------------------------------------------------------------------------
def _held64(rows):
    """What a cache in 4 bits holds for bf16 rows: nearest representable scale and
    nearest level by distance, the even one of two equally near."""
    x = rows.double()
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // 16, 16))
    want = torch.div(g.abs().amax(-1), torch.tensor([6.0], dtype=torch.float64, device=x.device))
    grid = torch.tensor([b * 2.0 ** -17 if b < 8 else (8 + b % 8) * 2.0 ** (b // 8 - 18)
                         for b in range(227)], dtype=torch.float64, device=x.device)
    level = torch.tensor(_LEVELS, dtype=torch.float64, device=x.device)

    def nearest(t, table):
        hi = torch.searchsorted(table, t.contiguous()).clamp_max(table.numel() - 1)
        lo = (hi - 1).clamp_min(0)
        up, down = table[hi] - t, t - table[lo]
        pick = (up < down) | ((up == down) & (hi % 2 == 0))
        return table[torch.where(pick, hi, lo)]

    s = nearest(want, grid)[..., None]
    held = torch.sign(g) * nearest(g.abs() / torch.where(s > 0, s, 1.0), level) * s
    return held.reshape(x.shape)


def exact(case, seed):
    c = case
    n, h, d = c["n_seq"], c["n_kv"], c["d"]
    if c["op"] == "attend" and c["n_seq"] * h * c["group"] * c["B"] * c["len0"] * d > 1 << 40:
        return None
    x = _inputs(c, seed)
    if c["op"] == "rope":
        half, n_q = c["rd"] // 2, c["n_q"]
        qkv = x["qkv"].double()
        if half:
            t = torch.arange(c["B"], device="cuda")[None, :] + x["first"].long()[:, None]
            turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                               t.double()[..., None, None] * x["freq"].double())
        got = []
        for lo, hi, w in ((0, n_q, x["qw"]), (n_q, n_q + h, x["kw"])):
            y = qkv[:, :, lo:hi].clone()
            if w is not None:
                y = y * torch.rsqrt((y * y).sum(-1, keepdim=True) / d + 1.0e-6) * w.double()
            if half:
                i = torch.arange(half, device="cuda")
                a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
                z = torch.complex(y[..., a], y[..., b]) * turn
                y[..., a], y[..., b] = z.real, z.imag
            got.append(y)
        return [got[0], got[1].permute(0, 2, 1, 3)[:, None],
                qkv[:, :, n_q + h:].permute(0, 2, 1, 3)[:, None]]
    lens = _lens(c)
    if c["op"] in ("append", "pack"):
        back = []
        for t in ("k", "v"):
            y = torch.zeros((n, c["n_layer"], h, c["cap"], d), dtype=torch.float64, device="cuda")
            for i, m in enumerate(lens):
                for layer in range(c["n_layer"]):
                    y[i, layer, :, :m] = _held64(x[t][i, layer, :, :m])
                    if c["op"] == "append":
                        y[i, layer, :, m:m + c["B"]] = _held64(x[t + "_new"][i, layer])
            back.append(y)
        return back + [None]
    B, G = c["B"], c["group"]
    out = torch.empty((n, B, h * G, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((n, B, h * G), dtype=torch.float64, device="cuda")
    for i, m in enumerate(lens):
        for j in range(h):
            ks, vs = _held64(x["k"][i, j, :m]), _held64(x["v"][i, j, :m])
            if c["new"]:
                ks = torch.cat((ks, x["k_new"][i, c["layer"], j].double()))
                vs = torch.cat((vs, x["v_new"][i, c["layer"], j].double()))
            for g in range(j * G, (j + 1) * G):
                for t0 in range(0, B, 128):
                    t1 = min(B, t0 + 128)
                    z = x["q"][i, t0:t1, g].double() @ ks.T / math.sqrt(d)
                    if c["new"]:
                        last = m + torch.arange(t0, t1, device="cuda")
                        z[torch.arange(ks.shape[0], device="cuda") > last[:, None]] = -math.inf
                    lse[i, t0:t1, g] = torch.logsumexp(z, 1)
                    out[i, t0:t1, g] = torch.softmax(z, 1) @ vs
    return [out, lse]

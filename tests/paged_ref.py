"""What the calls on a paged cache are held to, in 64 bits, and the caches that the tests run on."""
from __future__ import annotations

import math

import torch

import paper_2609_23314_gb300 as vd

FP8 = torch.float8_e4m3fn
FILL = 9.0  # what slots hold that no call may write


def raw(t):
    """A tensor with elements that torch indexes and compares: 8-bit floats as bytes."""
    return t.view(torch.uint8) if t.dtype == FP8 else t


def cache(lens, n_layer, h, d, page, dtype=torch.bfloat16, by_token=False, scales=True, extra=0,
          seed=0, spare=2, one_buffer=False):
    """A paged cache of random rows: pages in a random order, table places that are not needed -1,
    slots behind len (room for `extra` more) FILL, and so are `spare` pages that nobody has."""
    g = torch.Generator().manual_seed(seed)
    n = len(lens)
    need = [-(-(m + extra) // page) for m in lens]
    P, width = sum(need) + spare, max(max(need), 1) + 1
    order = torch.randperm(P, generator=g).int()
    table = torch.full((n, width), -1, dtype=torch.int32)
    at = 0
    for s, m in enumerate(need):
        table[s, :m] = order[at:at + m]
        at += m
    two = 2 if one_buffer else 1
    shape = (n_layer, P, page, h, two * d) if by_token else (n_layer, P, h, page, two * d)
    pools, scale = [], []
    for t in range(2):
        if t == 0 or not one_buffer:
            buf = raw(torch.full(shape, FILL, dtype=torch.float32).to(dtype)).cuda().view(dtype)
        pool = buf.transpose(2, 3) if by_token else buf
        pools.append(pool[..., t * d:(t + 1) * d] if one_buffer else pool)
        scale.append((0.02 + 0.03 * torch.rand((n_layer, h), generator=g)).cuda()
                     if dtype == FP8 and scales else None)
        for s, m in enumerate(lens):
            rows = torch.randn((n_layer, m, h, d), generator=g) * (1 + torch.rand(d, generator=g))
            if dtype == FP8:
                rows = (rows * 20).clamp(-448, 448)
            slot = torch.arange(m)
            raw(pools[t])[:, table[s, slot // page].long().cuda(), :, (slot % page).cuda()] = raw(
                rows.transpose(0, 1).contiguous().to(dtype)).cuda()
    return vd.PagedCache(pools[0], pools[1], table.cuda(),
                         torch.tensor(lens, dtype=torch.int32).cuda(), *scale)


def rows_of(c, pool, scale, s, m, layer):
    """[m, h, d] in 64 bits: the first m slots of a sequence."""
    slot = torch.arange(m, device=pool.device)
    x = raw(pool)[layer, c.page_table[s, slot // c.page_size].long(), :, slot % c.page_size]
    x = x.contiguous().view(pool.dtype).cpu().float().double()
    return x if scale is None else x * scale[layer].cpu().double()[None, :, None]


def attend(c, q, layer, causal, scale, news):
    """Per sequence (outputs [B, n_q, d], lse [B, n_q], how far each may be off)."""
    B, n_q, d = q.shape[1:]
    G = n_q // c.n_kv_head
    weight = 2.0 ** -16 if c.type == vd.VD_PAGED_BF16 else 2.0 ** -11
    outs = []
    for s, (n, add) in enumerate(zip(c.len.tolist(), news)):
        m = n + (add if causal else 0) if add else 0
        k, v = (rows_of(c, p, f, s, m, layer) for p, f in ((c.k, c.k_scale), (c.v, c.v_scale)))
        x = q[s, :add].cpu().double()
        kk, vv = (t.repeat_interleave(G, 1) for t in (k, v))          # [m, n_q, d]
        z = torch.einsum("bqd,mqd->bqm", x, kk) * scale
        size = torch.einsum("bqd,mqd->bqm", x.abs(), kk.abs()) * scale
        ends = n + (torch.arange(add) + 1 if causal else torch.zeros(add, dtype=torch.long))
        hidden = (torch.arange(m) >= ends[:, None])[:, None].expand_as(z)
        z = z.masked_fill(hidden, -math.inf)
        size = size.masked_fill(hidden, 0.0)
        lse = torch.logsumexp(z, -1) if m else torch.full((add, n_q), -math.inf).double()
        p = torch.exp(z - torch.where(lse.isinf(), 0.0, lse)[..., None])
        # rows that a token does not see reach nothing, whatever they hold
        seen = torch.where(hidden[..., None], 0.0, vv.transpose(0, 1)[None]) if m else None
        o = (p[..., None] * seen).sum(-2) if m else torch.zeros(add, n_q, d).double()
        mag = (p[..., None] * seen.abs()).sum(-2) if m else torch.zeros_like(o)
        # a score: d products and sums in fp32, four roundings of the size of the score on the way
        # to the exponent, for e4m3 pages queries in fp16 (2^-29 of the row's largest);  weights: 2^-20 for the exponential, `weight` for their rounding (and
        # 2^-36 of the largest, of every slot, where it drops them); m sums in fp32
        ds = ((d + 8) * 2.0 ** -23 * size).amax(-1) if m else torch.zeros(add, n_q).double()
        ls = torch.where(lse.isinf(), 0.0, lse.abs())
        ds = ds + 2.0 ** -21 * ls
        if m and c.type == vd.VD_PAGED_E4M3:
            ds = ds + d * 2.0 ** -29 * scale * x.abs().amax(-1) * k.abs().nan_to_num(0.0).amax()
        top = seen.abs().amax(-2) if m else mag
        tol = 2.0 ** -8 * o.abs() + (2 * ds + weight + 2.0 ** -20 + m * 2.0 ** -23)[..., None] * mag \
            + m * 2.0 ** -36 * top + 1e-30
        outs.append((o, lse, tol, ds + 2.0 ** -19 + m * 2.0 ** -23 + 2.0 ** -22 * ls))
    return outs


def check_attend(c, q, layer=0, causal=True, scale=None, n_new=None, call=None, lse=True):
    """Runs the call, holds it to the definition, and returns what it wrote."""
    n, B, n_q, d = q.shape
    news = [B] * n if n_new is None else n_new
    out = torch.full_like(q, FILL)
    e = torch.full((n, B, n_q), FILL, device="cuda") if lse else None
    size = vd.vd_paged_attend_workspace(c, n_q, B)
    work = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    new = None if n_new is None else torch.tensor(n_new, dtype=torch.int32).cuda()
    vd.vd_paged_attend(c, q, out, work, layer=layer, causal=causal, scale=scale, n_new=new,
                       lse_out=e)
    torch.cuda.synchronize()
    refs = attend(c, q, layer, causal, d ** -0.5 if scale is None else scale, news)
    for s, (o, z, tol, tol_z) in enumerate(refs):
        got = out[s, :news[s]].cpu().double()
        bad = torch.isnan(o) != torch.isnan(got)
        assert not bool(bad.any()), f"sequence {s}: NaN in other places"
        off = (got - o).abs() - tol
        assert not bool((off > 0).any()), f"sequence {s}: {off.nan_to_num(0).max()} more than allowed"
        assert bool((out[s, news[s]:] == FILL).all())
        if lse:
            got = e[s, :news[s]].cpu().double()
            same = (got == z) | ((got - z).abs() <= tol_z) | (torch.isnan(z) & torch.isnan(got))
            assert bool(same.all()), f"sequence {s}: log-sums {(got - z).abs().max()} off"
            assert bool((e[s, news[s]:] == FILL).all())
    return out, e

"""Plain 64-bit forms of the 4-bit cache's operators, on the CPU: the row format,
attention over cached and new rows, norms and rotation.  Shares no code with the
library."""
from __future__ import annotations

import torch

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
# scale bytes 0 .. 226: 5 exponent bits (bias 15), 3 mantissa bits
SCALES = torch.tensor([b / 8 * 2.0 ** -14 if b < 8 else (1 + (b % 8) / 8) * 2.0 ** (b // 8 - 15)
                       for b in range(227)], dtype=torch.float64)


def nearest_even(x, table):
    """Index of the table value nearest to x >= 0, the even index of two equally near."""
    hi = torch.searchsorted(table, x.contiguous()).clamp(max=table.numel() - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = table[hi] - x, x - table[lo]
    return torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


def quantise(rows):
    """bf16 [..., d] -> codes uint8 [..., d / 2], scale bytes uint8 [..., d / 16]."""
    x = rows.double().unflatten(-1, (-1, 16))
    bad = ~torch.isfinite(x).all(-1)
    x = torch.where(bad[..., None], 0.0, x)
    sb = nearest_even(x.abs().amax(-1) / 6, SCALES)
    s = SCALES[sb][..., None]
    q = torch.where(s > 0, x.abs() / torch.where(s > 0, s, 1.0), 0.0)
    code = nearest_even(q, LEVELS) + 8 * torch.signbit(x)
    code = code.flatten(-2).to(torch.uint8)
    return (code[..., 0::2] | (code[..., 1::2] << 4)), torch.where(bad, 255, sb).to(torch.uint8)


def values(codes, scales):
    """What codes [..., d / 2] and scale bytes [..., d / 16] stand for, in fp64."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    v = LEVELS[c & 7] * torch.where(c >= 8, -1.0, 1.0)
    s = torch.cat((SCALES, torch.full((29,), float("nan"), dtype=torch.float64)))[scales.long()]
    return (v.unflatten(-1, (-1, 16)) * s[..., None]).flatten(-2)


def attend(q, ks, vs, k_new, v_new, scale):
    """One KV head: q [B, G, d]; ks, vs [n, d] and k_new, v_new [B, d] (or None), fp64.
    Returns out [B, G, d], lse [B, G] and what the tolerances need: per output the
    weighted mean of |v| over cached and new rows, the mean weight-free sum of |v|, and
    per row the largest sum of |q_i k_i| * scale over its scores."""
    B, G, d = q.shape
    n = ks.shape[0]
    out, lse = torch.zeros(B, G, d).double(), torch.full((B, G), -float("inf")).double()
    a_old, a_new, a_abs = (torch.zeros(B, G, d).double() for _ in range(3))
    size = torch.zeros(B, G).double()
    for i in range(B):
        k, v = ks, vs
        if k_new is not None:
            k, v = torch.cat((ks, k_new[:i + 1])), torch.cat((vs, v_new[:i + 1]))
        if k.shape[0] == 0:
            continue
        s = q[i] @ k.T * scale
        m = s.amax(1, keepdim=True)
        p = torch.exp(s - m)
        l = p.sum(1, keepdim=True)
        out[i] = p @ v / l
        lse[i] = (m + torch.log(l)).squeeze(1)
        a_old[i] = p[:, :n] @ v[:n].abs() / l
        a_new[i] = p[:, n:] @ v[n:].abs() / l
        a_abs[i] = v.abs().sum(0)
        size[i] = (q[i].abs() @ k.abs().T).amax(1) * scale
    return out, lse, a_old, a_new, a_abs, size


def attend_tolerance(out, lse, a_old, a_new, a_abs, size, keys, d):
    """Bounds of the errors of out (bf16) and lse (fp32).

    A score: products exact, fp32 sums of d terms in the tensor core (each addition off
    by at most 2^-23 of the partial sums, which size bounds), then a scaling and the
    difference to the maximum: ds <= (d + 8) 2^-23 size.  A weight exp(s - m): off by
    the two scores' errors, 2^-21 for exp2 and the rescaling; then rounded to fp16, 2^-11
    (bf16 for new rows, 2^-8), or 2^-25 where it is subnormal in fp16.  The sums over
    tokens: fp32, 2^-23 of the partial sums per addition, keys / 8 + 64 additions in a
    chain.  The result: bf16, 2^-8 of itself."""
    ds = (d + 8) * 2.0 ** -23 * size
    rel = (2 * ds + 2.0 ** -20 + (keys / 8 + 64) * 2.0 ** -23)[..., None]
    # the quotient by l: the weights' common errors, once more, on the result itself
    t_out = 2.0 ** -8 * out.abs() + (rel + 2.0 ** -11) * a_old + (rel + 2.0 ** -8) * a_new + \
        rel * out.abs() + 2.0 ** -24 * a_abs
    t_lse = ds + (keys / 8 + 64) * 2.0 ** -23 + 2.0 ** -20 + 2.0 ** -22 * lse.abs()
    return t_out * (1 + 2.0 ** -7) + 1e-30, t_lse


def norm_rope(x, weight, eps, inv_freq, pos, interleaved):
    """x [B, heads, d] fp64, pos [B]; the rotated heads, and the size that the tolerance
    takes for every value: of a pair, the sum of both magnitudes."""
    y = x.clone()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double()
    size = y.abs()
    if inv_freq is not None:
        half = inv_freq.numel()
        t = pos.double()[:, None, None] * inv_freq.double()
        i = torch.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        ya, yb = y[..., a].clone(), y[..., b].clone()
        y[..., a] = ya * torch.cos(t) - yb * torch.sin(t)
        y[..., b] = yb * torch.cos(t) + ya * torch.sin(t)
        size[..., a] = size[..., b] = ya.abs() + yb.abs()
    return y, size


def norm_rope_tolerance(y, size):
    """bf16's 2^-8 of the result, and fp32: the norm's factor off by at most 2^-19 (a sum
    of 256 squares, a root, a quotient), two products, sine and cosine off by 2^-22 of one
    (their argument rounded to fp32 among it), the rotation's three roundings."""
    return 2.0 ** -8 * y.abs() + 2.0 ** -18 * size + 1e-38

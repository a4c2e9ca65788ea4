"""Attention over a 4-bit cache where its arithmetic can go wrong: scores, queries, factors
and weights far from one, on every kernel that vd_q4_attend chooses from.  Needs a GB300."""
from __future__ import annotations

import pytest
import torch

import paper_2609_23314_gb300 as vd
import q4_ref as ref
from paper_2609_23314_gb300 import build
from test_gpu_q4_attend import state

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    vd.load_library()
    torch.cuda.set_device(0)
    vd.vd_get_device_status()
    yield
    assert vd.vd_get_device_status() == 0


@pytest.fixture(params=["automatic", "streaming8", "streaming16", "block"], autouse=True)
def route(request, monkeypatch):
    kinds = {"streaming8": "0", "streaming16": "1", "block": "2"}
    if request.param in kinds:
        monkeypatch.setenv("VD_Q4_KERNEL", kinds[request.param])


def run(c, q, k_new, v_new, layer=0, scale=None):
    """out and lse in fp64, and the same from the definition."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    out = torch.full_like(q, 9.0)
    lse = torch.full(q.shape[:-1], 9.0, device="cuda")
    vd.vd_q4_attend(c, q, out, k_new, v_new, layer, scale, lse)
    want_o, want_l = (torch.empty(x.shape, dtype=torch.float64) for x in (out, lse))
    group = q.shape[2] // c.n_kv_head
    scale = float(torch.tensor(scale, dtype=torch.float32))  # what the C call gets
    for s, m in enumerate(c.len.tolist()):
        for h in range(c.n_kv_head):
            ks, vs = (ref.values(x[s, layer, h, :m].cpu(), y[s, layer, h, :m].cpu())
                      for x, y in ((c.k, c.k_scale), (c.v, c.v_scale)))
            new = [None, None] if k_new is None else \
                [x[s, layer, h].cpu().double() for x in (k_new, v_new)]
            hs = slice(h * group, (h + 1) * group)
            o, e = ref.attend(q[s, :, hs].cpu().double(), ks, vs, *new, scale)[:2]
            want_o[s, :, hs], want_l[s, :, hs] = o, e
    return out.cpu().double(), lse.cpu().double(), want_o, want_l


def near(got, want, tol, what):
    err = (got - want).abs() - tol
    assert bool((err <= 0).all()), f"{what} off by {(got - want).abs().max()}, " \
                                   f"{err.max()} more than allowed"


@pytest.mark.parametrize("scale", [1e6, 1e10, 1e20, 1e30])
@pytest.mark.parametrize("B", [1, 40])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_scores_of_any_size(d, B, scale):
    """A query picks one value of every key, so that products are exact and two scores are
    equal or at least 2^-9 of themselves apart, thousands of nats here: out is the mean of
    the values with the largest score.  Weights of 1, whose sums lose 2^-20 at most in fp32,
    and out's rounding; lse: six roundings of 2^-24 from the scale to the result."""
    c, q, k_new, v_new = state([70, 300], 1, 2, 4, d, B, 304)
    q.zero_()
    for h in range(q.shape[2]):
        q[:, :, h, (7 * h) % d] = 1.0 if h % 2 else -1.0
    o, e, want_o, want_l = run(c, q, k_new, v_new, scale=scale)
    most = max(float(ref.values(c.v[..., :70, :].cpu(), c.v_scale[..., :70, :].cpu()).abs().max()),
               float(ref.values(c.v[1].cpu(), c.v_scale[1].cpu()).nan_to_num().abs().max()),
               float(v_new.abs().max()))
    near(o, want_o, 2.0 ** -8 * want_o.abs() + 2.0 ** -20 * most, "out")
    near(e, want_l, 2.0 ** -21 * want_l.abs() + 2.0 ** -18, "lse")


def tolerance(want_o, want_l, a_old, a_new, a_abs, size, keys, d):
    """q4_ref.attend_tolerance, but a weight that is subnormal in fp16 is off by 2^-25 of
    2^-11 of the largest weight: weights are lifted by 2^11 at least before they are rounded."""
    t_out, t_lse = ref.attend_tolerance(want_o, want_l, a_old, a_new, 0 * a_abs, size, keys, d)
    return t_out + 2.0 ** -36 * a_abs, t_lse


@pytest.mark.parametrize("cluster", [None, "1"])
@pytest.mark.parametrize("sink", ["cached", "new"])
@pytest.mark.parametrize("gap", [12.0, 18.0, 20.0, 24.0])
@pytest.mark.parametrize("value", [0.0, 0.015625])
def test_weights_far_below_the_largest(gap, value, sink, cluster, monkeypatch):
    """One key lies `gap` nats above 32768 others, and its own value is small or zero: the
    others carry the output."""
    if cluster:
        monkeypatch.setenv("VD_Q4_CLUSTER", cluster)
    n, d, G = 32769, 64, 4
    g = torch.Generator().manual_seed(3)
    k = torch.zeros(n, d)
    k[:, 1:] = torch.randn(n, d - 1, generator=g)
    v = 1.0 + 0.25 * torch.randn(n, d, generator=g)
    k_new, v_new = torch.zeros(1, d), torch.ones(1, d)
    if sink == "cached":
        k[0], v[0] = 0.0, value
        k[0, 0] = gap
    else:
        k_new[0, 0], v_new[0] = gap, value
    c = vd.Q4Cache.empty(1, 1, 1, n + 7, d)
    for x, codes, scales in ((k, c.k, c.k_scale), (v, c.v, c.v_scale)):
        a, b = ref.quantise(x.to(torch.bfloat16))
        codes[0, 0, 0, :n].copy_(a)
        scales[0, 0, 0, :n].copy_(b)
    c.len.fill_(n)
    q = torch.zeros(1, 1, G, d)
    q[..., 0] = 1.0
    new = [x.to(torch.bfloat16).view(1, 1, 1, 1, d).cuda() for x in (k_new, v_new)]
    qc = q.to(torch.bfloat16).cuda()
    out, lse = torch.empty_like(qc), torch.empty(1, 1, G, device="cuda")
    vd.vd_q4_attend(c, qc, out, new[0], new[1], 0, 1.0, lse)
    ks, vs = (ref.values(x[0, 0, 0, :n].cpu(), y[0, 0, 0, :n].cpu())
              for x, y in ((c.k, c.k_scale), (c.v, c.v_scale)))
    # 20 is held as 6 times 3.25, the scale nearest to 20 / 6
    assert float(ks[:, 0].max()) == ((19.5 if gap == 20.0 else gap) if sink == "cached" else 0.0)
    got = ref.attend(q[0].double(), ks, vs, *(x[0, 0, 0].cpu().double() for x in new), 1.0)
    t_out, t_lse = tolerance(*got, n + 1, d)
    near(out[0].cpu().double(), got[0], t_out, "out")
    near(lse[0].cpu().double(), got[1], t_lse, "lse")


@pytest.mark.parametrize("B", [1, 40])
def test_new_values_up_to_the_limit(B):
    """Values of 2^95 and more in the new rows, which sums of lifted weights have to hold."""
    c, q, k_new, v_new = state([0, 33], 1, 2, 4, 128, B, 40)
    v_new = v_new.clamp(-1.875, 1.875) * 2.0 ** 95
    o, e, want_o, want_l = run(c, q, k_new, v_new)
    # weights in bf16, 2^-8 each, and out's rounding, of values up to 2^96
    near(o, want_o, torch.full_like(o, 2.0 ** -6 * 2.0 ** 96), "out")


@pytest.mark.parametrize("scale,size", [(3.3e38, 0.0), (3.3e38, 1e-36), (1e-44, 0.0), (1e-44, 1e36)])
@pytest.mark.parametrize("B", [1, 40])
def test_scales_of_any_size(B, scale, size):
    """Queries of zero, whose scores are zero at any scale, and queries that make up for the
    scale.  Ordinary tolerances: q4_ref.attend_tolerance."""
    c, q, k_new, v_new = state([70, 33], 1, 2, 4, 128, B, 72)
    q = (q.double() * size).to(torch.bfloat16)
    o, e, want_o, want_l = run(c, q, k_new, v_new, scale=scale)
    group = q.shape[2] // c.n_kv_head
    scale = float(torch.tensor(scale, dtype=torch.float32))
    for s, m in enumerate(c.len.tolist()):
        for h in range(c.n_kv_head):
            ks, vs = (ref.values(x[s, 0, h, :m].cpu(), y[s, 0, h, :m].cpu())
                      for x, y in ((c.k, c.k_scale), (c.v, c.v_scale)))
            hs = slice(h * group, (h + 1) * group)
            got = ref.attend(q[s, :, hs].cpu().double(), ks, vs, k_new[s, 0, h].cpu().double(),
                             v_new[s, 0, h].cpu().double(), scale)
            t_out, t_lse = tolerance(*got, m + B, 128)
            near(o[s, :, hs], got[0], t_out, "out")
            near(e[s, :, hs], got[1], t_lse, "lse")


@pytest.mark.parametrize("B", [2, 40])
def test_factors_below_the_smallest_normal_number(B):
    """New keys of 2^127 under a scale that brings their scores to 2^-6: what the scores are
    multiplied by is subnormal.  Its rounding, 2^-17 of itself, is far below the weights'."""
    d = 256
    c, q, k_new, v_new = state([0, 0], 1, 2, 4, d, B, 40)
    q = torch.full_like(q, 2.0 ** -20)
    sign = torch.where(torch.arange(B, device="cuda") % 2 == 0, 1.0, -1.0)
    k_new = (sign[:, None].expand(B, d) * 1.5 * 2.0 ** 126).to(torch.bfloat16).expand(
        k_new.shape).contiguous()
    o, e, want_o, want_l = run(c, q, k_new, v_new, scale=2.0 ** -121)
    # weights in bf16, 2^-8, out's rounding, the scores' own 2^-16 of at most 2^-5
    mean = v_new.double().abs().cpu().cumsum(3) / torch.arange(1, B + 1)[:, None]
    mean = mean[:, 0].transpose(1, 2).repeat_interleave(4, 2)
    near(o, want_o, 2.0 ** -8 * want_o.abs() + 2.0 ** -7 * mean, "out")
    near(e, want_l, torch.full_like(e, 2.0 ** -18) + 2.0 ** -21 * want_l.abs(), "lse")


@pytest.mark.parametrize("exponent", [0, 116])
@pytest.mark.parametrize("B", [1, 40])
def test_the_largest_queries(B, exponent):
    """Queries of the largest finite bf16 value, with ordinary new keys and with keys of up to
    2^117 (whose scores dwarf the cached ones').  Exact products, so that scores only lose what
    their sums and factor lose; tolerances as everywhere."""
    top = float(torch.finfo(torch.bfloat16).max)
    c, q, k_new, v_new = state([70, 33], 1, 2, 4, 128, B, 72)
    q = torch.where(q > 0, top, -top).to(torch.bfloat16)
    k_new = (k_new.double().clamp(-1.875, 1.875) * 2.0 ** exponent).to(torch.bfloat16)
    scale = 2.0 ** -132 if exponent == 0 else 2.0 ** -149
    o, e, want_o, want_l = run(c, q, k_new, v_new, scale=scale)
    group = q.shape[2] // c.n_kv_head
    for s, m in enumerate(c.len.tolist()):
        for h in range(c.n_kv_head):
            ks, vs = (ref.values(x[s, 0, h, :m].cpu(), y[s, 0, h, :m].cpu())
                      for x, y in ((c.k, c.k_scale), (c.v, c.v_scale)))
            hs = slice(h * group, (h + 1) * group)
            got = ref.attend(q[s, :, hs].cpu().double(), ks, vs, k_new[s, 0, h].cpu().double(),
                             v_new[s, 0, h].cpu().double(), scale)
            t_out, t_lse = tolerance(*got, m + B, 128)
            assert bool(torch.isfinite(o[s, :, hs]).all())
            near(o[s, :, hs], got[0], t_out, "out")
            near(e[s, :, hs], got[1], t_lse, "lse")


@pytest.mark.parametrize("lens", [[0, 3], [200, 70]])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("B", [1, 2, 7, 40, 150])
def test_weights_of_new_rows(B, d, lens):
    """A new row's weight is carried in two bf16 parts, 2^-8 of a weight twice over: 2^-16 at
    most, where q4_ref.attend_tolerance allows for one part."""
    c, q, k_new, v_new = state(lens, 1, 2, 4, d, B, 208)
    o, e, want_o, want_l = run(c, q, k_new, v_new)
    for s, m in enumerate(lens):
        for h in range(2):
            ks, vs = (ref.values(x[s, 0, h, :m].cpu(), y[s, 0, h, :m].cpu())
                      for x, y in ((c.k, c.k_scale), (c.v, c.v_scale)))
            hs = slice(h * 4, (h + 1) * 4)
            got = ref.attend(q[s, :, hs].cpu().double(), ks, vs, k_new[s, 0, h].cpu().double(),
                             v_new[s, 0, h].cpu().double(), d ** -0.5)
            t_out, t_lse = tolerance(*got, m + B, d)
            a_new = got[3]
            near(o[s, :, hs], got[0], t_out - (2.0 ** -8 - 2.0 ** -16) * a_new, "out")
            near(e[s, :, hs], got[1], t_lse, "lse")

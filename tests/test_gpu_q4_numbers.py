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
